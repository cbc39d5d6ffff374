"""A small token model trained by a learned optimizer, with everything that bounds such a loop by memory in this package's kernels:
layer norm forward and backward, the loss as token log probabilities with their gradient, clipping by the global gradient norm, and the
optimizer step, which takes the clipped gradients and the loss value.

    python examples/token_model.py [steps]

The optimizer's own weights are seeded random ones (no pretrained weights ship with this repository), so the loss is not
expected to fall; with meta-trained weights the loop is the same."""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import workloads as W                                    # noqa: E402
from paper_2506_10315_amd import LearnedOptTorch, ops    # noqa: E402

IGNORE = -100


class TokenModel(torch.nn.Module):
    """Embedding, `depth` residual blocks (layer norm, two linear layers), layer norm, head: a token from the one before."""

    def __init__(self, vocab: int = 1000, width: int = 256, depth: int = 2, seed: int = 0):
        super().__init__()
        gen = torch.Generator().manual_seed(seed)

        def weight(*shape):
            return torch.nn.Parameter(torch.randn(*shape, generator=gen) / shape[-1] ** 0.5)

        self.embed = weight(vocab, width)
        self.blocks = torch.nn.ModuleList()
        for _ in range(depth):
            b = torch.nn.Module()
            b.norm_w, b.norm_b = torch.nn.Parameter(torch.ones(width)), torch.nn.Parameter(torch.zeros(width))
            b.up, b.down = weight(4 * width, width), weight(width, 4 * width)
            self.blocks.append(b)
        self.norm_w, self.norm_b = torch.nn.Parameter(torch.ones(width)), torch.nn.Parameter(torch.zeros(width))
        self.head = weight(vocab, width)

    def forward(self, tokens: torch.Tensor) -> torch.Tensor:
        x = self.embed[tokens]
        for b in self.blocks:
            h = ops.layer_norm(x, b.norm_w, b.norm_b)
            x = x + torch.nn.functional.gelu(h @ b.up.t()) @ b.down.t()
        return ops.layer_norm(x, self.norm_w, self.norm_b) @ self.head.t()


def loss_of(logits: torch.Tensor, targets: torch.Tensor, entropy_weight: float = 0.0):
    """Mean of -log p over the targets that are not padding, less an entropy bonus."""
    r = ops.token_logprobs(logits, targets, ignore_index=IGNORE)
    kept = (targets != IGNORE).float()
    n = kept.sum().clamp_min(1.0)
    loss = -r.logp.sum() / n
    if entropy_weight:
        loss = loss - entropy_weight * (r.entropy * kept).sum() / n
    return loss


def train_step(model, optimizer, tokens, targets, max_norm: float = 1.0, entropy_weight: float = 0.01):
    """One step of training; (loss, gradient norm before clipping)."""
    loss = loss_of(model(tokens), targets, entropy_weight)
    optimizer.zero_grad()
    loss.backward()
    norm = ops.clip_grad_norm_(model.parameters(), max_norm)
    optimizer.step(loss)
    return float(loss.detach()), float(norm)


def batch(vocab: int, rows: int, length: int, seed: int, device):
    """Token sequences of different lengths, each token the one before plus a constant; the rest is padding."""
    gen = torch.Generator().manual_seed(seed)
    start, stride = torch.randint(0, vocab, (rows, 1), generator=gen), torch.randint(1, 4, (rows, 1), generator=gen)
    seq = (start + stride * torch.arange(length + 1)) % vocab
    tokens, targets = seq[:, :-1].contiguous(), seq[:, 1:].clone()
    lengths = torch.randint(1, length + 1, (rows, 1), generator=gen)
    targets[torch.arange(length) >= lengths] = IGNORE
    return tokens.to(device), targets.to(device)


def sample(model, tokens, length: int = 4, top: int = 5, temperature: float = 0.8):
    """Continues one sequence token by token from its best alternatives; (token, its log probability) of each."""
    out = []
    with torch.no_grad():
        for i in range(length):
            logits = model(tokens)[-1]
            r = ops.token_logprobs_forward(logits, None, scale=1.0 / temperature, top=top)
            pick = r.top_index[i % top].reshape(1)
            out.append((int(pick), float(r.top_logp[i % top])))
            tokens = torch.cat([tokens, pick])
    return out


def main(steps: int = 5):
    device = "cuda:0"
    model = TokenModel().to(device)
    optimizer = LearnedOptTorch(model.parameters(), W.velo_weights(0), kind="velo", lr=1e-3)
    for step in range(steps):
        loss, norm = train_step(model, optimizer, *batch(1000, 16, 64, step, device))
        print(f"step {step}: loss {loss:.4f}, gradient norm {norm:.4f}", flush=True)
    print("sampled:", sample(model, torch.tensor([3, 4, 5], device=device)))


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 5)
