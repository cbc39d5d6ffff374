"""A small token model trained by a learned optimizer, with everything that bounds such a loop by memory in this package's kernels:
layer norm forward and backward, with dropout and the residual addition in the same pass where there is dropout, the loss as token log probabilities with their
gradient, clipping by the global gradient norm, and the optimizer step, which takes the clipped gradients and the loss value. Beside the likelihood the model is trained
on pairs of answers and on sampled answers with advantages, against a frozen copy of itself.

    python examples/token_model.py [steps]

The optimizer's own weights are seeded random ones (no pretrained weights ship with this repository), so the loss is not
expected to fall; with meta-trained weights the loop is the same."""
from __future__ import annotations

import os
import sys
from typing import Optional

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import workloads as W                                    # noqa: E402
from paper_2506_10315_amd import LearnedOptTorch, ops    # noqa: E402

IGNORE = -100


class TokenModel(torch.nn.Module):
    """Embedding, `depth` residual blocks (layer norm, two linear layers), layer norm, head: a token from the one before."""

    def __init__(self, vocab: int = 1000, width: int = 256, depth: int = 2, seed: int = 0, dropout: float = 0.0):
        super().__init__()
        self.dropout = dropout
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

    def forward(self, tokens: torch.Tensor, seed: Optional[int] = None) -> torch.Tensor:
        """Logits. `seed`: that of this step's dropout, which has to be given in training with it."""
        x = self.embed[tokens]
        if self.dropout and self.training:
            return self._dropped(x, seed)
        for b in self.blocks:
            h = ops.layer_norm(x, b.norm_w, b.norm_b)
            x = x + torch.nn.functional.gelu(h @ b.up.t()) @ b.down.t()
        return ops.layer_norm(x, self.norm_w, self.norm_b) @ self.head.t()

    def _dropped(self, x: torch.Tensor, seed: Optional[int]) -> torch.Tensor:
        """The same with dropout of the embedding and of what every block adds: each with its number as offset, with the addition and the norm behind it."""
        x = ops.dropout(x, self.dropout, seed, 0)
        norms = [(b.norm_w, b.norm_b) for b in self.blocks] + [(self.norm_w, self.norm_b)]
        y = ops.layer_norm(x, *norms[0])
        for i, b in enumerate(self.blocks, 1):
            out = torch.nn.functional.gelu(y @ b.up.t()) @ b.down.t()
            y, x = ops.dropout_add_layer_norm(out, x, *norms[i], self.dropout, seed, i)
        return y @ self.head.t()


def loss_of(logits: torch.Tensor, targets: torch.Tensor, entropy_weight: float = 0.0):
    """Mean of -log p over the targets that are not padding, less an entropy bonus."""
    r = ops.token_logprobs(logits, targets, ignore_index=IGNORE)
    kept = (targets != IGNORE).float()
    n = kept.sum().clamp_min(1.0)
    loss = -r.logp.sum() / n
    if entropy_weight:
        loss = loss - entropy_weight * (r.entropy * kept).sum() / n
    return loss


def policy_loss_of(logits: torch.Tensor, ref_logits: torch.Tensor, targets: torch.Tensor, old_logp: torch.Tensor, advantages: torch.Tensor, kl_coef: float = 0.05,
                   entropy_coef: float = 0.01):
    """Clipped policy loss of sampled answers (targets that are not padding), with their distance from the reference and an entropy bonus; one advantage
    an answer."""
    kept = targets != IGNORE
    r = ops.token_logprobs(logits, targets, ignore_index=IGNORE)
    kl = ops.token_kl(logits, ref_logits, mask=kept)
    return ops.policy_loss(r.logp, old_logp, advantages, kept, kl=kl, kl_coef=kl_coef, entropy=r.entropy, entropy_coef=entropy_coef, reduction="sequences")


def preference_loss_of(logits: torch.Tensor, ref_logp: torch.Tensor, targets: torch.Tensor, beta: float = 0.1):
    """Loss of pairs of answers: the preferred ones in the first half of the rows, the others in the same order in the second."""
    r = ops.token_logprobs(logits, targets, ignore_index=IGNORE)
    return ops.preference_loss(r.logp, ref_logp, targets != IGNORE, beta)


def step_on(loss, model, optimizer, max_norm: float = 1.0):
    """The gradients of a loss, clipped, and the optimizer's step; (loss, gradient norm before clipping)."""
    optimizer.zero_grad()
    loss.backward()
    norm = ops.clip_grad_norm_(model.parameters(), max_norm)
    optimizer.step(loss)
    return float(loss.detach()), float(norm)


def train_step(model, optimizer, tokens, targets, max_norm: float = 1.0, entropy_weight: float = 0.01, seed: Optional[int] = None):
    """One step of training, its dropout drawn from `seed`, another one in every step; (loss, gradient norm before clipping)."""
    loss = loss_of(model(tokens, seed), targets, entropy_weight)
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
    reference = TokenModel().to(device).eval()
    for step in range(steps):
        loss, norm = train_step(model, optimizer, *batch(1000, 16, 64, step, device))
        print(f"step {step}: loss {loss:.4f}, gradient norm {norm:.4f}", flush=True)
    model.dropout = 0.1
    for step in range(steps):
        tokens, targets = batch(1000, 16, 64, 100 + step, device)
        with torch.no_grad():
            ref_logits = reference(tokens)
            ref_logp = ops.token_logprobs_forward(ref_logits, targets, ignore_index=IGNORE).logp
        loss, norm = train_step(model, optimizer, tokens, targets, seed=step)
        print(f"with dropout, step {step}: loss {loss:.4f}, gradient norm {norm:.4f}", flush=True)
        p = policy_loss_of(model(tokens, seed=1000 + step), ref_logits, targets, ref_logp, torch.linspace(-1.0, 1.0, 16, device=device))
        print(f"policy loss, gradient norm: {step_on(p.loss, model, optimizer)}, kl {float(p.stats[1]):.5f}", flush=True)
        q = preference_loss_of(model(tokens, seed=2000 + step), ref_logp, targets)
        print(f"preference loss, gradient norm: {step_on(q.loss, model, optimizer)}, right {float(q.stats[0]):.3f}", flush=True)
    model.eval()
    print("sampled:", sample(model, torch.tensor([3, 4, 5], device=device)))


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 5)
