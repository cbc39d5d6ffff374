"""The example's steps with dropout, on sampled answers and on pairs of answers against the same model in plain torch on the CPU in float64: losses and gradients."""
import pytest

from tests.test_gpu_example import _example
from tests.test_gpu_more_ops import EPS, U, host, keep_of

pytestmark = pytest.mark.gpu

# every value passes some 14 stages, each a sum of at most 501 terms: 14 * 501 roundings of 2^-24 at worst
REL = 14 * 501 * U


def _plain(params, depth, tokens, p, seed):
    """The example's logits from elementary operations, float64."""
    import numpy as np
    import torch

    def norm(x, w, b):
        d = x - x.mean(-1, keepdim=True)
        return d / (d.square().mean(-1, keepdim=True) + EPS).sqrt() * w + b

    def drop(x, offset):
        if not p:
            return x
        keep = keep_of(x.numel() // x.shape[-1], x.shape[-1], p, seed, offset).reshape(x.shape)
        return x * torch.from_numpy(keep) / (1 - float(np.float32(p)))

    x = drop(params["embed"][tokens], 0)
    for i in range(depth):
        q = {k: params[f"blocks.{i}.{k}"] for k in ("norm_w", "norm_b", "up", "down")}
        x = x + drop(torch.nn.functional.gelu(norm(x, q["norm_w"], q["norm_b"]) @ q["up"].t()) @ q["down"].t(), i + 1)
    return norm(x, params["norm_w"], params["norm_b"]) @ params["head"].t()


def _setup(dropout):
    ex = _example()
    model = ex.TokenModel(vocab=501, width=96, depth=2, dropout=dropout).cuda()
    reference = ex.TokenModel(vocab=501, width=96, depth=2, seed=1).cuda()
    tokens, targets = ex.batch(501, 6, 37, 1, "cuda:0")
    params = {k: v.detach().cpu().double().requires_grad_() for k, v in model.named_parameters()}
    return ex, model, reference, tokens, targets, params


def _compare(model, params, got, want):
    assert abs(float(got.detach()) - float(want.detach())) <= REL * (1 + abs(float(want.detach())))
    got.backward()
    want.backward()
    for k, v in model.named_parameters():
        g, e = host(v.grad), params[k].grad.numpy()
        assert abs(g - e).max() <= REL * abs(e).max(), k


@pytest.mark.parametrize("dropout", [0.0, 0.2])
def test_training_step_with_dropout(dropout):
    import torch
    ex, model, _, tokens, targets, params = _setup(dropout)
    got = ex.loss_of(model(tokens, seed=9), targets, 0.01)
    lp = torch.log_softmax(_plain(params, 2, tokens.cpu(), dropout, 9), -1)
    t = targets.cpu()
    kept = t != ex.IGNORE
    at = lp.gather(-1, t.clamp_min(0)[..., None])[..., 0]
    want = (-(at * kept).sum() - 0.01 * (-(lp.exp() * lp).sum(-1) * kept).sum()) / kept.sum()
    _compare(model, params, got, want)
    model.eval()
    with torch.no_grad():
        assert torch.equal(model(tokens, seed=1), model(tokens, seed=2))


def test_policy_step():
    import torch
    ex, model, reference, tokens, targets, params = _setup(0.1)
    t = targets.cpu()
    kept = t != ex.IGNORE
    adv = torch.linspace(-1.0, 1.5, 6)
    with torch.no_grad():
        ref_logits = reference(tokens)
        model.eval()
        old = ex.ops.token_logprobs_forward(model(tokens), targets, ignore_index=ex.IGNORE).logp
        model.train()
    p = ex.policy_loss_of(model(tokens, seed=4), ref_logits, targets, old, adv.cuda())
    lp, lq = torch.log_softmax(_plain(params, 2, tokens.cpu(), 0.1, 4), -1), torch.log_softmax(ref_logits.cpu().double(), -1)
    ratio = (lp.gather(-1, t.clamp_min(0)[..., None])[..., 0] - old.cpu().double()).exp()
    a = adv.double()[:, None]
    each = -torch.minimum(ratio * a, ratio.clamp(0.8, 1.2) * a) + 0.05 * (lp.exp() * (lp - lq)).sum(-1) + 0.01 * (lp.exp() * lp).sum(-1)
    n = kept.sum(1)
    want = ((each * kept).sum(1) / n.clamp_min(1)).sum() / (n > 0).sum()
    # a ratio so near its bound that the roundings decide on which side it lies would change its gradient: none is
    assert bool((((ratio - 1.2).abs() > 1e-3) & ((ratio - 0.8).abs() > 1e-3) | ~kept).all())
    _compare(model, params, p.loss, want)


def test_preference_step():
    import torch
    ex, model, reference, tokens, targets, params = _setup(0.1)
    t = targets.cpu()
    kept = t != ex.IGNORE
    with torch.no_grad():
        ref = ex.ops.token_logprobs_forward(reference(tokens), targets, ignore_index=ex.IGNORE).logp
    q = ex.preference_loss_of(model(tokens, seed=6), ref, targets)
    lp = torch.log_softmax(_plain(params, 2, tokens.cpu(), 0.1, 6), -1)
    s = ((lp.gather(-1, t.clamp_min(0)[..., None])[..., 0] - ref.cpu().double()) * kept).sum(1)
    _compare(model, params, q.loss, -torch.nn.functional.logsigmoid(0.1 * (s[:3] - s[3:])).mean())


def test_steps_run_with_the_optimizer(capsys):
    ex = _example()
    ex.main(1)
    out = capsys.readouterr().out
    assert out.count("gradient norm") == 4 and "nan" not in out
