"""The example's training step against the same model in plain torch on the CPU in float64: loss, gradient norm, clipped
gradients, and the optimizer step fed with them."""
import importlib.util
import os

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("token_model", os.path.join(ROOT, "examples", "token_model.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _plain_loss(params, depth, tokens, targets, entropy_weight, ignore):
    """The example's model and loss from elementary operations, float64."""
    import torch

    def norm(x, w, b):
        d = x - x.mean(-1, keepdim=True)
        return d / (d.square().mean(-1, keepdim=True) + float(np.float32(1e-5))).sqrt() * w + b

    x = params["embed"][tokens]
    for i in range(depth):
        p = {k: params[f"blocks.{i}.{k}"] for k in ("norm_w", "norm_b", "up", "down")}
        x = x + torch.nn.functional.gelu(norm(x, p["norm_w"], p["norm_b"]) @ p["up"].t()) @ p["down"].t()
    lp = torch.log_softmax(norm(x, params["norm_w"], params["norm_b"]) @ params["head"].t(), -1)
    kept = targets != ignore
    n = kept.sum().double()
    at = lp.gather(-1, targets.clamp_min(0)[..., None])[..., 0]
    return -(at * kept).sum() / n - entropy_weight * (-(lp.exp() * lp).sum(-1) * kept).sum() / n


def test_training_step_of_the_example():
    import torch
    import workloads as W
    ex = _example()
    from paper_2506_10315_amd import LearnedOptTorch, ops
    model = ex.TokenModel(vocab=501, width=96, depth=2).cuda()
    tokens, targets = ex.batch(501, 6, 37, 1, "cuda:0")
    params = {k: v.detach().cpu().double().requires_grad_() for k, v in model.named_parameters()}
    want = _plain_loss(params, 2, tokens.cpu(), targets.cpu(), 0.01, ex.IGNORE)
    want.backward()
    norm = float(torch.sqrt(sum((p.grad ** 2).sum() for p in params.values())))

    loss = ex.loss_of(model(tokens), targets, 0.01)
    loss.backward()
    # every value passes some 12 stages, each a sum of at most 501 terms: 12 * 501 roundings of 2^-24 at worst
    rel = 12 * 501 * 2.0 ** -24
    assert abs(float(loss.detach()) - float(want.detach())) <= rel * abs(float(want.detach()))
    before = {k: v.detach().clone() for k, v in model.named_parameters()}
    got = ops.clip_grad_norm_(model.parameters(), 0.25 * norm)
    assert abs(float(got) - norm) <= rel * norm
    c = 0.25 * norm / (norm + 1e-6)
    for k, p in model.named_parameters():
        a, b = p.grad.cpu().double(), c * params[k].grad
        assert float((a - b).norm()) <= rel * max(float(b.norm()), 1e-3 * c * norm), k
    opt = LearnedOptTorch(model.parameters(), W.velo_weights(0), kind="velo", lr=1e-3)
    opt.step(loss)
    moved = [not torch.equal(before[k], v) for k, v in model.named_parameters()]
    assert all(moved) and all(bool(torch.isfinite(v).all()) for v in model.parameters())


def test_example_trains_and_samples():
    import torch
    import workloads as W
    ex = _example()
    from paper_2506_10315_amd import LearnedOptTorch

    def run():
        model = ex.TokenModel(vocab=200, width=64, depth=1).cuda()
        opt = LearnedOptTorch(model.parameters(), W.velo_weights(0), kind="velo", lr=1e-3)
        out = [ex.train_step(model, opt, *ex.batch(200, 4, 16, s, "cuda:0")) for s in range(3)]
        return out, ex.sample(model, torch.tensor([1, 2], device="cuda:0"))

    steps, picks = run()
    assert all(np.isfinite(v) for s in steps for v in s) and len(picks) == 4
    assert all(lp <= 0 for _, lp in picks)
    assert abs(steps[0][0] - np.log(200)) < 1.5      # an untrained model: near the uniform distribution's loss
