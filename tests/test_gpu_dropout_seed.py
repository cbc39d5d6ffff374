"""Dropout without a seed is refused wherever it is drawn, by the fused calls as by the plain one, and needs none where p decides by itself."""
import pytest

from tests.test_gpu_ops import ops

pytestmark = pytest.mark.gpu


def test_fused_dropout_without_a_seed():
    import torch
    o = ops()
    x, m = torch.randn(4, 8, device="cuda:0"), torch.ones(4, device="cuda:0")
    for call in (lambda: o.dropout(x, 0.1, None), lambda: o.dropout_forward(x, 0.1, None), lambda: o.dropout_add_layer_norm(x, x, p=0.1),
                 lambda: o.dropout_add_layer_norm_forward(x, x, None, None, 0.1), lambda: o.dropout_add_layer_norm_forward(x, x, p=0.1, offset=3),
                 lambda: o.dropout_add_layer_norm_backward(x, None, x, None, m, m, 0.1)):
        with pytest.raises(ValueError, match="without a seed"):
            call()
    for p in (0.0, 1.0):
        for got, want in zip(o.dropout_add_layer_norm_forward(x, x, p=p), o.dropout_add_layer_norm_forward(x, x, p=p, seed=5)):
            assert torch.equal(got, want)
        a = x.clone().requires_grad_()
        y, h = o.dropout_add_layer_norm(a, x, p=p)
        (y.sum() + h.sum()).backward()
        b = x.clone().requires_grad_()
        y, h = o.dropout_add_layer_norm(b, x, p=p, seed=0)
        (y.sum() + h.sum()).backward()
        assert torch.equal(a.grad, b.grad)


def test_the_example_draws_by_its_steps_seed():
    import torch
    from tests.test_gpu_example import _example
    import workloads as W
    from paper_2506_10315_amd import LearnedOptTorch
    ex = _example()

    def step(**seed):
        model = ex.TokenModel(vocab=200, width=64, depth=2, dropout=0.3).cuda()
        opt = LearnedOptTorch(model.parameters(), W.velo_weights(0), kind="velo", lr=1e-3)
        return ex.train_step(model, opt, *ex.batch(200, 4, 16, 0, "cuda:0"), **seed)

    with pytest.raises(ValueError, match="without a seed"):
        step()
    first, again, other = step(seed=1), step(seed=1), step(seed=2)
    assert first == again and first != other
