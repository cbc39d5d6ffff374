"""KL divergence where the logits and the reference's are masked by different finite values, down to the types' lowest, in every layout of the kernels, against the definition in float64.
Rows and tolerances: those of the arithmetic's CPU test and of the kernels' own."""
import numpy as np
import pytest

from tests.test_gpu_more_ops import check_kl, kl_exact, kl_tolerance, logits_pair
from tests.test_gpu_ops import TYPES, close, dev, host, ops, tt
from tests.test_kl_sums_cpu import rows_that_x_masks, rows_with_unlikely_tokens_that_r_masks

pytestmark = pytest.mark.gpu

VOCABS = [9, 100, 200, 500, 1500, 3000, 20000, 140000]


def lowest(kind):
    import torch
    return torch.finfo(tt(kind)).min


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("vocab", VOCABS)
def test_tokens_that_x_masks_by_a_finite_value_and_r_by_the_lowest(vocab, kind):
    x, y = rows_that_x_masks(vocab, lowest(kind))
    for scale in (1.0,) if vocab > 3000 else (1.0, 0.5, 2.0):
        kl = host(check_kl(x, y, kind, scale, what=f"scale {scale}"))
        assert np.isfinite(kl).all()


def repeated(x, y, kind, rows):
    """kl and stats of `rows` rows, x's and y's over and over; each like the definition's."""
    import torch
    (a, av), (b, bv) = dev(x, kind), dev(y, kind)
    want = kl_exact(av, bv, 1.0)
    tol, _ = kl_tolerance(av, bv, 1.0, want)
    n = x.shape[0]
    at = torch.arange(rows, device="cuda:0") % n
    kl, stats = ops().token_kl_forward(a[at], b[at])
    k = np.arange(rows) % n
    close(kl, want[0][k], tol[k], "kl")
    close(stats[:, 4], want[1][k, 4], tol[k], "mean")


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("vocab", [9, 200, 500])
def test_many_short_rows_of_such_masks(vocab, kind):
    repeated(*rows_that_x_masks(vocab, lowest(kind)), kind, 8200)


@pytest.mark.parametrize("kind,vocab,rows", [("bf16", 262300, 70), ("fp32", 262300, 66), ("fp16", 20000, 3500), ("fp32", 20000, 1700), ("bf16", 20000, 3500)])
def test_rows_in_segments_and_beyond_the_cache_of_such_masks(kind, vocab, rows):
    """Some 70 rows of more than 2^18 logits are taken in segments; more than 256 MB of logits are read past the cache."""
    x, y = rows_that_x_masks(vocab, lowest(kind))
    repeated(x[::3], y[::3], kind, rows)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("vocab", VOCABS)
def test_unlikely_tokens_that_r_masks_by_the_lowest(vocab, kind):
    x, y = rows_with_unlikely_tokens_that_r_masks(vocab, lowest(kind))
    for scale in (1.0,) if vocab > 3000 else (1.0, 0.5):
        kl = host(check_kl(x, y, kind, scale, what=f"scale {scale}"))
        assert np.isfinite(kl).all()


@pytest.mark.parametrize("kind,vocab,rows", [("bf16", 9, 8200), ("fp32", 200, 8200), ("fp16", 500, 8200), ("bf16", 500, 8200), ("bf16", 262300, 70), ("fp32", 262300, 66),
                                             ("fp16", 20000, 3500), ("fp32", 20000, 1700), ("bf16", 20000, 3500)])
def test_many_rows_segments_and_rows_beyond_the_cache_of_such_tokens(kind, vocab, rows):
    for masked in (False, True):
        x, y = rows_with_unlikely_tokens_that_r_masks(vocab, lowest(kind), masked)
        repeated(x, y, kind, rows)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("vocab", VOCABS)
def test_gradient_of_tokens_of_no_probability_beside_such(vocab, kind):
    """x masks others by the lowest value: their gradient is 0, however large the mean difference is."""
    x, y = rows_with_unlikely_tokens_that_r_masks(vocab, lowest(kind), True)
    x, y = (v[::4] for v in (x, y)) if vocab > 3000 else (x, y)
    check_kl(x, y, kind)
    (xt, xv), (yt, _) = dev(x, kind), dev(y, kind)
    kl, stats = ops().token_kl_forward(xt, yt)
    dx = host(ops().token_kl_backward(xt, yt, stats, kl.new_ones(kl.shape))[0])
    assert np.isfinite(dx).all() and not dx[xv < xv.max(1, keepdims=True) - 200].any()


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("vocab", [9, 500, 3000, 140000])
def test_gradient_where_the_scale_takes_differences_beyond_the_type(vocab, kind):
    """scale (x - r) beyond 3.4e38 under tokens of p = 1e-6, whose gradient is a number."""
    x, y = rows_with_unlikely_tokens_that_r_masks(vocab, lowest(kind))
    x, y = x[2::3][:6], y[2::3][:6]
    r = np.random.default_rng(vocab)
    for scale in (1.0, 1.5, 2.0, 70.0, 1000.0):
        a, b = r.uniform(-1.0, 0.0, x.shape) * 9 / scale, r.uniform(-1.0, 0.0, x.shape) * 9 / scale
        run = y == np.float64(lowest(kind))
        a = np.where(run, a.max() - 14.0 / scale - np.log(vocab) / scale, a)
        check_kl(a, np.where(run, lowest(kind), b), kind, scale, what=f"scale {scale}")


@pytest.mark.parametrize("vocab", VOCABS)
def test_enormous_scales(vocab):
    for scale in (1e20, 1e30):
        s32 = float(np.float32(scale))
        for x, y in (logits_pair(8, vocab, 1), logits_pair(8, vocab, 2, 0.3, 2.0), rows_that_x_masks(vocab, lowest("fp32"))):
            (xt, xv), (yt, yv) = dev(x[:24], "fp32"), dev(y[:24], "fp32")
            want = kl_exact(xv, yv, s32)
            kl, stats = ops().token_kl_forward(xt, yt, scale=scale)
            close(kl, want[0], kl_tolerance(xv, yv, s32, want)[0], f"kl {scale}")
            dx = ops().token_kl_backward(xt, yt, stats, kl.new_zeros(kl.shape).fill_(1e-30), scale=scale)[0]
            assert bool(dx.isfinite().all())
