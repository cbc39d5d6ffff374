"""Dropout, dropout with residual and layer norm, the KL divergence of logits, the policy and the preference loss against their formulas in float64 on the host,
through the torch functions and the C boundary.

Tolerances are bounds derived from the order of the operations, with the names of test_gpu_ops: U is the unit roundoff of float32, depth(n) the longest
chain of additions that any of n terms goes through, ROUND a type's own rounding."""
import math

import numpy as np
import pytest

from tests.test_gpu_ops import (NORM_SHAPES, ROUND, TINY, TYPES, U, close, depth, dev, host, norm_back_exact, norm_back_tolerance, norm_exact, norm_tolerance, ops, tt)

pytestmark = pytest.mark.gpu

EPS = float(np.float32(1e-5))


# ---------------------------------------------------------------------------------------------- the generator and dropout

def philox(counter, key):
    """Philox4x32 of ten rounds: four words for each counter. uint64 arrays of 32-bit values."""
    c = [np.asarray(v, dtype=np.uint64) for v in counter]
    k = [np.uint64(v) for v in key]
    low = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ k[0], b & low, (a >> np.uint64(32)) ^ c[3] ^ k[1], a & low]
        k = [(k[0] + np.uint64(0x9E3779B9)) & low, (k[1] + np.uint64(0xBB67AE85)) & low]
    return c


def keep_of(rows, cols, p, seed, offset=0, first_row=0):
    """The mask of the definition in include/lopt.h."""
    k = np.arange((cols + 3) // 4, dtype=np.uint64)[None, :]
    r = np.arange(first_row, first_row + rows, dtype=np.uint64)[:, None]
    full = np.broadcast_to(np.uint64(0), (rows, k.shape[1]))
    words = philox((k + full, r + full, np.uint64(offset & 0xFFFFFFFF) + full, np.uint64(offset >> 32) + full), (seed & 0xFFFFFFFF, seed >> 32))
    word = np.stack(words, -1).reshape(rows, -1)[:, :cols]
    return word >= np.uint64(round(float(np.float32(p)) * 2.0 ** 32))


def dropped(x, keep, p):
    return np.where(keep, x / (1.0 - float(np.float32(p))) if p < 1 else 0.0, 0.0)


def test_generator_of_this_file():
    """Known answers of Philox4x32-10, as its authors publish them."""
    for counter, key, want in (((0,) * 4, (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
                               ((0xffffffff,) * 4, (0xffffffff,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
                               ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0), (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1))):
        assert tuple(int(v) for v in philox(counter, key)) == want


DROP_SHAPES = [(1, 1), (5, 1), (3, 2), (7, 3), (4, 4), (5, 7), (9, 8), (1000, 9), (33, 17), (3, 64), (21, 127), (300, 257), (70, 768), (5, 1531), (3, 4099), (2, 32769 * 4), (1, 300001)]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,cols", DROP_SHAPES)
def test_dropout(rows, cols, kind):
    import torch
    r = np.random.default_rng(rows * 1000 + cols)
    x, xv = dev(r.standard_normal((rows, cols)), kind)
    for p, seed, offset in ((0.1, 7, 0), (0.5, (1 << 63) + 12345, (1 << 63) + 5), (0.0, 7, 0), (1.0, 7, 3), (1e-7, 1 << 40, 1 << 33), (0.999, 3, 4)):
        y = ops().dropout_forward(x, p, seed, offset)
        want = dropped(xv, keep_of(rows, cols, p, seed, offset), p)
        # scale and product are rounded to 32 bits, then the output
        close(y, want, (2 * U + 1.01 * ROUND[kind]) * np.abs(want) + TINY[kind], f"p {p}")
        assert y.dtype is x.dtype and torch.equal(y, ops().dropout_forward(x, p, seed, offset))
        if seed < 1 << 63:
            assert torch.equal(y, ops().dropout_forward(x, p, torch.tensor(seed, device="cuda:0"), offset))
    if rows * cols > 200:
        assert not torch.equal(ops().dropout_forward(x, 0.5, 7, 0), ops().dropout_forward(x, 0.5, 8, 0))
        assert not torch.equal(ops().dropout_forward(x, 0.5, 7, 0), ops().dropout_forward(x, 0.5, 7, 1))


def test_dropout_beyond_32_bits_of_packs():
    import torch
    rows = (1 << 32) // 7 + 1000
    x, xv = dev(np.array([1.0, 2.0, 3.0, 4.0, 5.0, 6.0, 7.0]), "fp16")
    y = ops().dropout_forward(x[None].expand(rows, 7), 0.5, 11, 5)
    for first in (0, (1 << 31) // 7 - 50, (1 << 32) // 7 - 50, rows - 100):
        assert np.array_equal(host(y[first:first + 100]), dropped(np.broadcast_to(xv, (100, 7)), keep_of(100, 7, 0.5, 11, 5, first), 0.5))


def test_dropout_rate_and_independence():
    """Shares of kept elements, of neighbours, of rows and of calls kept together: within five standard deviations of a binomial."""
    import torch
    n = 1 << 22
    x = torch.ones(2048, n // 2048, device="cuda:0")
    for p in (0.1, 0.5):
        a, b = (ops().dropout_forward(x, p, 99, k) != 0 for k in (0, 1))
        c = ops().dropout_forward(x, p, 100, 0) != 0
        for both, q in ((a, 1 - p), (a & b, (1 - p) ** 2), (a & c, (1 - p) ** 2), (a[:, 1:] & a[:, :-1], (1 - p) ** 2), (a[1:] & a[:-1], (1 - p) ** 2)):
            m = both.numel()
            assert abs(int(both.sum()) - m * q) <= 5 * math.sqrt(m * q * (1 - q)), (p, q)


def test_dropout_is_a_selection():
    """What is dropped is 0 whatever it was; what stays is passed on."""
    import torch
    x = torch.full((50, 333), math.nan, device="cuda:0")
    x[::2] = math.inf
    y = ops().dropout_forward(x, 0.5, 11)
    keep = torch.from_numpy(keep_of(50, 333, 0.5, 11)).cuda()
    assert bool((y[~keep] == 0).all()) and bool(y[1::2][keep[1::2]].isnan().all()) and bool((y[::2][keep[::2]] == math.inf).all())
    assert bool((ops().dropout_forward(x, 1.0, 11) == 0).all())


@pytest.mark.parametrize("kind", TYPES)
def test_dropout_strides_dimensions_margins_and_in_place(kind):
    import ctypes as C
    import torch
    from paper_2506_10315_amd import lib
    r = np.random.default_rng(4)
    buf, bv = dev(r.standard_normal((40, 91)), kind)
    keep = keep_of(40, 77, 0.3, 5)
    flat = ops().dropout_forward(buf[:, 3:80].contiguous(), 0.3, 5)
    assert torch.equal(ops().dropout_forward(buf[:, 3:80], 0.3, 5), flat)                       # rows at a distance, off every grid
    assert torch.equal(ops().dropout_forward(buf[:, 3:80].reshape(5, 8, 77), 0.3, 5), flat.view(5, 8, 77))
    assert torch.equal(ops().dropout_forward(buf[:, 3:80].t().contiguous().t(), 0.3, 5), flat)  # columns at a distance
    one = ops().dropout_forward(buf[:1, 3:80].expand(40, 77), 0.3, 5)                           # one row for all
    want = dropped(np.broadcast_to(bv[0, 3:80], (40, 77)), keep, 0.3)
    close(one, want, (2 * U + 1.01 * ROUND[kind]) * np.abs(want) + TINY[kind], "one row")
    t = buf.clone()
    kinds = {"fp32": 0, "bf16": 1, "fp16": 2}
    at = t.data_ptr() + 3 * t.element_size()
    assert lib().lopt_dropout(at, 91, at, 91, 40, 77, kinds[kind], 0.3, 5, None, 0, C.c_void_p(torch.cuda.current_stream().cuda_stream)) == 0
    assert torch.equal(t[:, 3:80], flat) and torch.equal(t[:, :3], buf[:, :3]) and torch.equal(t[:, 80:], buf[:, 80:])
    assert ops().dropout_forward(buf[:0], 0.3, 5).shape == (0, 91)
    assert torch.equal(ops().dropout_forward(buf[0, 3:80], 0.3, 5), ops().dropout_forward(buf[:1, 3:80], 0.3, 5)[0])


def test_dropout_gradient():
    import torch
    r = np.random.default_rng(6)
    x, xv = dev(r.standard_normal((31, 45)), "fp32")
    g, gv = dev(r.standard_normal((31, 45)), "fp32")
    for seed in (17, torch.tensor(17, device="cuda:0")):
        x.grad = None
        x.requires_grad_()
        ops().dropout(x, 0.25, seed, 2).backward(g)
        assert torch.equal(x.grad, ops().dropout_forward(g, 0.25, 17, 2))
    # differences: the function is linear, so that they are its values
    keep = keep_of(31, 45, 0.25, 17, 2)
    d = r.standard_normal(xv.shape)
    slope = float((dropped(xv + d, keep, 0.25) * gv).sum() - (dropped(xv - d, keep, 0.25) * gv).sum()) / 2
    got = float((host(x.grad) * d).sum())
    assert abs(got - slope) <= 3 * U * float(np.abs(host(x.grad) * d).sum()) + 1e-12
    # a seed that changes before the backward pass is seen
    seed = torch.tensor(17, device="cuda:0")
    y = ops().dropout(x, 0.25, seed)
    seed += 1
    with pytest.raises(RuntimeError, match="modified"):
        y.sum().backward()


# ---------------------------------------------------------------------------------------------- dropout, residual, layer norm

PAIRS = [("fp32", "fp32"), ("bf16", "bf16"), ("bf16", "fp32"), ("fp16", "fp16"), ("fp16", "fp32")]
FUSED_SHAPES = [s for s in NORM_SHAPES if s not in ((2, 8200),)] + [(3, 9000), (4, 12), (2, 16385)]


def fused_case(r, rows, cols, kind, rkind):
    x, xv = dev(0.5 * r.standard_normal((rows, cols)), kind)
    res, rv = dev(r.standard_normal((rows, cols)) * np.exp(0.5 * r.standard_normal((rows, 1))) + r.standard_normal((rows, 1)), rkind)
    return x, xv, res, rv


@pytest.mark.parametrize("kind,rkind", PAIRS)
@pytest.mark.parametrize("rows,cols", FUSED_SHAPES)
def test_dropout_add_layer_norm_forward(rows, cols, kind, rkind):
    r = np.random.default_rng(rows * 1000 + cols)
    x, xv, res, rv = fused_case(r, rows, cols, kind, rkind)
    for p, wkind, have_w, have_b in ((0.2, "fp32", True, True), (0.0, kind, True, False), (1.0, "bf16", False, True), (0.5, "fp32", False, False)):
        w, wv = dev(1 + 0.3 * r.standard_normal(cols), wkind) if have_w else (None, None)
        b, bv = dev(0.3 * r.standard_normal(cols), wkind) if have_b else (None, None)
        y, h, mean, rstd = ops().dropout_add_layer_norm_forward(x, res, w, b, p, 21, 4, eps=1e-5)
        assert y.dtype is x.dtype and h.dtype is res.dtype
        drop = dropped(xv, keep_of(rows, cols, p, 21, 4), p)
        # scale and product, the sum, and the rounding as it is stored
        close(h, rv + drop, 2 * U * np.abs(drop) + (U + 1.01 * ROUND[rkind]) * np.abs(rv + drop) + TINY[rkind], f"h p {p}")
        hv = host(h)   # the norm is of what is stored
        for got, a, t, what in zip((y, mean, rstd), norm_exact(hv, wv, bv, EPS), norm_tolerance(hv, wv, bv, EPS, kind), ("y", "mean", "rstd")):
            close(got, a, t, f"{what} p {p} weights {wkind} {have_w} {have_b}")


@pytest.mark.parametrize("kind,rkind", PAIRS)
@pytest.mark.parametrize("rows,cols", FUSED_SHAPES + [(3000, 96), (1301, 333), (9000, 8)])
def test_dropout_add_layer_norm_backward(rows, cols, kind, rkind):
    import torch
    r = np.random.default_rng(rows * 1000 + cols)
    _, _, h, hv = fused_case(r, rows, cols, kind, rkind)
    dy, dyv = dev(r.standard_normal((rows, cols)), kind)
    dh, dhv = dev(r.standard_normal((rows, cols)), rkind)
    mean = torch.from_numpy(hv.mean(1).astype(np.float32)).cuda()
    rstd = torch.from_numpy((1 / np.sqrt(hv.var(1) + EPS)).astype(np.float32)).cuda()
    mv, rs = host(mean), host(rstd)
    for p, wkind, have_w, have_dh in ((0.2, "fp32", True, True), (0.0, kind, True, True), (0.5, "fp32", False, False)):
        w, wv = dev(1 + 0.3 * r.standard_normal(cols), wkind) if have_w else (None, None)
        got = ops().dropout_add_layer_norm_backward(dy, dh if have_dh else None, h, w, mean, rstd, p, 21, 4)
        norm_dx, dw, db = norm_back_exact(dyv, hv, wv, mv, rs)[:3]
        tol_norm, tol_w, tol_b = norm_back_tolerance(dyv, hv, wv, mv, rs, "fp32", wkind)
        d = norm_dx + (dhv if have_dh else 0.0)
        tol = tol_norm + U * np.abs(d)   # the gradient of h is added
        keep, scale = keep_of(rows, cols, p, 21, 4), 1.0 / (1.0 - float(np.float32(p)))
        want = (np.where(keep, d * scale, 0.0), d, dw, db)
        tols = (np.where(keep, scale * tol + (2 * U + 1.01 * ROUND[kind]) * np.abs(d * scale) + TINY[kind], 0.0), tol + 1.01 * ROUND[rkind] * np.abs(d) + TINY[rkind], tol_w, tol_b)
        for g, a, t, what in zip(got, want, tols, ("dx", "dresidual", "dw", "db")):
            close(g, a, t, f"{what} p {p} weights {wkind} {have_w} dh {have_dh}")
        assert (got[0] is got[1]) == (p == 0.0 and kind == rkind)
        again = ops().dropout_add_layer_norm_backward(dy, dh if have_dh else None, h, w, mean, rstd, p, 21, 4)
        assert all(torch.equal(a, b) for a, b in zip(got, again))
        for need in ((True, False, False, False), (False, True, False, False), (False, False, True, False), (False, False, False, True), (False,) * 4):
            part = ops().dropout_add_layer_norm_backward(dy, dh if have_dh else None, h, w, mean, rstd, p, 21, 4, need=need)
            for k in range(4):
                assert (part[k] is None) == (not need[k])
                assert part[k] is None or torch.equal(part[k], got[k]), (need, k)


@pytest.mark.parametrize("kind,rkind", [("bf16", "fp32"), ("fp16", "fp16")])
@pytest.mark.parametrize("cols", [77, 1531, 16391])
def test_dropout_add_layer_norm_strides_and_margins(cols, kind, rkind):
    import torch
    r = np.random.default_rng(9)
    big = [dev(r.standard_normal((7, cols + 14)), k)[0] for k in (kind, rkind, kind, rkind)]
    x, res, dy, dh = (t[:, 3 + i:3 + i + cols] for i, t in enumerate(big))
    w = dev(1 + 0.3 * r.standard_normal(cols), "fp32")[0]
    a = ops().dropout_add_layer_norm_forward(x, res, w, w, 0.3, 5)
    b = ops().dropout_add_layer_norm_forward(x.contiguous(), res.contiguous(), w, w, 0.3, 5)
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    y, h, mean, rstd = a
    g = ops().dropout_add_layer_norm_backward(dy, dh, res, w, mean, rstd, 0.3, 5)
    e = ops().dropout_add_layer_norm_backward(dy.contiguous(), dh.contiguous(), res.contiguous(), w, mean, rstd, 0.3, 5)
    assert all(torch.equal(p, q) for p, q in zip(g, e))
    # through the boundary: outputs into margins, in place of inputs
    import ctypes as C
    from paper_2506_10315_amd import lib
    kinds = {"fp32": 0, "bf16": 1, "fp16": 2}
    s = C.c_void_p(torch.cuda.current_stream().cuda_stream)
    bx, br = big[0].clone(), big[1].clone()
    px, pr = bx.data_ptr() + 3 * bx.element_size(), br.data_ptr() + 4 * br.element_size()
    ld = cols + 14
    m2, r2 = torch.empty(7, device="cuda:0"), torch.empty(7, device="cuda:0")
    assert lib().lopt_dropout_add_layer_norm(px, ld, pr, ld, w.data_ptr(), w.data_ptr(), px, ld, pr, ld, m2.data_ptr(), r2.data_ptr(), 7, cols, 1e-5, kinds[kind], kinds[rkind],
                                             0, 0.3, 5, None, 0, s) == 0
    assert torch.equal(bx[:, 3:3 + cols], y) and torch.equal(br[:, 4:4 + cols], h) and torch.equal(m2, mean) and torch.equal(r2, rstd)
    assert torch.equal(bx[:, :3], big[0][:, :3]) and torch.equal(bx[:, 3 + cols:], big[0][:, 3 + cols:])
    assert torch.equal(br[:, :4], big[1][:, :4]) and torch.equal(br[:, 4 + cols:], big[1][:, 4 + cols:])
    by, bh = big[2].clone(), big[3].clone()
    py, ph = by.data_ptr() + 5 * by.element_size(), bh.data_ptr() + 6 * bh.element_size()
    dw, db = torch.empty_like(w), torch.empty_like(w)
    ws = torch.empty(lib().lopt_dropout_add_layer_norm_workspace(7, cols), dtype=torch.uint8, device="cuda:0")
    assert lib().lopt_dropout_add_layer_norm_backward(py, ld, ph, ld, res.data_ptr(), ld, w.data_ptr(), mean.data_ptr(), rstd.data_ptr(), py, ld, ph, ld, dw.data_ptr(),
                                                      db.data_ptr(), 7, cols, kinds[kind], kinds[rkind], 0, 0.3, 5, None, 0, ws.data_ptr(), ws.numel(), s) == 0
    assert torch.equal(by[:, 5:5 + cols], g[0]) and torch.equal(bh[:, 6:6 + cols], g[1]) and torch.equal(dw, g[2]) and torch.equal(db, g[3])
    assert torch.equal(by[:, :5], big[2][:, :5]) and torch.equal(by[:, 5 + cols:], big[2][:, 5 + cols:])
    assert torch.equal(bh[:, :6], big[3][:, :6]) and torch.equal(bh[:, 6 + cols:], big[3][:, 6 + cols:])


def test_dropout_add_layer_norm_beyond_the_cache():
    """Arrays of more than 256 MB are read another way: the first rows with dropout, the last without, to the bit as by themselves."""
    import torch
    gen = torch.Generator(device="cuda:0").manual_seed(3)
    rows, cols, n = 25001, 1999, 65
    x, dy = (torch.randn(rows, cols, device="cuda:0", generator=gen).bfloat16() for _ in range(2))
    res, dh = (torch.randn(rows, cols, device="cuda:0", generator=gen) for _ in range(2))
    w = torch.randn(cols, device="cuda:0", generator=gen)
    for p, part in ((0.3, slice(0, n)), (0.0, slice(rows - n, rows))):
        y, h, mean, rstd = ops().dropout_add_layer_norm_forward(x, res, w, w, p, 5, 6)
        few = ops().dropout_add_layer_norm_forward(x[part], res[part], w, w, p, 5, 6)
        # the second rows start off the grid in the one and the other alike: their distance is odd in both
        for a, b in zip((y, h, mean, rstd), few):
            assert torch.equal(a[part], b), p
        got = ops().dropout_add_layer_norm_backward(dy, dh, h, w, mean, rstd, p, 5, 6)
        few = ops().dropout_add_layer_norm_backward(dy[part], dh[part], h[part], w, mean[part], rstd[part], p, 5, 6)
        assert torch.equal(got[0][part], few[0]) and torch.equal(got[1][part], few[1]), p
        xh = (h - mean[:, None]) * rstd[:, None]
        want = (dy.double() * xh).sum(0)
        # xh has two roundings, a column 25001 terms: up to 144 a lane, then the tree
        assert bool(((got[2].double() - want).abs() <= (144 + 30) * U * (dy.double() * xh).abs().sum(0)).all())


def test_one_tensor_as_block_and_residual():
    import torch
    x = torch.randn(7, 64, device="cuda:0", requires_grad=True)
    w = torch.randn(64, device="cuda:0")
    for p in (0.0, 0.5):
        x.grad = None
        y, h = ops().dropout_add_layer_norm(x, x, w, None, p, 3)
        (y.square().sum() + h.sum()).backward()
        a, b = x.detach().clone().requires_grad_(), x.detach().clone().requires_grad_()
        y, h = ops().dropout_add_layer_norm(a, b, w, None, p, 3)
        (y.square().sum() + h.sum()).backward()
        assert torch.equal(x.grad, a.grad + b.grad)


def test_dropout_add_layer_norm_zero_rows():
    import torch
    x = torch.empty(0, 64, device="cuda:0", dtype=torch.bfloat16)
    w = torch.ones(64, device="cuda:0")
    y, h, mean, rstd = ops().dropout_add_layer_norm_forward(x, x.float(), w, w, 0.1, 1)
    assert y.shape == h.shape == (0, 64) and mean.shape == (0,)
    dx, dres, dw, db = ops().dropout_add_layer_norm_backward(x, h, h, w, mean, rstd, 0.1, 1)
    assert dx.shape == dres.shape == (0, 64) and dw.tolist() == [0.0] * 64 and db.tolist() == [0.0] * 64


def test_dropout_add_layer_norm_autograd_against_differences():
    import torch
    r = np.random.default_rng(22)
    x, xv = dev(r.standard_normal((9, 37)), "fp32")
    res, rv = dev(r.standard_normal((9, 37)), "fp32")
    w, wv = dev(1 + 0.3 * r.standard_normal(37), "fp32")
    b, bv = dev(0.3 * r.standard_normal(37), "fp32")
    c, cv = dev(r.standard_normal((9, 37)), "fp32")
    e, ev = dev(r.standard_normal((9, 37)), "fp32")
    keep = keep_of(9, 37, 0.25, 8, 1)
    ts = (x, res, w, b)
    for use_y, use_h in ((True, True), (True, False), (False, True)):
        for t in ts:
            t.grad = None
            t.requires_grad_()
        y, h = ops().dropout_add_layer_norm(x, res, w, b, 0.25, 8, 1)
        ((y * c).sum() * use_y + (h * e).sum() * use_h if use_y and use_h else (y * c).sum() if use_y else (h * e).sum()).backward()

        def loss(xa, ra, wa, ba):
            ha = ra + dropped(xa, keep, 0.25)
            return use_y * float((norm_exact(ha, wa, ba, EPS)[0] * cv).sum()) + use_h * float((ha * ev).sum())
        step = 1e-5
        for k, t in enumerate(ts):
            for _ in range(4):
                args = [xv, rv, wv, bv]
                d = r.standard_normal(args[k].shape)
                args[k] = args[k] + step * d
                up = loss(*args)
                args[k] = args[k] - 2 * step * d
                slope = (up - loss(*args)) / (2 * step)
                grad = host(t.grad) if t.grad is not None else np.zeros(d.shape)
                got, scale = float((grad * d).sum()), float(np.abs(grad * d).sum())
                # as in the layer norm's test, with a sum and a product more
                assert abs(got - slope) <= 1e-8 * scale + 1e-8 + (3 * depth(37) * 4 + 4) * U * (scale + 37), (use_y, use_h, k, got, slope)


def test_block_of_fused_calls_trains_like_its_parts():
    """A stream through three fused calls against dropout, addition and layer norm one by one, in float64 on the host."""
    import torch
    r = np.random.default_rng(31)
    rows, cols = 64, 96
    xs = [dev(r.standard_normal((rows, cols)), "fp32") for _ in range(3)]
    ws = [dev(1 + 0.2 * r.standard_normal(cols), "fp32") for _ in range(3)]
    res, rv = dev(r.standard_normal((rows, cols)), "fp32")
    leaves = [t.requires_grad_() for t, _ in xs + ws] + [res.requires_grad_()]
    h, total = res, 0.0
    for i, ((x, _), (w, _)) in enumerate(zip(xs, ws)):
        y, h = ops().dropout_add_layer_norm(x, h, w, None, 0.1, 5, i)
        total = total + (y * y).sum() * (i + 1) + (ops().dropout(y, 0.5, 5, 100 + i)).sum()
    (total + h.sum()).backward()
    refs = [torch.from_numpy(v).requires_grad_() for _, v in xs + ws] + [torch.from_numpy(rv).requires_grad_()]
    h, want = refs[-1], 0.0
    for i in range(3):
        h = h + refs[i] * torch.from_numpy(keep_of(rows, cols, 0.1, 5, i)) / (1 - float(np.float32(0.1)))
        d = h - h.mean(-1, keepdim=True)
        y = d / (d.square().mean(-1, keepdim=True) + EPS).sqrt() * refs[3 + i]
        want = want + (y * y).sum() * (i + 1) + (y * torch.from_numpy(keep_of(rows, cols, 0.5, 5, 100 + i)) * 2).sum()
    (want + h.sum()).backward()
    for got, ref in zip(leaves, refs):
        a, b = host(got.grad), ref.grad.numpy()
        # three stages of sums of at most depth(96) roundings each, forwards and backwards, of terms as large as the rms of what comes out
        assert np.abs(a - b).max() <= 6 * depth(96) * 4 * U * (np.sqrt((b * b).mean()) + np.abs(b).max())


# ---------------------------------------------------------------------------------------------- KL divergence

def kl_exact(x, r, scale):
    """Row by row from the definition; float64 [rows, vocab]."""
    n = x.shape[0]
    kl, stats, p, q, d = np.zeros(n), np.zeros((n, 5)), np.zeros(x.shape), np.zeros(x.shape), np.zeros(x.shape)
    with np.errstate(all="ignore"):
        for i in range(n):
            mx, mr = x[i].max(), r[i].max()
            if np.isnan(x[i]).any() or np.isnan(r[i]).any() or mx == np.inf or mr == np.inf:
                kl[i], stats[i], p[i], q[i] = np.nan, np.nan, np.nan, np.nan
                continue
            e = np.exp(scale * (x[i] - (mx if mx > -np.inf else 0.0)))
            f = np.exp(scale * (r[i] - (mr if mr > -np.inf else 0.0)))
            sx, sr = e.sum(), f.sum()
            d[i] = scale * ((x[i] - r[i]) - (mx - mr))
            stats[i] = mx, np.log(sx), mr, np.log(sr), 0.0
            p[i], q[i] = e / sx if sx else 0.0, f / sr if sr else 0.0
            if sx == 0:
                continue
            if ((r[i] == -np.inf) & (x[i] > -np.inf)).any():
                kl[i] = stats[i, 4] = np.inf
                continue
            at = x[i] > -np.inf
            stats[i, 4] = (p[i][at] * d[i][at]).sum()
            kl[i] = max(stats[i, 4] + np.log(sr / sx), 0.0)
    return kl, stats, p, q, d


# A lane of a row of n logits adds up at most 128 + n / 256 of them one after the other, then 24 levels of lanes, wavefronts and pieces.
def kl_depth(n):
    return 152 + n // 256


def kl_tolerance(x, r, scale, want):
    """Of KL and of the mean difference. An exponential has the roundings of its exponent t, three of |t|, and its own: with |t| <= 40 where it counts (below, 2^-40 of the sum at
    most), 2.1 * 40 + 2 units. Both sums of a quotient have that and their additions', so that h / sx is off by that twice of the mean |d|, and a logarithm of a quotient by
    that twice; the d themselves by their three roundings, of which that of x - r is a unit of up to 32 more where such a constant lies between the rows (beyond, d goes by the
    maxima). Every sum counts what is lost of |t| > 40: nothing beside the others."""
    kl, stats, p, q, d = want
    with np.errstate(invalid="ignore"):
        spread = np.nansum(p * np.where(np.isfinite(d), np.abs(d), 0.0), 1)
        offset = np.where(np.isfinite(stats[:, 0]) & np.isfinite(stats[:, 2]), np.minimum(np.abs(stats[:, 0] - stats[:, 2]), 32.0), 0.0) * scale
    unit = 2 * (86 + kl_depth(x.shape[1])) * U
    tol = unit * (1.0 + spread) + 2 * U * offset + 3 * U * spread + 2 * U * np.abs(np.where(np.isfinite(kl), kl, 0.0)) + 1e-37
    tol_ln = unit + 2 * U * np.abs(np.where(np.isfinite(stats[:, 1::2][:, :2]), stats[:, 1::2][:, :2], 0.0))
    return tol, tol_ln


def check_kl(x, r, kind, scale=1.0, mask=None, what=""):
    import torch
    xt, xv = dev(x, kind) if isinstance(x, np.ndarray) else (x, host(x))
    rt, rv = dev(r, kind) if isinstance(r, np.ndarray) else (r, host(r))
    s32 = float(np.float32(scale))
    want = kl_exact(xv, rv, s32)
    tol, tol_ln = kl_tolerance(xv, rv, s32, want)
    keep = np.ones(xv.shape[0], bool) if mask is None else host(mask) > 0
    kl, stats = ops().token_kl_forward(xt, rt, scale=scale, mask=mask)
    close(kl, np.where(keep, want[0], 0.0), tol, f"kl {what}")
    sv, nan = host(stats), np.isnan(want[0])
    ws = np.where(keep[:, None], want[1], 0.0)
    rows = keep & ~nan
    assert np.array_equal(sv[rows][:, [0, 2]], ws[rows][:, [0, 2]]), what
    close(sv[rows][:, [1, 3]], ws[rows][:, [1, 3]], tol_ln[rows], f"stats {what}")
    close(sv[rows][:, 4], ws[rows][:, 4], tol[rows] + 2 * U * np.abs(np.where(np.isfinite(ws[rows][:, 4]), ws[rows][:, 4], 0.0)), f"mean {what}")
    assert not sv[~keep].any(), what
    again, stats2 = ops().token_kl_forward(xt, rt, scale=scale, mask=mask)
    assert torch.equal(torch.nan_to_num(kl), torch.nan_to_num(again)) and torch.equal(torch.nan_to_num(stats), torch.nan_to_num(stats2))
    # the gradients
    rr = np.random.default_rng(x.shape[1])
    g, gv = dev(rr.standard_normal(xv.shape[0]), "fp32")
    dx, dr = ops().token_kl_backward(xt, rt, stats, g, scale=scale, mask=mask, need=(True, True))
    _, st, p, q, d = want
    gs = np.where(keep & ~(want[1][:, 0] == -np.inf), gv * s32, 0.0)[:, None]
    with np.errstate(invalid="ignore", over="ignore"):
        ok = np.isfinite(want[0])[:, None] | (gs == 0)
        wx = np.where(p > 0, gs * p * (np.where(np.isfinite(d), d, 0.0) - np.where(np.isfinite(st[:, 4:5]), st[:, 4:5], 0.0)), 0.0)
        wr = gs * (q - p)
        # p: the exponent's roundings, at most 4 of its size up to 100 (below, p is 4e-44), those of ln S, the exponential's; d - mean: their roundings and the mean's
        lp = np.minimum(np.abs(np.where(p > 0, np.log(np.where(p > 0, p, 1.0)), 0.0)), 104.0)
        lq = np.minimum(np.abs(np.where(q > 0, np.log(np.where(q > 0, q, 1.0)), 0.0)), 104.0)
        big = 4 * U * (np.abs(st[:, 1]) + np.abs(st[:, 3]))[:, None]
        rp, rq = 4 * U * lp + 8 * U + tol_ln[:, :1] + big, 4 * U * lq + 8 * U + tol_ln[:, 1:] + big
        fd = np.where(np.isfinite(d), np.abs(d), 0.0)
        tx = np.abs(wx) * (rp + 6 * U) + np.abs(gs) * p * (4 * U * fd + tol[:, None] + 4 * U * np.abs(np.where(np.isfinite(st[:, 4:5]), st[:, 4:5], 0.0)))
        tr = np.abs(gs) * (p * rp + q * rq) + 3 * U * np.abs(wr)
        tiny = 2.0 ** -126 * np.abs(gs) * (1.0 + fd) * (p < 2.0 ** -100)   # where the exponential leaves the normal numbers
    wx, wr = np.where(ok, wx, np.nan), np.where(ok, wr, np.nan)
    clean = lambda t: np.where(np.isfinite(t), t, 0.0)
    close(dx, wx, clean(1.01 * tx + tiny + 1.01 * ROUND[kind] * np.abs(wx)) + TINY[kind], f"dlogits {what}")
    close(dr, wr, clean(1.01 * tr + 2.0 ** -126 * np.abs(gs) + 1.01 * ROUND[kind] * np.abs(wr)) + TINY[kind], f"dref {what}")
    for need in ((True, False), (False, True)):
        part = ops().token_kl_backward(xt, rt, stats, g, scale=scale, mask=mask, need=need)
        for k, whole in enumerate((dx, dr)):
            assert (part[k] is None) == (not need[k])
            assert part[k] is None or torch.equal(torch.nan_to_num(part[k]), torch.nan_to_num(whole)), (what, need)
    return kl


def logits_pair(rows, vocab, seed, masked=0.0, apart=0.3):
    r = np.random.default_rng(seed)
    x = 2.0 * r.standard_normal((rows, vocab))
    x[np.arange(rows), r.integers(0, vocab, rows)] += 8.0
    y = x + apart * r.standard_normal(x.shape) + r.standard_normal((rows, 1))
    if masked:
        off = r.random(x.shape) < masked
        off[np.arange(rows), x.argmax(1)] = False
        x[off] = y[off] = -np.inf
    return x, y


KL_SHAPES = [(1, 1), (3, 1), (5, 2), (4, 7), (9, 8), (3, 9), (33, 63), (6, 64), (5, 65), (13, 505), (4, 513), (11, 1017), (3, 1025), (5, 2041), (7, 2048), (3, 2500), (2, 8191), (260, 3001),
             (3, 50257), (2, 131065), (3, 131080), (1, 300007), (2100, 33000), (17, 121), (17, 122), (4100, 10), (4100, 130), (4099, 249), (4097, 505), (8193, 1)]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,vocab", KL_SHAPES)
def test_token_kl(rows, vocab, kind):
    import torch
    if rows * vocab > 10_000_000 and kind != "bf16":
        pytest.skip("one type is enough at this size")
    for scale, masked, apart in (((1.0, 0.0, 0.3),) if rows * vocab > 10_000_000 else ((1.0, 0.0, 0.3), (0.5, 0.5, 0.3), (1.25, 0.0, 5.0), (1.0, 0.2, 0.0))):
        x, y = logits_pair(rows, vocab, rows + vocab, masked, apart)
        if rows * vocab > 10_000_000:   # 16 of the rows by the definition, beside others
            xt, yt = (torch.from_numpy(a[:16].astype(np.float32)).to(tt(kind)).cuda() for a in (x, y))
            big = [torch.cat([t] * (rows // 16 + 1))[:rows].contiguous() for t in (xt, yt)]
            kl, stats = ops().token_kl_forward(*big, scale=scale)
            want = check_kl(xt, yt, kind, scale)
            tol = torch.from_numpy(2 * kl_tolerance(host(xt), host(yt), scale, kl_exact(host(xt), host(yt), scale))[0]).cuda()
            assert bool(((kl.double() - torch.cat([want] * (rows // 16 + 1))[:rows].double()).abs() <= torch.cat([tol] * (rows // 16 + 1))[:rows]).all())
            assert all(torch.equal(kl[k], kl[k % 16]) for k in (16, 33, rows - 1))
            continue
        check_kl(x, y, kind, scale, what=f"scale {scale} masked {masked} apart {apart}")
        if rows > 2:
            mask = torch.arange(rows, device="cuda:0") % 3 != 1
            check_kl(x, y, kind, scale, mask=mask, what="mask")


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("vocab", [5, 100, 1500, 3000, 20000, 140000])
def test_token_kl_special_rows(vocab, kind):
    low = -65504.0 if kind == "fp16" else -3.3895314e38
    inf, at = np.inf, np.arange(vocab)
    x, y = logits_pair(30, vocab, vocab)
    x[0] = y[0] = -inf                                # both masked whole
    x[1] = -inf                                       # the first
    y[2] = -inf                                       # the second: infinite
    y[3, vocab // 2] = -inf                           # one token that the reference masks alone
    x[4, vocab // 2] = -inf                           # one that the policy masks alone
    x[5, 0], y[6, vocab - 1], x[7, 1], y[8, 2] = np.nan, np.nan, inf, inf
    x[9], y[9] = np.where(at == 1, 0.5, -inf), np.where(at == 1, -7.0, -inf)     # one token is allowed
    x[10] = y[10] = 0.0
    x[11] = y[11] = low                               # the lowest value everywhere
    off = at % 3 != 1
    x[12], y[12] = np.where(off, low, x[12]), np.where(off, low, y[12])          # as a mask in both
    x[13] = np.where(off, low, x[13])                 # in the first alone
    y[14], x[14] = np.where(at == 0, low, y[14]), np.where(at == 0, -60.0, x[14])  # in the second, under an unlikely token
    x[15], y[15] = np.where(off, -1e4, x[15]), np.where(off, -1e4, y[15])
    x[16] = np.where(at < 1024, -inf, x[16]) if vocab > 1500 else x[16]          # whole pieces
    y[16] = np.where(at < 1024, -inf, y[16]) if vocab > 1500 else y[16]
    x[17] = np.where(at >= 1, -inf, x[17])            # x keeps one token
    x[18], y[18] = 100.0 * np.sign(x[18]), -100.0 * np.sign(x[18])               # far apart everywhere
    y[19] = -inf
    y[19, 0] = 3.0                                    # the reference keeps one token
    x[20] = np.where(at == 3, np.nan, -inf)
    y[21] = np.where(at == vocab // 2, np.nan, y[21])
    x[21] = np.where(at == vocab // 2, -inf, x[21])   # a NaN under a masked token
    if kind != "fp16":
        x[22], y[22] = 1e30 * (at % 5), 1e30 * (at % 4)                          # enormous logits
        x[23] = y[23] = 3e38 * np.where(at % 2, 1.0, -1.0)
        x[24], y[24] = x[24] + 65536.0, y[24] - 131072.0                         # far offsets
        x[25], y[25] = np.where(off, -1e9, x[25]), np.where(off, -1e9, y[25])
        x[26] = np.where(off, -1e9, x[26])
        y[27] = np.where(at == 0, -1e9, y[27])
        x[27, 0] = -90.0
    kl = host(check_kl(x, y, kind, what="special"))
    assert kl[0] == kl[1] == kl[10] == kl[11] == 0 and kl[2] == kl[3] == kl[19] == inf and np.isnan(kl[[5, 6, 7, 8, 20, 21]]).all() and np.isfinite(kl[[4, 9, 12, 13, 17]]).all()
    check_kl(x[:12], y[:12], kind, scale=2.0, what="special, scale 2")


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("vocab", [9, 100, 200, 500])
def test_token_kl_special_rows_among_many_short_ones(vocab, kind):
    """Rows that share a wavefront, special ones beside ordinary ones, against the definition; none of them changes another."""
    import torch
    x, y = logits_pair(70, vocab, 40 + vocab)
    a, b = (dev(v, kind)[0] for v in (x, y))
    a[3], a[5, 1], a[6, 2], a[9, :4], b[9, :3] = -math.inf, math.nan, math.inf, -math.inf, -math.inf
    b[11, 4], a[15], b[15], b[18] = -math.inf, a[15] + 512, b[15] - 512, -math.inf
    a[21, 1:], b[22, 2], a[30, 3] = -math.inf, torch.finfo(tt(kind)).min, torch.finfo(tt(kind)).min
    av, bv = host(a), host(b)
    want = kl_exact(av, bv, 1.0)
    tol, _ = kl_tolerance(av, bv, 1.0, want)
    kl, stats = ops().token_kl_forward(a.repeat(60, 1), b.repeat(60, 1))
    g = torch.ones_like(kl)
    grads = ops().token_kl_backward(a.repeat(60, 1), b.repeat(60, 1), stats, g, need=(True, True))
    for part in (kl[:70], kl[2100:2170], kl[-70:]):
        close(part, want[0], tol, "kl")
    few = ops().token_kl_forward(a, b)
    for got, w in zip(grads, ops().token_kl_backward(a, b, few[1], g[:70], need=(True, True))):
        assert torch.equal(got.reshape(60, 70, vocab)[-1].isnan(), w.isnan())
    special = [3, 5, 6, 9, 11, 15, 18, 21, 22, 30]
    plain = [i for i in range(70) if i not in special]
    c, e = a.clone(), b.clone()
    c[special], e[special] = a[0], b[0]
    other = ops().token_kl_forward(c.repeat(60, 1), e.repeat(60, 1))[0]
    assert torch.equal(kl.reshape(60, 70)[:, plain], other.reshape(60, 70)[:, plain])


@pytest.mark.parametrize("vocab", [300, 5000, 140000])
def test_token_kl_is_not_lost_where_it_is_small(vocab):
    """Logits that differ by 2^-10 here and there, of KL around 1e-7 to 1e-6: its error is less than it. Identical rows have 0."""
    r = np.random.default_rng(1)
    x = np.round(64 * 2 * r.standard_normal((16, vocab))) / 64
    y = x + np.where(r.random(x.shape) < 0.5, 2.0 ** -10, 0.0)
    xt, xv = dev(x, "fp32")
    yt, yv = dev(y, "fp32")
    want = kl_exact(xv, yv, 1.0)[0]
    kl = host(ops().token_kl_forward(xt, yt)[0])
    # sum p d - ln sum p e^d cancels all but d / 2 of its terms, which are of size d = 1.4e-3 in units of log 2: of rows of at most 2048 logits q - 1 has five roundings of its own
    # size, so that KL is off by 10 U d; in longer ones q has a rounding of its own, which is random from token to token: sqrt(sum p^2) of it, six standard deviations
    p = kl_exact(xv, yv, 1.0)[2]
    d = 2.0 ** -10
    tol = 30 * U * d + (0 if vocab <= 2040 else 6 * U * np.sqrt((p * p).sum(1))) + kl_depth(vocab) * U * d
    assert (np.abs(kl - want) <= tol).all() and (tol < want).all(), (kl, want, tol)   # the bound itself says something
    assert host(ops().token_kl_forward(xt, xt.clone())[0]).tolist() == [0.0] * 16


def test_token_kl_strides_dimensions_and_in_place():
    import ctypes as C
    import torch
    from paper_2506_10315_amd import lib
    for kind, vocab in (("bf16", 333), ("fp16", 3001), ("fp32", 2047), ("bf16", 140001)):
        x, y = logits_pair(6, vocab + 20, vocab)
        a, b = dev(x, kind)[0], dev(y, kind)[0]
        xs, ys = a[:, 3:3 + vocab], b[:, 10:10 + vocab]       # rows on different grids
        kl, stats = ops().token_kl_forward(xs, ys)
        # the grid that packs are counted from moves with the row: sums in another order
        want, wstats = ops().token_kl_forward(xs.contiguous(), ys.contiguous())
        tol, _ = kl_tolerance(host(xs), host(ys), 1.0, kl_exact(host(xs), host(ys), 1.0))
        close(kl, host(want), 2 * tol, "strided")
        nd, ns = ops().token_kl_forward(xs.reshape(2, 3, vocab), ys.reshape(2, 3, vocab))
        assert nd.shape == (2, 3) and ns.shape == (2, 3, 5) and torch.equal(nd.flatten(), want) and torch.equal(ns.view(6, 5), wstats)
        close(ops().token_kl_forward(xs[:1].expand(6, vocab), ys)[0][:1], host(want)[:1], 2 * tol[:1], "one row")
        g = torch.randn(6, device="cuda:0")
        dx, dr = ops().token_kl_backward(xs, ys, stats, g, need=(True, True))
        ex, er = ops().token_kl_backward(xs.contiguous(), ys.contiguous(), stats, g, need=(True, True))
        assert torch.equal(dx, ex) and torch.equal(dr, er)
        kinds = {"fp32": 0, "bf16": 1, "fp16": 2}
        px, py = a.data_ptr() + 3 * a.element_size(), b.data_ptr() + 10 * b.element_size()
        ca, cb = a.clone(), b.clone()
        s = C.c_void_p(torch.cuda.current_stream().cuda_stream)
        ld = vocab + 20
        assert lib().lopt_token_kl_backward(px, ld, py, ld, None, stats.data_ptr(), g.data_ptr(), px, ld, py, ld, 6, vocab, kinds[kind], 1.0, s) == 0   # in place
        assert torch.equal(a[:, 3:3 + vocab], dx) and torch.equal(b[:, 10:10 + vocab], dr)
        assert torch.equal(a[:, :3], ca[:, :3]) and torch.equal(a[:, 3 + vocab:], ca[:, 3 + vocab:]) and torch.equal(b[:, :10], cb[:, :10]) and torch.equal(b[:, 10 + vocab:], cb[:, 10 + vocab:])
    e = torch.empty(0, 5, device="cuda:0")
    kl, stats = ops().token_kl_forward(e, e)
    assert kl.shape == (0,) and ops().token_kl_backward(e, e, stats, kl)[0].shape == (0, 5)


def test_token_kl_autograd_against_differences():
    import torch
    r = np.random.default_rng(5)
    x, y = logits_pair(7, 41, 3, masked=0.2, apart=1.0)
    (xt, xv), (yt, yv), (c, cv) = dev(x, "fp32"), dev(y, "fp32"), dev(r.standard_normal(7), "fp32")
    mask = torch.tensor([True] * 5 + [False] + [True], device="cuda:0")
    xt.requires_grad_()
    yt.requires_grad_()
    (ops().token_kl(xt, yt, scale=0.75, mask=mask) * c).sum().backward()
    keep = host(mask)
    loss = lambda a, b: float((kl_exact(a, b, 0.75)[0] * cv * keep).sum())
    h = 1e-5
    for t, which in ((xt, 0), (yt, 1)):
        for _ in range(6):
            d = r.standard_normal(xv.shape)
            args = [xv, yv]
            args[which] = args[which] + h * d
            up = loss(*args)
            args[which] = args[which] - 2 * h * d
            slope = (up - loss(*args)) / (2 * h)
            got, scale = float((host(t.grad) * d).sum()), float(np.abs(host(t.grad) * d).sum())
            # the gradient's own tolerance is below 4 * 100 + 2 * (86 + 152) units of its terms
            assert abs(got - slope) <= 1e-8 * (scale + 1) + 900 * U * (scale + 1), (which, got, slope)


def test_token_kl_far_rows():
    import torch
    ld = (1 << 31) + 8
    buf = torch.zeros(2 * ld, dtype=torch.bfloat16, device="cuda:0")
    x = buf.as_strided((2, 999), (ld, 1))
    a, b = (dev(v, "bf16")[0] for v in logits_pair(2, 999, 8))
    a = torch.nn.functional.pad(a, (0, 1))[:, :999]     # rows on the same grid of 16 bytes as those at a distance
    x.copy_(a)
    kl, stats = ops().token_kl_forward(x, b)
    want, _ = ops().token_kl_forward(a, b)
    assert torch.equal(kl, want)
    g = torch.ones(2, device="cuda:0")
    assert torch.equal(ops().token_kl_backward(x, b, stats, g)[0], ops().token_kl_backward(a, b, stats, g)[0])
    assert torch.equal(ops().dropout_forward(x, 0.5, 3), ops().dropout_forward(a, 0.5, 3))
    for p, q in zip(ops().dropout_add_layer_norm_forward(x, x, None, None, 0.5, 3), ops().dropout_add_layer_norm_forward(a, a, None, None, 0.5, 3)):
        assert torch.equal(p, q)


def test_token_kl_of_very_many_rows():
    import torch
    x, y = (dev(v, "bf16")[0] for v in logits_pair(1, 520, 9))
    rows = (1 << 26) + 77
    kl, stats = ops().token_kl_forward(x.expand(rows, 520), y.expand(rows, 520))
    one, its = ops().token_kl_forward(x, y)
    assert bool((kl == one).all()) and bool((stats[-100:] == its).all()) and bool((stats[:100] == its).all())


# ---------------------------------------------------------------------------------------------- policy loss

def exp_rest(v):
    """e^v - 1 - v."""
    return np.where(np.abs(v) < 1e-3, v * v * (0.5 + v / 6 + v * v / 24 + v ** 3 / 120), np.expm1(v) - v)


def policy_exact(v, clip, kl_coef, entropy_coef, reduction):
    """From the formulas in include/lopt.h; v: float64 arrays [seqs, tokens], None where not given. Also the bounds of the errors."""
    logp, old, adv, keep = v["logp"], v["old"], v["adv"], v["mask"]
    adv = adv if adv.shape == logp.shape else np.broadcast_to(adv[:, None], logp.shape)
    with np.errstate(all="ignore"):
        d = logp - old
        ratio = np.exp(d)
        out = ((adv > 0) & (d > np.log1p(clip[1]))) | ((adv < 0) & (d < (np.log1p(-clip[0]) if clip[0] < 1 else -np.inf)))
        bound = np.where(adv > 0, 1 + clip[1], 1 - clip[0])
        surrogate = np.where(adv == 0, 0.0, -adv * np.where(out, bound, ratio))
        slope = np.where(out, 0.0, surrogate)
        kl, ent = np.zeros_like(logp), np.zeros_like(logp)
        # the ratio: d is rounded once; its polynomial, the square of half of it and the additions have eight units, the hardware's power of two two of its own and, of its exponent's product and
        # the constant in it, 1.3 of |d|; drift and kl: their argument's rounding, the polynomial's ten units or the exponential's
        r_ratio = U * (3 * np.abs(d) + 8)
        # ratios below 2^-126 are 0, as the hardware's power of two leaves out subnormal numbers
        t_sur = np.abs(surrogate) * (r_ratio + 2 * U) + 2.0 ** -126 * np.abs(adv)
        t_slope = np.abs(slope) * (r_ratio + 2 * U) + 2.0 ** -126 * np.abs(adv)
        rest = lambda u: 16 * U * np.abs(exp_rest(u)) + U * np.abs(u) * np.abs(np.expm1(u)) + np.where(np.abs(u) < 1.999, 0.0, U * ((2 * np.abs(u) + 4) * np.exp(u) + 2 * np.abs(u) + 2))
        t_kl = np.zeros_like(logp)
        if v["ref"] is not None:
            u = v["ref"] - logp
            kl, t_kl = exp_rest(u), rest(u)
            slope = slope - kl_coef * np.expm1(u)
            t_slope = t_slope + abs(kl_coef) * (t_kl + 3 * U * np.abs(np.expm1(u)) + 2 * U * np.abs(u) + U) + U * np.abs(slope)
        elif v["kl"] is not None:
            kl = v["kl"]
        if v["ent"] is not None:
            ent = v["ent"]
        n = keep.sum(1).astype(np.float64)
        N, S = n.sum(), float((n > 0).sum())
        w = np.where(keep, 1.0 / max(N, 1) if reduction == "tokens" else 1.0 / np.maximum(n * S, 1)[:, None], 0.0)
        terms = [surrogate, kl, ent, out.astype(float), ratio, exp_rest(d)]
        # ratios, less 1, and drifts are added up four at a time in 32 bits, three additions, the rest in 64
        tols = [t_sur, t_kl, 0 * ent, 0 * ent, ratio * r_ratio + 3 * U * np.abs(np.expm1(d)), rest(d) + 3 * U * exp_rest(d)]
        mean = lambda a: float(np.where(keep, w * a, 0.0).sum())
        means, t_means = [mean(a) for a in terms], [mean(t) + 2 * U * abs(mean(a)) + 1e-14 * mean(np.abs(a)) for t, a in zip(tols, terms)]
        has_kl = v["ref"] is not None or v["kl"] is not None
        loss = means[0] + (kl_coef * means[1] if has_kl else 0.0) - entropy_coef * means[2] * (v["ent"] is not None)
        t_loss = t_means[0] + abs(kl_coef) * t_means[1] + abs(entropy_coef) * t_means[2] + 2 * U * abs(loss)
        grads = [np.where(keep, w * slope, 0.0), w * kl_coef, -w * entropy_coef]
        t_grads = [np.where(keep, w * (t_slope + 4 * U * np.abs(slope)), 0.0), 6 * U * np.abs(grads[1]), 6 * U * np.abs(grads[2])]
    return loss, t_loss, np.array(means + [N, S]), np.array(t_means + [U * N, U * S]), grads, t_grads


def policy_inputs(seqs, tokens, seed, kl="ref", ent=True, each=True, lengths=True, kinds=("fp32", "fp32", "fp32"), spread=0.15):
    import torch
    r = np.random.default_rng(seed)
    n = lambda *s: r.standard_normal(s)
    logp = -np.exp(n(seqs, tokens))
    t, v = {}, {}
    t["logp"], v["logp"] = dev(logp, "fp32")
    t["old"], v["old"] = dev(logp + spread * n(seqs, tokens), kinds[0])
    t["adv"], v["adv"] = dev(n(seqs, tokens) if each else n(seqs), kinds[1])
    t["ref"], v["ref"] = dev(logp + 0.5 * n(seqs, tokens), kinds[2]) if kl == "ref" else (None, None)
    t["kl"], v["kl"] = dev(0.1 * n(seqs, tokens) ** 2, "fp32") if kl == "given" else (None, None)
    t["ent"], v["ent"] = dev(np.exp(n(seqs, tokens)), "fp32") if ent else (None, None)
    keep = np.arange(tokens) < r.integers(0, tokens + 1, (seqs, 1)) if lengths else np.ones((seqs, tokens), bool)
    t["mask"], v["mask"] = torch.from_numpy(keep).cuda(), keep
    return t, v


def check_policy(t, v, clip=(0.2, 0.28), kl_coef=0.05, entropy_coef=0.01, reduction="tokens", up=1.0, what="", mask=True):
    import torch
    args = dict(mask=t["mask"] if mask else None, clip=clip, ref_logp=t["ref"], kl=t["kl"], kl_coef=kl_coef if t["ref"] is not None or t["kl"] is not None else 0.0,
                entropy=t["ent"], entropy_coef=entropy_coef if t["ent"] is not None else 0.0, reduction=reduction)
    r = ops().policy_loss_forward(t["logp"], t["old"], t["adv"], **args)
    dl = torch.tensor(up, device="cuda:0")
    got = ops().policy_loss_backward(dl, r, t["logp"], t["old"], t["adv"], **args)
    loss, t_loss, stats, t_stats, grads, t_grads = policy_exact(v, clip, args["kl_coef"], args["entropy_coef"], reduction)
    close(r.loss, np.array(loss), t_loss + 1e-37, f"loss {what}")
    close(r.stats, stats, t_stats + 1e-37, f"stats {what}")
    if reduction == "sequences":
        assert np.array_equal(host(r.counts), v["mask"].sum(1)), what
    for g, a, tol, given, name in zip(got, grads, t_grads, (True, t["kl"] is not None, t["ent"] is not None), ("dlogp", "dkl", "dentropy")):
        assert (g is None) == (not given)
        if given:
            close(g.reshape(a.shape), up * a, 1.01 * abs(up) * tol + TINY["fp32"], f"{name} {what}")
    again = ops().policy_loss_forward(t["logp"], t["old"], t["adv"], **args)
    assert torch.equal(r.loss, again.loss) and torch.equal(r.stats, again.stats)
    assert torch.equal(got[0], ops().policy_loss_backward(dl, r, t["logp"], t["old"], t["adv"], need=(True, False, False), **args)[0])
    return r, got


POLICY_SHAPES = [(1, 1), (5, 1), (1, 3), (7, 5), (3, 64), (9, 65), (16, 257), (8, 128), (1, 16384), (1, 16385), (3, 5000), (4, 4097), (700, 3), (70000, 7), (20000, 10), (9000, 16), (40000, 3), (2048, 33), (2200, 130), (2100, 1001), (300, 300), (1000, 60), (5, 20000), (1, 300001),
                 (1023, 1100), (600, 2048), (2, 100003)]


@pytest.mark.parametrize("seqs,tokens", POLICY_SHAPES)
def test_policy_loss(seqs, tokens):
    for i, (kl, ent, each, reduction, kinds) in enumerate((("ref", True, True, "tokens", ("fp32", "fp32", "fp32")), ("given", False, False, "sequences", ("bf16", "fp16", "fp32")),
                                                           ("none", True, False, "tokens", ("fp16", "bf16", "fp32")), ("ref", False, True, "sequences", ("fp32", "fp32", "bf16")))):
        t, v = policy_inputs(seqs, tokens, seqs + tokens + i, kl, ent, each, kinds=kinds)
        check_policy(t, v, reduction=reduction, up=(1.0, -2.5)[i % 2], what=f"{kl} {reduction}")


def test_policy_loss_without_mask_strides_and_one_dimension():
    import torch
    t, v = policy_inputs(6, 90, 3, lengths=False)
    a, ga = check_policy(t, v, mask=False)
    b, gb = check_policy(t, v, mask=True)
    assert torch.equal(a.loss, b.loss) and torch.equal(ga[0], gb[0])
    big = {k: torch.nn.functional.pad(x, (i + 1, 9 - i)) for i, (k, x) in enumerate(t.items()) if x is not None}
    s = {k: big[k][:, i + 1:i + 91] if t[k] is not None else None for i, k in enumerate(t)}
    assert all(torch.equal(s[k], t[k]) for k in big)
    c, gc = check_policy(s, v)
    assert torch.equal(a.loss, c.loss) and torch.equal(a.stats, c.stats) and all(torch.equal(p, q) for p, q in zip(ga, gc) if p is not None)
    one = {k: x[2] if x is not None else None for k, x in t.items()}
    r, g = check_policy(one, {k: x[2:3] if x is not None else None for k, x in v.items()})
    assert g[0].shape == (90,)
    one["adv"] = t["adv"][2, 5]          # one advantage for the only sequence
    check_policy(one, {**{k: x[2:3] if x is not None else None for k, x in v.items()}, "adv": v["adv"][2, 5:6]})
    three = {k: x.view(2, 3, 90) if x is not None else None for k, x in t.items()}
    r, g = check_policy(three, v)
    assert g[0].shape == (2, 3, 90) and torch.equal(r.loss, a.loss)


def test_policy_loss_where_nothing_counts_and_what_is_masked():
    import torch
    for seqs, tokens in ((4, 30), (40, 3000)):
        t, v = policy_inputs(seqs, tokens, 1)
        t["mask"][:], v["mask"][:] = False, False
        for reduction in ("tokens", "sequences"):
            r, g = check_policy(t, v, reduction=reduction)
            assert float(r.loss) == 0 and not host(r.stats).any() and not any(host(x).any() for x in g if x is not None)
        # whatever lies in masked places
        t, v = policy_inputs(seqs, tokens, 2)
        t["mask"][1] = False
        v["mask"][1] = False
        want = check_policy(t, v, reduction="sequences")
        for bad in (math.nan, math.inf, -math.inf, 3e38):
            for k in ("logp", "old", "adv", "ref", "ent"):
                t[k][~t["mask"]] = bad
            got = ops().policy_loss_forward(t["logp"], t["old"], t["adv"], t["mask"], (0.2, 0.28), t["ref"], kl_coef=0.05, entropy=t["ent"], entropy_coef=0.01, reduction="sequences")
            assert torch.equal(got.loss, want[0].loss) and torch.equal(got.stats, want[0].stats)
            g = ops().policy_loss_backward(torch.tensor(1.0, device="cuda:0"), got, t["logp"], t["old"], t["adv"], t["mask"], (0.2, 0.28), t["ref"], kl_coef=0.05, entropy=t["ent"],
                                           entropy_coef=0.01, reduction="sequences")
            assert all(torch.equal(a, b) for a, b in zip(g, want[1]) if a is not None)
    e = torch.empty(0, 5, device="cuda:0")
    r = ops().policy_loss_forward(e, e, e)
    assert float(r.loss) == 0 and host(r.stats).tolist() == [0.0] * 8 and ops().policy_loss_backward(torch.ones((), device="cuda:0"), r, e, e, e)[0].shape == (0, 5)


def test_policy_loss_at_the_bounds():
    """Log ratios on both sides of the bounds, to the last bit that two float32 values can tell: the decision is that of 64 bits."""
    import torch
    r = np.random.default_rng(0)
    rows = []
    for edge in (np.log1p(0.28), np.log1p(-0.2), np.log1p(0.2)):
        base = -r.random(500).astype(np.float32) * 4 - 0.5
        lp = (base.astype(np.float64) + edge).astype(np.float32)
        for k in range(-2, 3):
            x = lp.copy()
            for _ in range(abs(k)):
                x = np.nextafter(x, np.float32(np.inf if k > 0 else -np.inf))
            rows.append((x, base))
    logp, old = np.stack([a for a, _ in rows]).astype(np.float64), np.stack([b for _, b in rows]).astype(np.float64)
    adv = np.where(np.arange(logp.shape[1]) % 3 == 0, 0.0, np.where(np.arange(logp.shape[1]) % 3 == 1, 1.5, -0.75)) + 0 * logp
    t = {"logp": dev(logp, "fp32")[0], "old": dev(old, "fp32")[0], "adv": dev(adv, "fp32")[0], "ref": None, "kl": None, "ent": None, "mask": torch.ones(logp.shape, dtype=torch.bool, device="cuda:0")}
    v = {"logp": logp, "old": old, "adv": adv, "ref": None, "kl": None, "ent": None, "mask": np.ones(logp.shape, bool)}
    for clip in ((0.2, 0.28), (0.2, 0.2), (1.0, math.inf), (0.0, 0.0)):
        check_policy(t, v, clip=clip, what=f"{clip}")


def test_policy_loss_far_ratios():
    import torch
    d = np.array([[-200.0, -100.0, -20.0, 0.0, 20.0, 80.0, 100.0, 200.0]])
    for a in (1.0, -1.0, 0.0):
        t, v = {}, {}
        t["logp"], v["logp"] = dev(-1.0 + 0 * d, "fp32")
        t["old"], v["old"] = dev(-1.0 - d, "fp32")
        t["adv"], v["adv"] = dev(a + 0 * d, "fp32")
        t.update(ref=None, kl=None, ent=None, mask=torch.ones(1, 8, dtype=torch.bool, device="cuda:0"))
        v.update(ref=None, kl=None, ent=None, mask=np.ones((1, 8), bool))
        r = ops().policy_loss_forward(t["logp"], t["old"], t["adv"])
        g = ops().policy_loss_backward(torch.tensor(1.0, device="cuda:0"), r, t["logp"], t["old"], t["adv"])[0]
        if a < 0:      # a ratio of e^100 and a negative advantage: beyond float32
            assert float(r.loss) == math.inf and host(g)[0, 6] == math.inf and np.isfinite(host(g)[0, :6]).all()
        else:
            check = policy_exact(v, (0.2, 0.2), 0, 0, "tokens")
            close(r.loss, np.array(check[0]), check[1] + 1e-37, "loss")
            close(g, check[4][0], check[5][0] + TINY["fp32"], "dlogp")
        assert float(r.stats[6]) == 8


def test_policy_terms_without_a_coefficient_are_only_reported():
    import torch
    for tokens in (5, 3000):
        v = {k: torch.rand(40, tokens, device="cuda:0") for k in ("logp", "old", "adv", "ent")}
        ref = torch.zeros_like(v["logp"])
        logp = -v["logp"]
        logp[3, 1] = -2000.0
        old = logp - 0.1 * v["old"]
        v["ent"][7, 2] = math.inf
        dl = torch.ones((), device="cuda:0")
        want = ops().policy_loss_forward(logp, old, v["adv"])
        gw = ops().policy_loss_backward(dl, want, logp, old, v["adv"])[0]
        for more in ({"ref_logp": ref}, {"kl": v["ent"]}):
            r = ops().policy_loss_forward(logp, old, v["adv"], entropy=v["ent"], **more)
            g = ops().policy_loss_backward(dl, r, logp, old, v["adv"], entropy=v["ent"], **more)
            assert torch.equal(r.loss, want.loss) and torch.equal(g[0], gw) and bool(torch.isfinite(gw).all())
            assert bool((g[2] == 0).all()) and (g[1] is None or bool((g[1] == 0).all()))
            assert float(r.stats[1]) == math.inf and float(r.stats[2]) == math.inf


def test_policy_loss_autograd_against_differences():
    import torch
    r = np.random.default_rng(12)
    for reduction in ("tokens", "sequences"):
        for kl in ("ref", "given"):
            t, v = policy_inputs(5, 23, 4, kl=kl, spread=0.5)
            leaves = [k for k in ("logp", "kl", "ent") if t[k] is not None]
            for k in leaves:
                t[k].requires_grad_()
            out = ops().policy_loss(t["logp"], t["old"], t["adv"], t["mask"], (0.2, 0.3), t["ref"], t["kl"], 0.5, t["ent"], 0.25, reduction)
            (3.0 * out.loss).backward()
            f = lambda w: 3.0 * policy_exact(w, (0.2, 0.3), 0.5, 0.25, reduction)[0]
            h = 1e-6
            for k in leaves:
                for _ in range(4):
                    d = r.standard_normal(v["logp"].shape)
                    slope = (f({**v, k: v[k] + h * d}) - f({**v, k: v[k] - h * d})) / (2 * h)
                    grad = host(t[k].grad)
                    got, scale = float((grad * d).sum()), float(np.abs(grad * d).sum())
                    # a ratio within h |d| of a bound would break the differences: none of these is; the gradient's terms have at most 40 units
                    assert abs(got - slope) <= 1e-8 * (1 + scale) + 40 * U * scale, (reduction, kl, k, got, slope)
    with pytest.raises(ValueError, match="advantages"):
        ops().policy_loss(t["logp"], t["old"], t["adv"].requires_grad_())


# ---------------------------------------------------------------------------------------------- preference loss

def preference_exact(logp, ref, keep, beta, kind, smooth, margin, average):
    pairs = logp.shape[0] // 2
    with np.errstate(all="ignore"):
        count = keep.sum(1).astype(float)
        lr = logp - (ref if ref is not None and ref.ndim == 2 else 0.0)
        s = np.where(keep, lr, 0.0).sum(1)
        if ref is not None and ref.ndim == 1:
            s = s - ref
        per = np.maximum(count, 1.0) if average else np.ones_like(count)
        s = s / per
        m = s[:pairs] - s[pairs:]
        z = beta * m - margin
        log_sigmoid = lambda a: -np.logaddexp(0.0, -a)
        if kind == "sigmoid":
            each = -(1 - smooth) * log_sigmoid(z) - smooth * log_sigmoid(-z)
            slope = beta * (1 / (1 + np.exp(-z)) - (1 - smooth))
        elif kind == "hinge":
            each, slope = np.maximum(1 - z, 0), np.where(z < 1, -beta, 0.0)
        else:
            each, slope = (m - 0.5 / beta) ** 2, 2 * (m - 0.5 / beta)
        coef = np.concatenate([slope, -slope]) / max(pairs, 1) / per
        stats = np.array([(m > 0).mean(), (beta * m).mean(), (beta * s[:pairs]).mean(), (beta * s[pairs:]).mean()]) if pairs else np.zeros(4)
    return each.mean() if pairs else 0.0, beta * s, stats, np.where(keep, coef[:, None], 0.0), np.abs(np.where(keep, lr, 0.0)).sum(1)


def check_preference(logp, ref, mask, beta=0.1, kind="sigmoid", smooth=0.0, margin=0.0, average=False, up=1.0, what=""):
    import torch
    r = ops().preference_loss_forward(logp, ref, mask, beta, kind, smooth, margin, average)
    dl = torch.tensor(up, device="cuda:0")
    g = ops().preference_loss_backward(dl, r, logp, mask)
    keep = np.ones(tuple(logp.shape), bool) if mask is None else host(mask) > 0
    loss, rewards, stats, grad, size = preference_exact(host(logp), None if ref is None else host(ref), keep, beta, kind, smooth, margin, average)
    # sums in 64 bits, their error n 2^-53 of the terms' sizes, which moves the loss by its slope; every output is rounded once to 32, the gradient twice
    slack = 1e-12 * (1 + np.abs(size).max(initial=0.0)) * (1 + (np.abs(rewards / beta).max(initial=0.0) + 1 / beta if kind == "squared" else beta))
    close(r.loss, np.array(loss), 1.01 * U * abs(loss) + slack + 1e-37, f"loss {what}")
    close(r.rewards, rewards, 1.01 * U * np.abs(rewards) + slack + 1e-37, f"rewards {what}")
    close(r.stats, stats, 1.01 * U * np.abs(stats) + slack + 1e-37, f"stats {what}")
    close(g, up * grad, 2.02 * U * np.abs(up * grad) + slack * abs(up) + TINY["fp32"], f"dlogp {what}")
    again = ops().preference_loss_forward(logp, ref, mask, beta, kind, smooth, margin, average)
    assert all(torch.equal(a, b) for a, b in zip(r, again))
    return r, g


def preference_inputs(pairs, tokens, seed, ref="tokens", rkind="fp32", spread=0.3):
    import torch
    r = np.random.default_rng(seed)
    lp = -np.exp(r.standard_normal((2 * pairs, tokens)))
    logp, lv = dev(lp, "fp32")
    keep = np.arange(tokens) < r.integers(0, tokens + 1, (2 * pairs, 1))
    rv = lp + spread * r.standard_normal(lp.shape)
    other = None if ref == "none" else dev(rv if ref == "tokens" else np.where(keep, rv, 0).sum(1), rkind)[0]
    return logp, other, torch.from_numpy(keep).cuda()


PREFERENCE_SHAPES = [(1, 1), (2, 3), (40000, 3), (9000, 20), (1100, 127), (1024, 1023), (2100, 1500), (1500, 1100), (5, 64), (3, 65), (8, 512), (2, 257), (1, 4097), (1, 8193), (2, 16385), (3000, 5), (700, 130), (511, 1100), (512, 1025), (9, 33333), (1, 500001)]


@pytest.mark.parametrize("pairs,tokens", PREFERENCE_SHAPES)
def test_preference_loss(pairs, tokens):
    for i, (kind, smooth, margin, average, ref, rkind) in enumerate((("sigmoid", 0.0, 0.0, False, "tokens", "fp32"), ("sigmoid", 0.1, 0.5, True, "sums", "fp32"),
                                                                     ("hinge", 0.0, -0.25, False, "none", "fp32"), ("squared", 0.0, 0.0, True, "tokens", "bf16"),
                                                                     ("sigmoid", 0.0, 0.0, False, "tokens", "fp16"), ("hinge", 0.0, 0.0, True, "sums", "bf16"))):
        logp, other, mask = preference_inputs(pairs, tokens, pairs + tokens + i, ref, rkind)
        check_preference(logp, other, mask, 0.1, kind, smooth, margin, average, (1.0, -3.0)[i % 2], what=f"{kind} {ref} {average}")


def test_preference_loss_without_mask_strides_and_zero_pairs():
    import torch
    logp, ref, mask = preference_inputs(4, 50, 1)
    check_preference(logp, ref, None)
    a, ga = check_preference(logp, ref, mask)
    big = [torch.nn.functional.pad(t, (i, 5 - i)) for i, t in enumerate((logp, ref, mask))]
    b, gb = check_preference(big[0][:, 0:50], big[1][:, 1:51], big[2][:, 2:52])
    assert all(torch.equal(p, q) for p, q in zip(a, b)) and torch.equal(ga, gb)
    e = torch.empty(0, 5, device="cuda:0")
    r = ops().preference_loss_forward(e)
    assert float(r.loss) == 0 and host(r.stats).tolist() == [0.0] * 4 and ops().preference_loss_backward(torch.ones((), device="cuda:0"), r, e).shape == (0, 5)


def test_preference_loss_special_values():
    import torch
    logp, ref, mask = preference_inputs(6, 700, 2)
    mask[1] = False                     # a chosen answer without tokens, a pair without any
    mask[2] = False
    mask[8] = False
    want, gw = check_preference(logp, ref, mask, average=True)
    for bad in (math.nan, math.inf, -math.inf):
        x, y = logp.clone(), ref.clone()
        x[~mask], y[~mask] = bad, bad
        r = ops().preference_loss_forward(x, y, mask, average=True)
        assert all(torch.equal(p, q) for p, q in zip(r, want)) and torch.equal(ops().preference_loss_backward(torch.ones((), device="cuda:0"), r, x, mask), gw)
    # margins that saturate the sigmoid either way
    far = logp.clone()
    far[0], far[6], far[3], far[9] = -5000.0, 0.0, 0.0, -5000.0
    for kind in ("sigmoid", "hinge", "squared"):
        r, g = check_preference(far, ref, mask, kind=kind)
        assert bool(torch.isfinite(r.loss)) and bool(torch.isfinite(g).all())
    # a token of a rejected answer that cannot be: the pair is as far apart as can be
    x = logp.clone()
    was = bool(mask[9, 0])
    x[9, 0], mask[9, 0] = -math.inf, True
    for kind, smooth, want in (("sigmoid", 0.0, False), ("sigmoid", 0.1, True), ("hinge", 0.0, False), ("squared", 0.0, True)):
        r = ops().preference_loss_forward(x, ref, mask, kind=kind, label_smoothing=smooth)
        g = ops().preference_loss_backward(torch.ones((), device="cuda:0"), r, x, mask)
        assert math.isinf(float(r.loss)) is want and not math.isnan(float(r.loss)), (kind, smooth)
        assert float(r.rewards[9]) == -math.inf and bool(torch.isfinite(g[[0, 1, 4, 5]]).all())
        if not want:
            assert bool((g[[3, 9]] == 0).all())
    mask[9, 0] = was
    # sums of the reference where an answer has no tokens
    sums = torch.where(mask, ref, 0.0).sum(1)
    a = ops().preference_loss_forward(logp, sums, mask)
    sums[~mask.any(1)] = math.nan
    b = ops().preference_loss_forward(logp, sums, mask)
    assert all(torch.equal(p, q) for p, q in zip(a, b)) and bool((b.rewards[~mask.any(1)] == 0).all())
    for kind in ("sigmoid", "hinge", "squared"):      # a NaN that counts
        x = logp.clone()
        x[5, 0] = math.nan
        mask[5, 0] = True
        r = ops().preference_loss_forward(x, ref, mask, kind=kind)
        g = ops().preference_loss_backward(torch.ones((), device="cuda:0"), r, x, mask)
        assert math.isnan(float(r.loss)) and bool(g[5][mask[5]].isnan().all()) and bool(torch.isfinite(g[[0, 3, 4]]).all())


def test_preference_loss_autograd_against_differences():
    import torch
    r = np.random.default_rng(3)
    for kind, smooth, margin, average in (("sigmoid", 0.1, 0.2, False), ("hinge", 0.0, 0.0, True), ("squared", 0.0, 0.0, False)):
        logp, ref, mask = preference_inputs(5, 31, 7)
        logp.requires_grad_()
        (2.0 * ops().preference_loss(logp, ref, mask, 0.7, kind, smooth, margin, average).loss).backward()
        f = lambda x: 2.0 * preference_exact(x, host(ref), host(mask) > 0, 0.7, kind, smooth, margin, average)[0]
        h = 1e-5
        for _ in range(6):
            d = r.standard_normal(logp.shape)
            slope = (f(host(logp) + h * d) - f(host(logp) - h * d)) / (2 * h)
            grad = host(logp.grad)
            got, scale = float((grad * d).sum()), float(np.abs(grad * d).sum())
            # h^2 of a third derivative of at most 0.1 (31 beta)^3, 2^-52 / h of the loss, and the gradient's three units
            assert abs(got - slope) <= 1e-7 * (1 + scale) + 4 * U * scale, (kind, got, slope)
    with pytest.raises(ValueError, match="ref_logp"):
        ops().preference_loss(logp, ref.requires_grad_(), mask)


# ---------------------------------------------------------------------------------------------- all of them, as they would be used

def _inputs():
    import torch
    gen = torch.Generator(device="cuda:0").manual_seed(4)
    n = lambda *s: torch.randn(*s, device="cuda:0", generator=gen)
    rows, cols, vocab = 8 * 24, 120, 501
    t = torch.randint(0, vocab, (rows,), device="cuda:0", generator=gen)
    return {"x": n(rows, cols), "res": n(rows, cols), "w": 1 + 0.1 * n(cols), "b": 0.1 * n(cols), "head": n(cols, vocab) / 8, "ref": n(cols, vocab) / 8, "t": t, "old": -n(8, 24).abs() - 4,
            "adv": n(8), "mask": torch.arange(24, device="cuda:0") < torch.randint(1, 25, (8, 1), device="cuda:0", generator=gen), "seed": torch.tensor(77, device="cuda:0")}


def _policy_pass(v):
    """Dropout and norm, both heads, log probabilities, KL, policy loss, a preference loss over the same rows, and all gradients, pass by pass."""
    import torch
    o = ops()
    y, h, mean, rstd = o.dropout_add_layer_norm_forward(v["x"], v["res"], v["w"], v["b"], 0.1, v["seed"], 1)
    z = o.dropout_forward(y, 0.2, v["seed"], 2)
    logits, ref = z @ v["head"], z @ v["ref"]
    flat = v["mask"].reshape(-1)
    r = o.token_logprobs_forward(logits, v["t"])
    kl, stats = o.token_kl_forward(logits, ref, mask=flat)
    logp, ent, k = r.logp.view(8, 24), r.entropy.view(8, 24), kl.view(8, 24)
    terms = dict(mask=v["mask"], clip=(0.2, 0.3), kl=k, kl_coef=0.1, entropy=ent, entropy_coef=0.01, reduction="sequences")
    p = o.policy_loss_forward(logp, v["old"], v["adv"], **terms)
    q = o.preference_loss_forward(logp, v["old"], v["mask"])
    one = torch.ones_like(p.loss)
    dlogp, dkl, dent = o.policy_loss_backward(one, p, logp, v["old"], v["adv"], **terms)
    dlogp = dlogp + o.preference_loss_backward(one, q, logp, v["mask"])
    dlogits = o.token_logprobs_backward(logits, v["t"], r.stats, r.entropy, dlogp.view(-1), dent.view(-1))
    dk, dref = o.token_kl_backward(logits, ref, stats, dkl.view(-1), mask=flat, need=(True, True))
    dz = (dlogits + dk) @ v["head"].t().contiguous() + dref @ v["ref"].t().contiguous()
    dy = o.dropout_forward(dz, 0.2, v["seed"], 2)
    grads = o.dropout_add_layer_norm_backward(dy, h, h, v["w"], mean, rstd, 0.1, v["seed"], 1)
    out, norm = o.clip_grads(list(grads), 0.5)
    return [y, h, mean, rstd, z, logits, r.logp, kl, stats, *p, *q, dlogp, dkl, dent, dlogits, dk, dref, *grads, norm, *out]


def test_more_operators_on_another_stream_and_twice_the_same():
    import torch
    v = _inputs()
    a = _policy_pass(v)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = _policy_pass(v)
    s.synchronize()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_more_operators_in_captured_graphs():
    """Two graphs of the whole pass in one memory pool, replayed in turn with other inputs and another seed each time, against the same pass outside."""
    import torch
    v = _inputs()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        _policy_pass(v)
    torch.cuda.current_stream().wait_stream(s)
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    outs = []
    for i, g in enumerate(graphs):
        with torch.cuda.graph(g, pool=graphs[0].pool() if i else None):
            outs.append(_policy_pass(v))
    for k in range(6):
        v["x"].copy_(torch.roll(v["x"], k + 1, 0) * 1.1)
        v["t"].copy_(torch.roll(v["t"], 1))
        v["seed"] += 1
        graphs[k % 2].replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs[k % 2]]
        want = _policy_pass(v)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want)), k
    assert not torch.equal(outs[0][4] == 0, outs[1][4] == 0)       # another seed, another mask


def test_training_pass_against_plain_torch():
    """The same through autograd, against torch in float64 with the masks of the definition."""
    import torch
    v = _inputs()
    o = ops()
    leaves = [v[k].requires_grad_() for k in ("x", "res", "w", "b", "head")]
    y, h = o.dropout_add_layer_norm(v["x"], v["res"], v["w"], v["b"], 0.1, v["seed"], 1)
    z = o.dropout(y, 0.2, v["seed"], 2)
    logits = z @ v["head"]
    with torch.no_grad():
        ref = z @ v["ref"]
    r = o.token_logprobs(logits, v["t"])
    kl = o.token_kl(logits, ref, mask=v["mask"].reshape(-1))
    logp = r.logp.view(8, 24)
    p = o.policy_loss(logp, v["old"], v["adv"], v["mask"], kl=kl.view(8, 24), kl_coef=0.1, entropy=r.entropy.view(8, 24), entropy_coef=0.01, reduction="sequences")
    q = o.preference_loss(logp, v["old"], v["mask"])
    (p.loss + q.loss + 1e-3 * h.square().sum()).backward()

    w = {k: (t.detach().cpu().double() if t.is_floating_point() else t.detach().cpu()) for k, t in v.items()}
    refs = [w[k].requires_grad_() for k in ("x", "res", "w", "b", "head")]
    keep = lambda pr, n, off: torch.from_numpy(keep_of(w["x"].shape[0], n, pr, 77, off)) / (1 - float(np.float32(pr)))
    h64 = w["res"] + w["x"] * keep(0.1, 120, 1)
    d = h64 - h64.mean(-1, keepdim=True)
    z64 = (d / (d.square().mean(-1, keepdim=True) + EPS).sqrt() * w["w"] + w["b"]) * keep(0.2, 120, 2)
    lp = torch.log_softmax(z64 @ w["head"], -1)
    lq = torch.log_softmax(z64.detach() @ w["ref"], -1)
    at = lp.gather(1, w["t"][:, None])[:, 0].view(8, 24)
    k64, e64 = (lp.exp() * (lp - lq)).sum(-1).view(8, 24), -(lp.exp() * lp).sum(-1).view(8, 24)
    m, a = w["mask"].double(), w["adv"][:, None]
    ratio = (at - w["old"]).exp()
    sur = -torch.minimum(ratio * a, ratio.clamp(0.8, 1.2) * a)
    loss = ((sur + 0.1 * k64 - 0.01 * e64) * m).sum(1).div(m.sum(1)).mean()
    s = ((at - w["old"]) * m).sum(1)
    pref = -torch.nn.functional.logsigmoid(0.1 * (s[:4] - s[4:])).mean()
    (loss + pref + 1e-3 * h64.square().sum()).backward()
    # a dozen stages in a row, each a sum of at most 501 terms: 12 * 501 roundings
    rel = 12 * 501 * U
    assert abs(float(p.loss.detach()) - float(loss.detach())) <= rel * (abs(float(loss.detach())) + 1)
    assert abs(float(q.loss.detach()) - float(pref.detach())) <= rel * (abs(float(pref.detach())) + 1)
    for got, want in zip(leaves, refs):
        g, e = host(got.grad), want.grad.numpy()
        assert np.abs(g - e).max() <= rel * np.abs(e).max()


def test_more_functions_refuse_what_they_cannot_take():
    import torch
    o = ops()
    x, m = torch.randn(4, 8, device="cuda:0"), torch.ones(4, 8, dtype=torch.bool, device="cuda:0")
    s = torch.zeros(4, 5, device="cuda:0")
    one = torch.ones((), device="cuda:0")
    r = o.policy_loss_forward(x, x, x)
    q = o.preference_loss_forward(x)
    for call in (lambda: o.dropout(x.double(), 0.1, 0), lambda: o.dropout(x, 0.1, -1), lambda: o.dropout(x, 0.1, 1 << 64), lambda: o.dropout(x, 0.1, 0, -1), lambda: o.dropout(x, 0.1, 0, 1 << 64),
                 lambda: o.dropout(x, 0.1, torch.zeros(2, dtype=torch.int64, device="cuda:0")), lambda: o.dropout(x, 0.1, torch.zeros((), device="cuda:0")),
                 lambda: o.dropout(x, 0.1, torch.zeros((), dtype=torch.int64)), lambda: o.dropout(x[:, :0], 0.1, 0), lambda: o.dropout(one, 0.1, 0),
                 lambda: o.dropout_add_layer_norm(x, x[:3]), lambda: o.dropout_add_layer_norm(x, x.cpu()), lambda: o.dropout_add_layer_norm(x, x.double()),
                 lambda: o.dropout_add_layer_norm(x, x, x[0, :7]), lambda: o.dropout_add_layer_norm(x, x, x[0], x[0].half()),
                 lambda: o.dropout_add_layer_norm_backward(x, x.half(), x, None, x[:, 0], x[:, 0]), lambda: o.dropout_add_layer_norm_backward(x, None, x[:3], None, x[:, 0], x[:, 0]),
                 lambda: o.dropout_add_layer_norm_backward(x, None, x, None, x[:3, 0], x[:, 0]),
                 lambda: o.token_kl(x, x[:3]), lambda: o.token_kl(x, x.half()), lambda: o.token_kl(x, x.cpu()), lambda: o.token_kl(x, x, mask=m), lambda: o.token_kl(x, x, mask=x[:, 0]),
                 lambda: o.token_kl_backward(x, x, s[:, :4], x[:, 0]), lambda: o.token_kl_backward(x, x, s, x[0]),
                 lambda: o.policy_loss(x.half(), x, x), lambda: o.policy_loss(x, x[:3], x), lambda: o.policy_loss(x, x, x[:3]), lambda: o.policy_loss(x, x, x, m[:, :7]),
                 lambda: o.policy_loss(x, x, x, x), lambda: o.policy_loss(x, x, x, ref_logp=x, kl=x, kl_coef=0.1), lambda: o.policy_loss(x, x, x, kl_coef=0.1),
                 lambda: o.policy_loss(x, x, x, entropy_coef=0.1), lambda: o.policy_loss(x, x, x, reduction="mean"), lambda: o.policy_loss(x, x, x, kl=x.half(), kl_coef=0.1),
                 lambda: o.policy_loss(x, x.double(), x), lambda: o.policy_loss(x, x, x[:, 0].double()),
                 lambda: o.policy_loss_backward(x, r, x, x, x), lambda: o.policy_loss_backward(one.cpu(), r, x, x, x),
                 lambda: o.preference_loss(x[:3]), lambda: o.preference_loss(x[0]), lambda: o.preference_loss(x.half()), lambda: o.preference_loss(x, x[:2]), lambda: o.preference_loss(x, x[:2, 0]),
                 lambda: o.preference_loss(x, mask=m[0]), lambda: o.preference_loss(x, kind="other"), lambda: o.preference_loss(x, x[:, 0].double()),
                 lambda: o.preference_loss_backward(one, q._replace(coef=q.coef[:3]), x), lambda: o.preference_loss_backward(x, q, x)):
        with pytest.raises(ValueError):
            call()
    from paper_2506_10315_amd import LoptError
    for call in (lambda: o.dropout(x, 1.5, 0), lambda: o.dropout(x, math.nan, 0), lambda: o.dropout_add_layer_norm(x, x, p=-0.1), lambda: o.dropout_add_layer_norm(x, x, eps=-1.0),
                 lambda: o.dropout_add_layer_norm(x.half(), x.bfloat16()), lambda: o.token_kl(x, x, scale=0.0), lambda: o.policy_loss(x, x, x, clip=(1.5, 0.2)),
                 lambda: o.policy_loss(x, x, x, clip=(0.2, -0.1)), lambda: o.preference_loss(x, beta=0.0), lambda: o.preference_loss(x, kind="hinge", label_smoothing=0.1)):
        with pytest.raises(LoptError):
            call()
