"""Refusals of the calls without a context, at the C boundary: every one comes before anything is launched, so no GPU is
needed and the pointers are never followed."""
import ctypes as C
import math

import pytest

EINVAL, ESHAPE = 1, 2
P = 0x10000     # an address that is never read


@pytest.fixture(scope="module")
def L():
    import paper_2506_10315_amd as pkg
    return pkg.lib()


def _refused(L, status, want, word):
    assert status == want, (status, L.lopt_last_error(None))
    assert word in L.lopt_last_error(None).decode(), L.lopt_last_error(None)


def _clip(L, counts=(10,), grads=(P,), types=(0,), out=(P,), out_types=(0,), max_norm=1.0, norm=P, ws=P, ws_bytes=1 << 20, n=None, null=()):
    n = len(counts) if n is None else n
    arr = lambda ty, v, name: None if name in null else (ty * max(len(v), 1))(*v)
    return L.lopt_clip_grads(n, arr(C.c_int64, counts, "counts"), arr(C.c_void_p, grads, "grads"), arr(C.c_uint32, types, "types"),
                             arr(C.c_void_p, out, "out"), arr(C.c_uint32, out_types, "out_types"), max_norm, norm, ws, ws_bytes, None)


def test_clip_refusals(L):
    _refused(L, _clip(L, norm=None), EINVAL, "norm")
    _refused(L, _clip(L, norm=P + 2), EINVAL, "norm")
    for bad in (-1.0, math.nan, -math.inf):
        _refused(L, _clip(L, max_norm=bad), EINVAL, "max_norm")
    for name in ("counts", "grads", "types", "out_types"):
        _refused(L, _clip(L, null=(name,)), EINVAL, "null")
    _refused(L, _clip(L, counts=(-1,)), ESHAPE, "counts")
    _refused(L, _clip(L, counts=(1 << 40,)), ESHAPE, "counts")
    _refused(L, _clip(L, types=(3,)), EINVAL, "type")
    _refused(L, _clip(L, out_types=(7,)), EINVAL, "type")
    _refused(L, _clip(L, grads=(None,)), EINVAL, "null")
    _refused(L, _clip(L, out=(None,)), EINVAL, "null")
    _refused(L, _clip(L, grads=(P + 2,)), EINVAL, "aligned")
    _refused(L, _clip(L, out=(P + 1,), out_types=(1,)), EINVAL, "aligned")
    _refused(L, _clip(L, types=(1,)), EINVAL, "in place")
    _refused(L, _clip(L, ws=None), EINVAL, "workspace")
    _refused(L, _clip(L, ws=P + 4), EINVAL, "workspace")
    _refused(L, _clip(L, ws_bytes=8), EINVAL, "workspace")
    counts = (C.c_int64 * 2)(1 << 30, 0)
    assert L.lopt_clip_workspace(2, counts) >= 16 and L.lopt_clip_workspace(0, None) >= 16


def test_clip_refuses_outputs_that_share_memory(L):
    """Two workgroups would read and write the same elements, in no order."""
    def clip(grads, out, counts=None, types=None, out_types=None, ws=None):
        n = len(grads)
        return _clip(L, counts=counts or (10,) * n, grads=grads, types=types or (0,) * n, out=out, out_types=out_types or (0,) * n, ws=ws)
    for grads, out in (((P, P), (P, P)), ((P, P, 2 * P), (P, P, 2 * P)), ((2 * P, P, 2 * P), (2 * P, P, 2 * P)), ((P, 2 * P), (3 * P, 3 * P)),
                       ((P, 2 * P), (3 * P, 3 * P + 36)), ((P, 2 * P), (3 * P + 36, 3 * P)), ((P, P + 36), (P, P + 36))):
        _refused(L, clip(grads, out), EINVAL, "overlap")
    for grads, out in (((P, 2 * P), (3 * P, P)), ((P, 2 * P), (2 * P, 3 * P)), ((P, 2 * P), (2 * P, P)), ((P, P), (P, 2 * P)), ((P,), (P + 8,)), ((P,), (P - 36,)),
                       ((P, 2 * P), (P, 2 * P + 4))):
        _refused(L, clip(grads, out), EINVAL, "overlap")
    _refused(L, clip((P, P + 20), (2 * P, 2 * P + 20), types=(1, 1)), EINVAL, "overlap")     # outputs twice as wide as the gradients
    # neighbours, gradients listed twice that go elsewhere, empty tensors, in place: on to the next check
    for grads, out in (((P, P + 40), (P, P + 40)), ((P + 40, P), (P + 40, P)), ((P, P), (2 * P, 2 * P + 40)), ((P,), (P + 40,)), ((P,), (P - 40,)),
                       ((P, 2 * P, 3 * P), (3 * P + 40, 2 * P, P + 40))):
        _refused(L, clip(grads, out), EINVAL, "workspace")
    _refused(L, clip((P, P, None), (P, P, None), counts=(10, 0, 0)), EINVAL, "workspace")
    _refused(L, _clip(L, counts=(10, 10), grads=(P, P), types=(0, 0), ws=None, null=("out", "out_types")), EINVAL, "workspace")     # the norm alone only reads


def _norm(L, x=P, ld_x=8, w=P, b=P, y=2 * P, ld_y=8, mean=P, rstd=P, rows=4, cols=8, eps=1e-5, kind=0, wkind=0):
    return L.lopt_layer_norm(x, ld_x, w, b, y, ld_y, mean, rstd, rows, cols, eps, kind, wkind, None)


def test_layer_norm_refusals(L):
    _refused(L, _norm(L, kind=3), EINVAL, "type")
    _refused(L, _norm(L, wkind=9), EINVAL, "weight_type")
    _refused(L, _norm(L, rows=-1), ESHAPE, "rows")
    _refused(L, _norm(L, rows=1 << 31), ESHAPE, "rows")
    for cols in (0, -3, 1 << 31):
        _refused(L, _norm(L, cols=cols, ld_y=1 << 40), ESHAPE, "cols")
    for eps in (-1e-9, math.nan, math.inf):
        _refused(L, _norm(L, eps=eps), EINVAL, "eps")
    _refused(L, _norm(L, ld_y=7), ESHAPE, "ld_y")
    _refused(L, _norm(L, ld_x=-8), ESHAPE, "ld_x")
    _refused(L, _norm(L, ld_x=1 << 62), ESHAPE, "ld_x")
    _refused(L, _norm(L, x=None), EINVAL, "x")
    _refused(L, _norm(L, y=None), EINVAL, "y")
    _refused(L, _norm(L, x=P + 2), EINVAL, "x")
    _refused(L, _norm(L, w=P + 1, wkind=1), EINVAL, "weight")
    _refused(L, _norm(L, b=P + 2), EINVAL, "bias")
    _refused(L, _norm(L, mean=P + 1), EINVAL, "mean")
    _refused(L, _norm(L, y=P, ld_y=9), EINVAL, "ld_y")
    _refused(L, _norm(L, y=P, ld_x=0), ESHAPE, "ld_x")
    assert _norm(L, rows=0, x=None, y=None) == 0


def _norm_back(L, dy=P, ld_dy=8, x=2 * P, ld_x=8, w=P, mean=P, rstd=P, dx=3 * P, ld_dx=8, dw=P, db=P, rows=4, cols=8, kind=0, wkind=0, ws=P,
               ws_bytes=1 << 30):
    return L.lopt_layer_norm_backward(dy, ld_dy, x, ld_x, w, mean, rstd, dx, ld_dx, dw, db, rows, cols, kind, wkind, ws, ws_bytes, None)


def test_layer_norm_backward_refusals(L):
    _refused(L, _norm_back(L, kind=3), EINVAL, "type")
    _refused(L, _norm_back(L, cols=0), ESHAPE, "cols")
    _refused(L, _norm_back(L, dy=None), EINVAL, "dy")
    _refused(L, _norm_back(L, x=None), EINVAL, "x")
    _refused(L, _norm_back(L, mean=None), EINVAL, "mean")
    _refused(L, _norm_back(L, rstd=P + 3), EINVAL, "rstd")
    _refused(L, _norm_back(L, ld_dx=7), ESHAPE, "ld_dx")
    _refused(L, _norm_back(L, dx=P, ld_dx=9), EINVAL, "ld_dx")
    _refused(L, _norm_back(L, dw=P + 2), EINVAL, "dweight")
    _refused(L, _norm_back(L, ws=None), EINVAL, "workspace")
    _refused(L, _norm_back(L, ws_bytes=3), EINVAL, "workspace")
    assert L.lopt_layer_norm_workspace(0, 8) == 0 and L.lopt_layer_norm_workspace(4, 8) > 0
    assert _norm_back(L, rows=0, dy=None, x=None, mean=None, rstd=None, dw=None, db=None) == 0


def _logp(L, x=P, ld=8, t=P, rows=4, vocab=8, kind=0, scale=1.0, ignore=-100, top=2, logp=P, ent=P, stats=P, tl=P, ti=P, ws=P, ws_bytes=1 << 30):
    return L.lopt_token_logprobs(x, ld, t, rows, vocab, kind, scale, ignore, top, logp, ent, stats, tl, ti, ws, ws_bytes, None)


def test_token_logprobs_refusals(L):
    _refused(L, _logp(L, kind=4), EINVAL, "type")
    _refused(L, _logp(L, vocab=0), ESHAPE, "vocab")
    _refused(L, _logp(L, vocab=1 << 31), ESHAPE, "vocab")
    _refused(L, _logp(L, rows=-2), ESHAPE, "rows")
    _refused(L, _logp(L, ld=-1), ESHAPE, "ld")
    for scale in (0.0, -1.0, math.nan, math.inf):
        _refused(L, _logp(L, scale=scale), EINVAL, "scale")
    _refused(L, _logp(L, top=9), EINVAL, "top")
    _refused(L, _logp(L, top=33, vocab=100, ld=100), EINVAL, "top")
    _refused(L, _logp(L, x=None), EINVAL, "logits")
    _refused(L, _logp(L, t=None), EINVAL, "targets")
    _refused(L, _logp(L, stats=None), EINVAL, "stats")
    _refused(L, _logp(L, tl=None), EINVAL, "top_logp")
    _refused(L, _logp(L, ti=None), EINVAL, "top_index")
    _refused(L, _logp(L, ti=P + 4), EINVAL, "top_index")
    _refused(L, _logp(L, logp=P + 1), EINVAL, "logp")
    need = L.lopt_token_logprobs_workspace(4, 50000, 20)
    if need:
        _refused(L, _logp(L, vocab=50000, ld=50000, top=20, ws_bytes=need - 1), EINVAL, "workspace")
    assert _logp(L, rows=0, x=None, t=None, stats=None, ws=None, ws_bytes=0) == 0


def _logp_back(L, x=P, ld=8, t=P, stats=P, ent=P, g=P, h=P, dx=2 * P, ld_d=8, rows=4, vocab=8, kind=0, scale=1.0, ignore=-100):
    return L.lopt_token_logprobs_backward(x, ld, t, stats, ent, g, h, dx, ld_d, rows, vocab, kind, scale, ignore, None)


def test_token_logprobs_backward_refusals(L):
    _refused(L, _logp_back(L, kind=4), EINVAL, "type")
    _refused(L, _logp_back(L, x=None), EINVAL, "logits")
    _refused(L, _logp_back(L, dx=None), EINVAL, "dlogits")
    _refused(L, _logp_back(L, stats=None), EINVAL, "stats")
    _refused(L, _logp_back(L, t=None), EINVAL, "targets")
    _refused(L, _logp_back(L, ent=None), EINVAL, "entropy")
    _refused(L, _logp_back(L, ld_d=7), ESHAPE, "ld_d")
    _refused(L, _logp_back(L, dx=P, ld_d=9), EINVAL, "ld_d")
    _refused(L, _logp_back(L, scale=-1.0), EINVAL, "scale")
    assert _logp_back(L, rows=0, x=None, dx=None, stats=None, t=None, ent=None) == 0


def test_functions_refuse_cpu_tensors():
    import torch
    from paper_2506_10315_amd import ops
    x = torch.randn(3, 4)
    for call in (lambda: ops.layer_norm(x), lambda: ops.token_logprobs(x, torch.zeros(3, dtype=torch.int64)), lambda: ops.clip_grads([x], 1.0),
                 lambda: ops.grad_norm([x]), lambda: ops.clip_grad_norm_([], 1.0)):
        with pytest.raises(ValueError):
            call()
