"""Refusals of dropout, of dropout with residual and layer norm, of the KL divergence and of the losses, at the C boundary and in the torch functions:
every one comes before anything is launched, so no GPU is needed and the pointers are never followed."""
import ctypes as C
import math
import os
import re

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


BAD_P = (-0.1, 1.0001, math.nan, math.inf)


def _dropout(L, x=P, ld_x=8, y=2 * P, ld_y=8, rows=4, cols=8, kind=0, p=0.1, seed=1, dev=None, offset=0):
    return L.lopt_dropout(x, ld_x, y, ld_y, rows, cols, kind, p, seed, dev, offset, None)


def test_dropout_refusals(L):
    _refused(L, _dropout(L, kind=3), EINVAL, "type")
    for p in BAD_P:
        _refused(L, _dropout(L, p=p), EINVAL, "p must")
    _refused(L, _dropout(L, rows=-1), ESHAPE, "rows")
    for cols in (0, 1 << 31):
        _refused(L, _dropout(L, cols=cols), ESHAPE, "cols")
    _refused(L, _dropout(L, ld_x=-1), ESHAPE, "ld_x")
    _refused(L, _dropout(L, ld_y=7), ESHAPE, "ld_y")
    _refused(L, _dropout(L, ld_y=1 << 60), ESHAPE, "ld_y")
    _refused(L, _dropout(L, x=None), EINVAL, "x")
    _refused(L, _dropout(L, y=None), EINVAL, "y")
    _refused(L, _dropout(L, y=P + 2), EINVAL, "aligned")
    _refused(L, _dropout(L, dev=P + 4), EINVAL, "seed_device")
    _refused(L, _dropout(L, y=P, ld_y=9), EINVAL, "ld_y")
    assert _dropout(L, rows=0, x=None, y=None) == 0


def _add_norm(L, x=P, ld_x=8, res=2 * P, ld_res=8, w=P, b=P, y=3 * P, ld_y=8, h=4 * P, ld_h=8, mean=P, rstd=P, rows=4, cols=8, eps=1e-5, kind=1, rkind=0, wkind=0,
              p=0.1, dev=None):
    return L.lopt_dropout_add_layer_norm(x, ld_x, res, ld_res, w, b, y, ld_y, h, ld_h, mean, rstd, rows, cols, eps, kind, rkind, wkind, p, 1, dev, 0, None)


def test_dropout_add_layer_norm_refusals(L):
    _refused(L, _add_norm(L, kind=3), EINVAL, "type")
    _refused(L, _add_norm(L, rkind=3), EINVAL, "residual_type")
    _refused(L, _add_norm(L, rkind=2), EINVAL, "residual_type")
    _refused(L, _add_norm(L, kind=0, rkind=1), EINVAL, "residual_type")
    _refused(L, _add_norm(L, wkind=7), EINVAL, "weight_type")
    for p in BAD_P:
        _refused(L, _add_norm(L, p=p), EINVAL, "p must")
    for eps in (-1e-9, math.nan, math.inf):
        _refused(L, _add_norm(L, eps=eps), EINVAL, "eps")
    _refused(L, _add_norm(L, cols=0), ESHAPE, "cols")
    _refused(L, _add_norm(L, rows=1 << 31), ESHAPE, "rows")
    for name in ("ld_y", "ld_h"):
        _refused(L, _add_norm(L, **{name: 7}), ESHAPE, name)
    for name in ("ld_x", "ld_res"):
        _refused(L, _add_norm(L, **{name: -1}), ESHAPE, name)
    for name, word in (("x", "x"), ("res", "residual"), ("y", "y"), ("h", "h")):
        _refused(L, _add_norm(L, **{name: None}), EINVAL, word)
        _refused(L, _add_norm(L, **{name: 5 * P + 1}), EINVAL, word)
    _refused(L, _add_norm(L, w=P + 2), EINVAL, "weight")
    _refused(L, _add_norm(L, b=P + 2), EINVAL, "bias")
    _refused(L, _add_norm(L, rstd=P + 2), EINVAL, "rstd")
    _refused(L, _add_norm(L, dev=P + 1), EINVAL, "seed_device")
    _refused(L, _add_norm(L, y=3 * P, h=3 * P, rkind=1), EINVAL, "same memory")
    _refused(L, _add_norm(L, y=2 * P), EINVAL, "another type")            # bf16 over the fp32 residual
    _refused(L, _add_norm(L, h=P), EINVAL, "another type")
    _refused(L, _add_norm(L, y=P, ld_y=9), EINVAL, "ld")
    _refused(L, _add_norm(L, h=2 * P, ld_h=9), EINVAL, "ld")
    _refused(L, _add_norm(L, h=2 * P, ld_res=0, ld_h=8), ESHAPE, "ld_res")  # a residual of one row for all is not written
    assert _add_norm(L, rows=0, x=None, res=None, y=None, h=None) == 0


def _add_norm_back(L, dy=P, ld_dy=8, dh=2 * P, ld_dh=8, h=3 * P, ld_h=8, w=P, mean=P, rstd=P, dx=4 * P, ld_dx=8, dres=5 * P, ld_dres=8, dw=P, db=P, rows=4, cols=8,
                   kind=1, rkind=0, wkind=0, p=0.1, dev=None, ws=P, ws_bytes=1 << 30):
    return L.lopt_dropout_add_layer_norm_backward(dy, ld_dy, dh, ld_dh, h, ld_h, w, mean, rstd, dx, ld_dx, dres, ld_dres, dw, db, rows, cols, kind, rkind, wkind, p, 1,
                                                  dev, 0, ws, ws_bytes, None)


def test_dropout_add_layer_norm_backward_refusals(L):
    _refused(L, _add_norm_back(L, kind=3), EINVAL, "type")
    _refused(L, _add_norm_back(L, rkind=2), EINVAL, "residual_type")
    _refused(L, _add_norm_back(L, wkind=3), EINVAL, "weight_type")
    for p in BAD_P:
        _refused(L, _add_norm_back(L, p=p), EINVAL, "p must")
    _refused(L, _add_norm_back(L, cols=0), ESHAPE, "cols")
    for name, word in (("dy", "dy"), ("h", "h"), ("mean", "mean"), ("rstd", "rstd")):
        _refused(L, _add_norm_back(L, **{name: None}), EINVAL, word)
    for name, word in (("dy", "dy"), ("dh", "dh"), ("h", "h"), ("dx", "dx"), ("dres", "dresidual"), ("dw", "dweight"), ("db", "dbias"), ("w", "weight")):
        _refused(L, _add_norm_back(L, **{name: 9 * P + 1}), EINVAL, word)
    for name in ("ld_dx", "ld_dres"):
        _refused(L, _add_norm_back(L, **{name: 7}), ESHAPE, name)
    for name in ("ld_dy", "ld_dh", "ld_h"):
        _refused(L, _add_norm_back(L, **{name: -1}), ESHAPE, name)
    _refused(L, _add_norm_back(L, dx=5 * P), EINVAL, "same memory")
    _refused(L, _add_norm_back(L, dx=3 * P), EINVAL, "another type")
    _refused(L, _add_norm_back(L, dres=P), EINVAL, "another type")
    _refused(L, _add_norm_back(L, dx=P, ld_dx=9), EINVAL, "ld")
    _refused(L, _add_norm_back(L, dres=2 * P, ld_dres=9), EINVAL, "ld")
    _refused(L, _add_norm_back(L, ws=None), EINVAL, "workspace")
    need = L.lopt_dropout_add_layer_norm_workspace(4, 8)
    assert need > 0 and L.lopt_dropout_add_layer_norm_workspace(0, 8) == 0
    _refused(L, _add_norm_back(L, ws_bytes=need - 1), EINVAL, "workspace")
    assert _add_norm_back(L, rows=0, dy=None, h=None, mean=None, rstd=None, dw=None, db=None) == 0


def _kl(L, x=P, ld=8, r=2 * P, ld_ref=8, mask=None, rows=4, vocab=8, kind=0, scale=1.0, kl=P, stats=P, ws=P, ws_bytes=1 << 30):
    return L.lopt_token_kl(x, ld, r, ld_ref, mask, rows, vocab, kind, scale, kl, stats, ws, ws_bytes, None)


def test_token_kl_refusals(L):
    _refused(L, _kl(L, kind=3), EINVAL, "type")
    _refused(L, _kl(L, vocab=0), ESHAPE, "vocab")
    _refused(L, _kl(L, vocab=0x7fff0001, ld=0x7fff0001, ld_ref=0x7fff0001), ESHAPE, "vocab")
    _refused(L, _kl(L, rows=-1), ESHAPE, "rows")
    _refused(L, _kl(L, ld=-1), ESHAPE, "ld")
    _refused(L, _kl(L, ld_ref=-1), ESHAPE, "ld_ref")
    for scale in (0.0, -1.0, math.nan, math.inf):
        _refused(L, _kl(L, scale=scale), EINVAL, "scale")
    for name, word in (("x", "logits"), ("r", "ref"), ("kl", "kl"), ("stats", "stats")):
        _refused(L, _kl(L, **{name: None}), EINVAL, word)
        _refused(L, _kl(L, **{name: P + 1}), EINVAL, word)
    need = L.lopt_token_kl_workspace(3, 1 << 20)
    assert need > 0 and L.lopt_token_kl_workspace(4, 50257) == 0 and L.lopt_token_kl_workspace(0, 8) == 0
    long = dict(rows=3, vocab=1 << 20, ld=1 << 20, ld_ref=1 << 20)
    _refused(L, _kl(L, ws=None, **long), EINVAL, "workspace")
    _refused(L, _kl(L, ws_bytes=need - 1, **long), EINVAL, "workspace")
    assert _kl(L, rows=0, x=None, r=None, kl=None, stats=None) == 0


def _kl_back(L, x=P, ld=8, r=2 * P, ld_ref=8, mask=None, stats=P, dkl=P, dx=3 * P, ld_d=8, dr=4 * P, ld_dr=8, rows=4, vocab=8, kind=0, scale=1.0):
    return L.lopt_token_kl_backward(x, ld, r, ld_ref, mask, stats, dkl, dx, ld_d, dr, ld_dr, rows, vocab, kind, scale, None)


def test_token_kl_backward_refusals(L):
    _refused(L, _kl_back(L, kind=3), EINVAL, "type")
    _refused(L, _kl_back(L, scale=0.0), EINVAL, "scale")
    for name, word in (("x", "logits"), ("r", "ref"), ("stats", "stats"), ("dkl", "dkl")):
        _refused(L, _kl_back(L, **{name: None}), EINVAL, word)
    _refused(L, _kl_back(L, dx=P + 1), EINVAL, "dlogits")
    _refused(L, _kl_back(L, dr=P + 2), EINVAL, "dref")
    _refused(L, _kl_back(L, ld_d=7), ESHAPE, "ld_d")
    _refused(L, _kl_back(L, ld_dr=7), ESHAPE, "ld_dref")
    _refused(L, _kl_back(L, dx=4 * P), EINVAL, "same memory")
    _refused(L, _kl_back(L, dx=P, ld_d=9), EINVAL, "ld")
    _refused(L, _kl_back(L, dr=P, ld_dr=9), EINVAL, "ld")
    assert _kl_back(L, dx=None, dr=None) == 0
    assert _kl_back(L, rows=0, x=None, r=None, stats=None, dkl=None) == 0


# lopt_policy and lopt_preference, as a caller's compiler lays them out
class Policy(C.Structure):
    _fields_ = [f for name in ("logp", "old", "adv", "ref", "kl", "ent", "mask") for f in ((name, C.c_void_p), ("ld_" + name, C.c_int64))] + [
        ("seqs", C.c_int64), ("tokens", C.c_int64), ("clip_low", C.c_double), ("clip_high", C.c_double), ("kl_coef", C.c_double), ("entropy_coef", C.c_double),
        ("old_type", C.c_uint32), ("adv_type", C.c_uint32), ("ref_type", C.c_uint32), ("adv_per_seq", C.c_uint32), ("per_sequence", C.c_uint32),
        ("reserved", C.c_uint32)]


class Preference(C.Structure):
    _fields_ = [f for name in ("logp", "ref", "mask") for f in ((name, C.c_void_p), ("ld_" + name, C.c_int64))] + [
        ("pairs", C.c_int64), ("tokens", C.c_int64), ("beta", C.c_double), ("smooth", C.c_double), ("margin", C.c_double),
        ("ref_type", C.c_uint32), ("ref_sums", C.c_uint32), ("kind", C.c_uint32), ("average", C.c_uint32)]


def test_packed_terms_are_the_headers_structs():
    """The bytes that ops.py packs against the structs that include/lopt.h declares, field by field."""
    from paper_2506_10315_amd import ops
    assert C.sizeof(Policy) == ops._POLICY.size and C.sizeof(Preference) == ops._PREFERENCE.size
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = open(os.path.join(root, "include", "lopt.h")).read()
    sizes = {"float*": "Q", "void*": "Q", "uint8_t*": "Q", "int64_t": "q", "double": "d", "uint32_t": "I"}
    for name, packed in (("lopt_policy", ops._POLICY), ("lopt_preference", ops._PREFERENCE)):
        body = re.search(r"typedef struct \{([^}]*)\} %s;" % name, text).group(1)
        body = re.sub(r"/\*.*?\*/", "", body, flags=re.S).replace("const ", "")
        codes = ""
        for decl in body.split(";"):
            if decl.strip():
                kind, names = decl.split(None, 1)
                codes += sizes[kind] * len(names.split(","))
        flat = re.sub(r"(\d+)(\w)", lambda m: m.group(2) * int(m.group(1)), packed.format.lstrip("="))
        assert codes == flat, name


def _policy_terms(**over):
    v = dict(logp=P, ld_logp=8, old=P, ld_old=8, adv=P, ld_adv=8, ref=None, ld_ref=8, kl=None, ld_kl=8, ent=None, ld_ent=8, mask=None, ld_mask=8, seqs=4, tokens=8,
             clip_low=0.2, clip_high=0.2, kl_coef=0.1, entropy_coef=0.1, per_sequence=1)
    v.update(over)
    return C.byref(Policy(**v))


def _policy(L, loss=P, stats=P, counts=P, ws=P, ws_bytes=1 << 30, **terms):
    return L.lopt_policy_loss(_policy_terms(**terms), loss, stats, counts, ws, ws_bytes, None)


def _policy_back(L, stats=P, counts=P, dloss=P, dlogp=P, dkl=None, dent=None, **terms):
    return L.lopt_policy_loss_backward(_policy_terms(**terms), stats, counts, dloss, dlogp, dkl, dent, None)


@pytest.mark.parametrize("call", [_policy, _policy_back])
def test_policy_loss_refusals(L, call):
    _refused(L, call(L, seqs=-1), ESHAPE, "rows")
    _refused(L, call(L, tokens=0), ESHAPE, "tokens")
    for name, word in (("logp", "logp"), ("old", "old_logp"), ("adv", "advantages")):
        _refused(L, call(L, **{name: None}), EINVAL, word)
        _refused(L, call(L, **{name: P + 2}), EINVAL, word)
    for name, word in (("ref", "ref_logp"), ("kl", "kl"), ("ent", "entropy")):
        _refused(L, call(L, **{name: P + 2}), EINVAL, word)
    for name in ("logp", "old", "adv", "ref", "kl", "ent", "mask"):
        given = {name: P} if name not in ("logp", "old", "adv") else {}
        _refused(L, call(L, **{"ld_" + name: -1}, **given), ESHAPE, "ld_")
    for name in ("old_type", "adv_type", "ref_type"):
        _refused(L, call(L, **{name: 3}), EINVAL, "type")
    _refused(L, call(L, ref=P, kl=P), EINVAL, "both")
    for bad in (-0.1, 1.1, math.nan):
        _refused(L, call(L, clip_low=bad), EINVAL, "clip_low")
    for bad in (-0.1, math.nan):
        _refused(L, call(L, clip_high=bad), EINVAL, "clip_high")
    for bad in (math.inf, math.nan):
        _refused(L, call(L, kl_coef=bad), EINVAL, "kl_coef")
        _refused(L, call(L, entropy_coef=bad), EINVAL, "entropy_coef")
    _refused(L, call(L, stats=None), EINVAL, "stats")
    _refused(L, call(L, counts=None), EINVAL, "counts")


def test_policy_loss_refusals_of_each_pass(L):
    _refused(L, L.lopt_policy_loss(None, P, P, P, P, 8, None), EINVAL, "terms_host")
    _refused(L, L.lopt_policy_loss_backward(None, P, P, P, P, P, P, None), EINVAL, "terms_host")
    _refused(L, _policy(L, loss=None), EINVAL, "loss")
    need = L.lopt_policy_loss_workspace(64, 4096)
    assert need > 0 and L.lopt_policy_loss_workspace(8, 128) == 0
    large = dict(seqs=64, tokens=4096, ld_logp=4096, ld_old=4096, ld_adv=4096)
    _refused(L, _policy(L, ws=None, **large), EINVAL, "workspace")
    _refused(L, _policy(L, ws_bytes=need - 1, **large), EINVAL, "workspace")
    _refused(L, _policy_back(L, dloss=None), EINVAL, "dloss")
    _refused(L, _policy_back(L, dlogp=P + 2), EINVAL, "dlogp")
    _refused(L, _policy_back(L, dkl=P), EINVAL, "kl")
    _refused(L, _policy_back(L, dent=P), EINVAL, "entropy")
    assert _policy_back(L, dlogp=None) == 0
    assert _policy_back(L, seqs=0, logp=None, old=None, adv=None) == 0


def _preference(L, loss=P, stats=P, rewards=P, coef=P, ws=P, ws_bytes=1 << 30, **over):
    v = dict(logp=P, ld_logp=8, ref=P, ld_ref=8, mask=None, ld_mask=8, pairs=4, tokens=8, beta=0.1)
    v.update(over)
    return L.lopt_preference_loss(C.byref(Preference(**v)), loss, stats, rewards, coef, ws, ws_bytes, None)


def test_preference_loss_refusals(L):
    _refused(L, L.lopt_preference_loss(None, P, P, P, P, P, 8, None), EINVAL, "terms_host")
    for pairs in (-1, 1 << 30):
        _refused(L, _preference(L, pairs=pairs), ESHAPE, "pairs")
    _refused(L, _preference(L, tokens=0), ESHAPE, "tokens")
    _refused(L, _preference(L, logp=None), EINVAL, "logp")
    _refused(L, _preference(L, logp=P + 2), EINVAL, "logp")
    _refused(L, _preference(L, ref=P + 2), EINVAL, "ref")
    _refused(L, _preference(L, ref_type=5), EINVAL, "ref_type")
    for name in ("ld_logp", "ld_ref"):
        _refused(L, _preference(L, **{name: -1}), ESHAPE, name)
    _refused(L, _preference(L, mask=P, ld_mask=-1), ESHAPE, "ld_mask")
    _refused(L, _preference(L, kind=3), EINVAL, "kind")
    for beta in (0.0, -1.0, math.nan, math.inf):
        _refused(L, _preference(L, beta=beta), EINVAL, "beta")
    for smooth in (-0.1, 1.1, math.nan):
        _refused(L, _preference(L, smooth=smooth), EINVAL, "label_smoothing")
    _refused(L, _preference(L, smooth=0.1, kind=1), EINVAL, "label_smoothing")
    _refused(L, _preference(L, margin=math.nan), EINVAL, "margin")
    _refused(L, _preference(L, margin=1.0, kind=2), EINVAL, "margin")
    for name in ("loss", "stats", "rewards", "coef"):
        _refused(L, _preference(L, **{name: None}), EINVAL, name)
        _refused(L, _preference(L, **{name: P + 2}), EINVAL, name)
    need = L.lopt_preference_loss_workspace(64, 4096)
    assert need > 0 and L.lopt_preference_loss_workspace(0, 8) == 0 and L.lopt_preference_loss_workspace(4, 8) == 0
    large = dict(pairs=64, tokens=4096, ld_logp=4096, ld_ref=4096)
    _refused(L, _preference(L, ws=None, **large), EINVAL, "workspace")
    _refused(L, _preference(L, ws_bytes=need - 1, **large), EINVAL, "workspace")


def test_preference_loss_backward_refusals(L):
    def back(coef=P, mask=P, ld_mask=8, dloss=P, dlogp=P, pairs=4, tokens=8):
        return L.lopt_preference_loss_backward(coef, mask, ld_mask, dloss, dlogp, pairs, tokens, None)
    _refused(L, back(pairs=-1), ESHAPE, "pairs")
    _refused(L, back(tokens=0), ESHAPE, "tokens")
    _refused(L, back(ld_mask=-1), ESHAPE, "ld_mask")
    for name in ("coef", "dloss", "dlogp"):
        _refused(L, back(**{name: None}), EINVAL, name)
    assert back(pairs=0, coef=None, dlogp=None) == 0


def test_functions_refuse_cpu_tensors():
    import torch
    from paper_2506_10315_amd import ops
    x, m = torch.randn(4, 6), torch.ones(4, 6, dtype=torch.bool)
    for call in (lambda: ops.dropout(x, 0.1, 0), lambda: ops.dropout_add_layer_norm(x, x), lambda: ops.token_kl(x, x), lambda: ops.policy_loss(x, x, x, m),
                 lambda: ops.preference_loss(x, x, m)):
        with pytest.raises(ValueError):
            call()
