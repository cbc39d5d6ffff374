"""The operators of a training loop around the optimizer step, on torch tensors: layer norm, token log probabilities with
entropy and top alternatives, dropout (alone, and with residual and layer norm), the KL divergence to a reference's logits, the clipped policy loss and the
preference loss, their gradients, and clipping by the global gradient norm.

Nothing numerical happens here: every function checks its tensors, allocates outputs and workspace, and hands pointers to the
call of the same name in include/lopt.h (formulas, masks and special values are described there) on the current stream.
Tensors are CUDA tensors of float32, bfloat16 or float16; `layer_norm`, `dropout`, `dropout_add_layer_norm`,
`token_logprobs`, `token_kl`, `policy_loss` and `preference_loss` take part in autograd, the `*_forward` and `*_backward` functions are the passes by themselves."""
from __future__ import annotations

import operator
import struct
from array import array
from typing import Iterable, List, NamedTuple, Optional, Sequence, Tuple, Union

import torch

from .binding import _check, lib

__all__ = ["clip_grads", "clip_grad_norm_", "grad_norm", "layer_norm", "layer_norm_forward", "layer_norm_backward",
           "dropout", "dropout_forward", "dropout_add_layer_norm", "dropout_add_layer_norm_forward", "dropout_add_layer_norm_backward",
           "TokenLogprobs", "token_logprobs", "token_logprobs_forward", "token_logprobs_backward", "TOP_MAX",
           "token_kl", "token_kl_forward", "token_kl_backward",
           "PolicyLoss", "policy_loss", "policy_loss_forward", "policy_loss_backward",
           "PreferenceLoss", "preference_loss", "preference_loss_forward", "preference_loss_backward"]

TOP_MAX = 32          # LOPT_TOP_MAX
_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}   # lopt_type


def _type(name: str, t: torch.Tensor) -> int:
    if not t.is_cuda:
        raise ValueError(f"{name} is not a CUDA tensor")
    k = _TYPES.get(t.dtype)
    if k is None:
        raise ValueError(f"{name} is of {t.dtype}; float32, bfloat16 or float16 is needed")
    return k


def _expect(name: str, t: torch.Tensor, like: torch.Tensor, dtype, shape) -> torch.Tensor:
    """`t` on `like`'s device with this type and shape, contiguous (copied where it is not)."""
    if t.get_device() != like.get_device():
        raise ValueError(f"{name} is on {t.device}, not on {like.device}")
    if t.dtype is not dtype or t.shape != shape:
        raise ValueError(f"{name} is {tuple(t.shape)} of {t.dtype}; {tuple(shape)} of {dtype} is needed")
    return t if t.is_contiguous() else t.contiguous()


def _matrix(name: str, t: torch.Tensor) -> Tuple[torch.Tensor, int, int, int]:
    """(tensor, rows, columns, elements from row to row) of `t` seen as rows of its last dimension. A 2-D tensor keeps its row
    stride; any other layout whose rows are not evenly spaced runs of adjacent elements is copied."""
    shape = t.shape
    if not shape:
        raise ValueError(f"{name} has no dimension")
    cols = shape[-1]
    if cols == 0:
        raise ValueError(f"{name} has rows of no elements")
    if not t.is_contiguous():
        if len(shape) == 2 and (t.stride(1) == 1 or cols == 1):
            return t, shape[0], cols, t.stride(0)
        t = t.contiguous()
    return t, t.numel() // cols, cols, cols


# the current stream's handle and device without the objects around them, which cost as much as the launch of a small kernel
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _run(fn, index: int, *args):
    """The call on GPU `index`, on its current stream."""
    if _current_device() == index:
        status = fn(*args, _raw_stream(index))
    else:
        with torch.cuda.device(index):
            status = fn(*args, _raw_stream(index))
    if status:
        _check(status)


def _floats(rows: int, shape: torch.Size, device) -> torch.Tensor:
    """float32 of `shape`, which has `rows` elements."""
    return torch.empty(rows if len(shape) == 1 else shape, dtype=torch.float32, device=device)


def _rows_of(rows: int, shape: torch.Size, n: int, dtype, device) -> torch.Tensor:
    """`n` elements for each of the `rows` that `shape` has."""
    if len(shape) == 1:
        return torch.empty(rows, n, dtype=dtype, device=device)
    return torch.empty(shape + (n,), dtype=dtype, device=device)


def _new(t: torch.Tensor) -> torch.Tensor:
    """A contiguous tensor of `t`'s shape and type."""
    return torch.empty_like(t) if t.is_contiguous() else torch.empty(t.shape, dtype=t.dtype, device=t.device)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _workspace(nbytes: int, device) -> Optional[torch.Tensor]:
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None


# ---------------------------------------------------------------------------------------------- gradient norm and clipping

def _dense(t: torch.Tensor) -> bool:
    """Whether the elements fill one run of memory, in any order of the dimensions."""
    if t.is_contiguous():
        return True
    run = 1
    for stride, size in sorted((st, sz) for st, sz in zip(t.stride(), t.shape) if sz != 1):
        if stride != run:
            return False
        run *= size
    return True


def _clip_list(name: str, ts: Sequence[torch.Tensor], device: torch.device):
    """(pointers, lopt_types, whether all are contiguous) of a list of tensors on `device`."""
    if set(map(torch.Tensor.get_device, ts)) != {device.index} or device.type != "cuda":
        raise ValueError(f"{name}: all tensors have to be on one CUDA device")
    dtypes = list(map(_DTYPE, ts))
    kinds = set(dtypes)
    for k in kinds:
        if k not in _TYPES:
            raise ValueError(f"{name}: a tensor of {k}; float32, bfloat16 or float16 is needed")
    contiguous = all(map(torch.Tensor.is_contiguous, ts))
    if not contiguous:
        for t in ts:
            if t.layout != torch.strided or not _dense(t):
                raise ValueError(f"{name}: a tensor that does not fill one run of memory")
    types = array("I", [_TYPES[dtypes[0]]]) * len(ts) if len(kinds) == 1 else array("I", [_TYPES[k] for k in dtypes])
    return array("Q", map(torch.Tensor.data_ptr, ts)), types, contiguous


_DTYPE, _SHAPE = operator.attrgetter("dtype"), operator.attrgetter("shape")


def _clip(grads: Sequence[torch.Tensor], out: Optional[Sequence[torch.Tensor]], max_norm: float) -> torch.Tensor:
    n = len(grads)
    if n == 0:
        raise ValueError("no gradients")
    device = grads[0].device
    gp, gt, contiguous = _clip_list("grads", grads, device)
    op = ot = None
    if out is grads:
        op, ot = gp, gt
    elif out is not None:
        if len(out) != n:
            raise ValueError(f"{len(out)} outputs for {n} gradients")
        op, ot, out_contiguous = _clip_list("out", out, device)
        if list(map(_SHAPE, grads)) != list(map(_SHAPE, out)):
            raise ValueError("an output's shape is not its gradient's")
        if not (contiguous and out_contiguous):
            for g, o in zip(grads, out):
                if g.stride() != o.stride() and not (g.is_contiguous() and o.is_contiguous()):
                    raise ValueError("an output's strides are not its gradient's")
    counts = array("q", map(torch.Tensor.numel, grads))
    at = [a and a.buffer_info()[0] for a in (counts, gp, gt, op, ot)]
    L = lib()
    norm = torch.empty((), dtype=torch.float32, device=device)
    nbytes = L.lopt_clip_workspace(n, at[0])
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    _run(L.lopt_clip_grads, device.index, n, *at, max_norm, norm.data_ptr(), ws.data_ptr(), nbytes)
    if out is not None:   # autograd has to see that they were written
        torch.autograd.graph.increment_version(out)
    return norm


def grad_norm(grads: Sequence[torch.Tensor]) -> torch.Tensor:
    """The Euclidean norm of all elements of all tensors: a float32 tensor without dimensions, on their device."""
    return _clip(list(grads), None, 0.0)


def clip_grads(grads: Sequence[torch.Tensor], max_norm: float,
               out: Optional[Sequence[torch.Tensor]] = None) -> Tuple[List[torch.Tensor], torch.Tensor]:
    """(clipped gradients, norm before clipping): every gradient times min(1, max_norm / (norm + 1e-6)). `out` receives
    them, in float32 or any type this module takes; by default new float32 tensors, which is what LearnedOptimizer.step takes.
    The gradients stay as they are."""
    grads = list(grads)
    out = [torch.empty_like(g, dtype=torch.float32) for g in grads] if out is None else list(out)
    return out, _clip(grads, out, max_norm)


def clip_grad_norm_(parameters: Union[torch.Tensor, Iterable[torch.Tensor]], max_norm: float) -> torch.Tensor:
    """Clips the `.grad` of the parameters in place and returns the norm before. Parameters without a gradient are
    skipped, and if none has one the norm is 0; a gradient that is listed twice is refused."""
    parameters = [parameters] if isinstance(parameters, torch.Tensor) else list(parameters)
    grads = [p.grad for p in parameters if p.grad is not None]
    if parameters and not grads:
        return torch.zeros((), dtype=torch.float32, device=parameters[0].device)
    return _clip(grads, grads, max_norm)


# ---------------------------------------------------------------------------------------------- layer norm

def layer_norm_forward(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
                       eps: float = 1e-5) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(y, mean, rstd) over the last dimension of `x`; y has x's type, mean and rstd are float32 of x's other dimensions."""
    kind = _type("x", x)
    x2, rows, cols, ld = _matrix("x", x)
    wtype = 0
    if weight is not None:
        wtype = _type("weight", weight)
        weight = _expect("weight", weight, x, weight.dtype, (cols,))
    if bias is not None:
        if weight is None:
            wtype = _type("bias", bias)
        bias = _expect("bias", bias, x, bias.dtype if weight is None else weight.dtype, (cols,))
    y = _new(x)
    mean = _floats(rows, x.shape[:-1], x.device)
    rstd = torch.empty_like(mean)
    _run(lib().lopt_layer_norm, x.get_device(), x2.data_ptr(), ld, _ptr(weight), _ptr(bias), y.data_ptr(), cols, mean.data_ptr(), rstd.data_ptr(),
         rows, cols, eps, kind, wtype)
    return y, mean, rstd


def layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, weight: Optional[torch.Tensor], mean: torch.Tensor, rstd: torch.Tensor,
                        need: Tuple[bool, bool, bool] = (True, True, True), bias_type: Optional[torch.dtype] = None):
    """(dx, dweight, dbias) of layer_norm_forward; `need` says which are wanted, the others are None. dweight and dbias have the
    weight's type (without a weight bias_type, by default float32)."""
    kind = _type("x", x)
    x2, rows, cols, ld = _matrix("x", x)
    if dy.shape != x.shape or dy.dtype is not x.dtype or dy.get_device() != x.get_device():
        raise ValueError(f"dy is {tuple(dy.shape)} of {dy.dtype} on {dy.device}; x is {tuple(x.shape)} of {x.dtype} on {x.device}")
    dy2, _, _, ld_dy = _matrix("dy", dy)
    wtype = weight.dtype if weight is not None else bias_type or torch.float32
    if wtype not in _TYPES:
        raise ValueError(f"weights of {wtype}; float32, bfloat16 or float16 is needed")
    if weight is not None:
        weight = _expect("weight", weight, x, wtype, (cols,))
    shape = x.shape[:-1]
    mean = _expect("mean", mean, x, torch.float32, shape)
    rstd = _expect("rstd", rstd, x, torch.float32, shape)
    dx = _new(x) if need[0] else None
    dw = db = None
    if need[1]:
        dw = torch.empty_like(weight) if weight is not None else torch.empty(cols, dtype=wtype, device=x.device)
    if need[2]:
        db = torch.empty_like(dw) if dw is not None else torch.empty(cols, dtype=wtype, device=x.device)
    L = lib()
    nbytes = L.lopt_layer_norm_workspace(rows, cols) if need[1] or need[2] else 0
    ws = _workspace(nbytes, x.device)
    _run(L.lopt_layer_norm_backward, x.get_device(), dy2.data_ptr(), ld_dy, x2.data_ptr(), ld, _ptr(weight), mean.data_ptr(), rstd.data_ptr(), _ptr(dx), cols,
         _ptr(dw), _ptr(db), rows, cols, kind, _TYPES[wtype], _ptr(ws), nbytes)
    return dx, dw, db


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        y, mean, rstd = layer_norm_forward(x, weight, bias, eps)
        ctx.save_for_backward(x, weight, mean, rstd)
        ctx.bias_type = None if bias is None else bias.dtype
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, weight, mean, rstd = ctx.saved_tensors
        dx, dw, db = layer_norm_backward(dy, x, weight, mean, rstd, ctx.needs_input_grad[:3], ctx.bias_type)
        return dx, dw, db, None


def layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, eps: float = 1e-5) -> torch.Tensor:
    """Layer norm over the last dimension, with gradients for x, weight and bias."""
    return _LayerNorm.apply(x, weight, bias, eps)


# ---------------------------------------------------------------------------------------------- dropout

Seed = Union[int, torch.Tensor]


def _seed(seed: Optional[Seed], offset: int, like: torch.Tensor, p: float) -> Tuple[int, Optional[torch.Tensor], int]:
    """(seed, tensor that holds it or None, offset) as the boundary takes them. Where p decides by itself there need be no seed."""
    if seed is None:
        if 0.0 < p < 1.0:
            raise ValueError(f"p={p} without a seed, which would drop the same elements in every step")
        seed = 0
    if not 0 <= offset < 1 << 64:
        raise ValueError(f"offset={offset} outside [0, 2^64)")
    if isinstance(seed, torch.Tensor):
        if seed.dtype is not torch.int64 or seed.numel() != 1 or seed.get_device() != like.get_device():
            raise ValueError(f"seed is {tuple(seed.shape)} of {seed.dtype} on {seed.device}; one int64 on {like.device} is needed")
        return 0, seed, offset
    if not 0 <= seed < 1 << 64:
        raise ValueError(f"seed={seed} outside [0, 2^64)")
    return seed, None, offset


def dropout_forward(x: torch.Tensor, p: float, seed: Seed, offset: int = 0) -> torch.Tensor:
    """x / (1 - p) where an element stays, else 0, in x's type. Which elements stay is a function of seed, offset and the element's row and column
    (rows of the last dimension) alone; nothing is stored, and the backward pass is the same call on the gradient. A seed that is one int64 on
    the device is read when the kernel runs."""
    kind = _type("x", x)
    x2, rows, cols, ld = _matrix("x", x)
    number, tensor, offset = _seed(seed, offset, x, p)
    y = _new(x)
    _run(lib().lopt_dropout, x.get_device(), x2.data_ptr(), ld, y.data_ptr(), cols, rows, cols, kind, p, number, _ptr(tensor), offset)
    return y


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, p, seed, offset):
        ctx.args = p, None if isinstance(seed, torch.Tensor) else seed, offset
        if isinstance(seed, torch.Tensor):
            ctx.save_for_backward(seed)
        return dropout_forward(x, p, seed, offset)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        p, seed, offset = ctx.args
        return dropout_forward(dy, p, ctx.saved_tensors[0] if seed is None else seed, offset), None, None, None


def dropout(x: torch.Tensor, p: float, seed: Seed, offset: int = 0) -> torch.Tensor:
    """dropout_forward with the gradient for x. A program gives every step another seed and every call within a step another
    offset."""
    return _Dropout.apply(x, p, seed, offset)


def dropout_add_layer_norm_forward(x: torch.Tensor, residual: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
                                   p: float = 0.0, seed: Optional[Seed] = None, offset: int = 0,
                                   eps: float = 1e-5) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor, torch.Tensor]:
    """(y, h, mean, rstd) with h = residual + dropout(x) and y = layer_norm(h): y has x's type, h the residual's, which is x's or
    float32. The norm is of h as it is stored. `seed`: as in dropout_forward, needed where 0 < p < 1."""
    kind = _type("x", x)
    x2, rows, cols, ld = _matrix("x", x)
    if residual.shape != x.shape or residual.get_device() != x.get_device():
        raise ValueError(f"residual is {tuple(residual.shape)} on {residual.device}; x is {tuple(x.shape)} on {x.device}")
    rkind = _type("residual", residual)
    r2, _, _, ld_res = _matrix("residual", residual)
    wtype = 0
    if weight is not None:
        wtype = _type("weight", weight)
        weight = _expect("weight", weight, x, weight.dtype, (cols,))
    if bias is not None:
        if weight is None:
            wtype = _type("bias", bias)
        bias = _expect("bias", bias, x, bias.dtype if weight is None else weight.dtype, (cols,))
    number, tensor, offset = _seed(seed, offset, x, p)
    y, h = _new(x), _new(residual)
    mean = _floats(rows, x.shape[:-1], x.device)
    rstd = torch.empty_like(mean)
    _run(lib().lopt_dropout_add_layer_norm, x.get_device(), x2.data_ptr(), ld, r2.data_ptr(), ld_res, _ptr(weight), _ptr(bias), y.data_ptr(), cols,
         h.data_ptr(), cols, mean.data_ptr(), rstd.data_ptr(), rows, cols, eps, kind, rkind, wtype, p, number, _ptr(tensor), offset)
    return y, h, mean, rstd


def dropout_add_layer_norm_backward(dy: torch.Tensor, dh: Optional[torch.Tensor], h: torch.Tensor, weight: Optional[torch.Tensor], mean: torch.Tensor,
                                    rstd: torch.Tensor, p: float = 0.0, seed: Optional[Seed] = None, offset: int = 0,
                                    need: Tuple[bool, bool, bool, bool] = (True, True, True, True), bias_type: Optional[torch.dtype] = None):
    """(dx, dresidual, dweight, dbias) of dropout_add_layer_norm_forward from the gradients of y and of h (None: 0); `need` says which are wanted,
    the others are None. dx has dy's type, dresidual h's. Without dropout dx and dresidual of one type are the same tensor."""
    kind, rkind = _type("dy", dy), _type("h", h)
    dy2, rows, cols, ld_dy = _matrix("dy", dy)
    for name, t in (("h", h), ("dh", dh)):
        if t is not None and (t.shape != dy.shape or t.dtype is not h.dtype or t.get_device() != dy.get_device()):
            raise ValueError(f"{name} is {tuple(t.shape)} of {t.dtype} on {t.device}; {tuple(dy.shape)} of {h.dtype} on {dy.device} is needed")
    h2, _, _, ld_h = _matrix("h", h)
    dh2, ld_dh = None, 0
    if dh is not None:
        dh2, _, _, ld_dh = _matrix("dh", dh)
    wtype = weight.dtype if weight is not None else bias_type or torch.float32
    if wtype not in _TYPES:
        raise ValueError(f"weights of {wtype}; float32, bfloat16 or float16 is needed")
    if weight is not None:
        weight = _expect("weight", weight, dy, wtype, (cols,))
    shape = dy.shape[:-1]
    mean = _expect("mean", mean, dy, torch.float32, shape)
    rstd = _expect("rstd", rstd, dy, torch.float32, shape)
    number, tensor, offset = _seed(seed, offset, dy, p)
    same = p == 0.0 and kind == rkind
    dres = _new(h) if need[1] or (need[0] and same) else None
    dx = _new(dy) if need[0] and not same else None
    dw = db = None
    if need[2]:
        dw = torch.empty_like(weight) if weight is not None else torch.empty(cols, dtype=wtype, device=dy.device)
    if need[3]:
        db = torch.empty_like(dw) if dw is not None else torch.empty(cols, dtype=wtype, device=dy.device)
    L = lib()
    nbytes = L.lopt_dropout_add_layer_norm_workspace(rows, cols) if need[2] or need[3] else 0
    ws = _workspace(nbytes, dy.device)
    _run(L.lopt_dropout_add_layer_norm_backward, dy.get_device(), dy2.data_ptr(), ld_dy, _ptr(dh2), ld_dh, h2.data_ptr(), ld_h, _ptr(weight), mean.data_ptr(),
         rstd.data_ptr(), _ptr(dx), cols, _ptr(dres), cols, _ptr(dw), _ptr(db), rows, cols, kind, rkind, _TYPES[wtype], p, number, _ptr(tensor), offset, _ptr(ws),
         nbytes)
    return (dres if same and need[0] else dx), (dres if need[1] else None), dw, db


class _DropoutAddLayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, weight, bias, p, seed, offset, eps):
        y, h, mean, rstd = dropout_add_layer_norm_forward(x, residual, weight, bias, p, seed, offset, eps)
        on_device = isinstance(seed, torch.Tensor)
        ctx.save_for_backward(h, weight, mean, rstd, seed if on_device else None)
        ctx.args = p, None if on_device else seed, offset
        ctx.like = x.dtype
        ctx.bias_type = None if bias is None else bias.dtype
        ctx.set_materialize_grads(False)
        return y, h

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy, dh):
        if dy is None and dh is None:
            return (None,) * 8
        h, weight, mean, rstd, tensor = ctx.saved_tensors
        p, seed, offset = ctx.args
        if dy is None:   # the norm's output was not used
            dy = torch.zeros(h.shape, dtype=ctx.like, device=h.device)
        grads = dropout_add_layer_norm_backward(dy, dh, h, weight, mean, rstd, p, tensor if seed is None else seed, offset, ctx.needs_input_grad[:4],
                                                ctx.bias_type)
        return (*grads, None, None, None, None)


def dropout_add_layer_norm(x: torch.Tensor, residual: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
                           p: float = 0.0, seed: Optional[Seed] = None, offset: int = 0, eps: float = 1e-5) -> Tuple[torch.Tensor, torch.Tensor]:
    """(y, h): the block's output x is dropped, joins the residual stream, h, and the stream is normalised for the next block, y. With gradients
    for x, residual, weight and bias."""
    return _DropoutAddLayerNorm.apply(x, residual, weight, bias, p, seed, offset, eps)


# ---------------------------------------------------------------------------------------------- token log probabilities

class TokenLogprobs(NamedTuple):
    logp: Optional[torch.Tensor]        # of the given tokens; 0 where ignored
    entropy: Optional[torch.Tensor]
    top_logp: Optional[torch.Tensor]    # [..., top], best first
    top_index: Optional[torch.Tensor]   # int64
    stats: torch.Tensor                 # [..., 2]: largest logit and ln sum e^z, for the backward pass


def token_logprobs_forward(logits: torch.Tensor, targets: Optional[torch.Tensor], scale: float = 1.0, top: int = 0, ignore_index: int = -100,
                           entropy: bool = True) -> TokenLogprobs:
    """Log probabilities of `targets` (int64, logits.shape[:-1]; None: not wanted) under softmax(scale * logits), the entropy
    and the `top` best alternatives of every row."""
    kind = _type("logits", logits)
    x, rows, vocab, ld = _matrix("logits", logits)
    shape = logits.shape[:-1]
    if targets is not None:
        targets = _expect("targets", targets, logits, torch.int64, shape)
    if not 0 <= top <= min(vocab, TOP_MAX):
        raise ValueError(f"top={top} outside [0, {min(vocab, TOP_MAX)}]")
    dev = logits.device
    logp = _floats(rows, shape, dev) if targets is not None else None
    ent = None
    if entropy:
        ent = torch.empty_like(logp) if logp is not None else _floats(rows, shape, dev)
    stats = _rows_of(rows, shape, 2, torch.float32, dev)
    top_logp = top_index = None
    if top:
        top_logp = _rows_of(rows, shape, top, torch.float32, dev)
        top_index = torch.empty_like(top_logp, dtype=torch.int64)
    L = lib()
    nbytes = L.lopt_token_logprobs_workspace(rows, vocab, top)
    ws = _workspace(nbytes, dev)
    _run(L.lopt_token_logprobs, dev.index, x.data_ptr(), ld, _ptr(targets), rows, vocab, kind, scale, ignore_index, top, _ptr(logp), _ptr(ent), stats.data_ptr(),
         _ptr(top_logp), _ptr(top_index), _ptr(ws), nbytes)
    return TokenLogprobs(logp, ent, top_logp, top_index, stats)


def token_logprobs_backward(logits: torch.Tensor, targets: Optional[torch.Tensor], stats: torch.Tensor, entropy: Optional[torch.Tensor],
                            dlogp: Optional[torch.Tensor], dentropy: Optional[torch.Tensor] = None, scale: float = 1.0,
                            ignore_index: int = -100) -> torch.Tensor:
    """The logits' gradient from those of logp and entropy (either may be None), in the logits' type. `stats` and `entropy` are
    the forward pass's; `entropy` is needed with `dentropy` only, `targets` with `dlogp` only."""
    kind = _type("logits", logits)
    x, rows, vocab, ld = _matrix("logits", logits)
    shape = logits.shape[:-1]
    stats = _expect("stats", stats, logits, torch.float32, shape + (2,))
    if dlogp is not None:
        dlogp = _expect("dlogp", dlogp, logits, torch.float32, shape)
        if targets is None:
            raise ValueError("dlogp without targets")
        targets = _expect("targets", targets, logits, torch.int64, shape)
    if dentropy is not None:
        dentropy = _expect("dentropy", dentropy, logits, torch.float32, shape)
        if entropy is None:
            raise ValueError("dentropy without entropy")
        entropy = _expect("entropy", entropy, logits, torch.float32, shape)
    dx = _new(logits)
    _run(lib().lopt_token_logprobs_backward, logits.get_device(), x.data_ptr(), ld, _ptr(targets), stats.data_ptr(), _ptr(entropy), _ptr(dlogp), _ptr(dentropy),
         dx.data_ptr(), vocab, rows, vocab, kind, scale, ignore_index)
    return dx


class _TokenLogprobs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, targets, scale, top, ignore_index):
        r = token_logprobs_forward(logits, targets, scale, top, ignore_index)
        ctx.save_for_backward(logits, targets, r.stats, r.entropy)
        ctx.scale, ctx.ignore_index = scale, ignore_index
        ctx.set_materialize_grads(False)
        ctx.mark_non_differentiable(*[t for t in (r.top_logp, r.top_index, r.stats) if t is not None])
        return r.logp, r.entropy, r.top_logp, r.top_index, r.stats

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dlogp, dentropy, *_):
        if dlogp is None and dentropy is None:
            return None, None, None, None, None
        logits, targets, stats, entropy = ctx.saved_tensors
        dx = token_logprobs_backward(logits, targets, stats, entropy, dlogp, dentropy, ctx.scale, ctx.ignore_index)
        return dx, None, None, None, None


def token_logprobs(logits: torch.Tensor, targets: Optional[torch.Tensor], scale: float = 1.0, top: int = 0,
                   ignore_index: int = -100) -> TokenLogprobs:
    """token_logprobs_forward with gradients for the logits from logp and entropy. The mean of -logp over the tokens that are
    not ignored is the loss that LearnedOptTorch.step takes."""
    return TokenLogprobs(*_TokenLogprobs.apply(logits, targets, scale, top, ignore_index))


# ---------------------------------------------------------------------------------------------- KL divergence to reference logits

def _mask(mask: Optional[torch.Tensor], like: torch.Tensor, shape) -> Optional[torch.Tensor]:
    return None if mask is None else _expect("mask", mask, like, torch.bool, shape)


def _two_logits(logits: torch.Tensor, ref: torch.Tensor):
    kind = _type("logits", logits)
    if ref.shape != logits.shape or ref.dtype is not logits.dtype or ref.get_device() != logits.get_device():
        raise ValueError(f"ref is {tuple(ref.shape)} of {ref.dtype} on {ref.device}; logits are {tuple(logits.shape)} of {logits.dtype} on {logits.device}")
    x, rows, vocab, ld = _matrix("logits", logits)
    r, _, _, ld_ref = _matrix("ref", ref)
    return kind, x, ld, r, ld_ref, rows, vocab


def token_kl_forward(logits: torch.Tensor, ref: torch.Tensor, scale: float = 1.0, mask: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(kl, stats): the KL divergence of softmax(scale * logits) from softmax(scale * ref) of every row, float32 of logits.shape[:-1], and what the
    backward pass needs of the rows. `mask` (bool, logits.shape[:-1]): rows that count, the others have 0."""
    kind, x, ld, r, ld_ref, rows, vocab = _two_logits(logits, ref)
    shape, dev = logits.shape[:-1], logits.device
    mask = _mask(mask, logits, shape)
    kl = _floats(rows, shape, dev)
    stats = _rows_of(rows, shape, 5, torch.float32, dev)
    L = lib()
    nbytes = L.lopt_token_kl_workspace(rows, vocab)
    ws = _workspace(nbytes, dev)
    _run(L.lopt_token_kl, dev.index, x.data_ptr(), ld, r.data_ptr(), ld_ref, _ptr(mask), rows, vocab, kind, scale, kl.data_ptr(), stats.data_ptr(), _ptr(ws), nbytes)
    return kl, stats


def token_kl_backward(logits: torch.Tensor, ref: torch.Tensor, stats: torch.Tensor, dkl: torch.Tensor, scale: float = 1.0, mask: Optional[torch.Tensor] = None,
                      need: Tuple[bool, bool] = (True, False)) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor]]:
    """(dlogits, dref) from the gradient of kl; `need` says which are wanted, the others are None. `stats` is the forward pass's."""
    kind, x, ld, r, ld_ref, rows, vocab = _two_logits(logits, ref)
    shape = logits.shape[:-1]
    mask = _mask(mask, logits, shape)
    stats = _expect("stats", stats, logits, torch.float32, shape + (5,))
    dkl = _expect("dkl", dkl, logits, torch.float32, shape)
    dx, dr = (_new(t) if wanted else None for t, wanted in zip((logits, ref), need))
    _run(lib().lopt_token_kl_backward, logits.get_device(), x.data_ptr(), ld, r.data_ptr(), ld_ref, _ptr(mask), stats.data_ptr(), dkl.data_ptr(), _ptr(dx), vocab,
         _ptr(dr), vocab, rows, vocab, kind, scale)
    return dx, dr


class _TokenKl(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, ref, scale, mask):
        kl, stats = token_kl_forward(logits, ref, scale, mask)
        ctx.save_for_backward(logits, ref, stats, mask)
        ctx.scale = scale
        return kl

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dkl):
        logits, ref, stats, mask = ctx.saved_tensors
        dx, dr = token_kl_backward(logits, ref, stats, dkl, ctx.scale, mask, ctx.needs_input_grad[:2])
        return dx, dr, None, None


def token_kl(logits: torch.Tensor, ref: torch.Tensor, scale: float = 1.0, mask: Optional[torch.Tensor] = None) -> torch.Tensor:
    """token_kl_forward's kl with gradients for logits and ref: as a policy's distance from its reference, which has no gradient, or, with a teacher's logits
    first and the student's second, as the loss of a distillation."""
    return _TokenKl.apply(logits, ref, scale, mask)


# ---------------------------------------------------------------------------------------------- losses of log probabilities

_POLICY = struct.Struct("=" + "Qq" * 7 + "2q4d6I")          # lopt_policy
_PREFERENCE = struct.Struct("=" + "Qq" * 3 + "2q3d4I")      # lopt_preference
_KINDS = {"sigmoid": 0, "hinge": 1, "squared": 2}           # lopt_preference_kind
_REDUCTIONS = {"tokens": 0, "sequences": 1}


def _token_rows(name: str, t: torch.Tensor, like: torch.Tensor, dev: int, cols: int, dtype: Optional[torch.dtype]) -> Tuple[torch.Tensor, int]:
    """(tensor, elements from row to row) of `t`, which has to be of `like`'s shape, on its device `dev`, and of this type (None: one of the module's)."""
    if t.shape != like.shape or t.get_device() != dev or (t.dtype is not dtype if dtype is not None else t.dtype not in _TYPES):
        raise ValueError(f"{name} is {tuple(t.shape)} of {t.dtype} on {t.device}; {tuple(like.shape)} of {dtype or 'float32, bfloat16 or float16'} "
                         f"on {like.device} is needed")
    if t.is_contiguous():
        return t, cols
    t, _, _, ld = _matrix(name, t)
    return t, ld


class PolicyLoss(NamedTuple):
    loss: torch.Tensor                  # one float32
    stats: torch.Tensor                 # [8]: means of surrogate, kl, entropy, clipped, ratio, drift; tokens and sequences that count
    counts: Optional[torch.Tensor]      # tokens of each sequence that count, with reduction="sequences"


def _policy_terms(logp, old_logp, advantages, mask, clip, ref_logp, kl, kl_coef, entropy, entropy_coef, reduction):
    """(lopt_policy as bytes, the tensors that it points to, sequences, tokens)"""
    if _type("logp", logp) != 0:
        raise ValueError(f"logp is of {logp.dtype}; float32 is needed")
    x, seqs, tokens, ld = _matrix("logp", logp)
    dev = logp.get_device()
    old, ld_old = _token_rows("old_logp", old_logp, logp, dev, tokens, None)
    each = advantages.shape == logp.shape
    if each:
        adv, ld_adv = _token_rows("advantages", advantages, logp, dev, tokens, None)
    else:   # one a sequence
        if advantages.dtype not in _TYPES:
            raise ValueError(f"advantages are of {advantages.dtype}; float32, bfloat16 or float16 is needed")
        adv, ld_adv = _expect("advantages", advantages, logp, advantages.dtype, logp.shape[:-1]), 1
    if reduction not in _REDUCTIONS:
        raise ValueError(f"reduction={reduction!r}; 'tokens' or 'sequences' is needed")
    ref = k = ent = m = None
    ref_at = ref_type = k_at = ent_at = m_at = ld_ref = ld_k = ld_ent = ld_m = 0
    if ref_logp is not None:
        if kl is not None:
            raise ValueError("ref_logp and kl are both given")
        ref, ld_ref = _token_rows("ref_logp", ref_logp, logp, dev, tokens, None)
        ref_at, ref_type = ref.data_ptr(), _TYPES[ref.dtype]
    elif kl is not None:
        k, ld_k = _token_rows("kl", kl, logp, dev, tokens, torch.float32)
        k_at = k.data_ptr()
    elif kl_coef:
        raise ValueError("kl_coef without ref_logp or kl")
    if entropy is not None:
        ent, ld_ent = _token_rows("entropy", entropy, logp, dev, tokens, torch.float32)
        ent_at = ent.data_ptr()
    elif entropy_coef:
        raise ValueError("entropy_coef without entropy")
    if mask is not None:
        m, ld_m = _token_rows("mask", mask, logp, dev, tokens, torch.bool)
        m_at = m.data_ptr()
    low, high = clip
    terms = _POLICY.pack(x.data_ptr(), ld, old.data_ptr(), ld_old, adv.data_ptr(), ld_adv, ref_at, ld_ref, k_at, ld_k, ent_at, ld_ent, m_at, ld_m, seqs, tokens,
                         low, high, kl_coef, entropy_coef, _TYPES[old.dtype], _TYPES[adv.dtype], ref_type, not each,
                         _REDUCTIONS[reduction], 0)
    return terms, (x, old, adv, ref, k, ent, m), seqs, tokens


def policy_loss_forward(logp: torch.Tensor, old_logp: torch.Tensor, advantages: torch.Tensor, mask: Optional[torch.Tensor] = None,
                        clip: Tuple[float, float] = (0.2, 0.2), ref_logp: Optional[torch.Tensor] = None, kl: Optional[torch.Tensor] = None,
                        kl_coef: float = 0.0, entropy: Optional[torch.Tensor] = None, entropy_coef: float = 0.0, reduction: str = "tokens") -> PolicyLoss:
    """Clipped policy loss of tokens' log probabilities `logp` (float32 [..., tokens]) against those they were drawn with, with a KL term, of which `ref_logp`
    gives an estimate and `kl` (of token_kl) the value, and an entropy bonus. `advantages`: one a token, or one a sequence (logp.shape[:-1]). `mask`
    (bool): tokens that count. `reduction`: mean over the tokens, or over the sequences of the mean over each. Formulas: lopt_policy_loss."""
    terms, alive, seqs, tokens = _policy_terms(logp, old_logp, advantages, mask, clip, ref_logp, kl, kl_coef, entropy, entropy_coef, reduction)
    dev = logp.device
    loss = torch.empty((), dtype=torch.float32, device=dev)
    stats = torch.empty(8, dtype=torch.float32, device=dev)
    counts = torch.empty(seqs, dtype=torch.float32, device=dev) if reduction == "sequences" else None
    L = lib()
    nbytes = L.lopt_policy_loss_workspace(seqs, tokens)
    ws = _workspace(nbytes, dev)
    _run(L.lopt_policy_loss, dev.index, terms, loss.data_ptr(), stats.data_ptr(), _ptr(counts), _ptr(ws), nbytes)
    return PolicyLoss(loss, stats, counts)


def policy_loss_backward(dloss: torch.Tensor, forward: PolicyLoss, logp: torch.Tensor, old_logp: torch.Tensor, advantages: torch.Tensor,
                         mask: Optional[torch.Tensor] = None, clip: Tuple[float, float] = (0.2, 0.2), ref_logp: Optional[torch.Tensor] = None,
                         kl: Optional[torch.Tensor] = None, kl_coef: float = 0.0, entropy: Optional[torch.Tensor] = None, entropy_coef: float = 0.0,
                         reduction: str = "tokens", need: Tuple[bool, bool, bool] = (True, True, True)):
    """(dlogp, dkl, dentropy) from the gradient of the loss and what policy_loss_forward of the same arguments gave; `need` says which are wanted, the
    others are None, as are those of tensors that are not given."""
    terms, alive, seqs, tokens = _policy_terms(logp, old_logp, advantages, mask, clip, ref_logp, kl, kl_coef, entropy, entropy_coef, reduction)
    dloss = _expect("dloss", dloss, logp, torch.float32, ())
    stats = _expect("stats", forward.stats, logp, torch.float32, (8,))
    counts = _expect("counts", forward.counts, logp, torch.float32, (seqs,)) if reduction == "sequences" else None
    dlogp = _new(logp) if need[0] else None
    dkl = _new(kl) if need[1] and kl is not None else None
    dentropy = _new(entropy) if need[2] and entropy is not None else None
    _run(lib().lopt_policy_loss_backward, logp.get_device(), terms, stats.data_ptr(), _ptr(counts), dloss.data_ptr(), _ptr(dlogp), _ptr(dkl), _ptr(dentropy))
    return dlogp, dkl, dentropy


class _PolicyLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logp, kl, entropy, old_logp, advantages, mask, ref_logp, args):
        r = policy_loss_forward(logp, old_logp, advantages, mask, ref_logp=ref_logp, kl=kl, entropy=entropy, **args)
        ctx.save_for_backward(logp, kl, entropy, old_logp, advantages, mask, ref_logp, r.stats, r.counts)
        ctx.args = args
        ctx.mark_non_differentiable(*[t for t in (r.stats, r.counts) if t is not None])
        return r.loss, r.stats, r.counts

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dloss, *_):
        logp, kl, entropy, old_logp, advantages, mask, ref_logp, stats, counts = ctx.saved_tensors
        grads = policy_loss_backward(dloss, PolicyLoss(None, stats, counts), logp, old_logp, advantages, mask, ref_logp=ref_logp, kl=kl, entropy=entropy,
                                     need=ctx.needs_input_grad[:3], **ctx.args)
        return (*grads, None, None, None, None, None)


def policy_loss(logp: torch.Tensor, old_logp: torch.Tensor, advantages: torch.Tensor, mask: Optional[torch.Tensor] = None,
                clip: Tuple[float, float] = (0.2, 0.2), ref_logp: Optional[torch.Tensor] = None, kl: Optional[torch.Tensor] = None, kl_coef: float = 0.0,
                entropy: Optional[torch.Tensor] = None, entropy_coef: float = 0.0, reduction: str = "tokens") -> PolicyLoss:
    """policy_loss_forward with gradients of the loss for logp, kl and entropy. The others are constants: one that asks for a gradient is refused."""
    for name, t in (("old_logp", old_logp), ("advantages", advantages), ("ref_logp", ref_logp)):
        if t is not None and t.requires_grad and torch.is_grad_enabled():
            raise ValueError(f"{name} asks for a gradient, which this loss does not give; detach it")
    args = {"clip": clip, "kl_coef": kl_coef, "entropy_coef": entropy_coef, "reduction": reduction}
    return PolicyLoss(*_PolicyLoss.apply(logp, kl, entropy, old_logp, advantages, mask, ref_logp, args))


class PreferenceLoss(NamedTuple):
    loss: torch.Tensor       # one float32
    rewards: torch.Tensor    # [2 * pairs]: beta times each answer's sum of log ratios
    stats: torch.Tensor      # [4]: share of right ones, mean margin of the rewards, mean reward of the chosen and of the rejected
    coef: torch.Tensor       # [2 * pairs]: the slope of each answer's tokens, for the backward pass


def preference_loss_forward(logp: torch.Tensor, ref_logp: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None, beta: float = 0.1,
                            kind: str = "sigmoid", label_smoothing: float = 0.0, margin: float = 0.0, average: bool = False) -> PreferenceLoss:
    """Loss of pairs of answers from their tokens' log probabilities `logp`, float32 [2 * pairs, tokens]: the chosen answers' rows first, then the rejected ones' in
    the same order. `ref_logp`: the reference's, of the same shape or summed up ([2 * pairs]); None: 0. `mask` (bool): tokens that count. `kind`: "sigmoid",
    "hinge" or "squared". `average`: log ratios a token instead of an answer. Formulas: lopt_preference_loss."""
    if _type("logp", logp) != 0 or logp.dim() != 2 or logp.shape[0] % 2:
        raise ValueError(f"logp is {tuple(logp.shape)} of {logp.dtype}; float32 of an even number of rows is needed")
    if kind not in _KINDS:
        raise ValueError(f"kind={kind!r}; one of {', '.join(map(repr, _KINDS))} is needed")
    x, rows, tokens, ld = _matrix("logp", logp)
    index = logp.get_device()
    ref = m = None
    ref_at = ref_type = m_at = ld_ref = ld_m = 0
    sums = False
    if ref_logp is not None:
        sums = ref_logp.dim() == 1
        if sums:
            if ref_logp.dtype not in _TYPES:
                raise ValueError(f"ref_logp is of {ref_logp.dtype}; float32, bfloat16 or float16 is needed")
            ref, ld_ref = _expect("ref_logp", ref_logp, logp, ref_logp.dtype, (rows,)), 1
        else:
            ref, ld_ref = _token_rows("ref_logp", ref_logp, logp, index, tokens, None)
        ref_at, ref_type = ref.data_ptr(), _TYPES[ref.dtype]
    if mask is not None:
        m, ld_m = _token_rows("mask", mask, logp, index, tokens, torch.bool)
        m_at = m.data_ptr()
    dev = logp.device
    loss = torch.empty((), dtype=torch.float32, device=dev)
    rewards = torch.empty(rows, dtype=torch.float32, device=dev)
    coef = torch.empty_like(rewards)
    stats = torch.empty(4, dtype=torch.float32, device=dev)
    L = lib()
    nbytes = L.lopt_preference_loss_workspace(rows // 2, tokens)
    ws = _workspace(nbytes, dev)
    terms = _PREFERENCE.pack(x.data_ptr(), ld, ref_at, ld_ref, m_at, ld_m, rows // 2, tokens, beta, label_smoothing, margin,
                             ref_type, sums, _KINDS[kind], bool(average))
    _run(L.lopt_preference_loss, index, terms, loss.data_ptr(), stats.data_ptr(), rewards.data_ptr(), coef.data_ptr(), _ptr(ws), nbytes)
    return PreferenceLoss(loss, rewards, stats, coef)


def preference_loss_backward(dloss: torch.Tensor, forward: PreferenceLoss, logp: torch.Tensor, mask: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dlogp from the gradient of the loss and what preference_loss_forward gave."""
    if _type("logp", logp) != 0 or logp.dim() != 2 or logp.shape[0] % 2:
        raise ValueError(f"logp is {tuple(logp.shape)} of {logp.dtype}; float32 of an even number of rows is needed")
    rows, tokens = logp.shape
    m, ld_m = (None, 0) if mask is None else _token_rows("mask", mask, logp, logp.get_device(), tokens, torch.bool)
    dloss = _expect("dloss", dloss, logp, torch.float32, ())
    coef = _expect("coef", forward.coef, logp, torch.float32, (rows,))
    dlogp = _new(logp)
    _run(lib().lopt_preference_loss_backward, logp.get_device(), coef.data_ptr(), _ptr(m), ld_m, dloss.data_ptr(), dlogp.data_ptr(), rows // 2, tokens)
    return dlogp


class _PreferenceLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logp, ref_logp, mask, args):
        r = preference_loss_forward(logp, ref_logp, mask, **args)
        ctx.save_for_backward(logp, mask, r.coef)
        ctx.mark_non_differentiable(r.rewards, r.stats, r.coef)
        return r.loss, r.rewards, r.stats, r.coef

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dloss, *_):
        logp, mask, coef = ctx.saved_tensors
        return preference_loss_backward(dloss, PreferenceLoss(None, None, None, coef), logp, mask), None, None, None


def preference_loss(logp: torch.Tensor, ref_logp: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None, beta: float = 0.1,
                    kind: str = "sigmoid", label_smoothing: float = 0.0, margin: float = 0.0, average: bool = False) -> PreferenceLoss:
    """preference_loss_forward with the gradient of the loss for logp. The reference is a constant: one that asks for a gradient is refused."""
    if ref_logp is not None and ref_logp.requires_grad and torch.is_grad_enabled():
        raise ValueError("ref_logp asks for a gradient, which this loss does not give; detach it")
    args = {"beta": beta, "kind": kind, "label_smoothing": label_smoothing, "margin": margin, "average": average}
    return PreferenceLoss(*_PreferenceLoss.apply(logp, ref_logp, mask, args))
