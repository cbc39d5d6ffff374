"""The operators of a training loop around the optimizer step, on torch tensors: layer norm, token log probabilities with
entropy and top alternatives, their gradients, and clipping by the global gradient norm.

Nothing numerical happens here: every function checks its tensors, allocates outputs and workspace, and hands pointers to the
call of the same name in include/lopt.h (formulas, masks and special values are described there) on the current stream.
Tensors are CUDA tensors of float32, bfloat16 or float16; `layer_norm` and `token_logprobs` take part in autograd, the
`*_forward` and `*_backward` functions are the passes by themselves."""
from __future__ import annotations

import operator
from array import array
from typing import Iterable, List, NamedTuple, Optional, Sequence, Tuple, Union

import torch

from .binding import _check, lib

__all__ = ["clip_grads", "clip_grad_norm_", "grad_norm", "layer_norm", "layer_norm_forward", "layer_norm_backward",
           "TokenLogprobs", "token_logprobs", "token_logprobs_forward", "token_logprobs_backward", "TOP_MAX"]

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
