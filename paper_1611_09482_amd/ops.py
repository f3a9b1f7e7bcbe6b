"""The token operators of libfwg.so (include/fwg.h) on torch tensors: embedding lookup and its gradient, 8-bit
rows with or without RMS norm, the 8-bit product, log probabilities and their gradient.

Argument marshalling only, as in binding.py: every call checks its tensors, enqueues the library's kernels on the
current stream of the current device and returns without waiting.  Matrices may have any number of leading
dimensions as long as their rows lie evenly apart (views of consecutive rows, every n-th row, expanded rows as
inputs); elements of a row are consecutive.  Nothing is copied to make an argument fit: what does not fit is
refused (TypeError, ValueError; sizes that the library refuses raise FwgError).  `out` takes the results' tensors
of an earlier call, so that a loop allocates nothing but the workspaces that some calls take from torch's
allocator.  The calls are no part of torch's autograd, whether or not a tensor asks for gradients: results have no
graph, and the gradients (embed_grad, log_probs_grad) are calls of their own.
"""
from __future__ import annotations

import ctypes
import functools
from typing import NamedTuple, Optional

import torch

from .binding import FWG_BF16, FWG_EINVAL, FWG_EUNSUPPORTED, FWG_F32, FwgError, _check, load_library

_TYPES = {torch.float32: FWG_F32, torch.bfloat16: FWG_BF16}
_lib = None


def _library():
    global _lib
    if _lib is None:
        _lib = load_library()
    return _lib


_device = torch.cuda.current_device
# a device's current stream as an address, without the object that torch.cuda.current_stream() makes (2.7 us a call)
_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda d: torch.cuda.current_stream(d).cuda_stream)


def _refuse(name: str, t, device: int):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} is not a tensor")
    raise ValueError(f"{name} is on {t.device}: the call runs on the current device, cuda:{device}")


def _typed(name: str, t, dtype, device: int) -> None:
    if not isinstance(t, torch.Tensor) or t.get_device() != device:
        _refuse(name, t, device)
    if t.dtype != dtype:
        raise TypeError(f"{name} is {t.dtype}: {dtype} is wanted")


_MOST = 2 ** 31 - 1


def _int32(name: str, n: int) -> int:
    """A size that the library takes in 32 bits: ctypes would pass on the low 32 bits of a larger one."""
    if n > _MOST:
        raise FwgError(FWG_EUNSUPPORTED, f"{name} is {n}: at most 2^31 - 1 is supported")
    if n < -_MOST:
        raise FwgError(FWG_EINVAL, f"{name} is {n}")
    return n


def _matrix(name: str, t, device: int, out: bool = False):
    """(element type, rows, width, stride) of a float32 or bfloat16 tensor seen as rows."""
    if not isinstance(t, torch.Tensor) or t.get_device() != device:
        _refuse(name, t, device)
    kind = _TYPES.get(t.dtype)
    if kind is None:
        raise TypeError(f"{name} is {t.dtype}: float32 or bfloat16 is wanted")
    shape = t.shape
    if len(shape) == 2 and t.is_contiguous():
        rows, width = shape
        if width > _MOST:
            _int32(f"{name}'s width", width)
        return kind, rows, width, width
    rows, width, stride = _rows(name, t, out)
    return kind, rows, width, stride


def _table(name: str, t, device: int):
    """_matrix() of a tensor of two dimensions whose rows are tokens."""
    sizes = _matrix(name, t, device)
    if t.dim() != 2:
        _flat(name, t)
    if sizes[1] > _MOST:
        _int32(f"{name}'s length", sizes[1])
    return sizes


def _rows(name: str, t, out: bool = False):
    """(rows, width, stride) of a tensor seen as rows of its last dimension."""
    shape, strides = t.shape, t.stride()
    if not shape:
        raise ValueError(f"{name} has no dimensions: rows are wanted")
    width = shape[-1]
    if width > _MOST:
        _int32(f"{name}'s width", width)
    if width > 1 and strides[-1] != 1:
        raise ValueError(f"{name}: the elements of a row have to be consecutive (stride {strides[-1]})")
    if len(shape) == 2:
        rows, stride = shape[0], strides[0]
    else:
        rows, stride = 1, width
        for n, s in zip(reversed(shape[:-1]), reversed(strides[:-1])):
            if n == 1:
                continue
            if rows > 1 and s != rows * stride:
                raise ValueError(f"{name}: the rows of shape {tuple(shape)}, strides {strides} do not lie evenly apart")
            if rows == 1:
                stride = s
            rows *= n
    if rows <= 1:
        stride = width
    elif out and stride < width:
        raise ValueError(f"{name}: its rows overlap (stride {stride}, width {width})")
    return rows, width, stride


def _vector(name: str, t, n: int, dtype, device: int) -> int:
    """Address of `n` consecutive elements."""
    if not isinstance(t, torch.Tensor) or t.get_device() != device:
        _refuse(name, t, device)
    if t.dtype != dtype:
        raise TypeError(f"{name} is {t.dtype}: {dtype} is wanted")
    if t.numel() != n:
        raise ValueError(f"{name} has {t.numel()} elements: {n} are wanted")
    if not t.is_contiguous():
        raise ValueError(f"{name} has to be contiguous")
    return t.data_ptr()


def _like(name: str, t, dtype, shape, device: int, out: bool = False):
    """(address, stride) of a tensor of this type and shape seen as rows."""
    if not isinstance(t, torch.Tensor) or t.get_device() != device:
        _refuse(name, t, device)
    if t.dtype != dtype:
        raise TypeError(f"{name} is {t.dtype}: {dtype} is wanted")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}: {tuple(shape)} is wanted")
    if t.is_contiguous() and shape:
        return t.data_ptr(), shape[-1]
    return t.data_ptr(), _rows(name, t, out)[2]


def _shaped(name: str, t, shape) -> None:
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}: {tuple(shape)} is wanted")


def _flat(name: str, t) -> None:
    if t.dim() != 2:
        raise ValueError(f"{name} has {t.dim()} dimensions: 2 are wanted")


def _workspace(need: int):
    return torch.empty(need, dtype=torch.uint8, device="cuda") if need else None


@functools.lru_cache(maxsize=1024)
def _bytes(call: str, *sizes) -> int:
    """Workspace bytes: a pure function of the sizes."""
    n = ctypes.c_size_t(0)
    function = getattr(_library(), call)
    for size, kind in zip(sizes, function.argtypes):
        if kind is ctypes.c_int32:
            _int32("a size", size)
    _check(function(*sizes, ctypes.byref(n)))
    return n.value


def embed(table, tokens, scale: float = 1.0, out=None):
    """scale * table[tokens].  table: float32 or bfloat16 [vocab][channels]; tokens: int32, any shape, contiguous;
    a token outside [0, vocab) is padding and gives a zero row.  out: [*tokens.shape][channels], float32 or bfloat16
    (default: of the table's type).  No part of autograd: the table's gradient is embed_grad()'s."""
    dev = _device()
    kind, vocab, channels, stride = _table("table", table, dev)
    n = tokens.numel() if isinstance(tokens, torch.Tensor) else 0
    ids = _vector("tokens", tokens, n, torch.int32, dev)
    shape = tokens.shape + (channels,)
    if out is None:
        out = torch.empty(shape, dtype=table.dtype, device=table.device)
    okind, _, _, ostride = _matrix("out", out, dev, True)
    _shaped("out", out, shape)
    _check(_library().fwg_embed(kind, okind, n, vocab, channels, table.data_ptr(), stride, ids, scale, out.data_ptr(),
                                ostride, _stream(dev)))
    return out


def embed_grad(grad, tokens, vocab: int, scale: float = 1.0, out=None):
    """The gradient of embed() with respect to the table: out[v] = scale * (sum of grad over the positions of token
    v), zero where there is none.  grad: float32 or bfloat16 [*tokens.shape][channels] (rows may be expanded); out:
    float32 (default) or bfloat16 [vocab][channels].  Sums in float32 in an order that depends on the tokens only:
    the same bits every time."""
    dev = _device()
    kind, rows, channels, stride = _matrix("grad", grad, dev)
    n = tokens.numel() if isinstance(tokens, torch.Tensor) else 0
    ids = _vector("tokens", tokens, n, torch.int32, dev)
    _shaped("grad", grad, tokens.shape + (channels,))
    need = _bytes("fwg_embed_grad_workspace", n, vocab, channels)
    if out is None:
        out = torch.empty((vocab, channels), dtype=torch.float32, device=grad.device)
    okind, _, _, ostride = _matrix("out", out, dev, True)
    _shaped("out", out, (vocab, channels))
    ws = _workspace(need)
    _check(_library().fwg_embed_grad(kind, okind, n, vocab, channels, grad.data_ptr(), stride, ids, scale, out.data_ptr(),
                              ostride, None if ws is None else ws.data_ptr(), need, _stream(dev)))
    return out


class QuantRows(NamedTuple):
    """8-bit rows: row r stands for q[r] * scale[r]."""
    q: torch.Tensor
    scale: torch.Tensor


class NormQuant(NamedTuple):
    """8-bit rows of a norm, the residual stream after the addition, and the values that the rows stand for in
    bfloat16 (None where they were not asked for)."""
    q: torch.Tensor
    scale: torch.Tensor
    summed: Optional[torch.Tensor]
    values: Optional[torch.Tensor]


def quant_rows(x, out=None) -> QuantRows:
    """Rows in 8 bits with a scale each: scale = max|x| / 127, q = x / scale to the nearest (ties to even).  For
    weights [outputs][inner] these are matmul_quant's w and w_scale."""
    dev = _device()
    kind, rows, width, stride = _matrix("x", x, dev)
    if out is None:
        out = QuantRows(torch.empty(x.shape, dtype=torch.int8, device=x.device),
                        torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device))
    q, scale = out
    qp, qstride = _like("out.q", q, torch.int8, x.shape, dev, True)
    _check(_library().fwg_quant_rows(kind, rows, width, x.data_ptr(), stride, qp, qstride,
                                     _vector("out.scale", scale, rows, torch.float32, dev), _stream(dev)))
    return out if isinstance(out, QuantRows) else QuantRows(*out)


def norm_quant(x, gain=None, residual=None, eps: float = 1e-6, values: bool = False, out=None) -> NormQuant:
    """h = x + residual; y = h / sqrt(mean(h^2) + eps) * gain; y's rows in 8 bits as in quant_rows.  x, residual:
    float32 or bfloat16 [..., channels]; gain: float32 [channels].  Results: q, scale, `summed` (h, rounded to x's
    type; with a residual only) and, where values is true, `values` (q * scale in bfloat16).  out: a NormQuant or
    the four tensors (None: not wanted); out's `summed` may be x or residual itself.  No part of autograd: rounding to
    8 bits has no gradient."""
    dev = _device()
    kind, rows, width, stride = _matrix("x", x, dev)
    shape, dtype = x.shape, x.dtype
    rp, rstride = (None, 0) if residual is None else _like("residual", residual, dtype, shape, dev)
    if out is None:
        out = NormQuant(torch.empty(shape, dtype=torch.int8, device=x.device),
                        torch.empty(shape[:-1], dtype=torch.float32, device=x.device),
                        None if residual is None else torch.empty(shape, dtype=dtype, device=x.device),
                        torch.empty(shape, dtype=torch.bfloat16, device=x.device) if values else None)
    q, scale, summed, vals = out
    qp, qstride = _like("out.q", q, torch.int8, shape, dev, True)
    sp, sstride = (None, 0) if summed is None else _like("out.summed", summed, dtype, shape, dev, True)
    vp, vstride = (None, 0) if vals is None else _like("out.values", vals, torch.bfloat16, shape, dev, True)
    gp = None if gain is None else _vector("gain", gain, width, torch.float32, dev)
    _check(_library().fwg_norm_quant(kind, rows, width, x.data_ptr(), stride, rp, rstride, gp, eps, sp, sstride, qp, qstride,
                                     _vector("out.scale", scale, rows, torch.float32, dev), vp, vstride, _stream(dev)))
    return out if isinstance(out, NormQuant) else NormQuant(*out)


def matmul_quant(x, x_scale, w, w_scale, bias=None, dtype=torch.bfloat16, out=None):
    """(x @ w.T) * x_scale[:, None] * w_scale + bias, the product of the 8-bit integers exact.  x: int8
    [..., inner] with x_scale float32 [...]; w: int8 [outputs][inner] with w_scale float32 [outputs]; bias: float32
    [outputs].  out: [..., outputs] of dtype (float32 or bfloat16)."""
    dev = _device()
    _typed("x", x, torch.int8, dev)
    _typed("w", w, torch.int8, dev)
    rows, inner, stride = _rows("x", x)
    _flat("w", w)
    outputs, winner, wstride = _rows("w", w)
    if outputs > _MOST:
        _int32("w's length", outputs)
    if winner != inner:
        raise ValueError(f"w has {winner} inner elements: {inner} are wanted")
    shape = x.shape[:-1] + (outputs,)
    if out is None:
        out = torch.empty(shape, dtype=dtype, device=x.device)
    okind, _, _, ostride = _matrix("out", out, dev, True)
    _shaped("out", out, shape)
    need = _bytes("fwg_matmul_quant_workspace", rows, outputs, inner)
    ws = _workspace(need)
    _check(_library().fwg_matmul_quant(okind, rows, outputs, inner, x.data_ptr(), stride,
                                _vector("x_scale", x_scale, rows, torch.float32, dev), w.data_ptr(), wstride,
                                _vector("w_scale", w_scale, outputs, torch.float32, dev),
                                None if bias is None else _vector("bias", bias, outputs, torch.float32, dev),
                                out.data_ptr(), ostride, None if ws is None else ws.data_ptr(), need, _stream(dev)))
    return out


class LogProbs(NamedTuple):
    """Per row: the given token's log probability, the entropy (nats), log sum exp, and the most probable tokens
    with their log probabilities ([..., top])."""
    logp: torch.Tensor
    entropy: torch.Tensor
    lse: torch.Tensor
    top_ids: torch.Tensor
    top_logp: torch.Tensor


def log_probs(logits, tokens, top: int = 0, out=None) -> LogProbs:
    """Log probabilities of tokens (int32 [...]) under logits (float32 or bfloat16 [..., vocab]), with entropy, log
    sum exp and the `top` (at most 64) most probable tokens, equal logits in the order of the tokens.  -inf masks
    a token; a token outside [0, vocab) is padding and has log probability 0.  No part of autograd: the logits'
    gradient is log_probs_grad()'s."""
    dev = _device()
    kind, rows, vocab, stride = _matrix("logits", logits, dev)
    lead = logits.shape[:-1]
    ids = _vector("tokens", tokens, rows, torch.int32, dev)
    _shaped("tokens", tokens, lead)
    need = _bytes("fwg_log_probs_workspace", kind, rows, vocab, top)
    if out is None:
        def new(dtype, *more):
            return torch.empty(lead + more, dtype=dtype, device=logits.device)
        out = LogProbs(new(torch.float32), new(torch.float32), new(torch.float32), new(torch.int32, top),
                       new(torch.float32, top))
    logp, entropy, lse, top_ids, top_logp = out
    ws = _workspace(need)
    _check(_library().fwg_log_probs(kind, rows, vocab, logits.data_ptr(), stride, ids, top,
                             _vector("out.logp", logp, rows, torch.float32, dev),
                             _vector("out.entropy", entropy, rows, torch.float32, dev),
                             _vector("out.lse", lse, rows, torch.float32, dev),
                             _vector("out.top_ids", top_ids, rows * top, torch.int32, dev),
                             _vector("out.top_logp", top_logp, rows * top, torch.float32, dev),
                             None if ws is None else ws.data_ptr(), need, _stream(dev)))
    return out if isinstance(out, LogProbs) else LogProbs(*out)


def log_probs_grad(logits, tokens, lse, entropy, grad_logp, grad_entropy=None, out=None):
    """The gradient of log_probs() with respect to the logits, from the gradients of logp and (optional) entropy;
    lse and entropy as log_probs() returned them (entropy may be None without grad_entropy).  out: of the logits'
    shape and type; may be the logits themselves."""
    dev = _device()
    kind, rows, vocab, stride = _matrix("logits", logits, dev)
    ids = _vector("tokens", tokens, rows, torch.int32, dev)
    if out is None:
        out = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
    op, ostride = _like("out", out, logits.dtype, logits.shape, dev, True)
    if grad_entropy is not None and entropy is None:
        raise ValueError("grad_entropy is given without entropy")
    _check(_library().fwg_log_probs_grad(
        kind, rows, vocab, logits.data_ptr(), stride, ids, _vector("lse", lse, rows, torch.float32, dev),
        None if entropy is None else _vector("entropy", entropy, rows, torch.float32, dev),
        _vector("grad_logp", grad_logp, rows, torch.float32, dev),
        None if grad_entropy is None else _vector("grad_entropy", grad_entropy, rows, torch.float32, dev),
        op, ostride, _stream(dev)))
    return out
