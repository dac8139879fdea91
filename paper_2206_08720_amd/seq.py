"""Operators of a sequence model's block: root-mean-square norm, rotary positions, attention.

    h = seq.rms_norm(x, weight)                                    # or (y, h) with residual=
    q, k = seq.rotary(q, table, positions, k=k)
    o = seq.attention(q, k, v, causal=True)                        # or one token over a cache: k_lens=

and their gradients (`rms_norm_backward`, `rotary(..., inverse=True)`, `attention_backward`).  Arrays are
float32, bfloat16 or float16 torch tensors on the GPU; only the last dimension has to be contiguous.  Every
call enqueues on the current stream, or on `stream`, and returns before the work is done.  As in `ntk`, PyTorch
supplies device memory and streams only: every step runs in libntk.so (include/ntk_seq.h has the
formulas, the limits and what each mask means).

autograd records none of these calls: their gradients are the calls above.  Where an argument requires a gradient (and
gradients are enabled) the results require one too, and asking for it raises an error that names the call to make.
"""
from __future__ import annotations

import contextlib
import ctypes
import math

import torch

from . import _lib

_DTYPES = {torch.float32: _lib.NTK_F32, torch.bfloat16: _lib.NTK_BF16, torch.float16: _lib.NTK_F16}
_NO_CONTEXT = contextlib.nullcontext()
_MOST = 0x7fffffff


def _check(t, name, dtype=None, ndim=None, device=None, shape=None):
    if not isinstance(t, torch.Tensor) or not t.is_cuda or (t.dtype not in _DTYPES if dtype is None else t.dtype != dtype):
        raise TypeError(f"{name} must be a GPU tensor of type {dtype or 'float32, bfloat16 or float16'}")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    if (ndim is not None and t.dim() != ndim) or (shape is not None and t.shape != shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape) if shape is not None else f'{ndim} dimensions'}")
    if not t.is_contiguous() and t.stride(-1) != 1 and t.shape[-1] > 1:
        raise ValueError(f"{name} must be contiguous in its last dimension")


def _sizes(*sizes):
    """The library's sizes are 32-bit integers, and ctypes would cut larger ones."""
    if max(sizes) > _MOST:
        raise _lib.NTKError(_lib.NTK_E_UNSUPPORTED, f"a size of {max(sizes)} does not fit 32 bits")


class _Unrecorded(torch.autograd.Function):
    """Passes results on; a backward pass that reaches them ends with `message`."""

    @staticmethod
    def forward(ctx, message, outs, *inputs):
        ctx.message = message
        return outs

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError(ctx.message)


_recording = torch.is_grad_enabled


def _wanted(*inputs):
    """Whether one of the tensors (or None) requires a gradient."""
    for t in inputs:
        if t is not None and t.requires_grad:
            return True
    return False


def _unrecorded(name, gradient, inputs, *outs):
    """The results of a call one of whose inputs requires a gradient."""
    inputs = [t for t in inputs if t is not None]
    return _Unrecorded.apply(f"autograd does not record seq.{name}: its gradient is {gradient}", outs, *inputs)


def _written(name, inputs, *outs):
    """Before arrays of the caller's are written: refused where a gradient would have to pass, and counted as a change."""
    if _recording() and _wanted(*inputs, *outs):
        raise RuntimeError(f"seq.{name} writes into its argument, which autograd does not record: an argument requires a gradient")
    for t in outs:
        if t is not None:
            torch.autograd.graph.increment_version(t)


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)


class _Call:
    """The device and stream of one call: outputs and workspaces are allocated for that stream, and tensors
    that come from another one are kept from reuse until it has passed this call."""

    __slots__ = ("handle", "_enter")

    def __init__(self, lead, stream, inputs):
        index = lead.device.index
        self._enter = ()
        if stream is None:
            self.handle = _raw_stream(index)
            if torch.cuda.current_device() != index:
                self._enter = (torch.cuda.device(index),)
        else:
            self.handle = stream.cuda_stream
            self._enter = (torch.cuda.device(index), torch.cuda.stream(stream))
            for t in inputs:
                if t is not None:
                    t.record_stream(stream)

    def __enter__(self):
        for c in self._enter:
            c.__enter__()
        return self

    def __exit__(self, *exc):
        for c in reversed(self._enter):
            c.__exit__(*exc)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _views(*tensors):
    """The tensors' [batch, position, head, dim] as ntk_view structs in one array, and a reference to each (None for None); the
    stride of a dimension of size 1 is never used and counts as 0."""
    values = []
    for t in tensors:
        if t is None:
            values += (0, 0, 0, 0)
        else:
            (b, n, h, _), (sb, sn, sh, _) = t.shape, t.stride()
            values += (t.data_ptr(), sb if b > 1 else 0, sn if n > 1 else 0, sh if h > 1 else 0)
    array = (ctypes.c_longlong * len(values))(*values)
    return [None if t is None else ctypes.byref(array, 32 * i) for i, t in enumerate(tensors)]


def _like(t, dtype=None):
    """A contiguous tensor of t's shape."""
    if dtype is None and t.is_contiguous():
        return torch.empty_like(t)
    return torch.empty(t.shape, dtype=dtype or t.dtype, device=t.device)


def _rows(t):
    """A tensor's rows [rows, width] as (tensor, row stride), without a copy where they are evenly spaced and apart (rows of an
    expanded tensor are not)."""
    if t.dim() != 2:
        t = t.reshape(-1, t.shape[-1])
    rows, width = t.shape
    if rows > 1 and t.stride(0) < width:
        t = t.contiguous()
    return t, t.stride(0) if rows > 1 else width


# ---- root-mean-square norm ----------------------------------------------------------------------------------

def _rms_norm(x, weight, residual, eps, stream, e4m3):
    lib = _lib.load()
    _check(x, "x")
    if x.dim() < 1:
        raise ValueError("x needs a last dimension")
    width = x.shape[-1]
    if width > _MOST:
        _sizes(width)
    if not isinstance(weight, torch.Tensor) or weight.dtype not in (torch.float32, x.dtype):
        raise TypeError(f"weight must be float32 or {x.dtype}")
    _check(weight, "weight", weight.dtype, device=x.device, shape=x.shape[-1:])
    if residual is not None:
        _check(residual, "residual", x.dtype, device=x.device, shape=x.shape)
    with _Call(x, stream, (x, weight, residual)) as call:
        xr, xs = _rows(x)
        rr, rs = (None, 0) if residual is None else _rows(residual)
        y = _like(x, torch.float8_e4m3fn if e4m3 else None)
        h = None if residual is None else _like(x)
        scale = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device) if e4m3 else None
        _lib.check(lib.ntk_rms_norm(_DTYPES[x.dtype], _DTYPES[weight.dtype], xr.shape[0], width, _ptr(xr), xs, _ptr(rr), rs,
                                    _ptr(weight), eps, _ptr(y), _ptr(h), _ptr(scale), call.handle))
    return y, h, scale


def rms_norm(x, weight, residual=None, eps=1e-6, stream=None):
    """y = h weight / sqrt(mean(h^2) + eps) over the last dimension, with h = x.  With `residual`, h = x + residual
    and (y, h) is returned: h is what the next block adds to and what the backward pass reads."""
    y, h, _ = _rms_norm(x, weight, residual, eps, stream, False)
    if _recording() and _wanted(x, weight, residual):
        y, h = _unrecorded("rms_norm", "rms_norm_backward", (x, weight, residual), y, h)
    return y if residual is None else (y, h)


def rms_norm_e4m3(x, weight, residual=None, eps=1e-6, stream=None):
    """The norm in 8 bits: (q, scale) or, with `residual`, (q, scale, h), where q (float8_e4m3fn) times its row's scale
    is y, and scale = max|y| / 448."""
    q, h, scale = _rms_norm(x, weight, residual, eps, stream, True)
    if _recording() and _wanted(x, weight, residual):
        q, scale, h = _unrecorded("rms_norm_e4m3", "not defined", (x, weight, residual), q, scale, h)
    return (q, scale) if residual is None else (q, scale, h)


def rms_norm_backward(dy, h, weight, dh=None, eps=1e-6, stream=None):
    """(dx, dweight) of `rms_norm`: dx is the gradient of x and of the residual alike.  `dh` is the gradient that
    reaches h from elsewhere (the next block's residual)."""
    lib = _lib.load()
    _check(h, "h")
    width = h.shape[-1]
    if width > _MOST:
        _sizes(width)
    _check(dy, "dy", h.dtype, device=h.device, shape=h.shape)
    if dh is not None:
        _check(dh, "dh", h.dtype, device=h.device, shape=h.shape)
    if not isinstance(weight, torch.Tensor) or weight.dtype not in (torch.float32, h.dtype):
        raise TypeError(f"weight must be float32 or {h.dtype}")
    _check(weight, "weight", weight.dtype, device=h.device, shape=h.shape[-1:])
    with _Call(h, stream, (dy, h, weight, dh)) as call:
        hr, hs = _rows(h)
        yr, ys = _rows(dy)
        dr, ds = (None, 0) if dh is None else _rows(dh)
        dx, dweight = _like(h), _like(weight)
        rows = hr.shape[0]
        need = lib.ntk_rms_norm_workspace(rows, width)
        if need < 0:
            _lib.check(need)
        work = torch.empty(need, dtype=torch.uint8, device=h.device)
        _lib.check(lib.ntk_rms_norm_bwd(_DTYPES[h.dtype], _DTYPES[weight.dtype], rows, width, _ptr(yr), ys, _ptr(hr), hs, _ptr(weight),
                                        _ptr(dr), ds, eps, _ptr(dx), _ptr(dweight), _ptr(work), need, call.handle))
    if _recording() and _wanted(dy, h, weight, dh):
        return _unrecorded("rms_norm_backward", "not defined", (dy, h, weight, dh), dx, dweight)
    return dx, dweight


# ---- rotary positions ---------------------------------------------------------------------------------------

def _gpu(device):
    """The GPU that `device` names; the current one for None and for "cuda" without a number."""
    dev = torch.device("cuda" if device is None else device)
    if dev.type != "cuda":
        raise ValueError(f"device {dev} is not a GPU")
    return torch.device("cuda", torch.cuda.current_device()) if dev.index is None else dev


def rotary_table(max_pos, rot, base=10000.0, scaling=None, factor=1.0, original=None, low=1.0, high=32.0, device=None,
                 stream=None):
    """[max_pos, rot / 2, 2] float32: the cosine and sine of every position and pair, angles in 64 bits.  For
    contexts longer than the trained one `scaling` is "linear", "base" or "ramp" with their `factor` (the ramp also
    with the trained length `original`, and the numbers of turns `low` and `high` between which it lies)."""
    lib = _lib.load()
    if not torch.cuda.is_available():
        raise RuntimeError("no GPU visible: the NTK library runs on an MI355X only")
    kinds = {None: _lib.NTK_ROTARY_PLAIN, "linear": _lib.NTK_ROTARY_LINEAR, "base": _lib.NTK_ROTARY_BASE, "ramp": _lib.NTK_ROTARY_RAMP}
    if scaling not in kinds:
        raise ValueError(f"scaling is one of {list(kinds)}")
    if scaling == "ramp" and original is None:
        raise ValueError('scaling="ramp" needs original')
    dev = _gpu(device)
    if max_pos < 1 or rot < 2 or rot % 2:
        raise ValueError("rotary_table: max_pos < 1, or rot odd or < 2")
    _sizes(max_pos, rot)
    s = _lib.ntk_rotary_scaling(kinds[scaling], float(factor), float(original or 1), float(low), float(high))
    with torch.cuda.device(dev), torch.cuda.stream(stream) if stream is not None else _NO_CONTEXT:
        table = torch.empty((max_pos, rot // 2, 2), dtype=torch.float32, device=dev)
        _lib.check(lib.ntk_rotary_table(max_pos, rot, float(base), ctypes.byref(s), _ptr(table),
                                        ctypes.c_void_p(torch.cuda.current_stream(dev).cuda_stream)))
    return table


def rotary(q, table, positions=0, k=None, interleaved=False, inverse=False, inplace=False, stream=None):
    """Turns the first 2 * table.shape[1] elements of every head of q [batch, length, heads, dim], and of k with head counts of
    its own, by their positions: int32 [batch, length], or the first position of every sequence.  Returns q, or
    (q, k).  `inverse` turns the other way, which is how the gradients pass; it undoes the turn unless the table is a "ramp",
    whose magnitude is not 1."""
    lib = _lib.load()
    _check(q, "q", ndim=4)
    _check(table, "table", torch.float32, ndim=3, device=q.device)
    b, n, heads, dim = q.shape
    if not table.is_contiguous() or table.shape[2] != 2:
        raise ValueError("table must be a contiguous [max_pos, rot / 2, 2] tensor")
    if k is not None:
        _check(k, "k", q.dtype, device=q.device, shape=(b, n, k.shape[2] if k.dim() == 4 else -1, dim))
    per_token = isinstance(positions, torch.Tensor)
    if per_token:
        _check(positions, "positions", torch.int32, device=q.device, shape=(b, n))
        if not positions.is_contiguous():
            raise ValueError("positions must be contiguous")
    elif not -1 < positions <= _MOST:
        raise _lib.NTKError(_lib.NTK_E_ARG, f"rotary: first position {positions}")
    if q.numel() > _MOST or table.numel() > _MOST or (k is not None and k.numel() > _MOST):
        _sizes(b, n, heads, 0 if k is None else k.shape[2], dim, table.shape[0], 2 * table.shape[1])
    if inplace:
        _written("rotary", (table,), q, k)
    with _Call(q, stream, (q, table, k, positions if per_token else None)) as call:
        qo = q if inplace else _like(q)
        ko = k if inplace or k is None else _like(k)
        qv, kv, qov, kov = _views(q, k, qo, ko)
        _lib.check(lib.ntk_rotary(_DTYPES[q.dtype], b, n, heads, 0 if k is None else k.shape[2], dim, 2 * table.shape[1],
                                  int(interleaved), int(inverse), qv, kv, _ptr(table), table.shape[0],
                                  _ptr(positions) if per_token else None, 0 if per_token else int(positions),
                                  qov, kov, call.handle))
    if not inplace and _recording() and _wanted(q, table, k):
        qo, ko = _unrecorded("rotary", "rotary with `inverse` turned round, its backward pass", (q, table, k), qo, ko)
    return qo if k is None else (qo, ko)


# ---- attention ----------------------------------------------------------------------------------------------

def _attention_desc(q, k, v, causal, softcap, scale, slopes, k_lens, prefix, docs):
    _check(q, "q", ndim=4)
    b, sq, heads, dim = q.shape
    _check(k, "k", q.dtype, ndim=4, device=q.device)
    sk, kv_heads = k.shape[1], k.shape[2]
    if k.shape[0] != b or k.shape[3] != dim:
        raise ValueError(f"k has shape {tuple(k.shape)}, expected ({b}, k_len, kv_heads, {dim})")
    _check(v, "v", q.dtype, device=q.device, shape=k.shape)
    if q.numel() > _MOST or k.numel() > _MOST:
        _sizes(b, sq, sk, heads, kv_heads, dim)
    for name, t, dtype, shape in (("k_lens", k_lens, torch.int32, (b,)), ("prefix", prefix, torch.int32, (b,)),
                                  ("docs", docs, torch.int32, (b, sk)), ("slopes", slopes, torch.float32, (heads,))):
        if t is not None:
            _check(t, name, dtype, device=q.device, shape=shape)
            if not t.is_contiguous():
                raise ValueError(f"{name} must be contiguous")
    return _lib.ntk_attention_desc(_DTYPES[q.dtype], b, sq, sk, heads, kv_heads, dim, 1 if causal else 0,
                                   1.0 / math.sqrt(max(dim, 1)) if scale is None else scale, softcap,
                                   _ptr(k_lens), _ptr(prefix), _ptr(docs), _ptr(slopes))


def _workspace(lib, desc, backward, device):
    need = lib.ntk_attention_workspace(ctypes.byref(desc), backward)
    if need < 0:
        _lib.check(need)
    return (torch.empty(need, dtype=torch.uint8, device=device) if need else None), need


def attention(q, k, v, causal=False, softcap=0.0, scale=None, slopes=None, k_lens=None, prefix=None, docs=None,
              return_lse=False, out=None, stream=None):
    """softmax(scores) v for q [batch, q_len, heads, dim], k and v [batch, k_len, kv_heads, dim] (heads a multiple of
    kv_heads); returns o like q, or (o, lse) for the backward pass.  Scores are softcap tanh(scale q.k / softcap) - slope
    |distance|; the queries are the last q_len of each sequence's k_lens positions.  See include/ntk_seq.h for
    what `causal`, `prefix` and `docs` hide."""
    lib = _lib.load()
    desc = _attention_desc(q, k, v, causal, softcap, scale, slopes, k_lens, prefix, docs)
    b, sq, heads, dim = q.shape
    if out is not None:
        _check(out, "out", q.dtype, device=q.device, shape=q.shape)
        _written("attention(out=)", (q, k, v, slopes), out)
    with _Call(q, stream, (q, k, v, slopes, k_lens, prefix, docs, out)) as call:
        o = _like(q) if out is None else out
        lse = torch.empty((b, heads, sq), dtype=torch.float32, device=q.device) if return_lse else None
        work, need = _workspace(lib, desc, 0, q.device)
        _lib.check(lib.ntk_attention(ctypes.byref(desc), *_views(q, k, v, o), _ptr(lse), _ptr(work), need, call.handle))
    if out is None and _recording() and _wanted(q, k, v, slopes):
        o, lse = _unrecorded("attention", "attention_backward", (q, k, v, slopes), o, lse)
    return (o, lse) if return_lse else o


def attention_backward(do, q, k, v, o, lse, causal=False, softcap=0.0, scale=None, slopes=None, k_lens=None, prefix=None,
                       docs=None, stream=None):
    """(dq, dk, dv) of `attention` from the gradient of o, with the o and lse that it returned and the same options."""
    lib = _lib.load()
    desc = _attention_desc(q, k, v, causal, softcap, scale, slopes, k_lens, prefix, docs)
    b, sq, heads, dim = q.shape
    _check(do, "do", q.dtype, device=q.device, shape=q.shape)
    _check(o, "o", q.dtype, device=q.device, shape=q.shape)
    _check(lse, "lse", torch.float32, device=q.device, shape=(b, heads, sq))
    if not lse.is_contiguous():
        raise ValueError("lse must be contiguous")
    with _Call(q, stream, (do, q, k, v, o, lse, slopes, k_lens, prefix, docs)) as call:
        dq, dk, dv = _like(q), _like(k), _like(v)
        work, need = _workspace(lib, desc, 1, q.device)
        views = _views(do, q, k, v, o, dq, dk, dv)
        _lib.check(lib.ntk_attention_bwd(ctypes.byref(desc), *views[:5], _ptr(lse), *views[5:], _ptr(work), need, call.handle))
    if _recording() and _wanted(do, q, k, v, o, lse, slopes):
        return _unrecorded("attention_backward", "not defined", (do, q, k, v, o, lse, slopes), dq, dk, dv)
    return dq, dk, dv
