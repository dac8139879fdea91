"""Operators of a sequence model's block: root-mean-square norm, rotary positions, attention; and of its answers.

    h = seq.rms_norm(x, weight)                                    # or (y, h) with residual=
    q, k = seq.rotary(q, table, positions, k=k)
    o = seq.attention(q, k, v, causal=True)                        # or one token over a cache: k_lens=

a cache in pages, in the arrays' type or in 8 bits, and the log probabilities of the tokens that come out

    cache = seq.paged_cache(pages, page_size, kv_heads, dim)       # dtype=torch.float8_e4m3fn
    q = seq.cache_append(cache, page_table, lens, k, v, q=q, table=table)
    o = seq.attention_cached(q, cache, page_table, lens + 1)
    logp, entropy, lse, top_logp, top_tokens = seq.token_logprobs(logits, tokens, top=5)

and their gradients (`rms_norm_backward`, `rotary(..., inverse=True)`, `attention_backward`, `token_logprobs_backward`).  Arrays are
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
from typing import NamedTuple, Optional

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
    torch.autograd.graph.increment_version([t for t in outs if t is not None])


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


# ---- a cache in pages ---------------------------------------------------------------------------------------

class PagedCache(NamedTuple):
    """Keys and values [pages, page_size, kv_heads, dim], only the last dimension contiguous; in float8_e4m3fn under a power of
    two a page and head in k_scale and v_scale [pages, kv_heads]."""
    k: torch.Tensor
    v: torch.Tensor
    k_scale: Optional[torch.Tensor] = None
    v_scale: Optional[torch.Tensor] = None


_E4M3 = torch.float8_e4m3fn


def paged_cache(pages, page_size, kv_heads, dim, dtype=torch.bfloat16, device=None):
    """A cache of zeros.  Each head's part of a page lies in one piece, which is what `attention_cached` reads in whole lines."""
    if dtype not in _DTYPES and dtype != _E4M3:
        raise TypeError("dtype must be float32, bfloat16, float16 or float8_e4m3fn")
    if min(pages, kv_heads, dim) < 1 or not 8 <= page_size <= 1024 or page_size & (page_size - 1):
        raise ValueError("paged_cache: a size is below 1, or page_size is no power of two from 8 to 1024")
    dev = _gpu(device)
    k, v = (torch.zeros((pages, kv_heads, page_size, dim), dtype=torch.uint8 if dtype == _E4M3 else dtype, device=dev) for _ in range(2))
    if dtype != _E4M3:
        return PagedCache(k.transpose(1, 2), v.transpose(1, 2))
    scales = (torch.full((pages, kv_heads), 2.0 ** -126, dtype=torch.float32, device=dev) for _ in range(2))
    return PagedCache(k.view(_E4M3).transpose(1, 2), v.view(_E4M3).transpose(1, 2), *scales)


def _ints(t, name, device, shape):
    if t is not None:
        _check(t, name, torch.int32, device=device, shape=shape)
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")


def _cache(cache, page_table, dtype, device, batch):
    """(An ntk_cache in one array of 64-bit numbers, which is quicker than the struct; its dtype; the shape of cache.k; places of a
    sequence.)"""
    k, v, k_scale, v_scale = cache
    cells = k.dtype if isinstance(k, torch.Tensor) else None
    if cells not in (dtype, _E4M3):
        raise TypeError(f"the cache must be of type {dtype} or {_E4M3}")
    _check(k, "cache.k", cells, ndim=4, device=device)
    shape = k.shape
    _check(v, "cache.v", cells, device=device, shape=shape)
    pages, size, heads, dim = shape
    if cells == _E4M3:
        code = _lib.NTK_E4M3
        for name, t in (("cache.k_scale", k_scale), ("cache.v_scale", v_scale)):
            _check(t, name, torch.float32, device=device, shape=(pages, heads))
            if not t.is_contiguous():
                raise ValueError(f"{name} must be contiguous")
        scales = k_scale.data_ptr(), v_scale.data_ptr()
    elif k_scale is not None or v_scale is not None:
        raise ValueError(f"a cache of type {dtype} has no scales")
    else:
        code, scales = _DTYPES[cells], (0, 0)
    _check(page_table, "page_table", torch.int32, ndim=2, device=device)
    rows, most = page_table.shape
    if rows != batch or not page_table.is_contiguous():
        raise ValueError(f"page_table must be a contiguous [{batch}, max_pages] tensor")
    if pages > _MOST or most > _MOST:
        _sizes(pages, most)
    _sizes(size, heads, dim, most * size)
    (kp, ks, kh, _), (vp, vs, vh, _) = k.stride(), v.stride()
    array = (ctypes.c_longlong * 15)(
        code | pages << 32, size | heads << 32, dim,
        k.data_ptr(), kp if pages > 1 else 0, ks if size > 1 else 0, kh if heads > 1 else 0,
        v.data_ptr(), vp if pages > 1 else 0, vs if size > 1 else 0, vh if heads > 1 else 0, *scales, page_table.data_ptr(), most)
    return array, code, shape, most * size


def cache_append(cache, page_table, lens, k, v, q=None, table=None, positions=None, new_lens=None, interleaved=False, stream=None):
    """Appends new tokens' k and v [batch, length, kv_heads, dim] to sequences that hold lens[b] (int32 [batch]): token i < new_lens[b]
    (all of them without new_lens) goes to place lens[b] + i, which lies in page page_table[b, place // page_size] (int32 [batch,
    max_pages]).  With `table`, k turns as in `rotary` to its place (or to positions, int32 [batch, length]).  Returns q
    [batch, length, heads, dim] turned alike, with zeros past new_lens, or None without q.  `lens` stays as it is.  Tokens
    whose place the table or the cache does not have are dropped.  See include/ntk_seq.h for how a cache in 8 bits is rounded."""
    lib = _lib.load()
    _check(k, "k", ndim=4)
    b, n, heads, dim = k.shape
    dev = k.device
    _check(v, "v", k.dtype, device=dev, shape=k.shape)
    if q is not None:
        _check(q, "q", k.dtype, device=dev, shape=(b, n, q.shape[2] if q.dim() == 4 else -1, dim))
    _sizes(b, n, heads, 0 if q is None else q.shape[2])
    if table is not None:
        _check(table, "table", torch.float32, ndim=3, device=dev)
        if not table.is_contiguous() or table.shape[2] != 2:
            raise ValueError("table must be a contiguous [max_pos, rot / 2, 2] tensor")
        _sizes(table.shape[0], 2 * table.shape[1])
    elif positions is not None:
        raise ValueError("positions need a table")
    _ints(lens, "lens", dev, (b,))
    if lens is None:
        raise TypeError("lens must be a GPU tensor of type int32")
    _ints(new_lens, "new_lens", dev, (b,))
    _ints(positions, "positions", dev, (b, n))
    desc, _, held, _ = _cache(cache, page_table, k.dtype, dev, b)
    if held[2] != heads or held[3] != dim:
        raise ValueError(f"the cache holds {held[2]} heads of {held[3]}, k has {heads} of {dim}")
    _written("cache_append", (k, v, table), *cache)
    with _Call(k, stream, (k, v, q, table, positions, lens, new_lens, page_table, *cache)) as call:
        qo = None if q is None else _like(q)
        kv, vv, qv, qov = _views(k, v, q, qo)
        _lib.check(lib.ntk_cache_append(_DTYPES[k.dtype], b, n, 0 if q is None else q.shape[2], ctypes.byref(desc), _ptr(lens),
                                        _ptr(new_lens), kv, vv, qv, qov, _ptr(table), 0 if table is None else table.shape[0],
                                        0 if table is None else 2 * table.shape[1], int(interleaved), _ptr(positions), call.handle))
    if q is not None and _recording() and _wanted(q):
        return _unrecorded("cache_append", "not defined", (q,), qo)[0]
    return qo


def attention_cached(q, cache, page_table, k_lens, q_lens=None, causal=True, softcap=0.0, scale=None, slopes=None,
                     return_lse=False, out=None, stream=None):
    """`attention` of q [batch, q_len, heads, dim] over a cache of which sequence b fills k_lens[b] places (int32 [batch], the
    queries' own tokens among them).  Queries i < q_lens[b] (all of them without q_lens) are its last ones; the rows of o past them
    are zeros.  Returns o like q, or (o, lse).  It has no backward pass."""
    lib = _lib.load()
    _check(q, "q", ndim=4)
    b, sq, heads, dim = q.shape
    dev = q.device
    desc, cells, held, places = _cache(cache, page_table, q.dtype, dev, b)
    if held[3] != dim:
        raise ValueError(f"the cache holds heads of {held[3]}, q has heads of {dim}")
    _sizes(b, sq, heads)
    if k_lens is None:
        raise TypeError("k_lens must be a GPU tensor of type int32")
    _ints(k_lens, "k_lens", dev, (b,))
    _ints(q_lens, "q_lens", dev, (b,))
    if slopes is not None:
        _check(slopes, "slopes", torch.float32, device=dev, shape=(heads,))
        if not slopes.is_contiguous():
            raise ValueError("slopes must be contiguous")
    if out is not None:
        _check(out, "out", q.dtype, device=dev, shape=q.shape)
        _written("attention_cached(out=)", (q, slopes, *cache), out)
    scores = _lib.ntk_attention_desc(_DTYPES[q.dtype], b, sq, places, heads, held[2], dim, 1 if causal else 0,
                                     1.0 / math.sqrt(max(dim, 1)) if scale is None else scale, softcap, _ptr(k_lens), None, None, _ptr(slopes))
    with _Call(q, stream, (q, k_lens, q_lens, slopes, out, page_table, *cache)) as call:
        o = _like(q) if out is None else out
        lse = torch.empty((b, heads, sq), dtype=torch.float32, device=dev) if return_lse else None
        need = lib.ntk_attention_cached_workspace(ctypes.byref(scores), cells)
        if need < 0:
            _lib.check(need)
        work = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
        _lib.check(lib.ntk_attention_cached(ctypes.byref(scores), ctypes.byref(desc), _ptr(q_lens), *_views(q, o), _ptr(lse), _ptr(work),
                                            need, call.handle))
    if out is None and _recording() and _wanted(q, slopes, *cache):
        o, lse = _unrecorded("attention_cached", "not defined", (q, slopes, *cache), o, lse)
    return (o, lse) if return_lse else o


# ---- log probabilities of given tokens ----------------------------------------------------------------------

class TokenLogprobs(NamedTuple):
    """logp and entropy [...] float32; lse [..., 2] float32: the largest logit m and log sum exp(scale (logits - m)); top_logp float32 and
    top_tokens int32 [..., top], None where none were asked for."""
    logp: torch.Tensor
    entropy: torch.Tensor
    lse: torch.Tensor
    top_logp: Optional[torch.Tensor] = None
    top_tokens: Optional[torch.Tensor] = None


def _per_row(t, name, dtype, logits, each=()):
    """Checks one number (or `each` of them) a row, at any strides, or None."""
    if t is None:
        return
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor of type {dtype}")
    if t.device != logits.device or t.shape != logits.shape[:-1] + each:
        raise ValueError(f"{name} is {tuple(t.shape)} on {t.device}, expected {tuple(logits.shape[:-1] + each)} on {logits.device}")


def _logits(logits):
    _check(logits, "logits")
    if logits.dim() < 1 or logits.shape[-1] < 1:
        raise ValueError("logits need a last dimension of at least 1")
    _sizes(logits.shape[-1])


def token_logprobs(logits, tokens, top=0, scale=1.0, stream=None):
    """TokenLogprobs of the rows of logits [..., vocab]: the log probability of tokens (int32 [...]; 0 for a negative one), the
    entropy, the parts of log sum exp, and the `top` most likely tokens with their log probabilities, the lower token first among equal
    logits.  Probabilities are softmax(scale * logits); logits of -inf are tokens that are ruled out."""
    lib = _lib.load()
    _logits(logits)
    lead, vocab = logits.shape[:-1], logits.shape[-1]
    if tokens is None:
        raise TypeError("tokens must be a GPU tensor of type int32")
    _per_row(tokens, "tokens", torch.int32, logits)
    if not 0 <= top <= min(vocab, 64):
        raise ValueError(f"top must be between 0 and {min(vocab, 64)}")
    with _Call(logits, stream, (logits, tokens)) as call:
        x, stride = _rows(logits)
        rows = x.shape[0]
        t = tokens.contiguous()
        logp, entropy = (torch.empty(lead, dtype=torch.float32, device=logits.device) for _ in range(2))
        lse = torch.empty((*lead, 2), dtype=torch.float32, device=logits.device)
        top_logp = torch.empty((*lead, top), dtype=torch.float32, device=logits.device) if top else None
        top_tokens = torch.empty((*lead, top), dtype=torch.int32, device=logits.device) if top else None
        need = lib.ntk_logprobs_workspace(_DTYPES[x.dtype], rows, vocab, top)
        if need < 0:
            _lib.check(need)
        work = torch.empty(need, dtype=torch.uint8, device=logits.device) if need else None
        _lib.check(lib.ntk_logprobs(_DTYPES[x.dtype], rows, vocab, _ptr(x), stride, _ptr(t), scale, top, _ptr(logp), _ptr(entropy), _ptr(lse),
                                    _ptr(top_logp), _ptr(top_tokens), _ptr(work), need, call.handle))
    if _recording() and _wanted(logits):
        logp, entropy, lse, top_logp = _unrecorded("token_logprobs", "token_logprobs_backward", (logits,), logp, entropy, lse, top_logp)
    return TokenLogprobs(logp, entropy, lse, top_logp, top_tokens)


def token_logprobs_backward(dlogp, dentropy, logits, tokens, lse, entropy, scale=1.0, inplace=False, stream=None):
    """The gradient of the logits from those of logp and entropy (float32 [...], either may be None), with the lse and entropy that
    `token_logprobs` returned.  `inplace` writes it over the logits."""
    lib = _lib.load()
    _logits(logits)
    vocab = logits.shape[-1]
    for name, t in (("tokens", tokens), ("lse", lse), ("entropy", entropy)):
        if t is None:
            raise TypeError(f"{name} must be a GPU tensor")
    _per_row(tokens, "tokens", torch.int32, logits)
    _per_row(lse, "lse", torch.float32, logits, (2,))
    for name, t in (("entropy", entropy), ("dlogp", dlogp), ("dentropy", dentropy)):
        _per_row(t, name, torch.float32, logits)
    if inplace:
        _written("token_logprobs_backward", (dlogp, dentropy), logits)
    with _Call(logits, stream, (dlogp, dentropy, logits, tokens, lse, entropy)) as call:
        x, stride = _rows(logits)
        if inplace and x.data_ptr() != logits.data_ptr():
            raise ValueError("inplace needs logits whose rows are evenly spaced and apart")
        t, lse, entropy, dlogp, dentropy = (d if d is None else d.contiguous() for d in (tokens, lse, entropy, dlogp, dentropy))
        out, out_stride = (logits, stride) if inplace else (_like(logits), vocab)
        _lib.check(lib.ntk_logprobs_bwd(_DTYPES[x.dtype], x.shape[0], vocab, _ptr(x), stride, _ptr(t), scale, _ptr(lse), _ptr(entropy),
                                        _ptr(dlogp), _ptr(dentropy), _ptr(out), out_stride, call.handle))
    if not inplace and _recording() and _wanted(dlogp, dentropy, logits, lse, entropy):
        return _unrecorded("token_logprobs_backward", "not defined", (dlogp, dentropy, logits, lse, entropy), out)[0]
    return out
