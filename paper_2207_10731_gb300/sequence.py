"""Operators of a sequence encoder over the pooled embeddings: layer norm,
dropout and attention over packed sequences (argument marshalling only, like
``binding``; the kernels are in libpss.so, their contracts in include/pss.h).

All tensors are CUDA tensors of the current device; calls are asynchronous on
``stream`` (a keyword of each; default: the current stream), to which the
results belong.  Nothing is kept between calls.  Gradients are explicit calls:
there is no autograd graph here.
"""
from __future__ import annotations

import struct
import threading

from . import binding

_lib = torch = None
_types = {}
_local = threading.local()
# pss_attention_shape, then up to ten pss_rows
_SHAPE = struct.Struct("5q4if4x")
_ROWS = struct.Struct("Pqq")


def _library():
    global _lib, torch
    if _lib is None:
        torch = binding._torch()
        torch.cuda.init()
        _types.update({torch.float32: 0, torch.bfloat16: 1, torch.float16: 2})   # pss_dtype
        _lib = binding.load_library()
    return _lib


def _under(stream, call, *args, **kwargs):
    """The call with ``stream`` as the current stream, so that what it allocates
    belongs to the stream that uses it."""
    _library()
    with torch.cuda.stream(stream):
        return call(*args, **kwargs)


def _device():
    """The current device, with the library loaded."""
    if _lib is None:
        _library()
    return torch._C._cuda_getDevice()


def _tensor(t, name, device):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.get_device() != device:
        raise ValueError(f"{name} must be on the current CUDA device")


def _rows(t, name, device, like=None, dtype=None):
    """(rows, cols, stride) of a tensor seen as rows of its last dimension,
    which must be dense; the leading dimensions must be one stride apart."""
    _tensor(t, name, device)
    if t.dtype not in _types:
        raise TypeError(f"{name} must be float32, bfloat16 or float16, got {t.dtype}")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    shape = t.shape
    if like is not None and shape != like.shape:
        raise ValueError(f"{name} must have shape {tuple(like.shape)}, got {tuple(shape)}")
    if not shape:
        raise ValueError(f"{name} must have at least one dimension")
    cols = shape[-1]
    if t.is_contiguous():
        return (t.numel() // cols if cols else 0), cols, cols
    strides = t.stride()
    if cols > 1 and strides[-1] != 1:
        raise ValueError(f"{name} must be dense in its last dimension")
    if t.numel() == 0:
        return 0, cols, max(cols, 1)
    rows, stride = 1, None
    for n, s in zip(reversed(shape[:-1]), reversed(strides[:-1])):
        if n == 1:
            continue
        if stride is None:
            stride = s
        elif s != stride * rows:
            raise ValueError(f"{name}'s rows must be evenly spaced")
        rows *= n
    if stride is None:
        stride = cols
    if stride < cols:
        raise ValueError(f"{name}'s rows must not overlap")
    return rows, cols, stride


def _vector(t, n, name, device):
    _tensor(t, name, device)
    if t.dtype != torch.float32:
        raise TypeError(f"{name} must be torch.float32, got {t.dtype}")
    if t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous with {n} values")
    return t.data_ptr()


def layer_norm_forward(x, weight, bias, eps: float = 1e-5, out=None, out_dtype=None, stream=None):
    """(y, mean, rstd) of the layer norm over x's last dimension
    (pss_layer_norm_forward).  ``x``: float32, bfloat16 or float16, rows evenly
    spaced; ``weight``, ``bias``: float32.  y has ``out_dtype`` (default: x's)
    or is ``out``; mean and rstd are float32, for the backward call."""
    if stream is not None:
        return _under(stream, layer_norm_forward, x, weight, bias, eps, out, out_dtype)
    device = _device()
    rows, cols, xs = _rows(x, "x", device)
    if out is None:
        out = torch.empty(x.shape, dtype=out_dtype or x.dtype, device=x.device)
        if out.dtype not in _types:
            raise TypeError(f"out_dtype must be float32, bfloat16 or float16, got {out.dtype}")
        ys = cols
    else:
        if out_dtype is not None and out.dtype != out_dtype:
            raise TypeError(f"out must be {out_dtype}, got {out.dtype}")
        _, _, ys = _rows(out, "out", device, like=x)
    mean = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
    rstd = torch.empty_like(mean)
    rc = _lib.pss_layer_norm_forward(
        x.data_ptr(), _types[x.dtype], xs, _vector(weight, cols, "weight", device),
        _vector(bias, cols, "bias", device), rows, cols, eps, out.data_ptr(), _types[out.dtype], ys,
        mean.data_ptr(), rstd.data_ptr(), torch._C._cuda_getCurrentRawStream(device))
    if rc:
        binding._check(rc, "pss_layer_norm_forward")
    return out, mean, rstd


def layer_norm_backward(grad, x, weight, mean, rstd, out=None, stream=None):
    """(dx, dweight, dbias) for the upstream gradient ``grad`` of the y of
    ``layer_norm_forward(x, weight, ...)`` (pss_layer_norm_backward).  dx has
    x's type or is ``out``; dweight and dbias are float32."""
    if stream is not None:
        return _under(stream, layer_norm_backward, grad, x, weight, mean, rstd, out)
    device = _device()
    rows, cols, xs = _rows(x, "x", device)
    _, _, gs = _rows(grad, "grad", device, like=x)
    if out is None:
        out, ds = torch.empty_like(x, memory_format=torch.contiguous_format), cols
    else:
        _, _, ds = _rows(out, "out", device, like=x, dtype=x.dtype)
    both = torch.empty((2, cols), dtype=torch.float32, device=x.device)
    size = _lib.pss_layer_norm_workspace(rows, cols)
    work = torch.empty(size, dtype=torch.uint8, device=x.device)
    rc = _lib.pss_layer_norm_backward(
        grad.data_ptr(), _types[grad.dtype], gs, x.data_ptr(), _types[x.dtype], xs,
        _vector(weight, cols, "weight", device), _vector(mean, rows, "mean", device),
        _vector(rstd, rows, "rstd", device), rows, cols, out.data_ptr(), ds, both.data_ptr(),
        both.data_ptr() + 4 * cols, work.data_ptr(), size,
        torch._C._cuda_getCurrentRawStream(device))
    if rc:
        binding._check(rc, "pss_layer_norm_backward")
    return out, both[0], both[1]


def dropout(x, p: float, seed: int, offset: int = 0, residual=None, out=None, stream=None):
    """x with each element zeroed with probability p and the others divided by
    1 - p, plus ``residual`` (pss_dropout).  The mask follows from (seed,
    offset, position) alone and is not stored: the backward pass is the same
    call on the gradient, without the residual.  seed and offset are unsigned
    64-bit; give each call of a step an offset of its own.  Both are values of
    the call: a captured CUDA graph repeats its mask at every replay."""
    if stream is not None:
        return _under(stream, dropout, x, p, seed, offset, residual, out)
    device = _device()
    rows, cols, xs = _rows(x, "x", device)
    more, rs = None, 0
    if residual is not None:
        _, _, rs = _rows(residual, "residual", device, like=x, dtype=x.dtype)
        more = residual.data_ptr()
    if out is None:
        out, ys = torch.empty_like(x, memory_format=torch.contiguous_format), cols
    else:
        _, _, ys = _rows(out, "out", device, like=x, dtype=x.dtype)
    if not (0 <= seed < 2**64 and 0 <= offset < 2**64):
        raise ValueError("seed and offset must be unsigned 64-bit integers")
    rc = _lib.pss_dropout(x.data_ptr(), xs, more, rs, rows, cols, p, seed, offset, _types[x.dtype],
                          out.data_ptr(), ys, torch._C._cuda_getCurrentRawStream(device))
    if rc:
        binding._check(rc, "pss_dropout")
    return out


def _heads(t, name, device, shape=None):
    """(data, token stride, head stride) of a bfloat16 tensor [tokens, heads,
    dim], dense in its last dimension."""
    _tensor(t, name, device)
    if t.dtype != torch.bfloat16:
        raise TypeError(f"{name} must be torch.bfloat16, got {t.dtype}")
    own = t.shape
    if len(own) != 3 or (shape is not None and own != shape):
        raise ValueError(f"{name} must have shape {tuple(shape) if shape else '[tokens, heads, dim]'}"
                         f", got {tuple(own)}")
    token, head, one = t.stride()
    if one != 1 and own[2] > 1:
        raise ValueError(f"{name} must be dense in its last dimension")
    # the stride over a size of one means nothing
    return t.data_ptr(), token if own[0] != 1 else 0, head if own[1] != 1 else 0


def _made(t):
    """The same of a tensor made here."""
    _, heads, dim = t.shape
    return t.data_ptr(), heads * dim if t.shape[0] != 1 else 0, dim if heads != 1 else 0


def _structs(shape, *rows):
    """Addresses of the structures of one call, in a buffer of this thread that
    the library reads before it returns."""
    try:
        buffer, start = _local.buffer
    except AttributeError:
        buffer = bytearray(_SHAPE.size + 10 * _ROWS.size)
        start = binding.ctypes.addressof(binding.ctypes.c_char.from_buffer(buffer))
        _local.buffer = buffer, start
    _SHAPE.pack_into(buffer, 0, *shape)
    at, where = _SHAPE.size, [start]
    for r in rows:
        _ROWS.pack_into(buffer, at, *r)
        where.append(start + at)
        at += _ROWS.size
    return where


def _offsets(t, name, device):
    _tensor(t, name, device)
    if t.dtype != torch.int64:
        raise TypeError(f"{name} must be torch.int64, got {t.dtype}")
    if t.dim() != 1 or t.numel() < 1 or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous with at least one entry")
    return t


def _attention_shape(q, k, q_offsets, kv_offsets, causal, scale, device):
    n = _offsets(q_offsets, "q_offsets", device).numel()
    if kv_offsets is None:
        kv_offsets = q_offsets
    elif _offsets(kv_offsets, "kv_offsets", device).numel() != n:
        raise ValueError("q_offsets and kv_offsets must have the same number of entries")
    tokens, heads, dim = q.shape
    k_tokens, kv_heads, k_dim = k.shape
    if k_dim != dim:
        raise ValueError(f"k must have rows of {dim} values, got {k_dim}")
    return (n - 1, q_offsets.data_ptr(), kv_offsets.data_ptr(), tokens, k_tokens, heads, kv_heads,
            dim, 1 if causal else 0, dim ** -0.5 if scale is None else scale)


def _status(status, device):
    if status is None:
        return None
    _tensor(status, "status", device)
    if status.dtype != torch.int64 or status.numel() != 1:
        raise TypeError("status must be a torch.int64 tensor of one value")
    return status.data_ptr()


def attention_forward(q, k, v, q_offsets, kv_offsets=None, causal: bool = True, scale=None,
                      out=None, status=None, stream=None):
    """(out, lse) of softmax(scale q k^T) v inside each packed sequence
    (pss_attention_forward).

    q: bfloat16 [query tokens, heads, dim]; k, v: [key tokens, kv heads, dim]
    (views with any token and head strides that are multiples of 8; heads a
    multiple of kv heads; dim a multiple of 8 up to 128).  Sequence s owns the
    rows q_offsets[s] .. q_offsets[s+1] and kv_offsets[s] .. (int64, on the
    device; kv_offsets defaults to q_offsets).  With ``causal`` the queries
    stand at the end of their sequence: one query per sequence is the serving
    step.  scale defaults to dim ** -0.5.  lse is float32 [query tokens,
    heads].  ``status`` (int64, one value on the device) receives -1, the first
    sequence with malformed offsets (no result is defined then), or -2 if a
    device wait gave up.  Rows outside every sequence are left as they are, in
    results made here whatever the memory held."""
    if stream is not None:
        return _under(stream, attention_forward, q, k, v, q_offsets, kv_offsets, causal, scale, out,
                      status)
    device = _device()
    rq, rk, rv = _heads(q, "q", device), _heads(k, "k", device), _heads(v, "v", device, k.shape)
    shape = _attention_shape(q, k, q_offsets, kv_offsets, causal, scale, device)
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        ro = _made(out)
    else:
        ro = _heads(out, "out", device, q.shape)
    at = _structs(shape, rq, rk, rv, ro)
    lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
    size = _lib.pss_attention_workspace(at[0], 0)
    work = torch.empty(size, dtype=torch.uint8, device=q.device)
    rc = _lib.pss_attention_forward(*at, lse.data_ptr(), work.data_ptr(), size,
                                    _status(status, device),
                                    torch._C._cuda_getCurrentRawStream(device))
    if rc:
        binding._check(rc, "pss_attention_forward")
    return out, lse


def attention_backward(grad, q, k, v, out, lse, q_offsets, kv_offsets=None, causal: bool = True,
                       scale=None, grads=None, status=None, stream=None):
    """(dq, dk, dv) for the upstream gradient ``grad`` of the out of
    ``attention_forward`` (pss_attention_backward); out and lse are that
    call's.  The gradients go to the three tensors ``grads`` if given (e.g.
    views of one buffer for a fused projection).  Rows outside every sequence
    are left as they are, as in the forward call."""
    if stream is not None:
        return _under(stream, attention_backward, grad, q, k, v, out, lse, q_offsets, kv_offsets,
                      causal, scale, grads, status)
    device = _device()
    rq, rk, rv = _heads(q, "q", device), _heads(k, "k", device), _heads(v, "v", device, k.shape)
    rg, ro = _heads(grad, "grad", device, q.shape), _heads(out, "out", device, q.shape)
    shape = _attention_shape(q, k, q_offsets, kv_offsets, causal, scale, device)
    if lse.shape != q.shape[:2]:
        raise ValueError(f"lse must have shape {tuple(q.shape[:2])}, got {tuple(lse.shape)}")
    pl = _vector(lse, lse.numel(), "lse", device)
    if grads is None:
        dq = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        dk = torch.empty(k.shape, dtype=k.dtype, device=k.device)
        dv = torch.empty(v.shape, dtype=v.dtype, device=v.device)
        to = _made(dq), _made(dk), _made(dv)
    else:
        dq, dk, dv = grads
        to = (_heads(dq, "dq", device, q.shape), _heads(dk, "dk", device, k.shape),
              _heads(dv, "dv", device, v.shape))
    at = _structs(shape, rg, rq, rk, rv, ro, *to)
    size = _lib.pss_attention_workspace(at[0], 1)
    work = torch.empty(size, dtype=torch.uint8, device=q.device)
    rc = _lib.pss_attention_backward(*at[:6], pl, *at[6:], work.data_ptr(), size,
                                     _status(status, device),
                                     torch._C._cuda_getCurrentRawStream(device))
    if rc:
        binding._check(rc, "pss_attention_backward")
    return dq, dk, dv
