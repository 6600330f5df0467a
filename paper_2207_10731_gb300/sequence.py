"""Operators of a sequence encoder over the pooled embeddings: layer norm,
dropout, attention over packed sequences, rows of a dense table, norms between
blocks with gate and residual, and products with bias, activation and residual
(argument marshalling only, like ``binding``; the kernels are in libpss.so, their
contracts in include/pss.h).

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


def _ids(ids, device):
    _tensor(ids, "ids", device)
    if ids.dtype != torch.int64:
        raise TypeError(f"ids must be torch.int64, got {ids.dtype}")
    if not ids.is_contiguous():
        raise ValueError("ids must be contiguous")
    return ids.data_ptr()


def _type_of(dtype, name):
    if dtype not in _types:
        raise TypeError(f"{name} must be float32, bfloat16 or float16, got {dtype}")
    return _types[dtype]


def _table(t, name, device, rows=None, cols=None):
    """The row stride of a two-dimensional tensor."""
    _tensor(t, name, device)
    if t.dim() != 2 or (rows is not None and (t.shape[0] != rows or t.shape[1] != cols)):
        raise ValueError(f"{name} must have shape {'[rows, cols]' if rows is None else [rows, cols]}"
                         f", got {list(t.shape)}")
    return _rows(t, name, device)[2]


def embedding_forward(weight, ids, scale: float = 1.0, out=None, out_dtype=None, status=None,
                      stream=None):
    """scale * weight[ids], the rows of a dense table (pss_embedding_forward).

    weight: [rows, cols] float32, bfloat16 or float16; ids: int64 of any shape.  The
    result has shape [*ids.shape, cols] and ``out_dtype`` (default: weight's), or is
    ``out``.  An id outside the table, say -1 for padding, gives a zero row;
    ``status`` (int64, one value on the device) receives the smallest position of
    one, or -1."""
    if stream is not None:
        return _under(stream, embedding_forward, weight, ids, scale, out, out_dtype, status)
    device = _device()
    ws = _table(weight, "weight", device)
    rows, cols = weight.shape
    at = _ids(ids, device)
    if out is None:
        out = torch.empty((*ids.shape, cols), dtype=out_dtype or weight.dtype, device=weight.device)
        os = cols
    else:
        _tensor(out, "out", device)
        if out_dtype is not None and out.dtype != out_dtype:
            raise TypeError(f"out must be {out_dtype}, got {out.dtype}")
        if out.shape != (*ids.shape, cols):
            raise ValueError(f"out must have shape {(*ids.shape, cols)}, got {tuple(out.shape)}")
        os = _rows(out, "out", device)[2]
    rc = _lib.pss_embedding_forward(
        weight.data_ptr(), _types[weight.dtype], ws, rows, cols, at, ids.numel(), scale,
        out.data_ptr(), _type_of(out.dtype, "out_dtype"), os, _status(status, device),
        torch._C._cuda_getCurrentRawStream(device))
    if rc:
        binding._check(rc, "pss_embedding_forward")
    return out


def embedding_backward(grad, ids, rows: int, scale: float = 1.0, out=None, out_dtype=None,
                       status=None, stream=None):
    """The gradient of ``embedding_forward``'s weight for the upstream gradient ``grad``
    [*ids.shape, cols] (pss_embedding_backward): [rows, cols], zeros where no id
    names the row, in ``out_dtype`` (default: float32) or in ``out``.  Equal inputs
    give equal bits."""
    if stream is not None:
        return _under(stream, embedding_backward, grad, ids, rows, scale, out, out_dtype, status)
    device = _device()
    at = _ids(ids, device)
    _, cols, gs = _rows(grad, "grad", device)
    if grad.shape[:-1] != ids.shape:
        raise ValueError(f"grad must have shape {(*ids.shape, cols)}, got {tuple(grad.shape)}")
    if out is None:
        out = torch.empty((rows, cols), dtype=out_dtype or torch.float32, device=grad.device)
        os = cols
    else:
        _tensor(out, "out", device)
        if out_dtype is not None and out.dtype != out_dtype:
            raise TypeError(f"out must be {out_dtype}, got {out.dtype}")
        os = _table(out, "out", device, rows, cols)
    tokens = ids.numel()
    size = _lib.pss_embedding_workspace(tokens, rows, cols)
    work = torch.empty(size, dtype=torch.uint8, device=grad.device)
    rc = _lib.pss_embedding_backward(
        grad.data_ptr(), _types[grad.dtype], gs, at, tokens, scale, rows, cols, out.data_ptr(),
        _type_of(out.dtype, "out_dtype"), os, work.data_ptr(), size, _status(status, device),
        torch._C._cuda_getCurrentRawStream(device))
    if rc:
        binding._check(rc, "pss_embedding_backward")
    return out


def _gate(gate, x, name, device):
    """(data, kind, stride) of a gate: one value to each of x's, or one to a row."""
    if gate is None:
        return None, 0, 0
    _tensor(gate, name, device)
    if gate.shape == x.shape and x.shape[-1] != 1:
        return gate.data_ptr(), 2, _rows(gate, name, device, dtype=x.dtype)[2]
    if gate.shape != (*x.shape[:-1], 1):
        raise ValueError(f"{name} must have shape {tuple(x.shape)} or {(*x.shape[:-1], 1)}, "
                         f"got {tuple(gate.shape)}")
    return gate.data_ptr(), 1, _rows(gate, name, device, dtype=x.dtype)[2]


def _stream_rows(t, x, name, device):
    """The stride of the residual stream's rows: x's shape; x's type or float32."""
    stride = _rows(t, name, device, like=x)[2]
    if t.dtype != x.dtype and t.dtype != torch.float32:
        raise TypeError(f"{name} must be {x.dtype} or torch.float32, got {t.dtype}")
    return stride


def residual_norm_forward(x, residual, post_weight=None, pre_weight=None, gate=None,
                          scale: float = 1.0, eps: float = 1e-5, total=None, y=None, stream=None):
    """(total, y, post_rstd, pre_rstd): what lies between two blocks
    (pss_residual_norm_forward).  With rms(v, w) = v / sqrt(mean(v^2) + eps) * w over
    the last dimension,

        total = residual + scale * sigmoid(gate) * rms(x, post_weight)
        y = rms(total, pre_weight)

    x: the block's output, float32, bfloat16 or float16; residual: the stream, x's
    type or float32; weights: float32, either may be None (no such norm; y and its
    rstd are None then); gate: None, or logits of x's type, one to a value or one to a
    row ([..., 1]).  total (residual's type) and y (x's) go to the tensors of that name
    if given: total may be residual, y may be x.  The rstd are float32, for the
    backward call."""
    if stream is not None:
        return _under(stream, residual_norm_forward, x, residual, post_weight, pre_weight, gate,
                      scale, eps, total, y)
    device = _device()
    rows, cols, xs = _rows(x, "x", device)
    rs = _stream_rows(residual, x, "residual", device)
    pg, gates, gs = _gate(gate, x, "gate", device)
    if total is None:
        total, ts = torch.empty_like(residual, memory_format=torch.contiguous_format), cols
    else:
        ts = _rows(total, "total", device, like=x, dtype=residual.dtype)[2]
    ys = cols
    if pre_weight is None:
        if y is not None:
            raise ValueError("y needs pre_weight")
    elif y is None:
        y = torch.empty_like(x, memory_format=torch.contiguous_format)
    else:
        ys = _rows(y, "y", device, like=x, dtype=x.dtype)[2]
    post = pre = post_rstd = pre_rstd = None
    if post_weight is not None:
        post = _vector(post_weight, cols, "post_weight", device)
        post_rstd = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
    if pre_weight is not None:
        pre = _vector(pre_weight, cols, "pre_weight", device)
        pre_rstd = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
    rc = _lib.pss_residual_norm_forward(
        x.data_ptr(), _types[x.dtype], xs, residual.data_ptr(), _types[residual.dtype], rs, pg,
        gates, gs, post, pre, rows, cols, scale, eps, total.data_ptr(), ts,
        None if y is None else y.data_ptr(), ys,
        None if post is None else post_rstd.data_ptr(),
        None if pre is None else pre_rstd.data_ptr(),
        torch._C._cuda_getCurrentRawStream(device))
    if rc:
        binding._check(rc, "pss_residual_norm_forward")
    return total, y, post_rstd, pre_rstd


def residual_norm_backward(grad_total, grad_y, x, total, post_rstd, pre_rstd, post_weight=None,
                           pre_weight=None, gate=None, scale: float = 1.0, dx=None,
                           dresidual=None, dgate=None, stream=None):
    """(dx, dresidual, dgate, dpost_weight, dpre_weight) of ``residual_norm_forward``
    (pss_residual_norm_backward); None for what was not there.  grad_total: the
    gradient of total (residual's type; None: zero); grad_y: that of y (x's type; None
    without pre_weight); x, total and the rstd as the forward call took and gave
    them.  The first three go to the tensors of that name if given: dx may be x or
    grad_y, dresidual may be grad_total, dgate may be gate.  The weights' gradients
    are float32."""
    if stream is not None:
        return _under(stream, residual_norm_backward, grad_total, grad_y, x, total, post_rstd,
                      pre_rstd, post_weight, pre_weight, gate, scale, dx, dresidual, dgate)
    device = _device()
    rows, cols, xs = _rows(x, "x", device)
    ts = _stream_rows(total, x, "total", device)
    pg, gates, gs = _gate(gate, x, "gate", device)
    pt = py = None
    gts = gys = cols
    if grad_total is not None:
        gts = _rows(grad_total, "grad_total", device, like=x, dtype=total.dtype)[2]
        pt = grad_total.data_ptr()
    if (grad_y is None) != (pre_weight is None):
        raise ValueError("grad_y and pre_weight go together")
    if grad_y is not None:
        gys = _rows(grad_y, "grad_y", device, like=x, dtype=x.dtype)[2]
        py = grad_y.data_ptr()
    dxs = drs = cols
    if dx is None:
        dx = torch.empty_like(x, memory_format=torch.contiguous_format)
    else:
        dxs = _rows(dx, "dx", device, like=x, dtype=x.dtype)[2]
    if dresidual is None:
        dresidual = torch.empty_like(total, memory_format=torch.contiguous_format)
    else:
        drs = _rows(dresidual, "dresidual", device, like=x, dtype=total.dtype)[2]
    if gate is None:
        if dgate is not None:
            raise ValueError("dgate needs gate")
        pdg, dgs = None, 0
    else:
        if dgate is None:
            dgate = torch.empty_like(gate, memory_format=torch.contiguous_format)
        dgs = _rows(dgate, "dgate", device, like=gate, dtype=x.dtype)[2]
        pdg = dgate.data_ptr()
    post = pre = ppost = ppre = dpost = dpre = None
    size = 0
    if post_weight is not None or pre_weight is not None:
        both = torch.empty((2, cols), dtype=torch.float32, device=x.device)
        size = _lib.pss_residual_norm_workspace(rows, cols)
    work = torch.empty(size, dtype=torch.uint8, device=x.device)
    if post_weight is not None:
        post = _vector(post_weight, cols, "post_weight", device)
        ppost, dpost = _vector(post_rstd, rows, "post_rstd", device), both[0]
    if pre_weight is not None:
        pre = _vector(pre_weight, cols, "pre_weight", device)
        ppre, dpre = _vector(pre_rstd, rows, "pre_rstd", device), both[1]
    rc = _lib.pss_residual_norm_backward(
        pt, gts, py, gys, x.data_ptr(), _types[x.dtype], xs, total.data_ptr(), _types[total.dtype],
        ts, pg, gates, gs, post, pre, ppost, ppre, rows, cols, scale, dx.data_ptr(), dxs,
        dresidual.data_ptr(), drs, pdg, dgs, None if dpost is None else dpost.data_ptr(),
        None if dpre is None else dpre.data_ptr(), work.data_ptr(), size,
        torch._C._cuda_getCurrentRawStream(device))
    if rc:
        binding._check(rc, "pss_residual_norm_backward")
    return dx, dresidual, dgate, dpost, dpre


# pss_linear_forward_args, pss_linear_backward_args; the activations of pss_activation
_FORWARD = struct.Struct("3qPqP2qPPqPqPq4i")
_BACKWARD = struct.Struct("3qPqPqP2qPqPqP2qP4i")
_ACTIVATIONS = {None: 0, "relu": 1, "gelu": 2, "silu": 3}


def _packed(form, *values):
    """Address of a call's structure, in a buffer of this thread that the library reads
    before it returns."""
    try:
        buffer, start = _local.linear
    except AttributeError:
        buffer = bytearray(max(_FORWARD.size, _BACKWARD.size))
        start = binding.ctypes.addressof(binding.ctypes.c_char.from_buffer(buffer))
        _local.linear = buffer, start
    form.pack_into(buffer, 0, *values)
    return start


def _activation(name):
    try:
        return _ACTIVATIONS[name]
    except (KeyError, TypeError):
        raise ValueError(f"activation must be None, 'relu', 'gelu' or 'silu', got {name!r}") from None


def _half(t, name):
    if t.dtype != torch.bfloat16 and t.dtype != torch.float16:
        raise TypeError(f"{name} must be bfloat16 or float16, got {t.dtype}")


def _weight(t, name, device, dtype, shape=None):
    """(data, stride of in, stride of out) of a matrix [in, out] with one dense dimension."""
    _tensor(t, name, device)
    if t.dtype not in dtype:
        raise TypeError(f"{name} must be {' or '.join(map(str, dtype))}, got {t.dtype}")
    if t.dim() != 2 or (shape is not None and t.shape != shape):
        raise ValueError(f"{name} must have shape {'[in, out]' if shape is None else list(shape)}, "
                         f"got {list(t.shape)}")
    return t.data_ptr(), *t.stride()


def _result(out, like, cols, dtype, name, device):
    """A tensor [..., cols] over the rows of ``like``, made here or given, and its row stride."""
    shape = (*like.shape[:-1], cols)
    if out is None:
        return torch.empty(shape, dtype=dtype, device=like.device), cols
    _tensor(out, name, device)
    if out.shape != shape:
        raise ValueError(f"{name} must have shape {shape}, got {tuple(out.shape)}")
    return out, _rows(out, name, device, dtype=dtype)[2]


def linear_forward(x, weight, bias=None, activation=None, residual=None, keep: bool = False,
                   out=None, out_dtype=None, status=None, stream=None):
    """act(x @ weight + bias) + residual (pss_linear_forward); (that, z) with ``keep``,
    where z = x @ weight + bias in x's type is what the backward call needs of an
    activation.

    x: bfloat16 or float16 [..., in], rows evenly spaced; weight: x's type, [in, out]
    with either dimension dense (the transpose of an [out, in] tensor will do); bias:
    float32 [out]; activation: None, "relu", "gelu" (the exact form) or "silu";
    residual: [..., out] of the result's type.  The result has ``out_dtype`` (x's type,
    the default, or float32) or is ``out``, which may be residual.  Sums are fp32;
    each result is rounded once.  ``status`` (int64, one value on the device)
    receives -1, or -2 if a device wait gave up (the results are undefined then)."""
    if stream is not None:
        return _under(stream, linear_forward, x, weight, bias, activation, residual, keep, out,
                      out_dtype, status)
    device = _device()
    act = _activation(activation)
    if keep and not act:
        raise ValueError("keep needs an activation")
    tokens, n, xs = _rows(x, "x", device)
    _half(x, "x")
    pw, wi, wo = _weight(weight, "weight", device, (x.dtype,))
    m = weight.shape[1]
    if weight.shape[0] != n:
        raise ValueError(f"weight must have {n} rows, got {weight.shape[0]}")
    if out is not None:
        _tensor(out, "out", device)
    kind = out.dtype if out is not None and out_dtype is None else out_dtype or x.dtype
    if kind != x.dtype and kind != torch.float32:
        raise TypeError(f"out_dtype must be {x.dtype} or torch.float32, got {kind}")
    out, ys = _result(out, x, m, kind, "out", device)
    pr = pz = None
    rs = zs = m
    if residual is not None:
        rs = _rows(residual, "residual", device, like=out, dtype=kind)[2]
        pr = residual.data_ptr()
    if keep:
        z = torch.empty(out.shape, dtype=x.dtype, device=x.device)
        pz = z.data_ptr()
    pb = None if bias is None else _vector(bias, m, "bias", device)
    at = _packed(_FORWARD, tokens, n, m, x.data_ptr(), xs, pw, wi, wo, pb or 0, pr or 0, rs,
                 out.data_ptr(), ys, pz or 0, zs, _types[x.dtype], _types[kind], act, 0)
    size = _lib.pss_linear_forward_workspace(at)
    work = torch.empty(size, dtype=torch.uint8, device=x.device) if size else None
    rc = _lib.pss_linear_forward(at, work.data_ptr() if size else None, size,
                                 _status(status, device),
                                 torch._C._cuda_getCurrentRawStream(device))
    if rc:
        binding._check(rc, "pss_linear_forward")
    return (out, z) if keep else out


def linear_backward(grad, x, weight, z=None, activation=None, dx=True, dweight=True, dbias=True,
                    dweight_dtype=None, status=None, stream=None):
    """(dx, dweight, dbias) of ``linear_forward`` for the upstream gradient ``grad``
    [..., out] (pss_linear_backward), which itself is the residual's gradient.

    grad: x's type or float32; z: the forward call's, with an activation.  Each of
    dx, dweight and dbias is True, False (not wanted: None is returned) or the
    tensor to fill.  dx has x's type and shape; dweight lies in memory as weight does,
    in ``dweight_dtype`` (weight's type, the default, or float32); dbias is float32.
    They may not overlap the inputs or each other.
    grad * act'(z) enters the products rounded to x's type, and dbias unrounded."""
    if stream is not None:
        return _under(stream, linear_backward, grad, x, weight, z, activation, dx, dweight, dbias,
                      dweight_dtype, status)
    device = _device()
    act = _activation(activation)
    tokens, n, xs = _rows(x, "x", device)
    _half(x, "x")
    pw, wi, wo = _weight(weight, "weight", device, (x.dtype,))
    m = weight.shape[1]
    if weight.shape[0] != n:
        raise ValueError(f"weight must have {n} rows, got {weight.shape[0]}")
    _, gm, gs = _rows(grad, "grad", device)
    if grad.shape[:-1] != x.shape[:-1] or gm != m:
        raise ValueError(f"grad must have shape {(*x.shape[:-1], m)}, got {tuple(grad.shape)}")
    if grad.dtype != x.dtype and grad.dtype != torch.float32:
        raise TypeError(f"grad must be {x.dtype} or torch.float32, got {grad.dtype}")
    pz, zs = 0, m
    if act:
        if z is None:
            raise ValueError("z is needed with an activation")
        zs = _rows(z, "z", device, like=grad, dtype=x.dtype)[2]
        pz = z.data_ptr()
    px = pdw = pb = 0
    dxs, dwi, dwo = n, 0, 0
    kind = weight.dtype
    if dx is False or dx is None:
        dx = None
    else:
        dx, dxs = _result(None if dx is True else dx, x, n, x.dtype, "dx", device)
        px = dx.data_ptr()
    if dweight is False or dweight is None:
        dweight = None
    else:
        if dweight is True:
            kind = dweight_dtype or weight.dtype
            if wo == 1 or m == 1:
                dweight = torch.empty((n, m), dtype=kind, device=x.device)
            else:
                dweight = torch.empty((m, n), dtype=kind, device=x.device).t()
        else:
            _tensor(dweight, "dweight", device)
            if dweight_dtype is not None and dweight.dtype != dweight_dtype:
                raise TypeError(f"dweight must be {dweight_dtype}, got {dweight.dtype}")
        pdw, dwi, dwo = _weight(dweight, "dweight", device, (x.dtype, torch.float32), weight.shape)
        kind = dweight.dtype
    if dbias is False or dbias is None:
        dbias = None
    else:
        if dbias is True:
            dbias = torch.empty(m, dtype=torch.float32, device=x.device)
        pb = _vector(dbias, m, "dbias", device)
    at = _packed(_BACKWARD, tokens, n, m, grad.data_ptr(), gs, x.data_ptr(), xs, pw, wi, wo, pz, zs,
                 px, dxs, pdw, dwi, dwo, pb, _types[x.dtype], _types[grad.dtype], _types[kind], act)
    size = _lib.pss_linear_backward_workspace(at)
    work = torch.empty(size, dtype=torch.uint8, device=x.device) if size else None
    rc = _lib.pss_linear_backward(at, work.data_ptr() if size else None, size,
                                  _status(status, device),
                                  torch._C._cuda_getCurrentRawStream(device))
    if rc:
        binding._check(rc, "pss_linear_backward")
    return dx, dweight, dbias
