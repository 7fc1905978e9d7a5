"""Operators of the models that the nodes train: dropout, residual root-mean-square norm, cross attention.

Bindings of the C entry points of the same names (include/swarm.h says what each computes): checks of torch tensors,
allocation of outputs and scratch through torch, the current stream. Forward and backward are separate calls; nothing
is recorded for automatic differentiation. Refused arguments raise ValueError or SwarmError before anything is
launched. There is no CPU path.
"""
import ctypes as C
import struct

import torch

from . import binding as _b

_DTYPES = {torch.float32: _b.F32, torch.bfloat16: _b.BF16, torch.float16: _b.F16}
_DESC = struct.Struct("=7ifq2Q24q")       # swarm_attention: 8 strided tensors of 3 strides at the end
_workspace_bytes = C.c_size_t()


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _check(rc, what):
    if rc != 0:
        raise _b.SwarmError(rc, what)


def _on_device(x, name, dtype=None):
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise ValueError(f"{name}: a CUDA tensor is needed; this library has no CPU path")
    if x.get_device() != torch.cuda.current_device():
        raise ValueError(f"{name}: not on the current CUDA device")
    if dtype is not None and x.dtype != dtype:
        raise ValueError(f"{name}: {dtype} is needed, got {x.dtype}")


def _rows(x, name, like=None):
    """(tensor, rows, cols, pitch) of a tensor whose last dimension is consecutive and whose others collapse into one."""
    _on_device(x, name, None if like is None else like.dtype)
    if like is not None and x.shape != like.shape:
        raise ValueError(f"{name}: shape {tuple(x.shape)}, expected {tuple(like.shape)}")
    if x.dtype not in _DTYPES:
        raise ValueError(f"{name}: float32, bfloat16 or float16 is needed, got {x.dtype}")
    if x.dim() == 0:
        raise ValueError(f"{name}: at least one dimension is needed")
    cols = x.shape[-1]
    if x.is_contiguous():
        return x, (x.numel() // cols if cols else 0), cols, cols
    if x.stride(-1) != 1 and cols > 1:
        raise ValueError(f"{name}: the last dimension has to be consecutive")
    try:
        flat = x.view(-1, cols)
    except RuntimeError:
        raise ValueError(f"{name}: the leading dimensions do not collapse into rows at one pitch") from None
    pitch = flat.stride(0) if flat.shape[0] > 1 else cols
    return flat, flat.shape[0], cols, pitch


def _mask(rate, seed, event):
    if not 0.0 <= rate <= 1.0:
        raise ValueError("rate: between 0 and 1")
    if not 0 <= seed < 2 ** 64 or not 0 <= event < 2 ** 32:
        raise ValueError("seed: 64 bits, event: 32 bits, unsigned")


def dropout(x, rate, seed, event, residual=None, out=None):
    """residual + m * x with the mask of (seed, event); rows of x are its last dimension. The gradient with respect
    to x is dropout(dout, rate, seed, event). `out` may be x or residual."""
    _mask(rate, seed, event)
    fx, rows, cols, px = _rows(x, "x")
    pr = cols
    if residual is not None:
        residual, _, _, pr = _rows(residual, "residual", x)
    if out is None:
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        po = cols
    else:
        _, _, _, po = _rows(out, "out", x)
    _check(_b.load().swarm_dropout(fx.data_ptr(), residual.data_ptr() if residual is not None else None, out.data_ptr(),
                                   rows, cols, px, pr, po, _DTYPES[x.dtype], rate, seed, event, _stream()), "swarm_dropout")
    return out


def add_rms_norm(x, weight, residual=None, eps=1e-6, rate=0.0, seed=0, event=0, eight_bit=False):
    """(y, total): total = residual + m * x and y = weight * total / rms(total). With `eight_bit` (codes, scales, total):
    y in e4m3 with one float32 scale for each 128 columns of a row, y ~ codes * scales. Without a residual and with
    rate 0 the total is x itself."""
    _mask(rate, seed, event)
    fx, rows, cols, px = _rows(x, "x")
    _on_device(weight, "weight", torch.float32)
    if weight.shape != (cols,) or (cols > 1 and weight.stride(0) != 1):
        raise ValueError("weight: cols consecutive values are needed")
    pr = cols
    if residual is not None:
        residual, _, _, pr = _rows(residual, "residual", x)
    plain = residual is None and rate == 0.0
    total = x if plain else torch.empty(x.shape, dtype=x.dtype, device=x.device)
    y = torch.empty(x.shape, dtype=torch.float8_e4m3fn if eight_bit else x.dtype, device=x.device)
    scales = torch.empty(x.shape[:-1] + ((cols + 127) // 128,), dtype=torch.float32, device=x.device) if eight_bit else None
    _check(_b.load().swarm_add_rms_norm(
        fx.data_ptr(), residual.data_ptr() if residual is not None else None, weight.data_ptr(),
        None if plain else total.data_ptr(), None if eight_bit else y.data_ptr(), y.data_ptr() if eight_bit else None,
        scales.data_ptr() if eight_bit else None, rows, cols, px, pr, cols, cols, _DTYPES[x.dtype], eps, rate, seed, event,
        _stream()), "swarm_add_rms_norm")
    return (y, scales, total) if eight_bit else (y, total)


def add_rms_norm_backward(dy, total, weight, dtotal=None, eps=1e-6, rate=0.0, seed=0, event=0):
    """(dx, dresidual, dweight) of add_rms_norm at the total that it returned; `dtotal` is the gradient that reaches
    the total past the norm. dx is dresidual itself when rate is 0."""
    _mask(rate, seed, event)
    fd, rows, cols, pd = _rows(dy, "dy")
    ft, _, _, pt = _rows(total, "total", dy)
    _on_device(weight, "weight", torch.float32)
    if weight.shape != (cols,) or (cols > 1 and weight.stride(0) != 1):
        raise ValueError("weight: cols consecutive values are needed")
    pa = cols
    if dtotal is not None:
        dtotal, _, _, pa = _rows(dtotal, "dtotal", dy)
    L = _b.load()
    dresidual = torch.empty(dy.shape, dtype=dy.dtype, device=dy.device)
    dx = torch.empty(dy.shape, dtype=dy.dtype, device=dy.device) if rate > 0.0 else None
    dweight = torch.empty(cols, dtype=torch.float32, device=dy.device)
    nbytes = L.swarm_add_rms_norm_workspace(rows, cols)
    work = torch.empty(nbytes, dtype=torch.uint8, device=dy.device)
    _check(L.swarm_add_rms_norm_backward(
        fd.data_ptr(), dtotal.data_ptr() if dtotal is not None else None, ft.data_ptr(), weight.data_ptr(),
        dresidual.data_ptr(), dx.data_ptr() if dx is not None else None, dweight.data_ptr(), rows, cols, pd, pa, pt, cols,
        cols, _DTYPES[dy.dtype], eps, rate, seed, event, work.data_ptr(), nbytes, _stream()), "swarm_add_rms_norm_backward")
    return (dx if dx is not None else dresidual), dresidual, dweight


def _heads(x, name, like=None, shape=None):
    _on_device(x, name, like)
    if x.dim() != 4:
        raise ValueError(f"{name}: [batch, tokens, heads, head_dim] is needed")
    if shape is not None and tuple(x.shape) != shape:
        raise ValueError(f"{name}: shape {tuple(x.shape)}, expected {shape}")
    s = x.stride()
    if s[3] != 1 and x.shape[3] > 1:
        raise ValueError(f"{name}: the values of a head have to be consecutive")
    return s[0], s[1], s[2]


def _lengths(x, name, batch):
    if x is None:
        return 0
    _on_device(x, name, torch.int32)
    if x.shape != (batch,) or (batch > 1 and x.stride(0) != 1):
        raise ValueError(f"{name}: one consecutive int32 for each sentence is needed")
    return x.data_ptr()


def _attention_desc(q, k, v, o, scale, query_lengths, key_lengths, wait_limit, grads=()):
    qs = _heads(q, "q")
    b, tq, h, d = q.shape
    ks = _heads(k, "k", q.dtype)
    tk, hk = k.shape[1], k.shape[2]
    kv = (b, tk, hk, d)
    if tuple(k.shape) != kv:
        raise ValueError(f"k: shape {tuple(k.shape)} does not go with q's {tuple(q.shape)}")
    vs = _heads(v, "v", q.dtype, kv)
    os_ = _heads(o, "o", q.dtype, (b, tq, h, d))
    extra = (0,) * 12
    if grads:
        do, dq, dk, dv = grads
        whole = tuple(q.shape)
        extra = (_heads(do, "do", q.dtype, whole) + _heads(dq, "dq", q.dtype, whole) + _heads(dk, "dk", q.dtype, kv)
                 + _heads(dv, "dv", q.dtype, kv))
    if q.dtype not in (torch.bfloat16, torch.float16):
        raise ValueError(f"q: bfloat16 or float16 is needed, got {q.dtype}")
    return _DESC.pack(b, h, hk, tq, tk, d, _DTYPES[q.dtype], d ** -0.5 if scale is None else scale, wait_limit,
                      _lengths(query_lengths, "query_lengths", b), _lengths(key_lengths, "key_lengths", b),
                      *qs, *ks, *vs, *os_, *extra)


def _workspace(L, desc, backward, device):
    _check(L.swarm_cross_attention_workspace(desc, backward, C.byref(_workspace_bytes)), "swarm_cross_attention_workspace")
    n = _workspace_bytes.value
    return (torch.empty(n, dtype=torch.uint8, device=device) if n else None), n


def cross_attention(q, k, v, scale=None, query_lengths=None, key_lengths=None, need_lse=False, out=None, wait_limit=-1):
    """o (or (o, lse) with `need_lse`) of q [batch, queries, heads, head_dim] over k, v [batch, keys, kv_heads,
    head_dim]; any strides over the first three dimensions that are multiples of 8 elements. scale: 1 / sqrt(head_dim)
    unless given. query_lengths, key_lengths: int32 [batch] on the device, or None. One to a few query rows (a decoding
    step) take the same call."""
    L = _b.load()
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    desc = _attention_desc(q, k, v, out, scale, query_lengths, key_lengths, wait_limit)
    lse = torch.empty(q.shape[0], q.shape[2], q.shape[1], dtype=torch.float32, device=q.device) if need_lse else None
    work, nbytes = _workspace(L, desc, 0, q.device)
    _check(L.swarm_cross_attention(desc, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
                                   lse.data_ptr() if need_lse else None, work.data_ptr() if nbytes else None, nbytes,
                                   _stream()), "swarm_cross_attention")
    return (out, lse) if need_lse else out


def cross_attention_backward(do, q, k, v, o, lse, scale=None, query_lengths=None, key_lengths=None, dq=None, dk=None,
                             dv=None, wait_limit=-1):
    """(dq, dk, dv) from the gradient of o and what the forward call took and returned. dq, dk, dv may be given (for
    example as views of one packed gradient); dk and dv of a key head are sums over its query heads."""
    L = _b.load()
    dq = torch.empty(q.shape, dtype=q.dtype, device=q.device) if dq is None else dq
    dk = torch.empty(k.shape, dtype=k.dtype, device=k.device) if dk is None else dk
    dv = torch.empty(v.shape, dtype=v.dtype, device=v.device) if dv is None else dv
    desc = _attention_desc(q, k, v, o, scale, query_lengths, key_lengths, wait_limit, (do, dq, dk, dv))
    _on_device(lse, "lse", torch.float32)
    if lse.shape != (q.shape[0], q.shape[2], q.shape[1]) or not lse.is_contiguous():
        raise ValueError("lse: contiguous [batch, heads, queries] as the forward call returned it")
    work, nbytes = _workspace(L, desc, 1, q.device)
    _check(L.swarm_cross_attention_backward(desc, do.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
                                            lse.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
                                            work.data_ptr() if nbytes else None, nbytes, _stream()),
           "swarm_cross_attention_backward")
    return dq, dk, dv


def check():
    """Waits for the current stream; raises SwarmError if a device-side wait of an operator has given up since the
    last check, or the stream holds a CUDA error."""
    _check(_b.load().swarm_operator_check(_stream()), "swarm_operator_check")
