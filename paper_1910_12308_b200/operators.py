"""Operators of the models that the nodes train: dropout, residual root-mean-square norm, cross attention.

Bindings of the C entry points of the same names (include/swarm.h says what each computes): checks of torch tensors,
allocation of outputs and scratch through torch, the current stream. Forward and backward are separate calls; nothing
is recorded for automatic differentiation. Refused arguments raise ValueError or SwarmError before anything is
launched. There is no CPU path.

A decoding step makes these calls in a loop on tiny tensors, where the host's time is all that counts: tensors are looked
at through the cheapest attributes that say enough, contiguous ones first.
"""
import ctypes as C
import struct

import torch

from . import binding as _b

_DTYPES = {torch.float32: _b.F32, torch.bfloat16: _b.BF16, torch.float16: _b.F16}
_DESC = struct.Struct("=7ifq2Q24q")                        # swarm_attention: 8 tensors of 3 strides at the end
_NO_GRADS = (0,) * 12

_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
if _raw_stream is None:
    def _raw_stream(device):
        return torch.cuda.current_stream(device).cuda_stream


def _check(rc, what):
    if rc != 0:
        raise _b.SwarmError(rc, what)


def _device(x, name):
    """The device of the call: that of its first tensor, which has to be the current one."""
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise ValueError(f"{name}: a CUDA tensor is needed; this library has no CPU path")
    device = x.get_device()
    if device != _current_device():
        raise ValueError(f"{name}: not on the current CUDA device")
    return device


def _same(x, name, device, dtype):
    if not isinstance(x, torch.Tensor) or x.get_device() != device:
        raise ValueError(f"{name}: a tensor on the call's CUDA device is needed")
    if x.dtype != dtype:
        raise ValueError(f"{name}: {dtype} is needed, got {x.dtype}")


def _rows(x, name):
    """(pointer, rows, cols, pitch) of a tensor whose last dimension is consecutive and whose others collapse into one."""
    if x.dim() == 0:
        raise ValueError(f"{name}: at least one dimension is needed")
    cols = x.shape[-1]
    if x.is_contiguous():
        return x.data_ptr(), (x.numel() // cols if cols else 0), cols, cols
    if x.stride(-1) != 1 and cols > 1:
        raise ValueError(f"{name}: the last dimension has to be consecutive")
    try:
        flat = x.view(-1, cols)
    except RuntimeError:
        raise ValueError(f"{name}: the leading dimensions do not collapse into rows at one pitch") from None
    return flat.data_ptr(), flat.shape[0], cols, flat.stride(0) if flat.shape[0] > 1 else cols


def _like(x, name, device, other, cols):
    """(pointer, pitch) of a tensor of the same shape and type as `other`; (None, cols) for None."""
    if x is None:
        return None, cols
    _same(x, name, device, other.dtype)
    if x.shape != other.shape:
        raise ValueError(f"{name}: shape {tuple(x.shape)}, expected {tuple(other.shape)}")
    if x.is_contiguous():
        return x.data_ptr(), cols
    ptr, _, _, pitch = _rows(x, name)
    return ptr, pitch


def _empty(x):
    return torch.empty_like(x) if x.is_contiguous() else torch.empty(x.shape, dtype=x.dtype, device=x.device)


def _dtype(x, name):
    code = _DTYPES.get(x.dtype)
    if code is None:
        raise ValueError(f"{name}: float32, bfloat16 or float16 is needed, got {x.dtype}")
    return code


def _mask(rate, seed, event):
    if not 0.0 <= rate <= 1.0:
        raise ValueError("rate: between 0 and 1")
    if not 0 <= seed < 2 ** 64 or not 0 <= event < 2 ** 32:
        raise ValueError("seed: 64 bits, event: 32 bits, unsigned")


def _weight(weight, device, cols):
    _same(weight, "weight", device, torch.float32)
    if weight.dim() != 1 or weight.shape[0] != cols or (cols > 1 and weight.stride(0) != 1):
        raise ValueError("weight: cols consecutive values are needed")
    return weight.data_ptr()


def dropout(x, rate, seed, event, residual=None, out=None):
    """residual + m * x with the mask of (seed, event); rows of x are its last dimension. The gradient with respect
    to x is dropout(dout, rate, seed, event). `out` may be x or residual."""
    _mask(rate, seed, event)
    device = _device(x, "x")
    dtype = _dtype(x, "x")
    px, rows, cols, pitch = _rows(x, "x")
    pr, res_pitch = _like(residual, "residual", device, x, cols)
    if out is None:
        out = _empty(x)
    po, out_pitch = _like(out, "out", device, x, cols)
    _check(_b.load().swarm_dropout(px, pr, po, rows, cols, pitch, res_pitch, out_pitch, dtype, rate, seed, event,
                                   _raw_stream(device)), "swarm_dropout")
    return out


def add_rms_norm(x, weight, residual=None, eps=1e-6, rate=0.0, seed=0, event=0, eight_bit=False):
    """(y, total): total = residual + m * x and y = weight * total / rms(total). With `eight_bit` (codes, scales, total):
    y in e4m3 with one float32 scale for each 128 columns of a row, y ~ codes * scales. Without a residual and with
    rate 0 the total is x itself."""
    _mask(rate, seed, event)
    device = _device(x, "x")
    dtype = _dtype(x, "x")
    px, rows, cols, pitch = _rows(x, "x")
    pw = _weight(weight, device, cols)
    pr, res_pitch = _like(residual, "residual", device, x, cols)
    if residual is None and rate == 0.0:
        total, pt = x, None
    else:
        total = _empty(x)
        pt = total.data_ptr()
    py = pc = ps = None
    if eight_bit:
        y = x.new_empty(x.shape, dtype=torch.float8_e4m3fn)
        scales = x.new_empty(x.shape[:-1] + ((cols + 127) // 128,), dtype=torch.float32)
        pc, ps = y.data_ptr(), scales.data_ptr()
    else:
        y = _empty(x)
        py = y.data_ptr()
    _check(_b.load().swarm_add_rms_norm(px, pr, pw, pt, py, pc, ps, rows, cols, pitch, res_pitch, cols, cols, dtype, eps,
                                        rate, seed, event, _raw_stream(device)), "swarm_add_rms_norm")
    return (y, scales, total) if eight_bit else (y, total)


def add_rms_norm_backward(dy, total, weight, dtotal=None, eps=1e-6, rate=0.0, seed=0, event=0):
    """(dx, dresidual, dweight) of add_rms_norm at the total that it returned; `dtotal` is the gradient that reaches
    the total past the norm. dx is dresidual itself when rate is 0."""
    _mask(rate, seed, event)
    device = _device(dy, "dy")
    dtype = _dtype(dy, "dy")
    pd, rows, cols, pitch = _rows(dy, "dy")
    if total is None:
        raise ValueError("total: the total of the forward call is needed")
    pt, total_pitch = _like(total, "total", device, dy, cols)
    pw = _weight(weight, device, cols)
    pa, past_pitch = _like(dtotal, "dtotal", device, dy, cols)
    L = _b.load()
    dresidual = _empty(dy)
    dx = _empty(dy) if rate > 0.0 else None
    dweight = torch.empty_like(weight)
    nbytes = L.swarm_add_rms_norm_workspace(rows, cols)
    work = dy.new_empty((nbytes,), dtype=torch.uint8)
    _check(L.swarm_add_rms_norm_backward(
        pd, pa, pt, pw, dresidual.data_ptr(), dx.data_ptr() if dx is not None else None, dweight.data_ptr(), rows, cols,
        pitch, past_pitch, total_pitch, cols, cols, dtype, eps, rate, seed, event, work.data_ptr(), nbytes,
        _raw_stream(device)), "swarm_add_rms_norm_backward")
    return (dx if dx is not None else dresidual), dresidual, dweight


def _heads(x, name, device, dtype, shape):
    """Strides over sentence, token and head."""
    _same(x, name, device, dtype)
    if x.shape != shape:
        raise ValueError(f"{name}: shape {tuple(x.shape)}, expected {tuple(shape)}")
    s = x.stride()
    if s[3] != 1 and shape[3] > 1:
        raise ValueError(f"{name}: the values of a head have to be consecutive")
    return s[:3]


def _lengths(x, name, device, batch):
    if x is None:
        return 0
    _same(x, name, device, torch.int32)
    if x.dim() != 1 or x.shape[0] != batch or (batch > 1 and x.stride(0) != 1):
        raise ValueError(f"{name}: one consecutive int32 for each sentence is needed")
    return x.data_ptr()


def _attention_desc(device, q, k, v, o, scale, query_lengths, key_lengths, wait_limit, grads=None):
    dtype, whole, states = q.dtype, q.shape, k.shape
    if len(whole) != 4 or len(states) != 4 or states[0] != whole[0] or states[3] != whole[3]:
        raise ValueError(f"q, k: [batch, tokens, heads, head_dim] are needed, got {tuple(whole)} and {tuple(states)}")
    if dtype != torch.bfloat16 and dtype != torch.float16:
        raise ValueError(f"q: bfloat16 or float16 is needed, got {dtype}")
    strides = (*_heads(q, "q", device, dtype, whole), *_heads(k, "k", device, dtype, states),
               *_heads(v, "v", device, dtype, states), *_heads(o, "o", device, dtype, whole))
    if grads is None:
        more = _NO_GRADS
    else:
        do, dq, dk, dv = grads
        more = (*_heads(do, "do", device, dtype, whole), *_heads(dq, "dq", device, dtype, whole),
                *_heads(dk, "dk", device, dtype, states), *_heads(dv, "dv", device, dtype, states))
    batch, dim = whole[0], whole[3]
    if dim == 0:
        raise ValueError("q, k: head_dim is 0")
    lengths = (_lengths(query_lengths, "query_lengths", device, batch), _lengths(key_lengths, "key_lengths", device, batch))
    try:
        return _DESC.pack(batch, whole[2], states[2], whole[1], states[1], dim, _DTYPES[dtype],
                          dim ** -0.5 if scale is None else scale, wait_limit, *lengths, *strides, *more)
    except (struct.error, OverflowError) as err:
        raise ValueError(f"sizes, scale or wait_limit: {err}") from None


def _workspace(L, desc, backward, x):
    size = C.c_size_t()
    _check(L.swarm_cross_attention_workspace(desc, backward, C.byref(size)), "swarm_cross_attention_workspace")
    n = size.value
    return (x.new_empty((n,), dtype=torch.uint8) if n else None), n


def cross_attention(q, k, v, scale=None, query_lengths=None, key_lengths=None, need_lse=False, out=None, wait_limit=-1):
    """o (or (o, lse) with `need_lse`) of q [batch, queries, heads, head_dim] over k, v [batch, keys, kv_heads,
    head_dim]; any strides over the first three dimensions that are multiples of 8 elements. scale: 1 / sqrt(head_dim)
    unless given. query_lengths, key_lengths: int32 [batch] on the device, or None. One to a few query rows (a decoding
    step) take the same call."""
    device = _device(q, "q")
    if out is None:
        out = _empty(q)
    desc = _attention_desc(device, q, k, v, out, scale, query_lengths, key_lengths, wait_limit)
    L = _b.load()
    lse = q.new_empty((q.shape[0], q.shape[2], q.shape[1]), dtype=torch.float32) if need_lse else None
    work, nbytes = _workspace(L, desc, 0, q)
    _check(L.swarm_cross_attention(desc, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
                                   lse.data_ptr() if need_lse else None, work.data_ptr() if nbytes else None, nbytes,
                                   _raw_stream(device)), "swarm_cross_attention")
    return (out, lse) if need_lse else out


def cross_attention_backward(do, q, k, v, o, lse, scale=None, query_lengths=None, key_lengths=None, dq=None, dk=None,
                             dv=None, wait_limit=-1):
    """(dq, dk, dv) from the gradient of o and what the forward call took and returned. dq, dk, dv may be given (for
    example as views of one packed gradient); dk and dv of a key head are sums over its query heads."""
    device = _device(q, "q")
    dq = _empty(q) if dq is None else dq
    dk = _empty(k) if dk is None else dk
    dv = _empty(v) if dv is None else dv
    desc = _attention_desc(device, q, k, v, o, scale, query_lengths, key_lengths, wait_limit, (do, dq, dk, dv))
    _same(lse, "lse", device, torch.float32)
    if lse.shape != (q.shape[0], q.shape[2], q.shape[1]) or not lse.is_contiguous():
        raise ValueError("lse: contiguous [batch, heads, queries] as the forward call returned it")
    L = _b.load()
    work, nbytes = _workspace(L, desc, 1, q)
    _check(L.swarm_cross_attention_backward(desc, do.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
                                            lse.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
                                            work.data_ptr() if nbytes else None, nbytes, _raw_stream(device)),
           "swarm_cross_attention_backward")
    return dq, dk, dv


def check():
    """Waits for the current stream; raises SwarmError if a device-side wait of an operator has given up since the
    last check, or the stream holds a CUDA error."""
    _check(_b.load().swarm_operator_check(torch.cuda.current_stream().cuda_stream), "swarm_operator_check")
