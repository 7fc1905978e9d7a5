"""Argument checks of the operators that need no device: refused before anything is launched."""
import ctypes as C
import struct

import pytest

from paper_1910_12308_b200 import binding as g
from paper_1910_12308_b200 import operators as ops

P = 1 << 20                                  # an address that no refused call may touch


def desc(batch=2, heads=4, kv_heads=2, queries=3, keys=5, dim=64, dtype=g.BF16, scale=0.125, strides=None):
    whole = (heads * dim * max(queries, 1), heads * dim, dim)
    kv = (kv_heads * dim * max(keys, 1), kv_heads * dim, dim)
    s = strides or [whole, kv, kv, whole, whole, whole, kv, kv]
    return struct.pack("=7ifq2Q24q", batch, heads, kv_heads, queries, keys, dim, dtype, scale, -1, 0, 0, *[x for t in s for x in t])


def test_descriptor_has_the_size_of_the_c_struct():
    class Strides(C.Structure):
        _fields_ = [(n, C.c_int64) for n in ("batch", "token", "head")]

    class Desc(C.Structure):
        _fields_ = ([(n, C.c_int32) for n in ("batch", "heads", "kv_heads", "queries", "keys", "head_dim", "dtype")]
                    + [("scale", C.c_float), ("wait_limit", C.c_int64), ("ql", C.c_void_p), ("kl", C.c_void_p)]
                    + [(n, Strides) for n in ("q", "k", "v", "o", "dout", "dq", "dk", "dv")])

    assert C.sizeof(Desc) == len(desc()) == ops._DESC.size
    d = Desc.from_buffer_copy(desc(keys=9, scale=0.5))
    assert (d.keys, d.scale, d.wait_limit, d.q.token, d.dv.head) == (9, 0.5, -1, 256, 64)


def test_dropout_refusals():
    L = g.load()

    def call(x=P, r=None, o=P, rows=4, cols=8, px=8, pr=8, po=8, dtype=g.F32, rate=0.5):
        return L.swarm_dropout(x, r, o, rows, cols, px, pr, po, dtype, rate, 1, 2, None)

    for bad in (dict(x=None), dict(o=None), dict(rows=-1), dict(cols=-1), dict(rows=1 << 31), dict(px=7), dict(po=7),
                dict(r=P, pr=7), dict(dtype=3), dict(dtype=-1), dict(rate=-0.1), dict(rate=1.1), dict(rate=float("nan")),
                dict(x=P + 2), dict(o=P + 1, dtype=g.BF16)):
        assert call(**bad) == g.EINVAL, bad
    assert call(rows=0, x=None, o=None) == g.OK


def test_norm_refusals():
    L = g.load()

    def call(x=P, r=None, w=P, t=P, y=P, c=None, s=None, rows=4, cols=8, pitch=8, yp=8, dtype=g.F32, eps=1e-6, rate=0.0):
        return L.swarm_add_rms_norm(x, r, w, t, y, c, s, rows, cols, pitch, pitch, pitch, yp, dtype, eps, rate, 1, 2, None)

    for bad in (dict(x=None), dict(w=None), dict(w=P + 2), dict(y=None), dict(c=P), dict(y=None, c=P), dict(yp=7),
                dict(y=None, c=P, s=P, yp=7), dict(pitch=7), dict(cols=32769, pitch=32769, yp=32769), dict(eps=-1.0),
                dict(eps=float("inf")), dict(rate=2.0), dict(dtype=7)):
        assert call(**bad) == g.EINVAL, bad

    def back(dy=P, t=P, w=P, dr=P, dx=None, dw=P, rows=4, cols=8, ws=P, n=1 << 20, eps=1e-6):
        return L.swarm_add_rms_norm_backward(dy, None, t, w, dr, dx, dw, rows, cols, 8, 8, 8, 8, 8, g.F32, eps, 0.0, 1, 2, ws, n, None)

    for bad in (dict(dy=None), dict(t=None), dict(w=None), dict(dr=None), dict(ws=None), dict(ws=P + 8), dict(n=4),
                dict(cols=9), dict(eps=-1.0), dict(dx=P + 2)):
        assert back(**bad) == g.EINVAL, bad
    assert L.swarm_add_rms_norm_workspace(0, 8) == 0 and L.swarm_add_rms_norm_workspace(4, 8) >= 32


def test_attention_refusals():
    L = g.load()
    n = C.c_size_t()

    def call(d, q=P, k=P, v=P, o=P, lse=None, ws=P, size=1 << 40):
        return L.swarm_cross_attention(d, q, k, v, o, lse, ws, size, None)

    def back(d, do=P, q=P, k=P, v=P, o=P, lse=P, dq=P, dk=P, dv=P, ws=P, size=1 << 40):
        return L.swarm_cross_attention_backward(d, do, q, k, v, o, lse, dq, dk, dv, ws, size, None)

    for bad in (dict(batch=-1), dict(heads=0), dict(kv_heads=0), dict(kv_heads=3), dict(queries=-1), dict(keys=-1), dict(dim=0),
                dict(dim=4), dict(dim=60), dict(dim=136), dict(dtype=g.F32), dict(dtype=5), dict(scale=0.0), dict(scale=-1.0),
                dict(scale=float("inf")), dict(scale=float("nan")), dict(batch=65536),
                dict(queries=(1 << 30) + 1), dict(keys=(1 << 30) + 1), dict(batch=60000, heads=60000, kv_heads=60000)):
        if bad.get("heads") == 0 or bad.get("dim") == 0:
            strides = [(64, 64, 64)] * 8
        else:
            strides = None
        d = desc(strides=strides, **bad)
        assert call(d) == g.EINVAL and back(d) == g.EINVAL, bad
        assert L.swarm_cross_attention_workspace(d, 0, C.byref(n)) == g.EINVAL
    good = desc()
    assert L.swarm_cross_attention_workspace(good, 1, C.byref(n)) == g.OK and n.value >= 2 * 4 * 3 * 4
    assert L.swarm_cross_attention_workspace(good, 0, None) == g.EINVAL
    assert call(None) == g.EINVAL and back(None) == g.EINVAL
    for bad in (dict(q=None), dict(k=None), dict(v=None), dict(o=None), dict(q=P + 8), dict(k=P + 2), dict(o=P + 8), dict(lse=P + 2)):
        assert call(good, **bad) == g.EINVAL, bad
    for bad in (dict(do=None), dict(lse=None), dict(dq=None), dict(dk=P + 8), dict(dv=None), dict(ws=None), dict(size=0), dict(ws=P + 4)):
        assert back(good, **bad) == g.EINVAL, bad
    whole, kv = (768, 256, 64), (640, 128, 64)
    for at, s in ((0, (768, 252, 64)), (1, (640, 128, 60)), (1, (-640, 128, 64)), (3, (0, 256, 64)), (3, (768, 0, 64)), (2, (1 << 40, 128, 64))):
        strides = [whole, kv, kv, whole, whole, whole, kv, kv]
        strides[at] = s
        assert call(desc(strides=strides)) == g.EINVAL, (at, s)
    for at, s in ((5, (768, 0, 64)), (6, (0, 128, 64)), (7, (640, 128, 0)), (4, (768, 250, 64))):
        strides = [whole, kv, kv, whole, whole, whole, kv, kv]
        strides[at] = s
        assert back(desc(strides=strides)) == g.EINVAL, (at, s)


def test_no_cpu_path():
    torch = pytest.importorskip("torch")
    x = torch.zeros(2, 8)
    with pytest.raises(ValueError):
        ops.dropout(x, 0.1, 1, 2)
    with pytest.raises(ValueError):
        ops.add_rms_norm(x, torch.ones(8))
    with pytest.raises(ValueError):
        ops.cross_attention(torch.zeros(1, 1, 1, 8), torch.zeros(1, 1, 1, 8), torch.zeros(1, 1, 1, 8))


def test_attention_gradient_refuses_scales_whose_statistics_leave_fp32():
    L, n = g.load(), C.c_size_t()
    for scale in (2.0 ** -121, 2.0 ** -149):
        args = [P] * 10 + [1 << 40, None]
        assert L.swarm_cross_attention_backward(desc(scale=scale), *args) == g.EINVAL
        assert L.swarm_cross_attention_workspace(desc(scale=scale), 0, C.byref(n)) == g.OK
