"""Argument checks of the paged cache and of the log probabilities that need no device: refused before anything is launched."""
import ctypes as C

import pytest

from paper_1910_12308_b200 import binding as g
from paper_1910_12308_b200 import operators as ops

P = 1 << 20                                  # an address that no refused call may touch


class Strides(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("batch", "token", "head")]


class Desc(C.Structure):
    _fields_ = ([(n, C.c_int32) for n in ("batch", "heads", "kv_heads", "tokens", "head_dim", "dtype", "pages", "page_size",
                                          "table_columns", "rotated", "interleaved", "window", "sinks")]
                + [("scale", C.c_float), ("table_pitch", C.c_int64)]
                + [(n, C.c_void_p) for n in ("table", "lengths", "counts")]
                + [(n, Strides) for n in ("k_pages", "v_pages", "q", "out", "k", "v")])


def desc(**changes):
    page, whole, kv = (16 * 2 * 64, 2 * 64, 64), (3 * 4 * 64, 4 * 64, 64), (3 * 2 * 64, 2 * 64, 64)
    values = dict(batch=2, heads=4, kv_heads=2, tokens=3, head_dim=64, dtype=g.BF16, pages=5, page_size=16, table_columns=2, rotated=64,
                  interleaved=0, window=0, sinks=0, scale=0.125, table_pitch=2, table=P, lengths=P, counts=None, k_pages=page,
                  v_pages=page, q=whole, out=whole, k=kv, v=kv)
    values.update(changes)
    return C.byref(Desc(**{n: Strides(*x) if isinstance(x, tuple) else x for n, x in values.items()}))


BAD_DESCRIPTORS = [
    dict(batch=-1), dict(batch=65536), dict(kv_heads=0), dict(kv_heads=65536, heads=65536), dict(tokens=-1), dict(head_dim=0), dict(head_dim=4),
    dict(head_dim=60), dict(head_dim=136), dict(dtype=g.F32), dict(dtype=7), dict(pages=-1), dict(page_size=0), dict(table_columns=-1),
    dict(table_pitch=1), dict(table_pitch=-2), dict(table=None), dict(table=P + 2), dict(lengths=None), dict(lengths=P + 1), dict(counts=P + 2),
    dict(heads=0), dict(heads=5), dict(heads=-4),
    dict(k_pages=(2048, 128, 60)), dict(k_pages=(0, 128, 64)), dict(v_pages=(2048, 0, 64)), dict(v_pages=(-2048, 128, 64)),
    dict(k_pages=(1 << 40, 128, 64)), dict(q=(768, 250, 64)), dict(out=(0, 256, 64)), dict(out=(768, 256, 0)),
]


def test_descriptor_has_the_size_of_the_c_struct():
    assert C.sizeof(Desc) == ops._PAGED.size
    packed = ops._PAGED.pack(*range(1, 14), 0.5, *range(15, 37))
    d = Desc.from_buffer_copy(packed)
    assert (d.batch, d.sinks, d.scale, d.table_pitch, d.counts, d.k_pages.batch, d.v.head) == (1, 13, 0.5, 15, 18, 19, 36)


def test_append_refusals():
    L = g.load()

    def call(d, k=P, v=P, kp=P, vp=P, q=P, out=P, f=P):
        return L.swarm_cache_append(d, k, v, kp, vp, q, out, f, None)

    for bad in BAD_DESCRIPTORS + [dict(tokens=(1 << 30) + 1), dict(rotated=-2), dict(rotated=63), dict(rotated=66),
                                  dict(k=(384, 128, 60)), dict(v=(384, 130, 64))]:
        assert call(desc(**bad)) == g.EINVAL, bad
    for bad in (dict(k=None), dict(v=None), dict(kp=None), dict(vp=None), dict(q=None), dict(out=None), dict(f=None), dict(f=P + 2),
                dict(k=P + 8), dict(v=P + 2), dict(kp=P + 8), dict(vp=P + 8), dict(q=P + 8), dict(out=P + 8)):
        assert call(desc(), **bad) == g.EINVAL, bad
    assert call(None) == g.EINVAL
    assert call(desc(batch=0)) == g.OK and call(desc(tokens=0)) == g.OK


def test_paged_attention_refusals():
    L, n = g.load(), C.c_size_t()

    def call(d, q=P, kp=P, vp=P, out=P, lse=None, work=P, size=1 << 40):
        return L.swarm_paged_attention(d, q, kp, vp, out, lse, work, size, None)

    for bad in BAD_DESCRIPTORS + [dict(tokens=65), dict(batch=8192, heads=4096), dict(window=-1), dict(sinks=-1), dict(scale=0.0), dict(scale=-1.0),
                                  dict(scale=float("inf")), dict(scale=float("nan"))]:
        assert call(desc(**bad)) == g.EINVAL, bad
    for bad in (dict(q=None), dict(kp=None), dict(vp=None), dict(out=None), dict(lse=P + 2), dict(q=P + 8), dict(kp=P + 8), dict(vp=P + 2),
                dict(out=P + 8)):
        assert call(desc(), **bad) == g.EINVAL, bad
    assert call(None) == g.EINVAL and L.swarm_paged_attention_workspace(None, C.byref(n)) == g.EINVAL
    assert L.swarm_paged_attention_workspace(desc(), None) == g.EINVAL
    assert L.swarm_paged_attention_workspace(desc(scale=0.0), C.byref(n)) == g.EINVAL
    assert L.swarm_paged_attention_workspace(desc(batch=0), C.byref(n)) == g.OK and n.value == 0
    big = dict(batch=8, pages=8192, table_columns=1024, table_pitch=1024)
    assert L.swarm_paged_attention_workspace(desc(**big), C.byref(n)) == g.OK
    if n.value:
        assert call(desc(**big), size=n.value - 1) == g.EINVAL
        assert call(desc(**big), work=None) == g.EINVAL and call(desc(**big), work=P + 8) == g.EINVAL
    assert call(desc(batch=0)) == g.OK and call(desc(tokens=0)) == g.OK


def test_log_probs_refusals():
    L = g.load()

    def call(x=P, t=P, lp=P, st=P, h=None, tl=None, tt=None, rows=4, cols=8, pitch=8, dtype=g.F32, scale=1.0, top=0):
        return L.swarm_token_log_probs(x, t, lp, st, h, tl, tt, rows, cols, pitch, dtype, scale, top, None)

    sizes = (dict(rows=-1), dict(rows=1 << 31), dict(cols=0), dict(cols=1 << 31, pitch=1 << 31), dict(pitch=7), dict(pitch=1 << 39), dict(dtype=3),
             dict(dtype=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(x=None), dict(x=P + 2))
    for bad in sizes + (dict(t=None), dict(lp=None), dict(t=P + 4), dict(lp=P + 2), dict(st=None), dict(st=P + 1), dict(h=P + 2), dict(top=-1),
                        dict(top=33, cols=40, pitch=40, tl=P, tt=P), dict(top=9, tl=P, tt=P), dict(top=2), dict(top=2, tl=P), dict(top=2, tl=P, tt=P + 4)):
        assert call(**bad) == g.EINVAL, bad
    assert call(rows=0, x=None, st=None) == g.OK

    def back(g_=P, h=P, x=P, t=P, st=P, e=P, o=P, rows=4, cols=8, pitch=8, po=8, dtype=g.F32, scale=1.0):
        return L.swarm_token_log_probs_backward(g_, h, x, t, st, e, o, rows, cols, pitch, po, dtype, scale, None)

    for bad in sizes + (dict(po=7), dict(o=None), dict(o=P + 2), dict(st=None), dict(t=None), dict(e=None), dict(g_=P + 2), dict(h=P + 2),
                        dict(t=P + 4), dict(pitch=16)):
        assert back(**bad) == g.EINVAL, bad
    assert back(rows=0) == g.OK


def test_no_cpu_path():
    torch = pytest.importorskip("torch")
    x, pages, table = torch.zeros(1, 1, 1, 8), torch.zeros(2, 4, 1, 8), torch.zeros(1, 2, dtype=torch.int32)
    lengths = torch.ones(1, dtype=torch.int32)
    for call in (lambda: ops.append_to_cache(x, x, pages, pages, table, lengths), lambda: ops.paged_attention(x, pages, pages, table, lengths),
                 lambda: ops.token_log_probs(torch.zeros(2, 8), torch.zeros(2, dtype=torch.int64)),
                 lambda: ops.token_log_probs_backward(torch.zeros(2), torch.zeros(2, 8), torch.zeros(2, dtype=torch.int64), torch.zeros(2, 2))):
        with pytest.raises(ValueError):
            call()


def test_paged_attention_refuses_every_workspace_that_does_not_do():
    """Room for 16384 positions of 8 sentences: items are cut, so there is a workspace, and it has to be there, whole and aligned."""
    L, n = g.load(), C.c_size_t()
    big = dict(batch=8, pages=8192, table_columns=1024, table_pitch=1024)
    assert L.swarm_paged_attention_workspace(desc(**big), C.byref(n)) == g.OK
    assert n.value > 0

    def call(work, size):
        return L.swarm_paged_attention(desc(**big), P, P, P, P, None, work, size, None)

    for work, size in ((P, 0), (P, n.value - 1), (None, n.value), (P + 8, n.value), (P + 4, 1 << 40)):
        assert call(work, size) == g.EINVAL, (work, size)
