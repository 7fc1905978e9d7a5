"""Operators of the models that the nodes train, against their formulas in 64 bits.

Tolerances are bounds, not observations. U is the largest relative rounding error of a type. A result that is rounded
once is held to U of itself; E = 2e-5 covers what fp32 arithmetic adds (128-term dot products of unit normals, base-2
exponentials, sums of a few thousand terms); an operand that is rounded to the type before a product contributes U times
the product's absolute sum.
"""
import math

import pytest

from paper_1910_12308_b200 import binding as g

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_1910_12308_b200 import operators as ops  # noqa: E402

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
U = {BF16: 2.0 ** -8, F16: 2.0 ** -11, F32: 2.0 ** -24}
TINY = {BF16: 1e-38, F16: 2.0 ** -24, F32: 1e-38}        # a result may fall among the subnormals of its type
E = 2e-5


def randn(*shape, dtype=F32, seed=0, std=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=gen, device="cuda") * std).to(dtype)


def within(got, want, bound, what=""):
    got, want = got.double(), want.double()
    assert got.shape == want.shape, what
    assert not torch.isnan(got).any(), what
    over = (got - want).abs() - bound
    assert over.max().item() <= 0 if over.numel() else True, (what, over.max().item(), (got - want).abs().max().item())


# ---- the mask ------------------------------------------------------------------------------------------------------


def philox(counter, key):
    c, k = list(counter), list(key)
    for _ in range(10):
        p0, p1 = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(p1 >> 32) ^ c[1] ^ k[0], p1 & 0xFFFFFFFF, (p0 >> 32) ^ c[3] ^ k[1], p0 & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def factors(rows, cols, rate, seed, event):
    """m of every element: 0, or 2^16 / (2^16 - T)."""
    drop = math.floor(rate * 65536 + 0.5)
    out = torch.zeros(rows, cols, dtype=torch.float64)
    for r in range(rows):
        for c0 in range(0, cols, 8):
            words = philox((c0 // 8, r, event, 13), (seed & 0xFFFFFFFF, seed >> 32))
            for c in range(c0, min(c0 + 8, cols)):
                u = words[(c % 8) // 2] >> (16 * (c % 2)) & 0xFFFF
                out[r, c] = 65536 / (65536 - drop) if u >= drop else 0.0
    return out.cuda()


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (2, 8), (5, 9), (4, 255), (3, 256), (2, 264), (9, 513), (3, 1001)])
@pytest.mark.parametrize("residual", [False, True])
def test_dropout(dtype, rows, cols, residual):
    seed, event, rate = 0xFEDCBA9876543210 + rows, 4000000000 + cols, 0.3
    x, r = randn(rows, cols, dtype=dtype, seed=1), randn(rows, cols, dtype=dtype, seed=2, std=3) if residual else None
    m = factors(rows, cols, rate, seed, event)
    want = x.double() * m + (r.double() if residual else 0.0)
    got = ops.dropout(x, rate, seed, event, residual=r)
    size = (x.double() * m).abs() + (r.double().abs() if residual else 0.0)
    within(got, want, U[dtype] * want.abs() + 2.0 ** -22 * size + TINY[dtype])
    if not residual:
        assert torch.equal(got == 0, (m == 0) | (x == 0))


def test_dropout_ends_of_the_rate_and_what_is_dropped():
    x = torch.full((4, 300), float("nan"), device="cuda")
    assert torch.equal(ops.dropout(x, 1.0, 1, 2), torch.zeros_like(x))          # nothing of a dropped element is used
    y = randn(4, 300)
    assert torch.equal(ops.dropout(y, 0.0, 1, 2), y)
    assert torch.equal(ops.dropout(y, 1.0, 1, 2, residual=y), y)
    kept = ops.dropout(torch.ones(512, 4096, device="cuda"), 0.25, 77, 3)
    share = (kept > 0).double().mean().item()
    assert abs(share - 0.75) < 6 * math.sqrt(0.75 * 0.25 / kept.numel())         # six standard deviations
    other = ops.dropout(torch.ones(512, 4096, device="cuda"), 0.25, 77, 4)
    assert abs(((kept > 0) == (other > 0)).double().mean().item() - (0.75 ** 2 + 0.25 ** 2)) < 6 / math.sqrt(kept.numel())
    assert ops.dropout(torch.empty(0, 5, device="cuda"), 0.5, 1, 2).shape == (0, 5)
    assert ops.dropout(torch.empty(5, 0, device="cuda"), 0.5, 1, 2).shape == (5, 0)


def test_dropout_does_not_depend_on_strides_alignment_or_place():
    x, r = randn(40, 520, dtype=BF16, seed=3), randn(40, 520, dtype=BF16, seed=4)
    want = ops.dropout(x, 0.4, 9, 5, residual=r)
    wide = torch.zeros(40, 1111, dtype=BF16, device="cuda")
    wide[:, 3:523] = x                                                          # neither the base nor the pitch on 16 bytes
    assert torch.equal(ops.dropout(wide[:, 3:523], 0.4, 9, 5, residual=r), want)
    assert torch.equal(ops.dropout(x.view(4, 10, 520), 0.4, 9, 5, residual=r.view(4, 10, 520)).view(40, 520), want)
    into = torch.zeros(40, 600, dtype=BF16, device="cuda")
    ops.dropout(x, 0.4, 9, 5, residual=r, out=into[:, 8:528])
    assert torch.equal(into[:, 8:528], want) and not into[:, :8].any() and not into[:, 528:].any()
    here = x.clone()
    assert torch.equal(ops.dropout(here, 0.4, 9, 5, residual=r, out=here), want)
    there = r.clone()
    assert torch.equal(ops.dropout(x, 0.4, 9, 5, residual=there, out=there), want)


def test_dropout_gradient_is_its_difference():
    x, dy, u = (randn(7, 333, dtype=F32, seed=s) for s in (5, 6, 7))
    dx = ops.dropout(dy, 0.2, 11, 12)
    up, down = (ops.dropout(x + h * u, 0.2, 11, 12).double() for h in (0.5, -0.5))
    lhs, rhs = ((up - down) * dy.double()).sum().item(), (dx.double() * u.double()).sum().item()
    assert abs(lhs - rhs) <= 2.0 ** -21 * (dx.double().abs() * (u.abs() + x.abs())).sum().item()


# ---- norm ----------------------------------------------------------------------------------------------------------


def norm_reference(x, r, w, eps, m):
    total = x.double() * m + (r.double() if r is not None else 0.0)
    return total, w.double() * total / (total.square().mean(1, keepdim=True) + eps).sqrt()


NORM_SHAPES = [(1, 1), (2, 5), (3, 64), (5, 255), (2, 256), (7, 257), (3, 512), (9, 1001), (2, 1024), (3, 1032), (2, 2048),
               (2, 4100), (2, 8192), (1, 16000), (1, 32768)]


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("rows,cols", NORM_SHAPES)
@pytest.mark.parametrize("rate,residual", [(0.0, True), (0.3, True), (0.0, False)])
def test_add_rms_norm(dtype, rows, cols, rate, residual):
    if rate and cols > 1100:
        pytest.skip("the mask is checked at the smaller widths; the reference draws it one call at a time")
    x, r = randn(rows, cols, dtype=dtype, seed=1), randn(rows, cols, dtype=dtype, seed=2, std=3) if residual else None
    w = 1 + 0.3 * randn(cols, seed=3)
    m = factors(rows, cols, rate, 5, 6) if rate else 1.0
    total, want = norm_reference(x, r, w, 1e-5, m)
    y, kept = ops.add_rms_norm(x, w, residual=r, eps=1e-5, rate=rate, seed=5, event=6)
    size = (x.double() * m).abs() + (r.double().abs() if residual else 0.0)
    within(kept, total, U[dtype] * total.abs() + 2.0 ** -22 * size + TINY[dtype])
    rstd = 1 / (total.square().mean(1, keepdim=True) + 1e-5).sqrt()
    within(y, want, (U[dtype] + E) * want.abs() + 2.0 ** -22 * size * rstd * w.double().abs() + TINY[dtype])
    if not residual and not rate:
        assert kept is x


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("rows,cols", NORM_SHAPES)
def test_add_rms_norm_in_8_bits(dtype, rows, cols):
    x, r = randn(rows, cols, dtype=dtype, seed=1), randn(rows, cols, dtype=dtype, seed=2)
    x[0] = 0
    r[0, : cols // 2] = 0                                                       # blocks of zeros
    w = 1 + 0.3 * randn(cols, seed=3)
    codes, scales, total = ops.add_rms_norm(x, w, residual=r, eight_bit=True)
    _, want = norm_reference(x, r, w, 1e-6, 1.0)
    assert codes.dtype == torch.float8_e4m3fn and scales.shape == (rows, (cols + 127) // 128)
    within(total, x.double() + r.double(), U[dtype] * (x.double() + r.double()).abs() + 2.0 ** -22 * (x.abs() + r.abs()).double() + TINY[dtype])
    for b in range(scales.shape[1]):
        part = want[:, 128 * b: 128 * b + 128]
        top = part.abs().amax(1)
        assert ((scales[:, b].double() * 448 - top).abs() <= E * top).all()
        s = scales[:, b].double().unsqueeze(1)
        got = codes[:, 128 * b: 128 * b + 128].double() * s
        # e4m3 keeps four significant bits, and steps of 2^-9 below 2^-6
        within(got, part, part.abs() * (2.0 ** -4 + E) + s * 2.0 ** -10 * (1 + E) + E * top.unsqueeze(1))
        assert (codes[:, 128 * b: 128 * b + 128].float()[top == 0] == 0).all()


def test_add_rms_norm_8_bits_of_values_that_are_not_finite():
    x = randn(3, 384, seed=1)
    x[1, 200] = float("nan")
    codes, scales, _ = ops.add_rms_norm(x, torch.ones(384, device="cuda"), eight_bit=True)
    assert torch.isfinite(codes[0].float()).all() and torch.isfinite(scales[[0, 2]]).all()
    assert torch.isnan(scales[1]).all() and torch.isnan(codes[1].float()).all()  # the norm of that row has no value


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (4, 64), (5, 255), (700, 256), (33, 257), (9, 1001), (1200, 1024),
                                       (40, 1032), (6, 2048), (3, 4100), (300, 8192), (2, 16000), (2, 32768)])
@pytest.mark.parametrize("rate,past", [(0.0, True), (0.3, True), (0.0, False)])
def test_add_rms_norm_backward(dtype, rows, cols, rate, past):
    if rate and rows * cols > 12000:
        pytest.skip("the mask is checked at the smaller sizes; the reference draws it one call at a time")
    total, dy = randn(rows, cols, dtype=dtype, seed=1, std=2), randn(rows, cols, dtype=dtype, seed=2)
    dtotal = randn(rows, cols, dtype=dtype, seed=3) if past else None
    w = 1 + 0.3 * randn(cols, seed=4)
    m = factors(rows, cols, rate, 5, 6) if rate else 1.0
    t, dyd, wd = total.double(), dy.double(), w.double()
    r = 1 / (t.square().mean(1, keepdim=True) + 1e-6).sqrt()
    first, second = r * wd * dyd, t * r ** 3 * (wd * dyd * t).mean(1, keepdim=True)
    want = first - second + (dtotal.double() if past else 0.0)
    size = first.abs() + t.abs() * r ** 3 * (wd * dyd * t).abs().mean(1, keepdim=True) + (dtotal.double().abs() if past else 0.0)
    dx, dres, dw = ops.add_rms_norm_backward(dy, total, w, dtotal=dtotal, rate=rate, seed=5, event=6)
    within(dres, want, U[dtype] * want.abs() + E * size + TINY[dtype])
    within(dx, want * m, U[dtype] * (want * m).abs() + E * size * 2 + TINY[dtype])
    within(dw, (dyd * t * r).sum(0), E * (dyd * t * r).abs().sum(0) + 1e-30)
    again = ops.add_rms_norm_backward(dy, total, w, dtotal=dtotal, rate=rate, seed=5, event=6)
    assert all(torch.equal(a, b) for a, b in zip(again, (dx, dres, dw)))          # one fixed order of addition


def test_norm_gradient_is_the_difference_of_the_norm():
    x, dy, u = (randn(6, 300, seed=s).double() for s in (1, 2, 3))
    w, v = 1 + 0.3 * randn(300, seed=4), randn(300, seed=5)
    h = 1e-4

    def loss(x_, w_):
        return (norm_reference(x_, None, w_, 1e-6, 1.0)[1] * dy).sum().item()

    dx, _, dw = ops.add_rms_norm_backward(dy.float(), x.float(), w)
    x, dy = x.float().double(), dy.float().double()
    num = (loss(x + h * u, w.double()) - loss(x - h * u, w.double())) / (2 * h)
    assert abs(num - (dx.double() * u).sum().item()) <= (E + 1e-6) * (dx.double().abs() * u.abs()).sum().item() + 1e-6
    num = (loss(x, w.double() + h * v.double()) - loss(x, w.double() - h * v.double())) / (2 * h)
    assert abs(num - (dw.double() * v.double()).sum().item()) <= (E + 1e-6) * (dw.double().abs() * v.double().abs()).sum().item() + 1e-6


def test_norm_does_not_depend_on_strides_and_alignment():
    x, r, w = randn(20, 520, dtype=BF16, seed=1), randn(20, 520, dtype=BF16, seed=2), 1 + 0.3 * randn(520, seed=3)
    store = torch.zeros(521, device="cuda")
    store[1:] = w
    y, total = ops.add_rms_norm(x, w, residual=r, rate=0.2, seed=1, event=2)
    c, s, _ = ops.add_rms_norm(x, w, residual=r, rate=0.2, seed=1, event=2, eight_bit=True)
    wide = torch.zeros(20, 777, dtype=BF16, device="cuda")
    wide[:, 5:525] = x
    y2, total2 = ops.add_rms_norm(wide[:, 5:525], store[1:], residual=r, rate=0.2, seed=1, event=2)
    assert torch.equal(total, total2)
    within(y2, y, 2 * U[BF16] * y.double().abs() + TINY[BF16])                   # another order of the sum of squares
    c2, s2, _ = ops.add_rms_norm(wide[:, 5:525], store[1:], residual=r, rate=0.2, seed=1, event=2, eight_bit=True)
    assert ((s - s2).abs() <= E * s).all() and ((c.float() - c2.float()).abs() <= 2.0 ** -3 * c.float().abs() + 2.0 ** -9).all()
    y3, _ = ops.add_rms_norm(x.view(4, 5, 520), store[1:], residual=r.view(4, 5, 520), rate=0.2, seed=1, event=2)
    assert torch.equal(y3.view(20, 520), y)
    g1 = ops.add_rms_norm_backward(r, total, w, dtotal=x, rate=0.2, seed=1, event=2)
    g2 = ops.add_rms_norm_backward(r, total, store[1:], dtotal=wide[:, 5:525], rate=0.2, seed=1, event=2)
    for a, b in zip(g1, g2):
        within(b, a, (2 * U[BF16] if a.dtype == BF16 else 1e-4) * a.double().abs().clamp_min(1e-2))


# ---- attention -----------------------------------------------------------------------------------------------------


def attention_reference(q, k, v, scale, nq, nk, do=None, u=0.0):
    """o, lse (and dq, dk, dv) in 64 bits with elementwise bounds for an implementation that rounds p and ds to a type
    with relative error u before their products."""
    b, tq, h, d = q.shape
    tk, hk = k.shape[1], k.shape[2]
    grp = h // hk
    out = {}
    res = {n: torch.zeros(b, tq, h, d, dtype=torch.float64, device="cuda") for n in ("o", "o_b", "dq", "dq_b")}
    res |= {n: torch.zeros(b, tk, hk, d, dtype=torch.float64, device="cuda") for n in ("dk", "dk_b", "dv", "dv_b")}
    res["lse"] = torch.full((b, h, tq), -math.inf, dtype=torch.float64, device="cuda")
    for i in range(b):
        n, m = int(nq[i]), int(nk[i])
        if not n or not m:
            continue
        for a in range(h):
            c = a // grp
            qd, kd, vd = q[i, :n, a].double(), k[i, :m, c].double(), v[i, :m, c].double()
            s = scale * qd @ kd.T
            lse = torch.logsumexp(s, 1)
            p = torch.exp(s - lse[:, None])
            o = p @ vd
            res["lse"][i, a, :n] = lse
            res["o"][i, :n, a] = o
            ob = (u + E) * (p @ vd.abs())
            res["o_b"][i, :n, a] = u * o.abs() + ob
            if do is None:
                continue
            g_ = do[i, :n, a].double()
            dp, delta = g_ @ vd.T, (g_ * o).sum(1, keepdim=True)
            ds = scale * p * (dp - delta)
            delta_b = (g_.abs() * (u * o.abs() + ob)).sum(1, keepdim=True) + E * (g_ * o).abs().sum(1, keepdim=True)
            ds_b = (u + E) * ds.abs() + scale * p * (E * (g_.abs() @ vd.abs().T) * 0.1 + delta_b)
            res["dq"][i, :n, a] = ds @ kd
            res["dq_b"][i, :n, a] = ds_b @ kd.abs()
            res["dk"][i, :m, c] += ds.T @ qd
            res["dk_b"][i, :m, c] += ds_b.T @ qd.abs()
            res["dv"][i, :m, c] += p.T @ g_
            res["dv_b"][i, :m, c] += (u + E) * (p.T @ g_.abs())
    for name in ("dq", "dk", "dv"):
        res[name + "_b"] += u * res[name].abs()
    return res


def attention_inputs(b, tq, tk, h, hk, d, dtype, seed=0, layout="tokens"):
    q, do = randn(b, tq, h, d, dtype=dtype, seed=seed, std=1.5), randn(b, tq, h, d, dtype=dtype, seed=seed + 3)
    if layout == "packed":
        kv = randn(b, tk, 2, hk, d, dtype=dtype, seed=seed + 1)
        return q, kv[:, :, 0], kv[:, :, 1], do
    if layout == "heads":
        k, v = (randn(b, hk, tk, d, dtype=dtype, seed=seed + s).transpose(1, 2) for s in (1, 2))
        return q.transpose(1, 2).contiguous().transpose(1, 2), k, v, do
    return q, randn(b, tk, hk, d, dtype=dtype, seed=seed + 1), randn(b, tk, hk, d, dtype=dtype, seed=seed + 2), do


def check_attention(q, k, v, do, nq=None, nk=None, scale=None, clean=None):
    """Forward and backward against the reference; `clean` holds (q, k, v, do) with finite values where the inputs
    themselves hold others past the ends."""
    b, tq, h, d = q.shape
    tk, dtype = k.shape[1], q.dtype
    cq, ck, cv, cdo = clean or (q, k, v, do)
    s = scale or d ** -0.5
    lq = nq.tolist() if nq is not None else [tq] * b
    lk = nk.tolist() if nk is not None else [tk] * b
    clamp = lambda n, most: [min(max(x, 0), most) for x in n]  # noqa: E731
    ref = attention_reference(cq, ck, cv, s, clamp(lq, tq), clamp(lk, tk), cdo, U[dtype])
    kw = dict(scale=scale, query_lengths=nq, key_lengths=nk)
    o, lse = ops.cross_attention(q, k, v, need_lse=True, **kw)
    within(o, ref["o"], ref["o_b"] + TINY[dtype], "o")
    assert torch.equal(torch.isinf(lse), torch.isinf(ref["lse"])) and not (lse == math.inf).any()
    fin = torch.isfinite(ref["lse"])
    within(lse[fin], ref["lse"][fin], E * (1 + ref["lse"][fin].abs()), "lse")
    assert torch.equal(ops.cross_attention(q, k, v, **kw), o)                    # with and without lse, and twice the same bits
    got = ops.cross_attention_backward(do, q, k, v, o, lse, **kw)
    for name, x in zip(("dq", "dk", "dv"), got):
        within(x, ref[name], ref[name + "_b"] + TINY[dtype], name)
    again = ops.cross_attention_backward(do, q, k, v, o, lse, **kw)
    assert all(torch.equal(x, y) for x, y in zip(got, again))                    # one fixed order of addition
    ops.check()
    return o, lse, got


LENGTHS = [(1, 1), (1, 2), (1, 77), (2, 63), (3, 64), (5, 65), (7, 127), (16, 128), (17, 129), (50, 61), (127, 40), (128, 128),
           (129, 130), (130, 257), (257, 200), (300, 513)]


@pytest.mark.parametrize("tq,tk", LENGTHS)
@pytest.mark.parametrize("dtype,d", [(BF16, 64), (F16, 128)])
def test_cross_attention_lengths(tq, tk, dtype, d):
    check_attention(*attention_inputs(2, tq, tk, 2, 2, d, dtype, seed=tq))


@pytest.mark.parametrize("d", [8, 16, 32, 40, 56, 64, 72, 80, 96, 120, 128])
@pytest.mark.parametrize("tq,tk", [(1, 150), (140, 150)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_cross_attention_head_dims(d, tq, tk, dtype):
    check_attention(*attention_inputs(2, tq, tk, 3, 3, d, dtype, seed=d))


@pytest.mark.parametrize("h,hk", [(2, 1), (3, 1), (6, 2), (8, 1), (8, 2), (12, 4), (24, 1), (40, 1)])
@pytest.mark.parametrize("tq,tk,d", [(1, 300, 64), (4, 129, 128), (150, 140, 64), (140, 150, 128)])
def test_cross_attention_shared_heads(h, hk, tq, tk, d):
    check_attention(*attention_inputs(2, tq, tk, h, hk, d, BF16, seed=h))


@pytest.mark.parametrize("layout", ["packed", "heads"])
@pytest.mark.parametrize("tq,tk", [(1, 200), (20, 130), (200, 333)])
def test_cross_attention_layouts(layout, tq, tk):
    check_attention(*attention_inputs(3, tq, tk, 4, 2, 64, BF16, seed=5, layout=layout))


@pytest.mark.parametrize("tq,tk,d", [(1, 300, 64), (3, 70, 128), (40, 100, 64), (200, 300, 64), (300, 260, 128), (150, 270, 72)])
def test_cross_attention_ends_empty_rows_and_what_lies_past_them(tq, tk, d):
    """Unequal lengths, an empty sentence, a length past the end and a negative one; NaN and infinities past the ends."""
    b, dtype = 6, BF16
    q, k, v, do = attention_inputs(b, tq, tk, 4, 2, d, dtype, seed=9, layout="packed")
    nk = torch.tensor([tk, 0, 1, max(1, tk - 129), tk + 7, -3], dtype=torch.int32, device="cuda")
    nq = torch.tensor([tq, tq, max(1, tq // 2), max(1, tq - 1), tq + 9, tq], dtype=torch.int32, device="cuda")
    if tq > 1:
        nq[0] = 0
    dirty = [x.clone() for x in (q, k, v, do)]
    for i in range(b):
        nqi, nki = min(max(int(nq[i]), 0), tq), min(max(int(nk[i]), 0), tk)
        for x, n in ((dirty[0], nqi), (dirty[1], nki), (dirty[2], nki), (dirty[3], nqi)):
            x[i, n:] = float("nan")
            x[i, n::2] = float("inf")
            x[i, n::3] = -float("inf")
    o, lse, grads = check_attention(*dirty, nq=nq, nk=nk, clean=(q, k, v, do))
    assert not o[1].any() and torch.isinf(lse[1]).all() and not grads[0][1].any()
    check_attention(q, k, v, do, nk=nk)
    check_attention(q, k, v, do, nq=nq)


@pytest.mark.parametrize("tq", [1, 150])
def test_cross_attention_of_nothing(tq):
    q, k, v, do = attention_inputs(2, tq, 0, 2, 1, 64, BF16)
    o, lse, (dq, dk, dv) = check_attention(q, k, v, do)
    assert not o.any() and not dq.any() and dk.shape == k.shape
    q, k, v, do = attention_inputs(2, 0, 5, 2, 1, 64, BF16)
    o, lse = ops.cross_attention(q, k, v, need_lse=True)
    dq, dk, dv = ops.cross_attention_backward(do, q, k, v, o, lse)
    assert o.numel() == 0 and not dk.any() and not dv.any()                       # no rows: the states' gradients are 0
    q, k, v, do = attention_inputs(0, 3, 5, 2, 1, 64, BF16)
    assert ops.cross_attention(q, k, v).numel() == 0


@pytest.mark.parametrize("tq,tk", [(1, 500), (130, 500)])
def test_cross_attention_large_scores(tq, tk):
    """Scores in the thousands of either sign, and in growing order: the running maximum has to move."""
    q, k, v, do = attention_inputs(1, tq, tk, 2, 2, 64, BF16, seed=3)
    k = (k.float() * torch.linspace(0.1, 30, tk, device="cuda").view(1, tk, 1, 1)).to(BF16)
    q = (q.float() * 8).to(BF16)
    scale = 0.25                                                                  # scores up to about 10^4; a power of two
    ref = attention_reference(q, k, v, scale, [tq], [tk], None, U[BF16])
    o, lse = ops.cross_attention(q, k, v, scale=scale, need_lse=True)
    # fp32 scores of that size are off by up to 2^-24 * 64 * (largest sum of |q k|), which exp turns into a relative error
    size = (scale * torch.einsum("bqhd,bkhd->bhqk", q.double().abs(), k.double().abs())).max().item()
    slack = 8 * 2.0 ** -24 * size
    vmax = v.double().abs().max().item()
    within(o, ref["o"], ref["o_b"] + 2 * slack * vmax, "o")
    within(lse, ref["lse"], slack + E * ref["lse"].abs(), "lse")


@pytest.mark.parametrize("tq", [1, 8, 200])
def test_cross_attention_broadcast_states(tq):
    """Encoder states shared by all sentences (a beam) or all heads through strides of 0."""
    q, k, v, do = attention_inputs(1, tq, 140, 4, 2, 64, BF16, seed=4)
    q, do = (randn(3, tq, 4, 64, dtype=BF16, seed=s) for s in (21, 22))
    check_attention(q, k.expand(3, -1, -1, -1), v.expand(3, -1, -1, -1), do)
    one = k[:, :, :1].expand(3, -1, 4, -1), v[:, :, :1].expand(3, -1, 4, -1)
    o, lse, (dq, dk, dv) = check_attention(q, one[0], one[1], do)
    assert dk.shape == (3, 140, 4, 64)


def test_cross_attention_gradients_into_a_packed_buffer():
    q, k, v, do = attention_inputs(2, 70, 90, 4, 2, 64, BF16, seed=6)
    o, lse = ops.cross_attention(q, k, v, need_lse=True)
    want = ops.cross_attention_backward(do, q, k, v, o, lse)
    dkv = torch.full((2, 90, 3, 2, 64), 7.0, dtype=BF16, device="cuda")
    got = ops.cross_attention_backward(do, q, k, v, o, lse, dk=dkv[:, :, 0], dv=dkv[:, :, 2])
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and (dkv[:, :, 1] == 7).all()
    wide = torch.full((2, 70, 5, 64), 7.0, dtype=BF16, device="cuda")
    assert torch.equal(ops.cross_attention(q, k, v, out=wide[:, :, :4]), o) and (wide[:, :, 4] == 7).all()


@pytest.mark.parametrize("tq", [1, 130])
def test_cross_attention_offsets_past_32_bits(tq):
    """Two sentences whose states lie more than 2^32 bytes and 2^31 elements apart."""
    far, tk = (1 << 31) + 4096, 200
    store = torch.empty(far + 2 * tk * 64, dtype=BF16, device="cuda")
    k, v = (store.as_strided((2, tk, 1, 64), (far, 64, 64, 1), at) for at in (0, tk * 64))
    k.copy_(randn(2, tk, 1, 64, dtype=BF16, seed=1))
    v.copy_(randn(2, tk, 1, 64, dtype=BF16, seed=2))
    q, do = randn(2, tq, 2, 64, dtype=BF16, seed=3), randn(2, tq, 2, 64, dtype=BF16, seed=4)
    check_attention(q, k, v, do)


def test_cross_attention_long_states():
    """More states than one CTA walks alone, and a length that ends inside a tile of the last part."""
    for h, hk, d, dtype in ((4, 1, 64, BF16), (2, 2, 128, F16)):
        q, k, v, do = attention_inputs(1, 1, 20011, h, hk, d, dtype, seed=8, layout="heads")
        nk = torch.tensor([19999], dtype=torch.int32, device="cuda")
        check_attention(q, k, v, do)
        check_attention(q, k, v, do, nk=nk)


@pytest.mark.parametrize("h,hk,d,dtype", [(4, 2, 64, BF16), (2, 2, 128, F16), (3, 1, 96, BF16)])
def test_cross_attention_split_states_of_many_rows(h, hk, d, dtype):
    """Few row tiles over many states, whole, and of lengths that leave some parts without states."""
    q, k, v, do = attention_inputs(2, 140, 4100, h, hk, d, dtype, seed=14, layout="packed")
    check_attention(q, k, v, do)
    nk = torch.tensor([4033, 130], dtype=torch.int32, device="cuda")
    nq = torch.tensor([129, 140], dtype=torch.int32, device="cuda")
    check_attention(q, k, v, do, nq=nq, nk=nk)


@pytest.mark.parametrize("h,hk,d,dtype", [(4, 2, 64, BF16), (2, 2, 128, F16), (3, 1, 96, BF16)])
def test_cross_attention_split_rows_of_few_states(h, hk, d, dtype):
    """Few tiles of states under many rows, whole, and of lengths that leave some parts without rows."""
    q, k, v, do = attention_inputs(2, 4100, 130, h, hk, d, dtype, seed=15, layout="packed")
    check_attention(q, k, v, do)
    nq = torch.tensor([4033, 70], dtype=torch.int32, device="cuda")
    nk = torch.tensor([129, 130], dtype=torch.int32, device="cuda")
    check_attention(q, k, v, do, nq=nq, nk=nk)


def test_cross_attention_gradient_is_the_difference():
    q, k, v, do = attention_inputs(1, 9, 150, 2, 1, 64, F16, seed=12)
    o, lse = ops.cross_attention(q, k, v, need_lse=True)
    grads = ops.cross_attention_backward(do, q, k, v, o, lse)
    ref = attention_reference(q, k, v, 0.125, [9], [150], do, U[F16])
    h = 1e-4

    def loss(q_, k_, v_):
        return (attention_reference(q_, k_, v_, 0.125, [9], [150])["o"] * do.double()).sum().item()

    base = [x.double() for x in (q, k, v)]
    for at, (grad, name) in enumerate(zip(grads, ("dq", "dk", "dv"))):
        step = randn(*grad.shape, seed=30 + at).double()
        up, down = ([x + s * h * step if i == at else x for i, x in enumerate(base)] for s in (1, -1))
        num = (loss(*up) - loss(*down)) / (2 * h)
        assert abs(num - (grad.double() * step).sum().item()) <= (ref[name + "_b"] * step.abs()).sum().item() + 1e-5


def test_operators_on_another_stream_and_in_a_graph():
    side = torch.cuda.Stream()
    q, k, v, do = attention_inputs(2, 140, 150, 4, 2, 64, BF16, seed=6)
    x, r, w = randn(64, 512, dtype=BF16, seed=1), randn(64, 512, dtype=BF16, seed=2), 1 + 0.3 * randn(512, seed=3)

    def everything():
        o, lse = ops.cross_attention(q, k, v, need_lse=True)
        y, total = ops.add_rms_norm(x, w, residual=r, rate=0.1, seed=3, event=4)
        return [o, lse, ops.cross_attention(q[:, :1], k, v), *ops.cross_attention_backward(do, q, k, v, o, lse), y, total,
                *ops.add_rms_norm_backward(r, total, w, dtotal=x, rate=0.1, seed=3, event=4), ops.dropout(x, 0.1, 3, 4)]

    want = everything()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got = everything()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = everything()
    for t in out:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    ops.check()


@pytest.mark.parametrize("d", [64, 128])
def test_waits_that_give_up_are_reported_and_leave_the_device_usable(d):
    """wait_limit 0: every device-side wait gives up at once. The kernels return, the next check says so, and the
    calls after it are right again."""
    q, k, v, do = attention_inputs(2, 150, 200, 2, 2, d, BF16, seed=5)
    o, lse = ops.cross_attention(q, k, v, need_lse=True)
    ops.check()
    ops.cross_attention(q, k, v, wait_limit=0)
    with pytest.raises(g.SwarmError) as err:
        ops.check()
    assert err.value.code == g.ECUDA and g.load().swarm_operator_error() == 702       # cudaErrorLaunchTimeout
    ops.check()                                                                       # reported once
    ops.cross_attention_backward(do, q, k, v, o, lse, wait_limit=0)
    with pytest.raises(g.SwarmError):
        ops.check()
    check_attention(q, k, v, do)


def test_refusals_of_the_tensor_checks():
    x, w = randn(4, 64, dtype=BF16), torch.ones(64, device="cuda")
    for bad in (lambda: ops.dropout(x, 1.5, 1, 1), lambda: ops.dropout(x, float("nan"), 1, 1), lambda: ops.dropout(x, 0.1, -1, 1),
                lambda: ops.dropout(x, 0.1, 1, 2 ** 32), lambda: ops.dropout(x.cpu(), 0.1, 1, 1),
                lambda: ops.dropout(x.double(), 0.1, 1, 1), lambda: ops.dropout(x, 0.1, 1, 1, residual=x.float()),
                lambda: ops.dropout(x, 0.1, 1, 1, residual=x[:2]), lambda: ops.dropout(x.t(), 0.1, 1, 1),
                lambda: ops.dropout(torch.zeros(4, 5, 64, device="cuda")[:, :4], 0.1, 1, 1),
                lambda: ops.add_rms_norm(x, w.to(BF16)), lambda: ops.add_rms_norm(x, w[:60]),
                lambda: ops.add_rms_norm(x, torch.ones(128, device="cuda")[::2]),
                lambda: ops.add_rms_norm_backward(x, x[:3], w)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: ops.add_rms_norm(x, w, eps=-1.0), lambda: ops.add_rms_norm(x, w, eps=float("inf")),
                lambda: ops.add_rms_norm(torch.zeros(1, 32769, device="cuda"), torch.ones(32769, device="cuda"))):
        with pytest.raises(g.SwarmError):
            bad()
    q, k, v, do = attention_inputs(2, 5, 7, 4, 2, 64, BF16)
    f = ops.cross_attention
    for bad in (lambda: f(q.float(), k.float(), v.float()), lambda: f(q, k.half(), v), lambda: f(q, k[:1], v),
                lambda: f(q, k, v[:, :5]), lambda: f(q[0], k, v), lambda: f(q.transpose(2, 3), k, v),
                lambda: f(q, k, v, key_lengths=torch.zeros(2, device="cuda")),
                lambda: f(q, k, v, key_lengths=torch.zeros(3, dtype=torch.int32, device="cuda")),
                lambda: f(q.cpu(), k, v), lambda: f(q, k, v, out=torch.empty(2, 5, 4, 32, dtype=BF16, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    off = torch.zeros(2 * 7 * 2 * 64 + 8, dtype=BF16, device="cuda")[1:1 + 2 * 7 * 2 * 64].view(2, 7, 2, 64)
    for bad in (lambda: f(q, off, v), lambda: f(q, k, v, scale=0.0), lambda: f(q, k, v, scale=float("nan")),
                lambda: f(q[:, :, :3], k, v), lambda: f(q[..., :60].contiguous(), k[..., :60].contiguous(), v[..., :60].contiguous()),
                lambda: f(randn(1, 2, 1, 136, dtype=BF16), randn(1, 2, 1, 136, dtype=BF16), randn(1, 2, 1, 136, dtype=BF16)),
                lambda: f(q, k, v, out=torch.empty(1, 5, 4, 64, dtype=BF16, device="cuda").expand(2, -1, -1, -1))):
        with pytest.raises(g.SwarmError):
            bad()
    torch.cuda.synchronize()


@pytest.mark.parametrize("b,tq,tk,h,hk,d", [(40, 150, 120, 4, 4, 64), (40, 150, 120, 4, 2, 128), (3, 300, 700, 4, 2, 64), (3, 300, 700, 4, 4, 128),
                                            (1, 140, 4100, 2, 1, 64), (1, 4100, 130, 2, 1, 128)])
def test_waits_that_give_up_in_mid_call_leave_nothing_in_flight(b, tq, tk, h, hk, d):
    """Small positive limits: some threads of a CTA give up while others have copies and products under way, or are already
    through. The call is either reported or right, and so are the calls whose CTAs follow on the same multiprocessors."""
    q, k, v, do = attention_inputs(b, tq, tk, h, hk, d, BF16, seed=5)
    o, lse = ops.cross_attention(q, k, v, need_lse=True)
    grads = ops.cross_attention_backward(do, q, k, v, o, lse)
    ops.check()
    for limit in (1, 2, 3, 5, 8, 13, 30, 100, 1000):
        for call, want in ((lambda **kw: ops.cross_attention(q, k, v, need_lse=True, **kw), (o, lse)),
                           (lambda **kw: ops.cross_attention_backward(do, q, k, v, o, lse, **kw), grads)):
            short, right = call(wait_limit=limit), call()
            assert all(torch.equal(x, y) for x, y in zip(right, want)), limit
            try:
                ops.check()
            except g.SwarmError as err:
                assert err.code == g.ECUDA and g.load().swarm_operator_error() == 702
            else:
                assert all(torch.equal(x, y) for x, y in zip(short, want)), limit
    ops.check()


# ---- gradients away from unit size ---------------------------------------------------------------------------------


def beside_rounding(got, want, factor, what):
    """The error of `got` as a whole is at most `factor` times what rounding the exact result to its type leaves."""
    assert torch.isfinite(got).all(), what
    alone = (want.to(got.dtype).double() - want).norm().item()
    off = (got.double() - want).norm().item()
    assert off <= factor * alone, (what, off / alone)


def check_gradients_beside_rounding(q, k, v, do, scale=None, nq=None, nk=None, sentences=None, names=("dq", "dk", "dv")):
    """p and ds are each rounded once before their products, o once before delta: independent errors of the size of the
    result's own rounding, so that four of them come to twice it, and three times bounds them on any sizes."""
    b, tq, tk = q.shape[0], q.shape[1], k.shape[1]
    lq, lk = nq.tolist() if nq is not None else [tq] * b, nk.tolist() if nk is not None else [tk] * b
    ref = attention_reference(q, k, v, scale or q.shape[3] ** -0.5, lq, lk, do, U[q.dtype])
    kw = dict(scale=scale, query_lengths=nq, key_lengths=nk)
    o, lse = ops.cross_attention(q, k, v, need_lse=True, **kw)
    got = dict(zip(("dq", "dk", "dv"), ops.cross_attention_backward(do, q, k, v, o, lse, **kw)))
    ops.check()
    for name in names:
        for i in sentences or range(b):
            beside_rounding(got[name][i], ref[name][i], 3.0, (name, i))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("d", [64, 128])
def test_cross_attention_split_states_of_short_sentences(dtype, d):
    """Sentences of 6 and of 64 states beside a long one, whose states are split over CTAs. The values share a large part,
    so that the rounding of o would show in dk if it were not taken out of delta."""
    q, k, v, do = attention_inputs(3, 140, 4100, 2, 1, d, dtype, seed=39)
    v = (v.float() + 16).to(dtype)
    nk = torch.tensor([4100, 6, 64], dtype=torch.int32, device="cuda")
    check_gradients_beside_rounding(q, k, v, do, nk=nk, sentences=(1, 2), names=("dq", "dk"))
    short = slice(1, 3)
    check_gradients_beside_rounding(q[short], k[short, :64], v[short, :64], do[short], nk=nk[short], names=("dq", "dk"))


@pytest.mark.parametrize("tq,d,scale,size", [(140, 128, 2.0 ** -20, 360.0), (140, 64, 2.0 ** -20, 420.0), (9, 128, 2.0 ** 12, 0.007)])
def test_cross_attention_gradients_of_large_and_small_scales_fp16(tq, d, scale, size):
    """lse / scale, in which one of the kernels keeps a row's statistics, far above and far below the scores of unit normals."""
    q, k, v, do = attention_inputs(2, tq, 200, 2, 1, d, F16, seed=31)
    q, k = (q.float() * (size / 1.5)).to(F16), (k.float() * size).to(F16)
    check_gradients_beside_rounding(q, k, v, (do.float() / 64).to(F16) if scale > 1 else do, scale=scale)


def test_cross_attention_gradients_of_scores_in_the_millions_fp16():
    """Rows that each attend to one state, their products with it 2^23: all of a row's weight is there."""
    gen = torch.Generator(device="cuda").manual_seed(32)
    k = (torch.randint(0, 2, (1, 150, 2, 128), generator=gen, device="cuda") * 512 - 256).to(F16)
    at = torch.randint(0, 150, (140,), generator=gen, device="cuda")
    q, scale = k[:, at].contiguous(), 2.0 ** -4
    v, do = randn(1, 150, 2, 128, dtype=F16, seed=33), randn(1, 140, 2, 128, dtype=F16, seed=34)
    o, lse = ops.cross_attention(q, k, v, scale=scale, need_lse=True)
    dq, dk, dv = ops.cross_attention_backward(do, q, k, v, o, lse, scale=scale)
    assert torch.equal(o, v[:, at]) and (lse == 2.0 ** 19).all()
    want = torch.zeros(1, 150, 2, 128, dtype=torch.float64, device="cuda").index_add_(1, at, do.double())
    # fp32 numbers of 2^23 are 1 apart: the product, lse / scale, its parts and their sum leave four of them, times the scale
    size = torch.zeros_like(want).index_add_(1, at, do.double().abs())
    within(dv, want, size * (math.exp(4 * scale) - 1) + U[F16] * want.abs(), "dv")


def test_cross_attention_gradients_with_a_large_common_part_fp16():
    """rowsum(dout * o) of 2^23, of which the differences between the states are a hundredth."""
    q, k, v, do = attention_inputs(2, 20, 30, 2, 1, 128, F16, seed=35)
    v, do = (v.float() + 8).to(F16), (do.float() * 64 + 8192).to(F16)
    s = 128 ** -0.5
    ref = attention_reference(q, k, v, s, [20] * 2, [30] * 2, do, U[F16])
    o, lse = ops.cross_attention(q, k, v, need_lse=True)
    got = dict(zip(("dq", "dk", "dv"), ops.cross_attention_backward(do, q, k, v, o, lse)))
    for name in ("dq", "dk"):
        within(got[name], ref[name], ref[name + "_b"], name)


DOUT_SHAPES = [(1, 300, 4096, 4, 2, 128), (1, 140, 4100, 2, 1, 64), (8, 300, 4000, 4, 4, 128), (8, 140, 4000, 20, 4, 64), (1, 4100, 130, 2, 1, 64),
               (2, 50, 61, 4, 2, 128)]


def check_gradients_of_size(shape, size, names):
    q, k, v, do = attention_inputs(*shape, F16, seed=36)
    check_gradients_beside_rounding(q, k, v, (do.float() * size).to(F16), sentences=range(min(shape[0], 2)), names=names)


def check_gradients_are_linear(tq, tk, d, power, names):
    """A power of two times dout is the same power of two times the gradients, but for where their last rounding falls:
    half a step of either side. dout holds multiples of 2^-6, so that all of its multiples here are exact."""
    q, k, v, do = attention_inputs(2, tq, tk, 2, 1, d, F16, seed=38)
    do, v = ((do.float() * 64).round() / 64).clamp(-3.5, 3.5).to(F16), (v.float() * 4).to(F16)
    o, lse = ops.cross_attention(q, k, v, need_lse=True)
    one = ops.cross_attention_backward(do, q, k, v, o, lse)
    scaled = (do.float() * 2.0 ** power).to(F16)
    assert torch.equal(scaled.double(), do.double() * 2.0 ** power)
    other = ops.cross_attention_backward(scaled, q, k, v, o, lse)
    for name, x, y in zip(("dq", "dk", "dv"), one, other):
        if name not in names:
            continue
        want = x.double() * 2.0 ** power
        room = want.abs() < 60000                                                   # what fits the type
        assert room.double().mean() > 0.5, name
        within(y[room], want[room], 2.01 * U[F16] * want[room].abs() + 2.0 ** (power - 25) + 2.0 ** -25, name)


@pytest.mark.parametrize("shape", DOUT_SHAPES)
@pytest.mark.parametrize("size", [1e-2, 1e-3, 1e-4, 64.0])
def test_cross_attention_dq_of_small_and_large_dout_fp16(shape, size):
    check_gradients_of_size(shape, size, ("dq", "dv"))


@pytest.mark.parametrize("tq,tk,d", [(4, 2, 128), (4, 130, 64), (140, 200, 128), (20, 4100, 64)])
@pytest.mark.parametrize("power", [-18, -6, 7, 13])
def test_cross_attention_dq_is_linear_in_dout_fp16(tq, tk, d, power):
    check_gradients_are_linear(tq, tk, d, power, ("dq", "dv"))


@pytest.mark.parametrize("tk", [700, 5000])
def test_cross_attention_dq_of_rows_of_unequal_size_fp16(tk):
    """Rows of dout 2^-14 of the others, and first steps of states that take e^-25 of the weight."""
    q, k, v, do = attention_inputs(1, 260, tk, 2, 1, 128, F16, seed=37)
    do, k = do.float(), k.float()
    do[:, 100:] *= 2.0 ** -14
    k[:, :130] -= 1.5
    q, k, do = (q.float() + 1.5).to(F16), k.to(F16), do.to(F16)
    ref = attention_reference(q, k, v, 128 ** -0.5, [260], [tk], do, U[F16])
    o, lse = ops.cross_attention(q, k, v, need_lse=True)
    dq = ops.cross_attention_backward(do, q, k, v, o, lse)[0]
    beside_rounding(dq[:, :100], ref["dq"][:, :100], 3.0, "large rows")
    beside_rounding(dq[:, 100:], ref["dq"][:, 100:], 3.0, "small rows")


@pytest.mark.parametrize("shape", DOUT_SHAPES)
@pytest.mark.parametrize("size", [1e-2, 1e-3, 1e-4, 64.0])
def test_cross_attention_dk_of_small_and_large_dout_fp16(shape, size):
    check_gradients_of_size(shape, size, ("dk",))


@pytest.mark.parametrize("tq,tk,d", [(4, 2, 128), (4, 130, 64), (140, 200, 128), (20, 4100, 64)])
@pytest.mark.parametrize("power", [-18, -6, 7, 13])
def test_cross_attention_dk_is_linear_in_dout_fp16(tq, tk, d, power):
    check_gradients_are_linear(tq, tk, d, power, ("dk",))


@pytest.mark.parametrize("tq,tk,h,hk,d", [(260, 700, 2, 1, 128), (140, 5000, 2, 2, 64), (4100, 200, 2, 1, 128)])
def test_cross_attention_dk_of_unequal_sizes_fp16(tq, tk, h, hk, d):
    """Rows of dout 2^-12 of the others, alone in the second sentence, and states that take e^-12 of the weight."""
    q, k, v, do = attention_inputs(2, tq, tk, h, hk, d, F16, seed=40)
    do, k, shift = do.float() * 1024, k.float(), 12 / 1.5 / d ** 0.5
    do[:, 100:] *= 2.0 ** -12
    do[1, :100] = 0
    k[:, :130] -= shift
    q, k, do = (q.float() + 1.5).to(F16), k.to(F16), do.to(F16)
    lengths = torch.tensor([tq, tq - 3], dtype=torch.int32, device="cuda")
    ref = attention_reference(q, k, v, d ** -0.5, lengths.tolist(), [tk] * 2, do, U[F16])
    o, lse = ops.cross_attention(q, k, v, need_lse=True, query_lengths=lengths)
    _, dk, dv = ops.cross_attention_backward(do, q, k, v, o, lse, query_lengths=lengths)
    for i in range(2):
        beside_rounding(dk[i, :130], ref["dk"][i, :130], 3.0, ("light states", i))
        beside_rounding(dk[i, 130:], ref["dk"][i, 130:], 3.0, ("the others", i))
        beside_rounding(dv[i], ref["dv"][i], 3.0, ("dv", i))


def test_refusals_of_numbers_that_the_call_cannot_hold():
    q, k, v, do = attention_inputs(2, 5, 7, 4, 2, 64, BF16)
    o, lse = ops.cross_attention(q, k, v, need_lse=True)
    for bad in (dict(scale=1e300), dict(scale=-1e300), dict(wait_limit=1 << 70), dict(scale="a")):
        with pytest.raises(ValueError):
            ops.cross_attention(q, k, v, **bad)
        with pytest.raises(ValueError):
            ops.cross_attention_backward(do, q, k, v, o, lse, **bad)
    with pytest.raises(ValueError):
        ops.cross_attention(q[..., :0], k[..., :0], v[..., :0])


def step_of_ds(q, k, v, do, scale):
    """Half a step of ds at its smallest in fp16, per key head, times scale and the sum of |q| that it meets in dk: ds is
    held so that its largest value, or 2^-7 of a row's sum of |dout|, lies between 2^13 and 2^14, in steps of 2^-24."""
    b, tq, h, d = q.shape
    hk = k.shape[2]
    q, k, v, do = (x.double().transpose(1, 2) for x in (q, k.repeat_interleave(h // hk, 2), v.repeat_interleave(h // hk, 2), do))
    p = torch.softmax(scale * q @ k.transpose(2, 3), -1)
    dp = do @ v.transpose(2, 3)
    ds = (p * (dp - (p * dp).sum(-1, keepdim=True))).abs().amax(-1)
    peak = torch.maximum(ds, do.abs().sum(-1) / 128).reshape(b, hk, -1).amax(-1)
    return 2.0 ** -38 * scale * peak[:, None, :, None] * q.abs().reshape(b, hk, -1, d).sum(2)[:, None]


@pytest.mark.parametrize("tk,sharp", [(1, 1.0), (2, 1.0), (2, 30.0), (3, 30.0), (40, 30.0), (64, 30.0)])
@pytest.mark.parametrize("tq,d", [(16, 64), (140, 64), (16, 128), (300, 128), (300, 96)])
def test_cross_attention_gradients_that_cancel_fp16(tk, sharp, tq, d):
    """One state, or rows that attend to one state alone: the gradients of the scores are 0 but for what rounding leaves,
    which differs between the kernels and says nothing about the size of the other's. What passes fp16's end is not compared."""
    q, k, v, do = attention_inputs(6, tq, tk, 4, 2, d, F16, seed=41)
    q, v = (q.float() * sharp).to(F16), (v.float() * 3 + 5).to(F16)
    o, lse = ops.cross_attention(q, k, v, need_lse=True)
    for dout in (do, (do.float() * 100 + 900).to(F16)):
        ref = attention_reference(q, k, v, d ** -0.5, [tq] * 6, [tk] * 6, dout, U[F16])
        ref["dk_b"] += step_of_ds(q, k, v, dout, d ** -0.5)
        for name, x in zip(("dq", "dk", "dv"), ops.cross_attention_backward(dout, q, k, v, o, lse)):
            assert not torch.isnan(x).any(), name
            room = ref[name].abs() + ref[name + "_b"] < 65504
            within(x[room], ref[name][room], ref[name + "_b"][room] + TINY[F16], name)


# ---- masks over whole grids and wide rows ---------------------------------------------------------------------------


def factors_at_once(rows, cols, rate, seed, event):
    """As `factors`, all generator calls side by side."""
    import numpy as np
    u, groups = np.uint64, (cols + 7) // 8
    low, half = u(0xFFFFFFFF), u(32)
    c = [np.tile(np.arange(groups, dtype=u), rows), np.repeat(np.arange(rows, dtype=u), groups), np.full(rows * groups, event, dtype=u),
         np.full(rows * groups, 13, dtype=u)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        p0, p1 = u(0xD2511F53) * c[0], u(0xCD9E8D57) * c[2]
        c = [(p1 >> half) ^ c[1] ^ u(k[0]), p1 & low, (p0 >> half) ^ c[3] ^ u(k[1]), p0 & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    draws = np.stack([w >> u(16 * i) & u(0xFFFF) for w in c for i in (0, 1)], 1).reshape(rows, groups * 8)[:, :cols]
    drop = math.floor(rate * 65536 + 0.5)
    return torch.from_numpy(np.where(draws >= u(drop), 65536 / (65536 - drop), 0.0)).cuda()


def test_the_two_ways_to_draw_a_mask_agree():
    assert torch.equal(factors(5, 83, 0.3, 0xFEDCBA9876543210, 4000000000), factors_at_once(5, 83, 0.3, 0xFEDCBA9876543210, 4000000000))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols", [(70001, 48), (30011, 128), (9001, 1000), (5003, 1001), (1201, 8200), (901, 4099)])
def test_dropout_over_several_passes_of_the_grid(dtype, rows, cols):
    x = torch.ones(rows, cols, dtype=dtype, device="cuda")
    got = ops.dropout(x, 0.3, 41, 42)
    m = factors_at_once(rows, cols, 0.3, 41, 42)
    within(got, m, U[dtype] * m + 2.0 ** -22 * m)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("rows,cols", [(5, 1201), (900, 2048), (3, 3000), (400, 4096), (3, 4100), (300, 8192), (2, 16000), (40, 16384), (2, 32768)])
def test_norm_masks_of_wide_rows(dtype, rows, cols):
    rate, seed, event = 0.3, 2 ** 40 + 5, 6
    x, r, dy = (randn(rows, cols, dtype=dtype, seed=s) for s in (1, 2, 3))
    w = 1 + 0.3 * randn(cols, seed=4)
    m = factors_at_once(rows, cols, rate, seed, event)
    total, want = norm_reference(x, r, w, 1e-6, m)
    how = dict(rate=rate, seed=seed, event=event)
    y, kept = ops.add_rms_norm(x, w, residual=r, **how)
    size = (x.double() * m).abs() + r.double().abs()
    within(kept, total, U[dtype] * total.abs() + 2.0 ** -22 * size + TINY[dtype])
    rstd = 1 / (total.square().mean(1, keepdim=True) + 1e-6).sqrt()
    within(y, want, (U[dtype] + E) * want.abs() + 2.0 ** -22 * size * rstd * w.double().abs() + TINY[dtype])
    assert torch.equal(ops.add_rms_norm(x, w, residual=r, eight_bit=True, **how)[2], kept)
    t, wdy = kept.double(), w.double() * dy.double()
    rt = 1 / (t.square().mean(1, keepdim=True) + 1e-6).sqrt()
    grad = rt * wdy - t * rt ** 3 * (wdy * t).mean(1, keepdim=True)
    size = rt * wdy.abs() + t.abs() * rt ** 3 * (wdy * t).abs().mean(1, keepdim=True)
    dx, dres, _ = ops.add_rms_norm_backward(dy, kept, w, **how)
    within(dres, grad, U[dtype] * grad.abs() + E * size + TINY[dtype])
    within(dx, grad * m, U[dtype] * (grad * m).abs() + E * size * 2 + TINY[dtype])
    assert ((dx == 0) | (m > 0)).all()


@pytest.mark.parametrize("tq,tk,d,dtype", [(40, 100, 64, F16), (200, 300, 128, F16), (150, 270, 72, F16), (1, 300, 128, F16), (140, 4100, 64, F16),
                                           (140, 4100, 128, BF16), (2100, 130, 64, BF16), (2100, 130, 128, F16)])
def test_cross_attention_takes_nothing_from_past_the_ends_in_its_other_forms(tq, tk, d, dtype):
    """NaN and infinities past the ends, in fp16 and where states or rows are split: the same bits as without them."""
    clean = attention_inputs(2, tq, tk, 2, 1, d, dtype, seed=9, layout="packed")
    nk = torch.tensor([tk - 3, max(1, tk // 3)], dtype=torch.int32, device="cuda")
    nq = torch.tensor([max(1, tq // 2 - 1), max(1, tq - 5)], dtype=torch.int32, device="cuda")
    dirty = [x.clone() for x in clean]
    for i in range(2):
        for x, n in zip(dirty, (nq, nk, nk, nq)):
            x[i, int(n[i]):] = float("nan")
            x[i, int(n[i])::2] = float("inf")
            x[i, int(n[i])::3] = -float("inf")
    ends = dict(query_lengths=nq, key_lengths=nk)
    results = []
    for q, k, v, do in (clean, dirty):
        o, lse = ops.cross_attention(q, k, v, need_lse=True, **ends)
        results.append([o, lse, *ops.cross_attention_backward(do, q, k, v, o, lse, **ends)])
    assert all(torch.equal(x, y) for x, y in zip(*results))
