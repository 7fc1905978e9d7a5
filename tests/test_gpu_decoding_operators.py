"""The paged cache, attention over it and the log probabilities of tokens, against their formulas in 64 bits.

Tolerances are bounds, not observations. U is the largest relative rounding error of a type. What fp32 arithmetic adds:
  rotation      two products, a sum, and a sine and a cosine that are off by 2^-23 at most: 2^-21 (|x| + |y|); angles that leave a
                double's 53 bits add their last place
  attention     E = 2e-5 (128-term dot products, base-2 exponentials) times the sum of the weighted magnitudes, and 2^-16 for
                weights that go into their products as two numbers of the type
  log probs     sums of n positive terms, each thread a run of n / 256, or of n / 32 where a warp may take the row (n <= 16384):
                (run + 16) 2^-24; exponentials of d: (|d| + 4) 2^-23
"""
import math

import pytest

from paper_1910_12308_b200 import binding as g

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_1910_12308_b200 import operators as ops  # noqa: E402

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
U = {BF16: 2.0 ** -8, F16: 2.0 ** -11, F32: 2.0 ** -24}
TINY = {BF16: 1e-38, F16: 2.0 ** -24, F32: 1e-37}        # a result may fall among the subnormals of its type
E = 2e-5 + 2.0 ** -16


def run(n):
    return n / (32 if n <= 16384 else 256)


def randn(*shape, dtype=F32, seed=0, std=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=gen, device="cuda") * std).to(dtype)


def ints(*values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def within(got, want, bound, what=""):
    got, want = got.double(), want.double()
    assert got.shape == want.shape, what
    assert not torch.isnan(got).any(), what
    over = (got - want).abs() - bound
    assert over.max().item() <= 0 if over.numel() else True, (what, over.max().item(), (got - want).abs().max().item())


def make_cache(lengths, page_size, kv_heads, dim, dtype, layout="tokens", seed=0, fill=None, spare=3):
    """Pages in a shuffled order, just as many as the lengths need; the rest of the table is -1."""
    need = [-(-n // page_size) for n in lengths]
    pages, columns = sum(need) + spare, max(need + [0]) + 1
    shape = (pages, page_size, kv_heads, dim) if layout == "tokens" else (pages, kv_heads, page_size, dim)

    def one(s):
        x = randn(*shape, dtype=dtype, seed=seed + s) if fill is None else torch.full(shape, fill, dtype=dtype, device="cuda")
        return x if layout == "tokens" else x.transpose(1, 2)

    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed))
    table, at = torch.full((len(lengths), columns), -1, dtype=torch.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n].to(torch.int32)
        at += n
    return one(1), one(2), table.cuda()


def held(pages, table, b, length):
    """The tokens of a sentence, in order."""
    at = torch.arange(length, device="cuda")
    return pages[table[b][at // pages.shape[1]].long(), at % pages.shape[1]]


# ---- appending -----------------------------------------------------------------------------------------------------


def rotated(x, positions, frequencies, interleaved):
    """The first values of x [n, heads, dim] turned by position * frequency, in 64 bits; also |x| + |y| of each pair."""
    x = x.double().clone()
    size = x.abs()
    half = 0 if frequencies is None else len(frequencies)
    if half:
        angle = (positions.double().unsqueeze(1) * frequencies.double()).unsqueeze(1)
        first, second = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
        a, b = x[..., first].clone(), x[..., second].clone()
        x[..., first], x[..., second] = a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()
        size[..., first] = size[..., second] = a.abs() + b.abs()
    return x, size


def check_append(q, k, v, caches, table, lengths, counts, frequencies, interleaved, got_q, after, far=0.0):
    """after: the pages when the call has been made, caches: before."""
    dtype = k.dtype
    want = [c.double().clone() for c in caches]
    room = [torch.zeros(c.shape, dtype=torch.float64, device="cuda") for c in caches]
    slack = 2.0 ** -21 + far
    for b in range(k.shape[0]):
        n = min(max(counts[b], 0), k.shape[1], max(lengths[b], 0))
        at = torch.arange(lengths[b] - n, lengths[b], device="cuda")
        if q is not None:
            wq, size = rotated(q[b, :n], at, frequencies, interleaved)
            within(got_q[b, :n], wq, U[dtype] * wq.abs() + slack * size + TINY[dtype], "q")
            assert not got_q[b, n:].any()
        if not n:
            continue
        page, slot = table[b][at // k_size(caches)].long(), at % k_size(caches)
        wk, size = rotated(k[b, :n], at, frequencies, interleaved)
        want[0][page, slot], want[1][page, slot] = wk, v[b, :n].double()
        room[0][page, slot] = U[dtype] * wk.abs() + slack * size + TINY[dtype]
    for x, w, r in zip(after, want, room):
        within(x, w, r, "pages")


def k_size(caches):
    return caches[0].shape[1]


@pytest.mark.parametrize("dtype,dim,rot,interleaved,page,layout", [
    (BF16, 64, 64, False, 16, "tokens"), (F16, 128, 128, False, 64, "heads"), (BF16, 128, 64, True, 24, "heads"), (F16, 80, 80, False, 7, "tokens"),
    (BF16, 40, 40, False, 1, "tokens"), (F16, 72, 36, True, 5, "heads"), (BF16, 8, 8, True, 3, "tokens"), (F16, 96, 6, False, 33, "tokens"),
    (BF16, 48, 2, False, 16, "heads"), (F16, 64, 0, False, 10, "tokens"), (BF16, 104, 104, True, 128, "tokens"), (F16, 128, 16, False, 8, "tokens")])
def test_append(dtype, dim, rot, interleaved, page, layout):
    tokens, heads, kv_heads = 9, 6, 2
    lengths, counts = [9, 40, 3, 0, 100, 5, 17], [9, 3, 9, 4, 0, 5, -2]
    caches = make_cache(lengths, page, kv_heads, dim, dtype, layout, seed=dim)
    q, k, v = (randn(7, tokens, h, dim, dtype=dtype, seed=s) for s, h in ((1, heads), (2, kv_heads), (3, kv_heads)))
    freq = 10000.0 ** (-torch.arange(rot // 2, device="cuda") / max(rot // 2, 1)) if rot else None
    before = [c.clone() for c in caches[:2]]
    got = ops.append_to_cache(k, v, *caches, ints(*lengths), counts=ints(*counts), q=q, frequencies=freq, interleaved=interleaved)
    check_append(q, k, v, before, caches[2], lengths, counts, freq, interleaved, got, caches[:2])
    ops.check()


@pytest.mark.parametrize("tokens,batch,heads,kv_heads", [(1, 1, 1, 1), (1, 3, 33, 11), (1, 200, 8, 8), (700, 2, 8, 2), (33, 5, 1, 1)])
def test_append_whole_calls(tokens, batch, heads, kv_heads):
    lengths = [tokens + 3 * b for b in range(batch)]
    caches = make_cache(lengths, 16, kv_heads, 64, BF16, seed=5)
    q, k, v = (randn(batch, tokens, h, 64, dtype=BF16, seed=s) for s, h in ((1, heads), (2, kv_heads), (3, kv_heads)))
    freq = 10000.0 ** (-torch.arange(32, device="cuda") / 32)
    before = [c.clone() for c in caches[:2]]
    got = ops.append_to_cache(k, v, *caches, ints(*lengths), q=q, frequencies=freq)
    check_append(q, k, v, before, caches[2], lengths, [tokens] * batch, freq, False, got, caches[:2])
    again = [c.clone() for c in before]
    assert ops.append_to_cache(k, v, *again, caches[2], ints(*lengths), frequencies=freq) is None       # without queries
    assert torch.equal(again[0], caches[0]) and torch.equal(again[1], caches[1])


def test_append_takes_strides_and_writes_over_its_queries():
    b, t, h, hk, d = 3, 5, 4, 2, 48
    lengths = [5, 20, 11]
    qkv = randn(b, t, h + 2 * hk, d, dtype=BF16, seed=7)                        # one projection's output
    q, k, v = qkv[:, :, :h], qkv[:, :, h:h + hk], qkv[:, :, h + hk:]
    both = randn(9, 2, 16, hk, d, dtype=BF16, seed=8)                           # pages of keys and values side by side
    table = torch.tensor([[3, 0], [5, 1], [8, 7]], dtype=torch.int32, device="cuda")
    wide = torch.full((3, 5), -1, dtype=torch.int32, device="cuda")
    wide[:, 1:3] = table
    freq = 100.0 ** (-torch.arange(24, device="cuda") / 24)
    plain = [both[:, i].clone() for i in range(2)]
    want = ops.append_to_cache(k.contiguous(), v.contiguous(), *plain, table, ints(*lengths), q=q.contiguous(), frequencies=freq)
    got = ops.append_to_cache(k, v, both[:, 0], both[:, 1], wide[:, 1:3], ints(*lengths), q=q, frequencies=freq, out=q)
    assert got.data_ptr() == q.data_ptr() and torch.equal(q, want)
    assert torch.equal(both[:, 0], plain[0]) and torch.equal(both[:, 1], plain[1])
    one = k[:, :, :1].expand(b, t, hk, d)                                       # a key head repeated by a stride of 0
    ops.append_to_cache(one, v, both[:, 0], both[:, 1], table, ints(*lengths), frequencies=freq)
    assert torch.equal(both[3, 0, :5, 0], both[3, 0, :5, 1])


def test_append_at_far_positions():
    size, d = 1 << 20, 8
    last = 2 ** 31 - 1                                                          # tokens of the longest sentence there can be
    table = torch.full((1, 2048), -1, dtype=torch.int32, device="cuda")
    table[0, 2047] = 0
    freq = torch.tensor([1.0, 0.7531, 3.1e-3, 2.0 ** -20], device="cuda")
    q, k, v = (randn(1, 4, 1, d, dtype=F16, seed=s) for s in (1, 2, 3))
    caches = [torch.zeros(1, size, 1, d, dtype=F16, device="cuda") for _ in range(2)]
    got = ops.append_to_cache(k, v, *caches, table, ints(last), q=q, frequencies=freq)
    before = [torch.zeros_like(c) for c in caches]
    # an angle of 2^31 keeps 22 bits behind the point in 64 bits, whichever way it is formed
    check_append(q, k, v, before, table, [last], [4], freq, False, got, caches, far=2.0 ** -20)


def test_pages_that_do_not_exist_are_not_followed():
    lengths, hk, d = [20, 20, 20, 20], 2, 64
    k_pages, v_pages = (randn(6, 8, hk, d, dtype=BF16, seed=s) for s in (1, 2))
    table = torch.tensor([[0, 1, 2], [3, 6, 4], [-1, 5, -2 ** 31], [2 ** 31 - 1, -7, 99]], dtype=torch.int32, device="cuda")
    before = k_pages.clone(), v_pages.clone()
    q, k, v = (randn(4, 20, h, d, dtype=BF16, seed=s) for s, h in ((3, 4), (4, hk), (5, hk)))
    ops.append_to_cache(k, v, k_pages, v_pages, table, ints(*lengths))
    with pytest.raises(g.SwarmError) as err:
        ops.check()
    assert err.value.code == g.ERANGE
    ops.check()                                                                 # told once
    want = [x.clone() for x in before]
    for b, column, page, n in ((0, 0, 0, 8), (0, 1, 1, 8), (0, 2, 2, 4), (1, 0, 3, 8), (1, 2, 4, 4), (2, 1, 5, 8)):
        want[0][page, :n], want[1][page, :n] = k[b, 8 * column:8 * column + n], v[b, 8 * column:8 * column + n]
    assert torch.equal(k_pages, want[0]) and torch.equal(v_pages, want[1])
    o, lse = ops.paged_attention(q[:, -1:], k_pages, v_pages, table, ints(*lengths), need_lse=True)
    with pytest.raises(g.SwarmError):
        ops.check()
    for b, seen in ((0, range(20)), (1, [*range(8), *range(16, 20)]), (2, range(8, 16)), (3, [])):
        wo, wl, size = attention_of(q[b, -1], k[b, list(seen)], v[b, list(seen)], d ** -0.5)
        within(o[b, 0], wo, U[BF16] * wo.abs() + E * size, b)
        assert torch.equal(torch.isinf(lse[b, :, 0]), torch.isinf(wl))
    far = ints(20, 24, 30, 25)                                                  # longer than the table: positions from 24 have no page
    ops.append_to_cache(k[:, :1], v[:, :1], k_pages, v_pages, torch.arange(3, dtype=torch.int32, device="cuda").expand(4, 3).contiguous(), far)
    with pytest.raises(g.SwarmError):
        ops.check()


def test_append_refusals():
    q, k, v = (randn(2, 3, h, 64, dtype=BF16) for h in (4, 2, 2))
    pages, table, lengths = randn(5, 16, 2, 64, dtype=BF16), torch.zeros(2, 2, dtype=torch.int32, device="cuda"), ints(3, 3)
    freq = torch.ones(32, device="cuda")
    for bad in (dict(k=k.half()), dict(v=v.half()), dict(k=k.float(), v=v.float()), dict(k=k[0]), dict(v=v[:, :2]), dict(k=k[:, :, :1]), dict(k_pages=pages.half()),
                dict(k_pages=pages[:, :, :1]), dict(v_pages=pages[:4]), dict(k_pages=pages[..., :32]), dict(table=table.long()), dict(table=table[:1]),
                dict(table=table.t()), dict(table=table[0]), dict(lengths=ints(3)), dict(lengths=lengths.long()), dict(lengths=None), dict(counts=ints(1)),
                dict(q=q[:, :2]), dict(q=q.half()), dict(q=q[..., :32]), dict(out=q.half()), dict(out=q[:, :, :2]), dict(q=None, out=q),
                dict(frequencies=freq.double()), dict(frequencies=freq[None]), dict(frequencies=freq[::2]), dict(frequencies=freq.cpu()),
                dict(k=k.cpu()), dict(table=table.cpu()), dict(out=q.transpose(1, 2).contiguous().transpose(1, 2).as_strided(q.shape, (768, 64, 192, 1))[:0])):
        args = dict(k=k, v=v, k_pages=pages, v_pages=pages.clone(), table=table, lengths=lengths, counts=None, q=q, frequencies=freq)
        args.update(bad)
        with pytest.raises(ValueError):
            ops.append_to_cache(**args)
    for bad in (dict(frequencies=torch.ones(33, device="cuda")), dict(q=randn(2, 3, 3, 64, dtype=BF16)), dict(k=randn(2, 3, 2, 68, dtype=BF16)[..., 4:]),
                dict(k_pages=pages[:1].expand(5, 16, 2, 64))):
        args = dict(k=k, v=v, k_pages=pages, v_pages=pages.clone(), table=table, lengths=lengths, q=q, frequencies=freq)
        args.update(bad)
        with pytest.raises(g.SwarmError):
            ops.append_to_cache(**args)
    ops.check()


# ---- attention -----------------------------------------------------------------------------------------------------


def attention_of(q, k, v, scale):
    """(o, lse, sum of weighted magnitudes) of one token's heads [heads, dim] over k, v [n, kv_heads, dim]."""
    heads, group = q.shape[0], q.shape[0] // max(k.shape[1], 1)
    if not len(k):
        zero = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
        return zero, torch.full((heads,), -math.inf, dtype=torch.float64, device="cuda"), zero
    k, v = (x.double().repeat_interleave(group, 1) for x in (k, v))
    s = torch.einsum("hd,nhd->hn", q.double(), k) * scale
    p = torch.softmax(s, -1)
    return torch.einsum("hn,nhd->hd", p, v), torch.logsumexp(s, -1), torch.einsum("hn,nhd->hd", p, v.abs())


def check_attention(got, lse, q, caches, lengths, counts, window=0, sinks=0, scale=None, what=""):
    b_, t_, h_, d = q.shape
    scale = d ** -0.5 if scale is None else scale
    for b in range(b_):
        length = max(lengths[b], 0)
        n = min(max(counts[b], 0), t_, length)
        assert not got[b, n:].any(), what
        assert lse is None or torch.isneginf(lse[b, :, n:]).all(), what
        k, v = (held(c, caches[2], b, length) for c in caches[:2])
        for t in range(n):
            p = length - n + t
            seen = torch.arange(p + 1, device="cuda")
            if window:
                seen = seen[(seen > p - window) | (seen < sinks)]
            o, l, size = attention_of(q[b, t], k[seen], v[seen], scale)
            within(got[b, t], o, U[q.dtype] * o.abs() + E * size + TINY[q.dtype], (what, b, t))
            if lse is not None:
                within(lse[b, :, t], l, E * (1 + l.abs()), (what, b, t))


@pytest.mark.parametrize("dtype,heads,kv_heads,dim,page,layout", [
    (BF16, 1, 1, 8, 1, "tokens"), (F16, 4, 4, 64, 16, "tokens"), (BF16, 8, 2, 128, 64, "heads"), (F16, 6, 2, 80, 24, "heads"), (BF16, 16, 1, 128, 7, "tokens"),
    (F16, 20, 1, 40, 100, "tokens"), (BF16, 34, 2, 72, 5, "heads"), (F16, 3, 3, 104, 17, "tokens")])
@pytest.mark.parametrize("tokens", [1, 2, 7])
def test_paged_attention(dtype, heads, kv_heads, dim, page, layout, tokens):
    lengths = [1, 2, 15, 16, 17, 0, 33, 64, 127, 300, 1000, tokens]
    counts = [tokens, 1, tokens, 0, tokens, 3, tokens, -1, tokens, tokens, 1, tokens + 5]
    caches = make_cache(lengths, page, kv_heads, dim, dtype, layout, seed=dim + tokens)
    q = randn(len(lengths), tokens, heads, dim, dtype=dtype, seed=3, std=1.5)
    o, lse = ops.paged_attention(q, *caches, ints(*lengths), counts=ints(*counts), need_lse=True)
    check_attention(o, lse, q, caches, lengths, counts)
    ops.check()


@pytest.mark.parametrize("batch,length,heads,kv_heads,dim", [(1, 20011, 2, 1, 128), (2, 5000, 16, 16, 64), (300, 40, 4, 2, 64), (1, 1, 1, 1, 64), (70, 700, 8, 1, 128)])
def test_paged_attention_splits(batch, length, heads, kv_heads, dim):
    """Long sentences among short ones, so that the parts of one sentence are taken by several warps, and of several by one."""
    lengths = [length if b % 7 == 0 else max(1, length * (b % 5) // 5) for b in range(batch)]
    caches = make_cache(lengths, 32, kv_heads, dim, BF16, seed=batch)
    q = randn(batch, 1, heads, dim, dtype=BF16, seed=3, std=2.0)
    o, lse = ops.paged_attention(q, *caches, ints(*lengths), need_lse=True)
    check_attention(o, lse, q, caches, lengths, [1] * batch)
    again, lse2 = ops.paged_attention(q, *caches, ints(*lengths), need_lse=True)
    assert torch.equal(o, again) and torch.equal(lse, lse2)                     # one order of every sum


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 5), (15, 0), (16, 4), (17, 1), (40, 16), (33, 17), (100, 64), (299, 1), (300, 1), (1000, 4), (5, 1000), (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("tokens", [1, 5])
def test_windows_and_first_tokens(window, sinks, tokens):
    lengths = [300, 1, 16, 17, 64, 4, 0, 101, 299]
    caches = make_cache(lengths, 16, 2, 64, F16, seed=window % 1000)
    q = randn(len(lengths), tokens, 4, 64, dtype=F16, seed=3, std=1.5)
    o, lse = ops.paged_attention(q, *caches, ints(*lengths), window=window, sinks=sinks, need_lse=True)
    check_attention(o, lse, q, caches, lengths, [tokens] * len(lengths), window, sinks)


@pytest.mark.parametrize("tokens", [1, 4, 64])
@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 3)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_what_a_row_does_not_see_is_not_used(tokens, window, sinks, dtype):
    """Everything that no row sees is NaN; of a sentence's newest tokens, that the earlier rows do not see, the last is."""
    lengths = [64, 70, 200, 129, 65]
    caches = make_cache(lengths, 24, 2, 64, dtype, seed=9)
    q = randn(5, tokens, 6, 64, dtype=dtype, seed=4)
    want = ops.paged_attention(q, *caches, ints(*lengths), window=window, sinks=sinks)
    bad = [torch.full_like(c, float("nan")) for c in caches[:2]]
    for b, n in enumerate(lengths):
        at = torch.arange(n, device="cuda")
        if window:
            at = at[(at > n - tokens - window) | (at < sinks)]
        page, slot = caches[2][b][at // 24].long(), at % 24
        for x, y in zip(bad, caches):
            x[page, slot] = y[page, slot]
    table = caches[2].clone()
    if window:                                                                  # pages that the window has left behind are given up
        for b, n in enumerate(lengths):
            for column in range(table.shape[1]):
                if column * 24 >= sinks and (column + 1) * 24 <= n - tokens - window + 1:
                    table[b, column] = -1
    assert torch.equal(ops.paged_attention(q, *bad, table, ints(*lengths), window=window, sinks=sinks), want)
    ops.check()
    if tokens > 1:
        for value in (float("nan"), float("inf"), -float("inf")):
            for b, n in enumerate(lengths):
                bad[1][caches[2][b, (n - 1) // 24].long(), (n - 1) % 24] = value
            got = ops.paged_attention(q, *bad, table, ints(*lengths), window=window, sinks=sinks)
            assert torch.equal(got[:, :-1], want[:, :-1])
            assert not torch.isfinite(got[:, -1]).any()
        for b, n in enumerate(lengths):
            bad[1][caches[2][b, (n - 1) // 24].long(), (n - 1) % 24] = 0
            bad[0][caches[2][b, (n - 1) // 24].long(), (n - 1) % 24] = float("nan")
        got = ops.paged_attention(q, *bad, table, ints(*lengths), window=window, sinks=sinks)
        assert torch.equal(got[:, :-1], want[:, :-1]) and torch.isnan(got[:, -1]).all()


def test_scores_without_a_finite_maximum_and_large_ones():
    lengths, d = [40, 40], 64
    caches = make_cache(lengths, 16, 1, d, F16, seed=2)
    q = randn(2, 1, 2, d, dtype=F16, seed=4, std=40.0)                          # scores in the thousands
    o, lse = ops.paged_attention(q, *caches, ints(*lengths), scale=2.0, need_lse=True)
    for b in range(2):
        k, v = (held(c, caches[2], b, 40) for c in caches[:2])
        s = torch.einsum("hd,nd->hn", q[b, 0].double(), k[:, 0].double()) * 2
        w, l, size = attention_of(q[b, 0], k, v, 2.0)
        # a score of fp32 terms is off by 64 of their roundings, and the weights by a factor of the exponential of that
        off = 64 * 2.0 ** -24 * (q[b, 0].double().abs() @ k[:, 0].double().abs().T).max().item() * 2
        within(o[b, 0], w, U[F16] * w.abs() + (E + 2 * math.expm1(2 * off)) * v.double().abs().max(), b)
        within(lse[b, :, 0], l, 2 * off + 2.0 ** -22 * l.abs(), b)
    low = caches[0].clone()
    low[:] = -65504.0
    q = torch.full((2, 1, 2, d), 65504.0, dtype=F16, device="cuda")             # every score is the lowest there is
    o = ops.paged_attention(q, low, caches[1], caches[2], ints(*lengths))
    for b in range(2):
        mean = held(caches[1], caches[2], b, 40).double().mean(0)
        within(o[b, 0], mean.expand(2, d), U[F16] * mean.abs() + E * 4, b)


def test_sentences_share_pages():
    lengths = [50, 60, 37]
    caches = make_cache(lengths, 16, 2, 64, BF16, seed=3)
    caches[2][:, :2] = caches[2][0, :2]                                         # one beginning of 32 tokens
    q = randn(3, 2, 4, 64, dtype=BF16, seed=4)
    check_attention(ops.paged_attention(q, *caches, ints(*lengths)), None, q, caches, lengths, [2] * 3)


def test_attention_takes_strides_and_another_place_for_its_output():
    lengths, d = [33, 80], 64
    both = randn(12, 2, 2, 16, d, dtype=BF16, seed=1)                           # [pages, k or v, heads, slots, values]
    table = torch.randperm(12, device="cuda").to(torch.int32).view(2, 6)
    k_pages, v_pages = both[:, 0].transpose(1, 2), both[:, 1].transpose(1, 2)
    wide = randn(2, 3, 9, d, dtype=BF16, seed=2)
    q, out = wide[:, :, 1:5], torch.zeros(2, 4, 3, 72, dtype=BF16, device="cuda")
    into = out.transpose(1, 2)[..., :d]
    want = ops.paged_attention(q.contiguous(), k_pages.contiguous(), v_pages.contiguous(), table, ints(*lengths))
    assert ops.paged_attention(q, k_pages, v_pages, table, ints(*lengths), out=into) is into
    assert torch.equal(into, want) and not out[..., d:].any()
    same = q[:, :, :1].expand(2, 3, 4, d)                                       # query heads repeated by a stride of 0
    assert torch.equal(ops.paged_attention(same, k_pages, v_pages, table, ints(*lengths)),
                       ops.paged_attention(same.contiguous(), k_pages, v_pages, table, ints(*lengths)))


def test_paged_attention_agrees_with_cross_attention_over_the_same_states():
    n, d = 77, 128
    k, v = (randn(3, n, 2, d, dtype=F16, seed=s) for s in (1, 2))
    q = randn(3, 1, 8, d, dtype=F16, seed=3)
    caches = make_cache([n] * 3, 16, 2, d, F16, fill=0.0)
    ops.append_to_cache(k, v, *caches, ints(n, n, n))
    a, b = ops.paged_attention(q, *caches, ints(n, n, n)).double(), ops.cross_attention(q, k, v).double()
    size = max(attention_of(q[i, 0], k[i], v[i], d ** -0.5)[2].max().item() for i in range(3))
    within(a, b, 2 * U[F16] * b.abs() + (U[F16] + 2 * E) * size)                # there the weights are rounded to fp16


def test_cache_beyond_32_bits():
    """More than 2^32 values in each tensor: offsets of pages need 64 bits."""
    pages, size, hk, d = 33000, 128, 8, 128
    if torch.cuda.mem_get_info()[0] < 24 * 2 ** 30:
        pytest.skip("needs 24 GiB")
    caches = [torch.empty(pages, size, hk, d, dtype=BF16, device="cuda") for _ in range(2)]
    table = torch.tensor([[32999, 0, 32768], [16384, 32990, 1]], dtype=torch.int32, device="cuda")
    lengths, n = [300, 290], 300
    q, k, v = (randn(2, n, h, d, dtype=BF16, seed=s) for s, h in ((1, 8), (2, hk), (3, hk)))
    ops.append_to_cache(k, v, *caches, table, ints(*lengths), counts=ints(*lengths))
    o = ops.paged_attention(q[:, :1], *caches, table, ints(*lengths))
    for b in range(2):
        assert torch.equal(held(caches[0], table, b, lengths[b]), k[b, :lengths[b]])
        w, _, size_ = attention_of(q[b, 0], k[b, :lengths[b]], v[b, :lengths[b]], d ** -0.5)
        within(o[b, 0], w, U[BF16] * w.abs() + E * size_)
    ops.check()


def test_a_window_far_into_a_sentence_of_2_31_tokens():
    size, d, last = 1 << 20, 8, 2 ** 31 - 1
    table = torch.full((1, 2048), -1, dtype=torch.int32, device="cuda")
    table[0, 2047], table[0, 0] = 0, 1
    k_pages, v_pages = (randn(2, size, 1, d, dtype=BF16, seed=s) for s in (1, 2))
    q = randn(1, 2, 2, d, dtype=BF16, seed=3)
    o = ops.paged_attention(q, k_pages, v_pages, table, ints(last), window=1000, sinks=5)
    for t in range(2):
        p = last - 2 + t
        at = torch.arange(p - 999, p + 1, device="cuda") % size
        k, v = (torch.cat([x[1, :5], x[0, at]]) for x in (k_pages, v_pages))
        w, _, s = attention_of(q[0, t], k, v, d ** -0.5)
        within(o[0, t], w, U[BF16] * w.abs() + E * s)
    ops.check()


@pytest.mark.parametrize("window,sinks", [(0, 0), (10, 0), (10, 5), (1000, 30)])
@pytest.mark.parametrize("heads,kv_heads,dim", [(2, 2, 64), (16, 2, 128)])
def test_lengths_beyond_the_table_add_nothing(window, sinks, heads, kv_heads, dim):
    """Positions that the table has no room for are not there: what a row sees of the others is, and nothing is waited for."""
    page, columns = 8, 40
    lengths = [columns * page, columns * page + 3, columns * page + 500, 2 ** 31 - 1, 100]
    table = torch.randperm(5 * columns, generator=torch.Generator().manual_seed(1)).to(torch.int32).view(5, columns).cuda()
    k_pages, v_pages = (randn(5 * columns, page, kv_heads, dim, dtype=F16, seed=s) for s in (1, 2))
    q = randn(5, 2, heads, dim, dtype=F16, seed=3)
    o, lse = ops.paged_attention(q, k_pages, v_pages, table, ints(*lengths), window=window, sinks=sinks, need_lse=True)
    with pytest.raises(g.SwarmError):
        ops.check()
    for b, n in enumerate(lengths):
        room = min(n, columns * page)
        k, v = (held(x, table, b, room) for x in (k_pages, v_pages))
        for t in range(2):
            p, seen = n - 2 + t, torch.arange(room, device="cuda")
            seen = seen[seen <= p]
            if window:
                seen = seen[(seen > p - window) | (seen < sinks)]
            w, l, size = attention_of(q[b, t], k[seen], v[seen], dim ** -0.5)
            within(o[b, t], w, U[F16] * w.abs() + E * size + TINY[F16], (b, t))
            assert torch.equal(torch.isneginf(lse[b, :, t]), torch.isneginf(l))
    ops.paged_attention(q, k_pages, v_pages, table, ints(320, 0, 5, 319, 100), window=window, sinks=sinks)
    ops.check()


def test_keys_and_values_of_different_layouts_and_a_wide_table():
    lengths, hk, d = [50, 7, 200], 4, 64
    k_pages, v_pages, table = make_cache(lengths, 16, hk, d, BF16)
    q = randn(3, 1, 8, d, dtype=BF16, seed=5)
    want = ops.paged_attention(q, k_pages, v_pages, table, ints(*lengths))
    by_head = v_pages.transpose(1, 2).contiguous().transpose(1, 2)
    wide = torch.full((3, table.shape[1] + 9), 2 ** 30, dtype=torch.int32, device="cuda")
    wide[:, 5:5 + table.shape[1]] = table
    assert torch.equal(ops.paged_attention(q, k_pages, by_head, wide[:, 5:5 + table.shape[1]], ints(*lengths)), want)
    k_by_head = k_pages.transpose(1, 2).contiguous().transpose(1, 2)
    other = ops.paged_attention(q, k_by_head, by_head, table, ints(*lengths))   # heads one by one instead of in pairs
    size = torch.stack([attention_of(q[b, 0], held(k_pages, table, b, n), held(v_pages, table, b, n), d ** -0.5)[2] for b, n in enumerate(lengths)])
    within(other[:, 0], want[:, 0], 2 * U[BF16] * want[:, 0].double().abs() + 2 * E * size)
    ops.check()


def test_attention_refusals():
    q, pages = randn(2, 3, 4, 64, dtype=BF16), randn(5, 16, 2, 64, dtype=BF16)
    table, lengths = torch.zeros(2, 2, dtype=torch.int32, device="cuda"), ints(3, 3)
    for bad in (dict(q=q.half()), dict(q=q.float()), dict(q=q[0]), dict(q=q[..., :32]), dict(k_pages=pages[..., :32]), dict(v_pages=pages[:4]),
                dict(k_pages=pages[0]), dict(table=table.long()), dict(table=table[:1]), dict(lengths=ints(1)), dict(lengths=None),
                dict(counts=lengths.float()), dict(out=q.half()), dict(out=q[:, :2]), dict(window=2 ** 31), dict(sinks=-2 ** 40),
                dict(scale=1e300), dict(q=q.cpu()), dict(q=q.transpose(2, 3).contiguous().transpose(2, 3))):
        args = dict(q=q, k_pages=pages, v_pages=pages, table=table, lengths=lengths)
        args.update(bad)
        with pytest.raises(ValueError):
            ops.paged_attention(**args)
    for bad in (dict(window=-1), dict(sinks=-1), dict(scale=0.0), dict(scale=float("nan")), dict(q=randn(2, 65, 4, 64, dtype=BF16)),
                dict(q=randn(2, 3, 3, 64, dtype=BF16)), dict(out=torch.empty(2, 3, 4, 68, dtype=BF16, device="cuda")[..., 4:])):
        args = dict(q=q, k_pages=pages, v_pages=pages, table=table, lengths=lengths)
        args.update(bad)
        with pytest.raises(g.SwarmError):
            ops.paged_attention(**args)
    assert ops.paged_attention(q[:0], pages, pages, table[:0], lengths[:0]).shape == (0, 3, 4, 64)
    assert ops.paged_attention(q[:, :0], pages, pages, table, lengths).shape == (2, 0, 4, 64)
    none = ops.paged_attention(q, pages[:0], pages[:0], table[:, :0], ints(0, 0))
    assert not none.any()
    ops.check()


# ---- log probabilities ---------------------------------------------------------------------------------------------


def reference(logits, tokens, scale):
    """(log probs of tokens, stats, entropy, log probs, largest |d| weighted) in 64 bits."""
    raw = logits.double()
    most = raw.max(-1, keepdim=True).values
    base = torch.where(torch.isinf(most), torch.zeros_like(most), most)
    d = (raw - base) * scale
    total = torch.exp(d).sum(-1, keepdim=True)
    logp = d - torch.log(total)
    p = torch.exp(logp)
    finite = torch.where(p > 0, logp, torch.zeros_like(logp))
    given = torch.gather(logp, -1, tokens.clamp(0, logits.shape[-1] - 1).unsqueeze(-1)).squeeze(-1)
    given = torch.where((tokens >= 0) & (tokens < logits.shape[-1]), given, torch.zeros_like(given))
    spread = (p * torch.where(p > 0, d.abs(), torch.zeros_like(d))).sum(-1)
    return given, torch.cat([most, torch.log(total)], -1), -(p * finite).sum(-1), logp, spread


def within_fp32(got, want, off, what):
    """Log probabilities of fp32: a value past its range (1.25 times bf16's or fp32's lowest, 4.2e38 > 2^128) is -infinity there."""
    out = want < -2.0 ** 128
    assert torch.equal(torch.isneginf(got), out), what
    want = torch.where(out, 0.0, want)
    within(torch.where(out, 0.0, got.double()), want, off + 2.0 ** -22 * (want.abs() + 1), what)


def check_log_probs(got, logits, tokens, scale, top):
    n = logits.shape[-1]
    lp, stats, entropy, logp, spread = reference(logits, tokens, scale)
    off = (run(n) + 16) * 2.0 ** -24 + (spread + 4) * 2.0 ** -23               # of the logarithm of the sum
    assert torch.equal(got.stats[..., 0].double(), stats[..., 0])
    within(got.stats[..., 1], stats[..., 1], off + 2.0 ** -23 * stats[..., 1].abs(), "log of the sum")
    within_fp32(got.log_probs, lp, off, "log probs")
    if got.entropy is not None:
        within(got.entropy, entropy, (off + 2.0 ** -22) * (4 + 2 * spread + entropy.abs()), "entropy")
    if top:
        order = torch.sort(logits.double(), dim=-1, descending=True, stable=True).indices[..., :top]
        assert torch.equal(got.top_tokens, order)
        within_fp32(got.top_log_probs, logp.gather(-1, order), off.unsqueeze(-1), "top")


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("rows,cols,top", [(1, 1, 1), (3, 2, 2), (5, 7, 0), (2, 33, 32), (9, 100, 5), (1, 255, 1), (300, 256, 8), (2, 2049, 20), (4, 10007, 32),
                                           (1, 50000, 3), (3, 131072, 32), (40, 32000, 0), (700, 1000, 1), (2, 300001, 16),
                                           (1100, 1025, 0), (1024, 1025, 0), (2600, 2500, 0), (2600, 2500, 6), (4100, 4099, 0)])
def test_log_probs(dtype, rows, cols, top):
    logits = randn(rows, cols, dtype=dtype, seed=cols, std=3.0)
    tokens = torch.randint(cols, (rows,), generator=torch.Generator().manual_seed(1)).cuda()
    scale = 1.0 if cols % 2 else 0.7
    got = ops.token_log_probs(logits, tokens, scale=scale, top=top, entropy=rows != 40)
    check_log_probs(got, logits, tokens, scale, top)
    assert (got.top_tokens is None) == (top == 0)
    alone = ops.token_log_probs(logits, scale=scale, top=top)                   # without tokens and entropy
    assert alone.log_probs is None and alone.entropy is None and torch.equal(alone.stats, got.stats)
    if top:
        assert torch.equal(alone.top_tokens, got.top_tokens) and torch.equal(alone.top_log_probs, got.top_log_probs)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("cols", [5, 300, 20000])
def test_equal_logits_and_other_orders(dtype, cols):
    rows = torch.zeros(8, cols, dtype=dtype, device="cuda")
    up = torch.linspace(-9, 9, cols, device="cuda")
    rows[1], rows[2] = up.to(dtype), up.flip(0).to(dtype)                       # ascending and descending, with many equal ones
    rows[3, ::2] = -0.0                                                         # zeros of either sign are equal
    rows[4] = -math.inf
    rows[4, cols // 2] = 1.0                                                    # one token is left
    rows[5] = torch.finfo(dtype).min                                            # all at the type's lowest value
    rows[6, 1::3] = torch.finfo(dtype).min
    rows[7, cols - 1] = 5.0
    tokens = torch.full((8,), cols // 2, device="cuda")
    got = ops.token_log_probs(rows, tokens, top=min(5, cols), entropy=True, scale=1.25)
    check_log_probs(got, rows, tokens, 1.25, min(5, cols))


@pytest.mark.parametrize("cols,top", [(4, 4), (5000, 32), (70000, 7)])
def test_rows_without_a_token_and_padded_places(cols, top):
    logits = randn(6, cols, seed=3)
    logits[1] = -math.inf
    logits[4, :-1] = -math.inf
    tokens = torch.tensor([-1, 0, cols, 2 ** 40, cols - 1, -2 ** 62], device="cuda")
    got = ops.token_log_probs(logits, tokens, top=top, entropy=True)
    assert got.log_probs[[0, 2, 3, 5]].tolist() == [0.0] * 4
    assert got.log_probs[1] == -math.inf and got.entropy[1] == 0 and got.stats[1, 0] == -math.inf
    assert got.top_tokens[1].tolist() == list(range(top)) and torch.isneginf(got.top_log_probs[1]).all()
    assert abs(got.log_probs[4].item()) < 1e-6 and abs(got.entropy[4].item()) < 1e-6
    assert got.top_tokens[4].tolist() == [cols - 1, *range(top - 1)]
    dx = ops.token_log_probs_backward(torch.ones(6, device="cuda"), logits, tokens, got.stats, got.entropy, torch.zeros(6, device="cuda"))
    assert not dx[[0, 1, 2, 3, 5]].any() and not torch.isnan(dx).any() and dx[4].abs().max() < 1e-6
    dx = ops.token_log_probs_backward(None, logits, None, got.stats, got.entropy, torch.ones(6, device="cuda"))
    assert not torch.isnan(dx).any() and not dx[1].any()


def test_nan_and_infinity_stay_in_their_row():
    logits = randn(4, 3000, seed=4)
    logits[1, 17], logits[2, 100] = float("nan"), math.inf
    logits[1, 200] = -float("nan")
    tokens = torch.tensor([1, 2, 3, 4], device="cuda")
    got = ops.token_log_probs(logits, tokens, top=4, entropy=True)
    assert torch.isnan(got.log_probs).tolist() == [False, True, True, False]
    assert torch.isnan(got.entropy).tolist() == [False, True, True, False]
    assert got.top_tokens[1, :2].tolist() == [17, 200] and got.top_tokens[2, 0] == 100
    dx = ops.token_log_probs_backward(torch.ones(4, device="cuda"), logits, tokens, got.stats)
    assert torch.isnan(dx).all(1).tolist() == [False, True, True, False] and not torch.isnan(dx[[0, 3]]).any()


def check_gradient(dx, logits, tokens, scale, g_, h):
    n = logits.shape[-1]
    _, _, entropy, logp, spread = reference(logits, tokens, scale)
    p = torch.exp(logp)
    finite = torch.where(p > 0, logp, torch.zeros_like(logp))
    some = ((tokens >= 0) & (tokens < n)).double()
    here = torch.zeros_like(p).scatter_(-1, tokens.clamp(0, n - 1).unsqueeze(-1), some.unsqueeze(-1))
    first = torch.zeros_like(p) if g_ is None else (g_.double() * some).unsqueeze(-1) * (here - p)
    second = torch.zeros_like(p) if h is None else -h.double().unsqueeze(-1) * p * (finite + entropy.unsqueeze(-1))
    want = scale * (first + second)
    off = ((run(n) + 16) * 2.0 ** -24 + (spread + 4) * 2.0 ** -23).unsqueeze(-1) + 2.0 ** -22 * (finite.abs() + 1)
    size = p * (0 if g_ is None else g_.double().abs().unsqueeze(-1))
    size = size + p * (0 if h is None else h.double().abs().unsqueeze(-1) * (finite.abs() + entropy.abs().unsqueeze(-1) + 8 + 2 * spread.unsqueeze(-1)))
    bound = U[dx.dtype] * want.abs() + scale * size * 2 * off + 2.0 ** -22 * (first.abs() + second.abs()) * scale + TINY[dx.dtype]
    within(dx, want, bound, "gradient")


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (2, 256), (5, 1001), (30, 4099), (2, 70001), (1100, 1025), (2600, 2501)])
@pytest.mark.parametrize("parts", ["token", "entropy", "both"])
def test_gradient(dtype, rows, cols, parts):
    logits = randn(rows, cols, dtype=dtype, seed=cols, std=2.0)
    if cols > 10:
        logits[:, ::5] = -math.inf
    tokens = torch.randint(cols, (rows,), generator=torch.Generator().manual_seed(1)).cuda()
    tokens[rows // 2] = -100
    got = ops.token_log_probs(logits, tokens, scale=0.8, entropy=True)
    g_ = randn(rows, seed=5) if parts != "entropy" else None
    h = randn(rows, seed=6) if parts != "token" else None
    dx = ops.token_log_probs_backward(g_, logits, tokens if g_ is not None else None, got.stats, got.entropy if h is not None else None, h, scale=0.8)
    check_gradient(dx, logits, tokens, 0.8, g_, h)


def test_gradient_is_the_difference():
    """Along a direction u: differences of the calls' own outputs against their gradient."""
    rows, cols, scale = 6, 777, 0.9
    logits, u = randn(rows, cols, seed=1, std=1.5), randn(rows, cols, seed=2)
    tokens = torch.randint(cols, (rows,), generator=torch.Generator().manual_seed(3)).cuda()
    g_, h, step = randn(rows, seed=4), randn(rows, seed=5), 2.0 ** -6
    got = ops.token_log_probs(logits, tokens, scale=scale, entropy=True)
    dx = ops.token_log_probs_backward(g_, logits, tokens, got.stats, got.entropy, h, scale=scale)
    up, down = (ops.token_log_probs(logits + s * step * u, tokens, scale=scale, entropy=True) for s in (1, -1))
    lhs = ((up.log_probs - down.log_probs).double() * g_ + (up.entropy - down.entropy).double() * h).sum() / (2 * step)
    # the third derivative along u is at most a few times |u|^3 log n where p is spread out; outputs are off by 2e-6 each
    assert abs(lhs - (dx.double() * u.double()).sum()).item() < 100 * step ** 2 * (g_.abs() + h.abs()).sum().item() + 4e-6 / step * rows


def test_log_probs_take_strides_and_gradients_overwrite_logits():
    wide = randn(12, 1111, dtype=BF16, seed=3)
    part = wide[:, 3:1004]                                                      # neither the base nor the pitch on 16 bytes
    tokens = torch.arange(12, device="cuda") * 80
    a, b = ops.token_log_probs(part, tokens, top=6, entropy=True), ops.token_log_probs(part.contiguous(), tokens, top=6, entropy=True)
    n = part.shape[1]
    off = (run(n) + 16) * 2.0 ** -23 + 40 * 2.0 ** -22                         # another alignment may take another order
    within(a.log_probs, b.log_probs, off)
    assert torch.equal(a.top_tokens, b.top_tokens)
    c = ops.token_log_probs(part.contiguous().view(3, 4, n), tokens.view(3, 4), top=6, entropy=True)
    assert torch.equal(c.log_probs.view(12), b.log_probs) and torch.equal(c.top_tokens.view(12, 6), b.top_tokens) and c.stats.shape == (3, 4, 2)
    g_ = randn(12, seed=5)
    want = ops.token_log_probs_backward(g_, part, tokens, a.stats, a.entropy, g_)
    check_gradient(want, part, tokens, 1.0, g_, g_)
    into = torch.zeros(12, 1017, dtype=BF16, device="cuda")
    ops.token_log_probs_backward(g_, part, tokens, a.stats, a.entropy, g_, dlogits=into[:, 9:1010])
    assert torch.equal(into[:, 9:1010], want) and not into[:, :9].any() and not into[:, 1010:].any()
    before = wide.clone()
    assert ops.token_log_probs_backward(g_, part, tokens, a.stats, a.entropy, g_, dlogits=part) is part
    assert torch.equal(part, want) and torch.equal(wide[:, :3], before[:, :3]) and torch.equal(wide[:, 1004:], before[:, 1004:])


def test_log_probs_beyond_32_bits():
    rows, cols = 33000, 131072                                                  # more than 2^32 logits
    if torch.cuda.mem_get_info()[0] < 24 * 2 ** 30:
        pytest.skip("needs 24 GiB")
    logits = torch.zeros(rows, cols, dtype=BF16, device="cuda")
    logits[-2:] = randn(2, cols, dtype=BF16, seed=1)
    tokens = torch.zeros(rows, dtype=torch.int64, device="cuda")
    tokens[-1] = cols - 1
    got = ops.token_log_probs(logits, tokens, entropy=True)
    want, _, entropy, _, _ = reference(logits[-2:], tokens[-2:], 1.0)
    within(got.log_probs[-2:], want, 1e-3 * torch.ones_like(want))
    within(got.log_probs[:-2], torch.full((rows - 2,), -math.log(cols), device="cuda"), (cols / 256 + 64) * 2.0 ** -23)
    g_ = torch.ones(rows, device="cuda")
    ops.token_log_probs_backward(g_, logits, tokens, got.stats, dlogits=logits)
    assert abs(logits[-1, -1].item() - (1 - math.exp(want[-1]))) < 2.0 ** -8 and abs(logits[-3, 0].item() - 1) < 2.0 ** -8
    assert abs(logits[-3, 1].item() * cols + 1) < 2.0 ** -7


def test_log_probs_refusals():
    x, t = randn(3, 40), torch.zeros(3, dtype=torch.int64, device="cuda")
    for bad in (dict(logits=x.double()), dict(logits=x.t()), dict(logits=x[:, ::2]), dict(logits=torch.tensor(1.0, device="cuda")), dict(tokens=t.int()), dict(tokens=t[:2]),
                dict(tokens=t.cpu()), dict(top=-1), dict(top=33), dict(top=41), dict(top=2.0), dict(logits=x.cpu())):
        with pytest.raises(ValueError):
            ops.token_log_probs(**{**dict(logits=x, tokens=t), **bad})
    for bad in (dict(scale=0.0), dict(scale=-1.0), dict(scale=1e300), dict(scale=float("nan")), dict(logits=x[:, :0])):
        with pytest.raises(g.SwarmError):
            ops.token_log_probs(**{**dict(logits=x, tokens=t), **bad})
    assert ops.token_log_probs(x[:0], t[:0], top=3).top_tokens.shape == (0, 3)
    s, r = torch.zeros(3, 2, device="cuda"), torch.zeros(3, device="cuda")
    for bad in (dict(dlog_probs=r[:2]), dict(dlog_probs=r.double()), dict(tokens=None), dict(stats=None), dict(stats=s[:2]), dict(stats=s.double()),
                dict(dentropy=r), dict(dentropy=r[:2], entropy=r), dict(dlogits=x.half()), dict(dlogits=x[:2]), dict(dlogits=x.t().contiguous().t())):
        with pytest.raises(ValueError):
            ops.token_log_probs_backward(**{**dict(dlog_probs=r, logits=x, tokens=t, stats=s), **bad})
    wide = randn(6, 40)
    with pytest.raises(ValueError):
        ops.token_log_probs_backward(r, wide[:3], t, s, dlogits=wide[::2])
    ops.check()


# ---- streams, graphs, a run of them together -----------------------------------------------------------------------


def step_of(state):
    """One step of a decoder over its cache: append, attend, score."""
    q = ops.append_to_cache(state["k"], state["v"], *state["caches"], state["lengths"], q=state["q"], frequencies=state["freq"])
    o = ops.paged_attention(q, *state["caches"], state["lengths"], window=state["window"], sinks=4)
    got = ops.token_log_probs(o.flatten(1) @ state["w"], state["tokens"], top=4, entropy=True)
    return q, o, *got


def make_state(batch=5, heads=4, kv_heads=2, dim=64, window=0, seed=0):
    lengths = [100 + 37 * b for b in range(batch)]
    return {"k": randn(batch, 1, kv_heads, dim, dtype=BF16, seed=seed + 1), "v": randn(batch, 1, kv_heads, dim, dtype=BF16, seed=seed + 2),
            "q": randn(batch, 1, heads, dim, dtype=BF16, seed=seed + 3), "caches": make_cache([n + 64 for n in lengths], 16, kv_heads, dim, BF16, seed=seed),
            "lengths": ints(*lengths), "freq": 10000.0 ** (-torch.arange(dim // 2, device="cuda") / (dim // 2)), "window": window,
            "w": randn(heads * dim, 5000, dtype=BF16, seed=seed + 4, std=0.1), "tokens": torch.arange(batch, device="cuda")}


def test_calls_run_on_the_current_stream():
    state = make_state()
    want = [x.clone() for x in step_of(state)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        late = {**state, "q": state["q"].clone()}
        late["q"].copy_(randn(*late["q"].shape, dtype=BF16, seed=99))
        late["q"].copy_(state["q"])
        got = step_of(late)
    side.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("window", [0, 60])
def test_captured_steps_follow_lengths_and_two_graphs_do_not_meet(window):
    states = [make_state(window=window, seed=s) for s in (10, 20)]
    graphs, outs = [], []
    for s in states:
        step_of(s)                                                              # loads the kernels
    torch.cuda.synchronize()
    for s in states:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(step_of(s))
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in states]
    for i in range(3):
        for s in states:
            s["lengths"] += 5
            s["q"].copy_(randn(*s["q"].shape, dtype=BF16, seed=30 + i))
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, streams):                              # side by side
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for s, out in zip(states, outs):
            for a, b in zip(step_of(s), out):
                assert torch.equal(a, b)
    ops.check()


def test_a_run_of_steps_is_the_attention_over_all_that_was_appended():
    """Prompts of unequal lengths appended at once, then tokens one by one: against attention over the whole of it in 64 bits."""
    b, h, hk, d, steps, page = 4, 6, 2, 64, 20, 8
    prompt = [0, 5, 17, 30]
    keys, values, queries = ([randn(prompt[i] + steps, x, d, dtype=F16, seed=10 * i + s) for i in range(b)] for s, x in ((1, hk), (2, hk), (3, h)))
    freq = 1000.0 ** (-torch.arange(d // 2, device="cuda") / (d // 2))
    caches = make_cache([n + steps for n in prompt], page, hk, d, F16, fill=float("nan"))
    k, v = (torch.zeros(b, 30, hk, d, dtype=F16, device="cuda") for _ in range(2))
    for i, n in enumerate(prompt):
        k[i, :n], v[i, :n] = keys[i][:n], values[i][:n]
    lengths = ints(*prompt)
    ops.append_to_cache(k, v, *caches, lengths, counts=lengths, frequencies=freq)
    for step in range(steps):
        k, v, q = (torch.stack([x[i][prompt[i] + step] for i in range(b)]).unsqueeze(1) for x in (keys, values, queries))
        lengths += 1
        q = ops.append_to_cache(k, v, *caches, lengths, q=q, frequencies=freq)
        o = ops.paged_attention(q, *caches, lengths)
        for i in range(b):
            n = prompt[i] + step + 1
            at = torch.arange(n, device="cuda")
            wq, wk = rotated(queries[i][n - 1:n], at[-1:], freq, False)[0][0], rotated(keys[i][:n], at, freq, False)[0]
            w, _, size = attention_of(wq, wk, values[i][:n], d ** -0.5)
            # q and k were rounded to fp16 on the way: scores are off by two roundings of their magnitudes' sum
            off = 2 * U[F16] * (wq.abs().view(hk, h // hk, d) @ wk.abs().permute(1, 2, 0)).max().item() * d ** -0.5
            within(o[i, 0], w, U[F16] * w.abs() + (E + 2 * off) * size + 2 * off * w.abs(), (step, i))
    ops.check()
