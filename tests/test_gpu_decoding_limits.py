"""The decoding operators where their sums are long, their values infinite, their rows few; against their formulas in 64 bits.

U is the largest relative rounding error of a type, E what fp32 arithmetic adds to attention over a cache: 2e-5 (128-term dot products,
base-2 exponentials) and 2^-16 for weights that go into their products as two numbers of the type.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_1910_12308_b200 import operators as ops  # noqa: E402

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
U = {BF16: 2.0 ** -8, F16: 2.0 ** -11, F32: 2.0 ** -24}
E = 2e-5 + 2.0 ** -16


def randn(*shape, dtype=F32, seed=0, std=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=gen, device="cuda") * std).to(dtype)


def within(got, want, bound, what=""):
    got, want = got.double(), want.double()
    assert got.shape == want.shape, what
    assert not torch.isnan(got).any(), what
    over = (got - want).abs() - bound
    assert over.max().item() <= 0, (what, over.max().item(), (got - want).abs().max().item())


@pytest.mark.parametrize("dtype,dim", [(F16, 8), (F16, 128), (BF16, 64)])
def test_sums_of_a_million_positions(dtype, dim):
    """More sentences than the device has warps, so that each sentence of 2^20 positions is one running sum; they share their pages.

    Such a sum rounds n times, each time by at most 2^-24 of what it has grown to, up or down: 6 sqrt(n) 2^-24 is six times
    the spread of what that adds up to; n = 2^17 for the weights (eight lanes share them), fewer for the values."""
    n, batch, page = 1 << 20, 1200, 4096
    k, v = randn(n // page, page, 1, dim, dtype=dtype, seed=1), (0.5 + randn(n // page, page, 1, dim, seed=2).abs()).to(dtype)
    table = torch.arange(n // page, dtype=torch.int32, device="cuda").expand(batch, -1).contiguous()
    q = randn(batch, 1, 1, dim, dtype=dtype, seed=3, std=0.1)
    o, lse = ops.paged_attention(q, k, v, table, torch.full((batch,), n, dtype=torch.int32, device="cuda"), need_lse=True)
    slack = E + 2 * 6 * math.sqrt(1 << 17) * 2.0 ** -24
    for b in (0, 1, 600, 1198, 1199):
        s = k.view(n, dim).double() @ q[b, 0, 0].double() * dim ** -0.5
        want = torch.softmax(s, 0) @ v.view(n, dim).double()
        within(o[b, 0, 0], want, (U[dtype] + slack) * want, (b, "o"))
        within(lse[b, 0, 0], torch.logsumexp(s, 0), slack * 20, (b, "lse"))
    ops.check()


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("dim,page,kv_heads", [(64, 16, 2), (64, 24, 1), (128, 64, 1), (40, 10, 2)])
@pytest.mark.parametrize("tokens,window,std", [(1, 0, 0.3), (4, 0, 0.3), (5, 70, 0.3), (1, 0, 60.0), (3, 300, 60.0)])
def test_infinite_values_that_a_row_sees_make_it_infinite(dtype, dim, page, kv_heads, tokens, window, std):
    """What the formula says: +infinity, -infinity, NaN where both meet or a NaN is seen; all else as if they were 0."""
    lengths = [tokens, 33, 200, 5000]                                           # one weight of 1 alone (tokens 1), and cut sentences
    columns = -(-max(lengths) // page)
    table = torch.randperm(4 * columns, generator=torch.Generator().manual_seed(1)).to(torch.int32).view(4, columns).cuda()
    k, v = (randn(4 * columns, page, kv_heads, dim, dtype=dtype, seed=s) for s in (1, 2))
    q = randn(4, tokens, 3 * kv_heads, dim, dtype=dtype, seed=3, std=std)       # 60: weights that are 0 in fp32 beside the largest
    clean = v.clone()
    inf, nan = math.inf, math.nan
    # (position from the end, value's place, what stands there): the newest token is seen by the last row alone
    spoiled = [(0, 0, inf), (0, 1, -inf), (0, 2, nan), (tokens, 3, inf), (tokens, 4, -inf), (tokens, 5, nan), (tokens, 6, inf), (0, 6, -inf),
               (17, 8, inf), (60, 9, -inf), (150, 10, inf), (4000, 11, -inf), (4500, 7, inf), (16, 7, inf)]
    for b, n in enumerate(lengths):
        for back, d, x in spoiled:
            p = n - 1 - back
            if p >= 0:
                page_of, slot = table[b, p // page].long(), p % page
                v[page_of, slot, :, d], clean[page_of, slot, :, d] = x, 0.0
    length = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    got, lse = ops.paged_attention(q, k, v, table, length, window=window, need_lse=True)
    base, lse2 = ops.paged_attention(q, k, clean, table, length, window=window, need_lse=True)
    assert torch.isfinite(base).all() and torch.equal(lse, lse2)
    for b, n in enumerate(lengths):
        for t in range(tokens):
            own = n - tokens + t
            seen = [[] for _ in range(dim)]
            for back, d, x in spoiled:
                p = n - 1 - back
                if 0 <= p <= own and (not window or p > own - window):
                    seen[d].append(x)
            want = base[b, t].clone()
            for d, xs in enumerate(seen):
                if xs:
                    want[:, d] = sum(xs)
            assert torch.equal(torch.isnan(got[b, t]), torch.isnan(want)), (b, t)
            assert torch.equal(torch.nan_to_num(got[b, t], nan=1.0, posinf=2e4, neginf=-2e4), torch.nan_to_num(want, nan=1.0, posinf=2e4, neginf=-2e4)), (b, t)
    ops.check()


def run(rows, cols, top):
    """Terms that one thread adds up of a row: a warp walks short rows, and longer ones where there are as many and nothing is searched for."""
    warp = cols <= 1024 or (cols <= 16384 and rows >= cols and not top)
    return cols / (32 if warp else 256)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("rows,cols,top", [(3, 700, 4), (2, 1025, 0), (4, 10007, 0), (4, 10007, 32), (1, 16384, 0), (1024, 1025, 0), (1100, 1025, 3), (2600, 2500, 0),
                                           (5, 131072, 0), (40, 32000, 20)])
def test_log_probs_are_as_near_as_their_threads_runs(dtype, rows, cols, top):
    """A sum of n positive terms is off by n 2^-24 of it, an exponential of d by (|d| + 4) 2^-23, the joining of threads by 16 2^-24."""
    scale = 0.9
    logits = randn(rows, cols, dtype=dtype, seed=cols, std=3.0)
    tokens = torch.randint(cols, (rows,), generator=torch.Generator().manual_seed(1)).cuda()
    got = ops.token_log_probs(logits, tokens, scale=scale, top=top, entropy=True)
    x = logits.double() * scale
    logp = torch.log_softmax(x, -1)
    p, most = logp.exp(), x.max(-1).values
    spread = (p * (x - most.unsqueeze(-1)).abs()).sum(-1)
    off = (run(rows, cols, top) + 16) * 2.0 ** -24 + (spread + 4) * 2.0 ** -23
    log_sum = torch.logsumexp(x, -1) - most
    assert torch.equal(got.stats[:, 0].double(), logits.double().max(-1).values)
    within(got.stats[:, 1], log_sum, off + 2.0 ** -23 * log_sum.abs(), "log of the sum")
    want = logp.gather(1, tokens[:, None])[:, 0]
    within(got.log_probs, want, off + 2.0 ** -22 * (want.abs() + 1), "log probs")
    entropy = -(p * logp).sum(-1)
    within(got.entropy, entropy, (off + 2.0 ** -22) * (4 + 2 * spread + entropy.abs()), "entropy")
    if top:
        order = torch.sort(logits.double(), dim=-1, descending=True, stable=True).indices[:, :top]
        assert torch.equal(got.top_tokens, order)
        want = logp.gather(1, order)
        within(got.top_log_probs, want, off[:, None] + 2.0 ** -22 * (want.abs() + 1), "top")


@pytest.mark.parametrize("cols,top", [(700, 20), (131072, 20), (32000, 32), (5000, 3)])
def test_likeliest_tokens_of_rows_with_fewer_that_are_allowed(cols, top):
    """Rows in which almost everything is ruled out, and rows of equal logits: the bound of the search leaves them all."""
    logits = torch.full((6, cols), -math.inf, dtype=BF16, device="cuda")
    allowed = [0, cols // 3, cols - 1]
    logits[0, allowed] = torch.tensor([1.0, 3.0, 1.0], dtype=BF16, device="cuda")
    logits[1, 7] = -2.0
    logits[3], logits[4] = 0.0, torch.finfo(BF16).min
    logits[5, ::5] = 0.5
    got = ops.token_log_probs(logits, torch.zeros(6, dtype=torch.int64, device="cuda"), top=top)
    order = torch.sort(logits.double(), dim=-1, descending=True, stable=True).indices[:, :top]
    assert torch.equal(got.top_tokens, order)
    want = torch.log_softmax(logits.double(), -1).gather(1, order)
    want[2] = -math.inf                                                         # nothing is allowed
    assert torch.equal(torch.isneginf(got.top_log_probs), torch.isneginf(want))
    here = ~torch.isneginf(want)
    assert (got.top_log_probs.double() - want)[here].abs().max().item() <= (cols / 32 + 64) * 2.0 ** -23


@pytest.mark.parametrize("dtype,heads,kv_heads,dim,page", [(BF16, 4, 2, 64, 16), (F16, 12, 1, 64, 48), (F16, 6, 2, 128, 16), (BF16, 16, 1, 128, 32), (BF16, 9, 3, 40, 10),
                                                           (F16, 32, 2, 96, 7)])
@pytest.mark.parametrize("tokens", [1, 3])
def test_tables_with_room_for_long_sentences(dtype, heads, kv_heads, dim, page, tokens):
    """Room for 2^20 tokens of each sentence, as a loop has it that is captured once: the kernel for long runs, over short sentences."""
    lengths = [tokens, 17, 1024, 1023, 2500, 0, 33, 700, 2049, 64, 1, 100]
    batch, columns = len(lengths), -(-(1 << 20) // page)
    need = [-(-n // page) for n in lengths]
    pages = sum(need)
    order, at = torch.randperm(pages, generator=torch.Generator().manual_seed(1)).to(torch.int32), 0
    table = torch.full((batch, columns), -1, dtype=torch.int32)
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    table = table.cuda()
    k, v = (randn(pages, page, kv_heads, dim, dtype=dtype, seed=s) for s in (1, 2))
    q = randn(batch, tokens, heads, dim, dtype=dtype, seed=3, std=1.5)
    length = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    for window, sinks in ((0, 0), (1 << 19, 5)):
        o, lse = ops.paged_attention(q, k, v, table, length, window=window, sinks=sinks, need_lse=True)
        for b, n in enumerate(lengths):
            here, p = min(n, tokens), torch.arange(n, device="cuda")
            assert not o[b, here:].any() and torch.isneginf(lse[b, :, here:]).all()
            kb, vb = (x[table[b][p // page].long(), p % page].double().repeat_interleave(heads // kv_heads, 1) for x in (k, v))
            for t in range(here):
                m = n - here + t + 1
                s = torch.einsum("hd,nhd->hn", q[b, t].double(), kb[:m]) * dim ** -0.5
                w = torch.softmax(s, -1)
                want, size = torch.einsum("hn,nhd->hd", w, vb[:m]), torch.einsum("hn,nhd->hd", w, vb[:m].abs())
                within(o[b, t], want, U[dtype] * want.abs() + E * size + 2.0 ** -24, (b, t))
                l = torch.logsumexp(s, -1)
                within(lse[b, :, t], l, E * (1 + l.abs()), (b, t))
    if tokens > 1:                                                              # what earlier rows do not see: the same bits
        bad = v.clone()
        for b, n in enumerate(lengths):
            if n > 1:
                bad[table[b, (n - 1) // page].long(), (n - 1) % page] = math.inf
        again = ops.paged_attention(q, k, bad, table, length)
        plain = ops.paged_attention(q, k, v, table, length)
        for b, n in enumerate(lengths):
            here = min(n, tokens)
            if n > 1:
                assert torch.equal(again[b, :here - 1], plain[b, :here - 1]) and torch.isposinf(again[b, here - 1]).all()
    ops.check()


@pytest.mark.parametrize("dim", [64, 128])
def test_rows_that_are_none_stay_so_beside_infinite_values(dim):
    """A NaN in one query head makes that head's rows NaN, whatever the values; the others see the infinities."""
    n, page = 3000, 16
    k, v = (randn(n // page + 1, page, 1, dim, dtype=BF16, seed=s) for s in (1, 2))
    v[7, 3, 0, 5], v[90, 0, 0, 6] = math.inf, -math.inf
    table = torch.arange(n // page + 1, dtype=torch.int32, device="cuda")[None]
    q = randn(1, 2, 6, dim, dtype=BF16, seed=3)
    q[0, 1, 2, 0] = math.nan
    o, lse = ops.paged_attention(q, k, v, table, torch.tensor([n], dtype=torch.int32, device="cuda"), need_lse=True)
    none = torch.zeros(1, 2, 6, dtype=torch.bool, device="cuda")
    none[0, 1, 2] = True
    assert torch.equal(torch.isnan(o).all(-1), none) and torch.equal(torch.isnan(o).any(-1), none) and torch.equal(torch.isnan(lse).transpose(1, 2), none)
    seen = o[~none]
    assert (seen[:, 5] == math.inf).all() and (seen[:, 6] == -math.inf).all()
    rest = [d for d in range(dim) if d not in (5, 6)]
    assert torch.isfinite(seen[:, rest]).all()
