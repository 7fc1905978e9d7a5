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
