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
