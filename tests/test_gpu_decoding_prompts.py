"""Prompts that the decoding example is given: what it refuses, and those longer than one call of attention takes."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture()
def example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import decoding_swarm
        yield decoding_swarm
    finally:
        sys.path.pop(0)


def make(example):
    decoder = example.Decoder(vocabulary=97, width=64, heads=4, kv_heads=2, head_dim=32)
    flat = torch.empty(decoder.size, device="cuda")
    decoder.init(flat, torch.Generator(device="cuda").manual_seed(3))
    return decoder, flat


@pytest.mark.parametrize("counts", [(0, 5), (5, -1), (7, 8), (-3, 9)])
def test_counts_outside_the_prompts_are_refused(example, counts):
    decoder, flat = make(example)
    prompts = example.sequences(decoder, 0, 1, batch=2, n=7)
    with pytest.raises(ValueError):
        decoder.answer(flat, prompts, torch.tensor(counts, dtype=torch.int32, device="cuda"), 2)
    tokens, _ = decoder.answer(flat, prompts, torch.tensor((1, 7), dtype=torch.int32, device="cuda"), 2)
    assert tokens.shape == (2, 2)


def whole(decoder, flat, tokens):
    """(logits, leaf) of all positions of [batch, n] tokens in 64 bits, differentiable in the flat model."""
    leaf = flat.double().requires_grad_()
    norm, w = decoder.views(leaf)
    h = decoder.embedding[tokens].double()
    b, n = tokens.shape
    heads = (h @ decoder.qkv.double()).view(b, n, -1, decoder.head_dim)
    q, k, v = heads.split((decoder.heads, decoder.kv_heads, decoder.kv_heads), 2)
    angle = (torch.arange(n, device="cuda").double()[:, None] * decoder.frequencies.double())[:, None]

    def turn(x):
        x1, x2 = x.chunk(2, -1)
        return torch.cat([x1 * angle.cos() - x2 * angle.sin(), x2 * angle.cos() + x1 * angle.sin()], -1)

    group = decoder.heads // decoder.kv_heads
    q, k, v = turn(q), turn(k).repeat_interleave(group, 2), v.repeat_interleave(group, 2)
    s = torch.einsum("bthd,bshd->bhts", q, k) * decoder.head_dim ** -0.5
    s = s.masked_fill(torch.ones(n, n, device="cuda").triu(1).bool(), float("-inf"))
    o = torch.einsum("bhts,bshd->bthd", torch.softmax(s, -1), v).flatten(2)
    total = h + o @ decoder.o.double()
    return (norm * total / (total.square().mean(-1, keepdim=True) + 1e-6).sqrt()) @ w, leaf


def test_prompts_of_several_pieces_are_answered(example):
    """Every tensor on the way is rounded to bf16 (2^-8 each at most, about ten in a row): 6 % of the logits' size is above that."""
    decoder, flat = make(example)
    flat.mul_(4.0)
    prompts = example.sequences(decoder, 2, 5, batch=5, n=150)
    counts = torch.tensor([150, 64, 65, 1, 128], dtype=torch.int32, device="cuda")
    tokens, log_probs = decoder.answer(flat, prompts, counts, 4)
    for i in range(5):
        line = torch.cat([prompts[i, :counts[i]], tokens[i]])
        logits, _ = whole(decoder, flat, line[None, :-1])
        x = torch.log_softmax(logits[0, counts[i] - 1:], -1).detach()
        got = x.gather(1, tokens[i][:, None])[:, 0]
        slack = 0.06 * logits.abs().max()
        assert (x.max(1).values - got).max() <= slack
        assert (got - log_probs[i]).abs().max() <= slack


def test_pieces_are_what_one_call_each_gives(example):
    """Rows of every piece against attention of single tokens over the cache as it was then."""
    from paper_1910_12308_b200 import operators as ops
    decoder, _ = make(example)
    counts = torch.tensor([130, 64, 3, 129], dtype=torch.int32, device="cuda")
    cache = example.Cache(decoder, 4, 150)
    for x in (cache.k, cache.v):
        x.copy_(torch.randn(x.shape, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda"))
    cache.lengths += counts + 20
    q = torch.randn(4, 130, 4, 32, generator=torch.Generator(device="cuda").manual_seed(6), device="cuda").to(example.DTYPE)
    got = decoder.look(q, cache, counts)
    for t in (0, 2, 3, 63, 64, 127, 128, 129):
        live = counts > t
        one = ops.paged_attention(q[:, t:t + 1], cache.k, cache.v, cache.table, 20 + counts.clamp(max=t) + live.int(), counts=live.int())
        # two orders of the same sums, each rounded once, of values that stay below 4
        assert (got[:, t].double() - one[:, 0].double()).abs().max().item() <= 2 * 4 * (2.0 ** -8 + 4e-5)
        assert not got[~live, t].any()


def test_gradients_over_several_pieces(example):
    decoder, flat = make(example)
    tokens = example.sequences(decoder, 1, 2, batch=3, n=100)
    grad = torch.empty_like(flat)
    loss = decoder.loss(flat, grad, tokens)
    logits, leaf = whole(decoder, flat, tokens[:, :-1])
    want = torch.nn.functional.cross_entropy(logits.flatten(0, 1), tokens[:, 1:].flatten())
    ref, = torch.autograd.grad(want, leaf)
    assert abs(loss.item() - want.item()) < 0.03 * want.item()                  # 3 % of the norm: see above
    for a, b in zip(decoder.views(grad.double()), decoder.views(ref)):
        assert (a - b).norm() < 0.03 * b.norm()
