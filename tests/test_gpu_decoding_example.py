"""The decoding operators together, as the example uses them: nodes train what a decoder answers with, its mean model answers."""
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


def whole(decoder, flat, tokens):
    """(logits, leaf) of all positions of [batch, n] tokens in 64 bits, differentiable in the flat model."""
    leaf = flat.double().requires_grad_()
    norm, w = decoder.views(leaf)
    h = decoder.embedding[tokens].double()
    b, n = tokens.shape
    heads = (h @ decoder.qkv.double()).view(b, n, -1, decoder.head_dim)
    q, k, v = heads.split((decoder.heads, decoder.kv_heads, decoder.kv_heads), 2)
    angle = torch.arange(n, device="cuda").double()[:, None] * decoder.frequencies.double()

    def turn(x):
        x1, x2 = x.chunk(2, -1)
        c, s = angle.cos()[:, None], angle.sin()[:, None]
        return torch.cat([x1 * c - x2 * s, x2 * c + x1 * s], -1)

    group = decoder.heads // decoder.kv_heads
    q, k, v = turn(q), turn(k).repeat_interleave(group, 2), v.repeat_interleave(group, 2)
    s = torch.einsum("bthd,bshd->bhts", q, k) * decoder.head_dim ** -0.5
    s = s.masked_fill(torch.ones(n, n, device="cuda").triu(1).bool(), float("-inf"))
    o = torch.einsum("bhts,bshd->bthd", torch.softmax(s, -1), v).flatten(2)
    total = h + o @ decoder.o.double()
    return (norm * total / (total.square().mean(-1, keepdim=True) + 1e-6).sqrt()) @ w, leaf


def make(example):
    decoder = example.Decoder(vocabulary=97, width=64, heads=4, kv_heads=2, head_dim=32)
    flat = torch.empty(decoder.size, device="cuda")
    decoder.init(flat, torch.Generator(device="cuda").manual_seed(3))
    return decoder, flat


def test_gradients_are_those_of_automatic_differentiation(example):
    decoder, flat = make(example)
    tokens = example.sequences(decoder, 1, 2, batch=3, n=21)
    grad = torch.empty_like(flat)
    loss = decoder.loss(flat, grad, tokens)
    logits, leaf = whole(decoder, flat, tokens[:, :-1])
    want = torch.nn.functional.cross_entropy(logits.flatten(0, 1), tokens[:, 1:].flatten())
    ref, = torch.autograd.grad(want, leaf)
    # every tensor on the way is rounded to bf16 (2^-9 each, about ten of them in a row): 3 % of the norm is far above
    assert abs(loss.item() - want.item()) < 0.03 * want.item()
    for a, b in zip(decoder.views(grad.double()), decoder.views(ref)):
        assert (a - b).norm() < 0.03 * b.norm()


def test_answers_are_the_likeliest_tokens_of_the_whole_pass(example):
    """Prompts of unequal lengths continued token by token, each step held against all positions at once in 64 bits."""
    decoder, flat = make(example)
    flat.mul_(4.0)                                                              # distributions with a likeliest token
    prompts = example.sequences(decoder, 2, 5, batch=4, n=20)
    counts = torch.tensor([20, 3, 1, 17], dtype=torch.int32, device="cuda")
    tokens, log_probs = decoder.answer(flat, prompts, counts, 24)               # over ends of pages of 16
    for i in range(4):
        line = torch.cat([prompts[i, :counts[i]], tokens[i]])
        logits, _ = whole(decoder, flat, line[None, :-1])
        x = torch.log_softmax(logits[0, counts[i] - 1:], -1).detach()
        got = x.gather(1, tokens[i][:, None])[:, 0]
        # a logit is a sum of roundings like those of the gradients' test, 3 % of its size: so far may the chosen one be behind
        slack = 0.06 * logits.abs().max()
        assert (x.max(1).values - got).max() <= slack
        assert (got - log_probs[i]).abs().max() <= slack


def test_a_swarm_trains_and_answers(example):
    got = example.train(nodes=4, rounds=6, log=None)
    model = got["swarm"].mean_model()
    assert torch.isfinite(model).all() and got["last"] == got["last"]
    prompts = example.sequences(got["decoder"], 0, 7, batch=3, n=9)
    counts = torch.tensor([9, 1, 4], dtype=torch.int32, device="cuda")
    tokens, log_probs = got["decoder"].answer(model, prompts, counts, 5)
    assert tokens.shape == log_probs.shape == (3, 5) and (log_probs <= 0).all()
    assert ((tokens >= 0) & (tokens < got["decoder"].vocabulary)).all()
