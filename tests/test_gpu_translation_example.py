"""The operators together, as the example uses them: nodes of a swarm train a cross-attention sublayer."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture()
def example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import translation_swarm
        yield translation_swarm
    finally:
        sys.path.pop(0)


def test_swarm_of_sublayers_learns_and_decodes(example):
    got = example.train(nodes=4, rounds=30, log=None)
    assert got["last"] < 0.7 * got["first"]                       # the nodes learn from the teacher
    assert got["gamma"] < got["gamma0"]                           # and agree more than at the start
    layer = got["layer"]
    off, size = example.serve(layer, layer.views(got["swarm"].mean_model()))
    assert off < 0.1 * size                                       # rows in 8 bits (2^-4 each) against rows in bf16


def test_sublayer_gradients_are_those_of_automatic_differentiation(example):
    import torch
    layer = example.Sublayer(width=64, heads=2, kv_heads=1, head_dim=32)
    flat = torch.empty(layer.size, device="cuda")
    layer.init(flat, torch.Generator(device="cuda").manual_seed(3))
    p = layer.views(flat)
    x, residual, e, lengths, target = example.batch(layer, p, 1, 2, sentences=3, queries=5, keys=9)
    target = torch.zeros_like(target)
    out, saved = layer.forward(p, x, residual, e, lengths)
    flat_grad = torch.empty(layer.size, device="cuda")
    grad = layer.views(flat_grad)
    dx, dresidual = layer.backward(p, out, saved, x, e, lengths, grad)
    leaf = flat.double().requires_grad_()
    w = layer.views(leaf)
    xd, rd = x.double().requires_grad_(), residual.double().requires_grad_()
    total = rd + xd
    y = w["norm"] * total / (total.square().mean(-1, keepdim=True) + 1e-6).sqrt()
    q = (y @ w["q"]).view(3, 5, 2, 32)
    kv = (e.double() @ w["kv"]).view(3, 9, 2, 1, 32)
    s = torch.einsum("bthd,bsd->bhts", q, kv[:, :, 0, 0]) * 32 ** -0.5
    s = s.masked_fill(torch.arange(9, device="cuda")[None, None, None] >= lengths[:, None, None, None], float("-inf"))
    o = torch.einsum("bhts,bsd->bthd", torch.softmax(s, -1), kv[:, :, 1, 0]).reshape(3, 5, 64)
    loss = 0.5 * (total + o @ w["o"] - target.double()).square().sum()
    want = torch.autograd.grad(loss, (leaf, xd, rd))
    for got, ref in zip((flat_grad, dx, dresidual), want):
        # every tensor on the way is rounded to bf16 (2^-9 each, about ten of them in a row): 3 % of the norm is far above
        assert (got.double() - ref).norm() < 0.03 * ref.norm()
