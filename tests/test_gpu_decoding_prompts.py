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
