"""A swarm whose nodes train what a decoder answers with, and its mean model answering token by token.

The decoder has one attention sublayer over what it has said so far, a norm and a projection onto the vocabulary:

    h = embedding[token],  q, k, v = h Wq, h Wk, h Wv (q and k rotated by their positions),
    y, total = norm(h + attention(q, k, v) Wo),  logits = y W

Embedding and attention are the same for all nodes and stay as they are; each node's model is the norm's weight and W, one
flat vector of the swarm. A local step takes sequences of the node's own data: their keys and values are appended to a paged
cache at once, all positions attend to what came before them, and the loss is the mean negative log probability of each next
token. Between steps, pairs of nodes exchange 8-bit codes of their models and average (swarm_interact). At the end the mean model
continues prompts of unequal lengths: each step appends one token to every sequence, attends through the cache, and takes
the likeliest next token.

    python examples/decoding_swarm.py [--nodes 8] [--rounds 40]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1910_12308_b200 import BLOCKING, Swarm  # noqa: E402
from paper_1910_12308_b200 import operators as ops  # noqa: E402

DTYPE = torch.bfloat16
PIECE = 64                                  # tokens of a sequence that one call of attention over the cache takes


class Cache:
    """Pages of keys and values for `batch` sequences of up to `most` tokens, handed out in order."""

    def __init__(self, decoder, batch, most, page_size=16):
        columns = -(-most // page_size)
        shape = (batch * columns, page_size, decoder.kv_heads, decoder.head_dim)
        self.k, self.v = (torch.empty(shape, dtype=DTYPE, device="cuda") for _ in range(2))
        self.table = torch.arange(batch * columns, dtype=torch.int32, device="cuda").view(batch, columns)
        self.lengths = torch.zeros(batch, dtype=torch.int32, device="cuda")


class Decoder:
    """The part that all nodes share, and the shapes of the part that they train."""

    def __init__(self, vocabulary=512, width=256, heads=8, kv_heads=2, head_dim=64, seed=0):
        self.vocabulary, self.width, self.heads, self.kv_heads, self.head_dim = vocabulary, width, heads, kv_heads, head_dim
        g = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*shape, std):
            return (torch.randn(*shape, generator=g, device="cuda") * std).to(DTYPE)

        self.embedding = normal(vocabulary, width, std=1.0)
        self.qkv = normal(width, (heads + 2 * kv_heads) * head_dim, std=width ** -0.5)
        self.o = normal(heads * head_dim, width, std=(heads * head_dim) ** -0.5)
        self.frequencies = 10000.0 ** (-torch.arange(head_dim // 2, device="cuda") / (head_dim // 2))
        self.size = width + width * vocabulary

    def views(self, flat):
        return flat[:self.width], flat[self.width:self.size].view(self.width, self.vocabulary)

    def init(self, flat, generator):
        norm, w = self.views(flat)
        norm.fill_(1.0)
        w.copy_(torch.randn(w.shape, generator=generator, device="cuda") * 0.5 * self.width ** -0.5)

    def attend(self, tokens, cache, counts=None):
        """What the norm takes, h and the attention's output, for the newest tokens [batch, n] of the sequences in the cache
        (counts: how many of n are a sequence's). They are appended to the cache first."""
        h = self.embedding[tokens]
        heads = (h @ self.qkv).view(*tokens.shape, self.heads + 2 * self.kv_heads, self.head_dim)
        q, k, v = heads.split((self.heads, self.kv_heads, self.kv_heads), 2)
        cache.lengths += tokens.shape[1] if counts is None else counts
        q = ops.append_to_cache(k, v, cache.k, cache.v, cache.table, cache.lengths, counts=counts, q=q, frequencies=self.frequencies)
        return h, self.look(q, cache, counts).flatten(2) @ self.o

    def look(self, q, cache, counts):
        """Attention of the newest tokens, which are in the cache, piece by piece: a piece ends the cache for its own call."""
        n = q.shape[1]
        if n <= PIECE:
            return ops.paged_attention(q, cache.k, cache.v, cache.table, cache.lengths, counts=counts)
        counts = torch.full_like(cache.lengths, n) if counts is None else counts
        before, pieces = cache.lengths - counts, []
        for at in range(0, n, PIECE):
            here = (counts - at).clamp(0, PIECE)
            pieces.append(ops.paged_attention(q[:, at:at + PIECE], cache.k, cache.v, cache.table, before + counts.clamp(max=at + PIECE), counts=here))
        return torch.cat(pieces, 1)

    def logits(self, flat, h, a):
        norm, w = self.views(flat)
        y, total = ops.add_rms_norm(a, norm, residual=h)
        return y @ w.to(DTYPE), y, total

    def loss(self, flat, grad, tokens):
        """Mean negative log probability of tokens[:, 1:], the gradient of the node's part into the flat vector `grad`."""
        inputs, targets = tokens[:, :-1].contiguous(), tokens[:, 1:].contiguous()
        h, a = self.attend(inputs, Cache(self, *inputs.shape))
        logits, y, total = self.logits(flat, h, a)
        got = ops.token_log_probs(logits, targets)
        dlogits = ops.token_log_probs_backward(torch.full_like(got.log_probs, -1.0 / targets.numel()), logits, targets, got.stats, dlogits=logits)
        norm, w = self.views(flat)
        dnorm, dw = self.views(grad)
        rows = targets.numel()
        dw.copy_(y.view(rows, -1).T @ dlogits.view(rows, -1))
        dy = dlogits @ w.to(DTYPE).T
        dnorm.copy_(ops.add_rms_norm_backward(dy, total, norm)[2])
        return -got.log_probs.mean()

    def answer(self, flat, prompts, counts, steps):
        """Continues prompts [batch, n], of which counts [batch] tokens, one at least, are each sequence's: (tokens, their log
        probabilities), [batch, steps]."""
        if counts.min().item() < 1 or counts.max().item() > prompts.shape[1]:
            raise ValueError("counts: between 1 and the prompts' width")
        cache = Cache(self, prompts.shape[0], prompts.shape[1] + steps)
        h, a = self.attend(prompts, cache, counts)
        last = (counts.long() - 1).view(-1, 1, 1).expand(-1, 1, self.width)
        h, a = h.gather(1, last), a.gather(1, last)
        tokens, log_probs = [], []
        for step in range(steps):
            got = ops.token_log_probs(self.logits(flat, h, a)[0], top=1)
            tokens.append(got.top_tokens[..., 0])
            log_probs.append(got.top_log_probs[..., 0])
            if step + 1 < steps:
                h, a = self.attend(tokens[-1], cache)
        return torch.cat(tokens, 1), torch.cat(log_probs, 1)


def sequences(decoder, node, step, batch=16, n=33):
    """Data of a node: each token follows from the one before it by the node's rule half of the time, else by the common one."""
    g = torch.Generator(device="cuda").manual_seed(1000003 * node + step)
    tokens = torch.randint(decoder.vocabulary, (batch, n), generator=g, device="cuda")
    own = torch.rand(batch, n, generator=g, device="cuda") < 0.5
    for t in range(1, n):
        common, of_node = (tokens[:, t - 1] * 5 + 1) % decoder.vocabulary, (tokens[:, t - 1] + 7 * node + 3) % decoder.vocabulary
        tokens[:, t] = torch.where(own[:, t], of_node, common)
    return tokens


def train(nodes=8, rounds=40, steps=2, lr=2.0, bits=8, seed=1, log=print):
    decoder = Decoder()
    swarm = Swarm(nodes, decoder.size, "complete", seed=seed, stream=torch.cuda.current_stream())
    models = swarm.model_tensor()
    for i in range(nodes):
        decoder.init(models[i], torch.Generator(device="cuda").manual_seed(seed))
    grad = torch.empty(decoder.size, device="cuda")
    taken, first, last = [0] * nodes, None, None
    for r in range(rounds):
        pairs = swarm.sample_pairs(nodes // 2)
        losses = []
        for node in pairs.reshape(-1).tolist():
            for _ in range(steps):
                losses.append(decoder.loss(models[node], grad, sequences(decoder, node, taken[node])))
                models[node, :decoder.size].add_(grad, alpha=-lr)
                taken[node] += 1
        rc = swarm.interact(pairs, bits, BLOCKING)
        if rc != 0:
            raise RuntimeError(f"swarm_interact: {rc}")
        last = torch.stack(losses).mean().item()
        first = last if first is None else first
        if log and (r % 10 == 0 or r == rounds - 1):
            log(f"round {r:3d}: loss {last:.4f}, potential {swarm.potential():.1f}")
    ops.check()
    return {"first": first, "last": last, "swarm": swarm, "decoder": decoder}


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--nodes", type=int, default=8)
    ap.add_argument("--rounds", type=int, default=40)
    args = ap.parse_args()
    got = train(args.nodes, args.rounds)
    print(f"loss {got['first']:.4f} -> {got['last']:.4f}")
    decoder, model = got["decoder"], got["swarm"].mean_model()
    prompts = sequences(decoder, 0, 12345, batch=4, n=12)
    counts = torch.tensor([12, 5, 1, 8], dtype=torch.int32, device="cuda")
    tokens, log_probs = decoder.answer(model, prompts, counts, 8)
    for i in range(4):
        print(prompts[i, :counts[i]].tolist(), "->", tokens[i].tolist(), f"log probability {log_probs[i].sum().item():.2f}")
