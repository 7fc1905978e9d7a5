"""A swarm whose nodes train the cross-attention sublayer of a translation model.

Each node's model is one flat vector of the swarm: the norm's weight and the projections of queries, keys, values and
output. A local step runs the sublayer forward and backward on a minibatch of the node's own data

    y, total = norm(residual + dropout(x)),  q = y Wq,  k = e Wk,  v = e Wv,  out = total + dropout(attention(q, k, v) Wo)

with the operators of paper_1910_12308_b200.operators between plain matrix products, and moves the model in place;
between steps, pairs of nodes exchange 8-bit codes of their models and average (swarm_interact). The data are synthetic:
decoder states x and encoder states e of unequal lengths from the node's own distribution, targets from a fixed teacher
sublayer. At the end the mean model decodes token by token over cached keys and values.

    python examples/translation_swarm.py [--nodes 8] [--rounds 60]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1910_12308_b200 import BLOCKING, Swarm  # noqa: E402
from paper_1910_12308_b200 import operators as ops  # noqa: E402

DTYPE = torch.bfloat16


class Sublayer:
    """Shapes of the sublayer and its parameters as views of a flat fp32 vector."""

    def __init__(self, width=256, heads=8, kv_heads=4, head_dim=64):
        self.width, self.heads, self.kv_heads, self.head_dim = width, heads, kv_heads, head_dim
        inner, kv = heads * head_dim, kv_heads * head_dim
        self.shapes = {"norm": (width,), "q": (width, inner), "kv": (width, 2 * kv), "o": (inner, width)}
        self.size = sum(torch.Size(s).numel() for s in self.shapes.values())

    def views(self, flat):
        out, at = {}, 0
        for name, shape in self.shapes.items():
            n = torch.Size(shape).numel()
            out[name] = flat[at:at + n].view(shape)
            at += n
        return out

    def init(self, flat, generator):
        p = self.views(flat)
        for name, w in p.items():
            if name == "norm":
                w.fill_(1.0)
            else:
                w.copy_(torch.randn(w.shape, generator=generator, device=w.device) * w.shape[0] ** -0.5)

    def project(self, y, e, p):
        """Queries of the decoder's rows; keys and values of the encoder's states, side by side in one product."""
        q = (y @ p["q"].to(DTYPE)).view(*y.shape[:2], self.heads, self.head_dim)
        kv = (e @ p["kv"].to(DTYPE)).view(*e.shape[:2], 2, self.kv_heads, self.head_dim)
        return q, kv

    def forward(self, p, x, residual, e, lengths, rate=0.0, seed=0, event=0):
        y, total = ops.add_rms_norm(x, p["norm"], residual=residual, rate=rate, seed=seed, event=2 * event)
        q, kv = self.project(y, e, p)
        o, lse = ops.cross_attention(q, kv[:, :, 0], kv[:, :, 1], key_lengths=lengths, need_lse=True)
        a = o.flatten(2) @ p["o"].to(DTYPE)
        out = ops.dropout(a, rate, seed, 2 * event + 1, residual=total)
        return out, (y, total, q, kv, o, lse)

    def backward(self, p, dout, saved, x, e, lengths, grad, rate=0.0, seed=0, event=0):
        """Gradients of all parameters into the views `grad`; returns the gradients of x and of the residual."""
        y, total, q, kv, o, lse = saved
        rows = y.shape[0] * y.shape[1]
        da = ops.dropout(dout, rate, seed, 2 * event + 1)
        grad["o"].copy_(o.view(rows, -1).T @ da.view(rows, -1))
        do = (da @ p["o"].to(DTYPE).T).view(q.shape)
        dkv = torch.empty_like(kv)                       # gradients of keys and values side by side, as they were made
        dq, _, _ = ops.cross_attention_backward(do, q, kv[:, :, 0], kv[:, :, 1], o, lse, key_lengths=lengths,
                                                dk=dkv[:, :, 0], dv=dkv[:, :, 1])
        grad["q"].copy_(y.view(rows, -1).T @ dq.view(rows, -1))
        grad["kv"].copy_(e.flatten(0, 1).T @ dkv.view(e.shape[0] * e.shape[1], -1))
        dy = dq.flatten(2) @ p["q"].to(DTYPE).T
        dx, dresidual, dnorm = ops.add_rms_norm_backward(dy, total, p["norm"], dtotal=dout, rate=rate, seed=seed, event=2 * event)
        grad["norm"].copy_(dnorm)
        return dx, dresidual

    def decode(self, p, x, residual, kv, lengths):
        """One token for each sentence over cached keys and values; the normalised rows travel in 8 bits."""
        codes, scales, total = ops.add_rms_norm(x, p["norm"], residual=residual, eight_bit=True)
        y = (codes.float() * scales.repeat_interleave(128, -1)[..., :self.width]).to(DTYPE)
        q = (y @ p["q"].to(DTYPE)).view(*x.shape[:2], self.heads, self.head_dim)
        o = ops.cross_attention(q, kv[:, :, 0], kv[:, :, 1], key_lengths=lengths)
        return ops.dropout(o.flatten(2) @ p["o"].to(DTYPE), 0.0, 0, 0, residual=total)


def batch(layer, teacher, node, step, sentences=16, queries=24, keys=40):
    """Minibatch `step` of a node: its own mean state, encoder states of unequal lengths, the teacher's outputs."""
    g = torch.Generator(device="cuda").manual_seed(1000003 * node + step)
    shift = torch.randn(layer.width, generator=torch.Generator(device="cuda").manual_seed(node), device="cuda") * 0.3
    x, residual = ((torch.randn(sentences, queries, layer.width, generator=g, device="cuda") + shift).to(DTYPE) for _ in range(2))
    e = (torch.randn(sentences, keys, layer.width, generator=g, device="cuda") + shift).to(DTYPE)
    lengths = torch.randint(keys // 2, keys + 1, (sentences,), generator=g, device="cuda", dtype=torch.int32)
    target, _ = layer.forward(teacher, x, residual, e, lengths)
    return x, residual, e, lengths, target


def train(nodes=8, rounds=60, steps=2, lr=0.02, rate=0.1, bits=8, seed=1, log=print):
    """Returns the mean loss of the first and of the last round, the potential before and after, the swarm and layer."""
    layer = Sublayer()
    swarm = Swarm(nodes, layer.size, "complete", seed=seed, stream=torch.cuda.current_stream())
    models = swarm.model_tensor()
    make = torch.Generator(device="cuda").manual_seed(seed)
    for i in range(nodes):
        layer.init(models[i], make)
    flat_teacher = torch.empty(layer.size, device="cuda")
    layer.init(flat_teacher, make)
    teacher = layer.views(flat_teacher)
    flat_grad = torch.empty(layer.size, device="cuda")
    grad = layer.views(flat_grad)
    taken = [0] * nodes
    first = last = None
    gamma0 = swarm.potential()
    for r in range(rounds):
        pairs = swarm.sample_pairs(nodes // 2)
        losses = []
        for node in pairs.reshape(-1).tolist():
            p = layer.views(models[node])
            for _ in range(steps):
                event, mask = taken[node], {"rate": rate, "seed": seed + node, "event": taken[node]}
                x, residual, e, lengths, target = batch(layer, teacher, node, event)
                out, saved = layer.forward(p, x, residual, e, lengths, **mask)
                error = out.float() - target.float()
                losses.append(error.square().mean())
                layer.backward(p, (error / (error.shape[0] * error.shape[1])).to(DTYPE), saved, x, e, lengths, grad, **mask)
                models[node, :layer.size].add_(flat_grad, alpha=-lr)
                taken[node] += 1
        rc = swarm.interact(pairs, bits, BLOCKING)
        if rc != 0:
            raise RuntimeError(f"swarm_interact: {rc}")
        loss = torch.stack(losses).mean().item()
        first = loss if first is None else first
        last = loss
        if log and (r % 10 == 0 or r == rounds - 1):
            log(f"round {r:3d}: loss {loss:.4f}, potential {swarm.potential():.1f}")
    ops.check()
    return {"first": first, "last": last, "gamma0": gamma0, "gamma": swarm.potential(), "swarm": swarm, "layer": layer, "teacher": teacher}


def serve(layer, p, tokens=5):
    """Largest difference between the outputs of the decoding steps and of the whole forward pass."""
    x, residual, e, lengths, _ = batch(layer, p, 3, 7, queries=tokens)
    whole, _ = layer.forward(p, x, residual, e, lengths)
    _, kv = layer.project(x[:, :1], e, p)                # keys and values are made once and kept
    one = [layer.decode(p, x[:, t:t + 1], residual[:, t:t + 1], kv, lengths) for t in range(tokens)]
    return (torch.cat(one, 1).float() - whole.float()).abs().max().item(), whole.float().abs().max().item()


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--nodes", type=int, default=8)
    ap.add_argument("--rounds", type=int, default=60)
    a = ap.parse_args()
    got = train(a.nodes, a.rounds)
    print(f"loss {got['first']:.4f} -> {got['last']:.4f}, potential {got['gamma0']:.1f} -> {got['gamma']:.1f}")
    off, size = serve(got["layer"], got["layer"].views(got["swarm"].mean_model()))
    print(f"decoding with 8-bit rows: {off:.3f} off the whole pass, whose largest value is {size:.3f}")
