"""The operators of a decoder's cross-attention sublayer at sizes of real use: their cases, their inputs, their
plain forms and their definitions in 64 bits.

  dropout     out = residual + mask * x / (1 - p), the mask drawn from the counter-based generator
  norm        total = residual + dropout(x), y = weight * total / rms(total), y in the inputs' type or in 8 bits
  attention   attention of a decoder's rows to an encoder's states of another length

`run` computes them with elementary tensor operations in 32 bits where `own` is false, and through the package's
calls where it is true. A "train" case is the forward and the backward pass of a training step.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-6
STREAM = 13                     # generator stream of the dropout masks
E4M3_MAX = 448.0


def _dropout(name, rows, cols, kind, residual, form):
    return {"name": name, "op": "dropout", "rows": rows, "cols": cols, "type": kind, "rate": 0.1, "residual": residual,
            "form": form}


def _norm(name, rows, cols, kind, rate, form):
    return {"name": name, "op": "norm", "rows": rows, "cols": cols, "type": kind, "rate": rate, "form": form}


def _attention(name, batch, heads, kv_heads, queries, keys, dim, kind, form, ragged, layout):
    return {"name": name, "op": "attention", "batch": batch, "heads": heads, "kv_heads": kv_heads, "queries": queries,
            "keys": keys, "dim": dim, "type": kind, "form": form, "ragged": ragged, "layout": layout}


def listed():
    return [
        # a few sentences of odd length and width: launches count, not bytes
        _dropout("dropout small odd f16", 77, 1001, "f16", True, "train"),
        # a training batch of 32768 target tokens, dropout in front of a residual connection, and its gradient
        _dropout("dropout batch bf16", 32768, 1024, "bf16", True, "train"),
        # one token for each of 8 sentences, normalised for a projection with 8-bit operands
        _norm("norm token 8bit", 8, 512, "bf16", 0.0, "8bit"),
        # models in fp32 of an odd width
        _norm("norm odd f32", 1500, 1001, "f32", 0.1, "train"),
        # a training batch, residual connection with dropout and norm, forward and backward
        _norm("norm batch bf16", 16384, 1024, "bf16", 0.1, "train"),
        # a long batch of a wide model, normalised for a projection with 8-bit operands
        _norm("norm wide 8bit", 16384, 4096, "bf16", 0.0, "8bit"),
        # one new token for each of 4 sentences over short encoder states: the smallest call of a decoding loop
        _attention("attention token small", 4, 8, 8, 1, 77, 64, "bf16", "forward", False, "packed"),
        # a decoding batch of 128 sentences of unequal lengths
        _attention("attention token batch", 128, 16, 16, 1, 1024, 64, "bf16", "forward", True, "packed"),
        # few long documents, four query heads to each key head, states kept head by head
        _attention("attention token long", 8, 32, 8, 1, 16384, 128, "f16", "forward", False, "heads"),
        # training on short sentences of unequal lengths, one of them empty
        _attention("attention train small", 8, 8, 8, 50, 61, 64, "bf16", "train", True, "packed"),
        # an ordinary training batch of sentence pairs of unequal lengths
        _attention("attention train batch", 32, 16, 16, 512, 512, 64, "bf16", "train", True, "packed"),
        # long documents with four query heads to each key head
        _attention("attention train long", 4, 16, 4, 2048, 4096, 128, "f16", "train", False, "packed"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["dropout", "norm", "norm", "attention", "attention", "attention"])
    if op == "dropout":
        cols = _log(rng, 33, 8192)
        rows = _log(rng, 1, max(2, min(32768, 2 ** 25 // cols)))
        c = _dropout("", rows, cols, rng.choice(["bf16", "f16", "f32"]), rng.random() < 0.5, rng.choice(["train", "forward"]))
        if c["type"] == "f32":
            c["rows"] = max(1, rows // 2)
    elif op == "norm":
        form = rng.choice(["train", "forward", "8bit"])
        cols = _log(rng, 33, 8192)
        if rng.random() < 0.6:
            cols = max(64, cols // 64 * 64)
        rows = _log(rng, 1, max(2, min(16384, 2 ** 24 // cols)))
        c = _norm("", rows, cols, rng.choice(["bf16", "bf16", "f16", "f32"]), rng.choice([0.0, 0.1, 0.3]), form)
        if c["type"] == "f32":
            c["rows"] = max(1, rows // 2)
    else:
        kind, dim = rng.choice(["bf16", "bf16", "f16"]), rng.choice([32, 40, 64, 64, 80, 96, 128, 128])
        kv_heads, group = rng.choice([1, 2, 4, 6, 8, 16]), rng.choice([1, 1, 2, 3, 4, 8])
        heads = kv_heads * group
        form = rng.choice(["token", "forward", "train"])
        layout = rng.choice(["packed", "heads"])
        if form == "token":
            keys = _log(rng, 1, 16384)
            batch = _log(rng, 1, max(2, min(256, 2 ** 26 // (keys * kv_heads * dim))))
            c = _attention("", batch, heads, kv_heads, rng.choice([1, 1, 1, 2, 4]), keys, dim, kind, "forward",
                           rng.random() < 0.5, layout)
        else:
            queries, keys = _log(rng, 5, 2048), _log(rng, 5, 4096)
            queries = min(queries, 2 ** 28 // (heads * keys))
            batch = _log(rng, 1, max(1, min(64, 2 ** 28 // (heads * queries * keys), 2 ** 25 // (heads * max(queries, keys) * dim))))
            c = _attention("", batch, heads, kv_heads, queries, keys, dim, kind, form, rng.random() < 0.5, layout)
    del c["name"]
    return c


# ---- inputs --------------------------------------------------------------------------------------------------------


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = TYPES[case["type"]]

    def normal(*shape, std=1.0, dtype=dt):
        return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)

    s = {"case": case, "seed": (seed * 0x9E3779B97F4A7C15 + 0x1234567) % 2 ** 64, "event": seed % 1000003}
    if case["op"] in ("dropout", "norm"):
        rows, cols = case["rows"], case["cols"]
        s["x"] = normal(rows, cols)
        s["residual"] = normal(rows, cols, std=2.0) if case.get("residual", True) else None
        if case["op"] == "norm":
            s["weight"] = 1.0 + 0.2 * normal(cols, dtype=torch.float32)
        if case["form"] == "train":
            s["dy"] = normal(rows, cols)
            if case["op"] == "norm":
                s["dtotal"] = normal(rows, cols)
        return s
    b, h, hk, tq, tk, d = (case[k] for k in ("batch", "heads", "kv_heads", "queries", "keys", "dim"))
    s["q"] = normal(b, tq, h, d, std=1.5)
    if case["layout"] == "packed":             # one projection writes keys and values side by side
        kv = normal(b, tk, 2, hk, d)
        s["k"], s["v"] = kv[:, :, 0], kv[:, :, 1]
    else:                                      # states kept head by head
        s["k"], s["v"] = (normal(b, hk, tk, d).transpose(1, 2) for _ in range(2))
    s["query_lengths"] = s["key_lengths"] = None
    if case["ragged"]:
        def lengths(most):
            n = torch.randint(most - most // 2, most + 1, (b,), generator=g, device="cuda", dtype=torch.int32)
            n[0] = most
            return n
        s["key_lengths"] = lengths(tk)
        if b > 4:
            s["key_lengths"][b // 2] = 0       # a sentence without encoder states
        if tq > 4:
            s["query_lengths"] = lengths(tq)
    if case["form"] == "train":
        s["do"] = normal(b, tq, h, d)
    return s


def work(case):
    size = 4 if case["type"] == "f32" else 2
    if case["op"] == "dropout":
        n = case["rows"] * case["cols"]
        tensors = (3 if case["residual"] else 2) + (2 if case["form"] == "train" else 0)
        return {"bytes": n * size * tensors, "flops": 4 * n}
    if case["op"] == "norm":
        n, blocks = case["rows"] * case["cols"], case["rows"] * -(-case["cols"] // 128)
        if case["form"] == "8bit":
            return {"bytes": n * (3 * size + 1) + 4 * blocks + 4 * case["cols"], "flops": 8 * n}
        # x, residual -> total, y; dy, dtotal, total -> dx, dresidual
        extra = (4 + (case["rate"] > 0)) if case["form"] == "train" else 0
        return {"bytes": n * size * (4 + extra) + 8 * case["cols"], "flops": 8 * n + (12 * n if extra else 0)}
    b, h, hk, tq, tk, d = (case[k] for k in ("batch", "heads", "kv_heads", "queries", "keys", "dim"))
    share_k = 0.75 if case["ragged"] else 1.0
    share_q = 0.75 if case["ragged"] and tq > 4 else 1.0
    q, kv = b * tq * h * d * size, b * tk * hk * d * size * share_k
    product = 2 * b * h * tq * share_q * tk * share_k * d
    if case["form"] == "train":                # q, k, v, do -> o, dq, dk, dv; two products forward, five backward
        return {"bytes": 4 * q + 4 * kv + 4 * b * h * tq, "flops": 7 * product}
    return {"bytes": 2 * q + 2 * kv, "flops": 2 * product}


# ---- plain forms ---------------------------------------------------------------------------------------------------


def _keep(rows, cols, rate, seed, event):
    """Whether each element is kept: Philox-4x32 (10 rounds) keyed by the seed, one call for 8 consecutive columns of
    a row (counter = column div 8, row, event, stream), 16 bits an element, kept where they reach rate * 2^16."""
    low = 0xFFFFFFFF
    groups = -(-cols // 8)
    c0 = torch.arange(groups, device="cuda").expand(rows, groups)
    c1 = torch.arange(rows, device="cuda").unsqueeze(1).expand(rows, groups)
    c2, c3 = torch.full_like(c0, event), torch.full_like(c0, STREAM)
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57        # the low 64 bits, as signed numbers
        c0, c1, c2, c3 = ((p1 >> 32) & low) ^ c1 ^ k0, p1 & low, ((p0 >> 32) & low) ^ c3 ^ k1, p0 & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack([c0 & 0xFFFF, c0 >> 16, c1 & 0xFFFF, c1 >> 16, c2 & 0xFFFF, c2 >> 16, c3 & 0xFFFF, c3 >> 16], -1)
    return words.reshape(rows, groups * 8)[:, :cols] >= _threshold(rate)


def _threshold(rate):
    return int(math.floor(rate * 65536.0 + 0.5))


def _plain_dropout(x, case, s):
    x = x.float()
    if case["rate"] == 0.0:
        return x
    factor = 65536.0 / (65536 - _threshold(case["rate"]))
    return torch.where(_keep(case["rows"], case["cols"], case["rate"], s["seed"], s["event"]), x * factor, torch.zeros_like(x))


def _plain_dropout_pass(s, case, dt):
    out = _plain_dropout(s["x"], case, s)
    if s["residual"] is not None:
        out = s["residual"].float() + out
    out = out.to(dt)
    if case["form"] == "train":
        return {"out": out, "dx": _plain_dropout(s["dy"], case, s).to(dt)}
    return {"out": out}


def _plain_norm_pass(s, case, dt):
    total32 = s["residual"].float() + _plain_dropout(s["x"], case, s)
    total, w = total32.to(dt), s["weight"]
    y = total32 * torch.rsqrt(total32.square().mean(1, keepdim=True) + EPS) * w
    if case["form"] == "8bit":
        rows, cols = y.shape
        blocks = -(-cols // 128)
        wide = torch.zeros(rows, blocks * 128, device=y.device)
        wide[:, :cols] = y
        wide = wide.view(rows, blocks, 128)
        scales = wide.abs().amax(2) / E4M3_MAX
        codes = torch.where(scales.unsqueeze(2) > 0, wide / scales.unsqueeze(2), wide)
        return {"codes": codes.view(rows, blocks * 128)[:, :cols].contiguous().to(torch.float8_e4m3fn), "scales": scales,
                "total": total}
    if case["form"] == "forward":
        return {"y": y.to(dt), "total": total}
    # the backward pass is taken at the total as it is kept
    t, dy = total.float(), s["dy"].float()
    r = torch.rsqrt(t.square().mean(1, keepdim=True) + EPS)
    wdy = dy * w
    dtotal = s["dtotal"].float() + r * wdy - t * (r ** 3 * (wdy * t).mean(1, keepdim=True))
    return {"y": y.to(dt), "total": total, "dx": _plain_dropout(dtotal, case, s).to(dt), "dresidual": dtotal.to(dt),
            "dweight": (dy * t * r).sum(0)}


def _plain_attention_pass(s, case, dt):
    b, h, hk, tq, tk, d = (case[k] for k in ("batch", "heads", "kv_heads", "queries", "keys", "dim"))
    scale, group = d ** -0.5, h // hk
    rows = group * tq                          # the query heads of a key head side by side

    def by_kv_head(x):
        return x.float().view(b, tq, hk, group, d).permute(0, 2, 3, 1, 4).reshape(b, hk, rows, d)

    def back(x):
        return x.view(b, hk, group, tq, d).permute(0, 3, 1, 2, 4).reshape(b, tq, h, d)

    q, k, v = by_kv_head(s["q"]), s["k"].float().transpose(1, 2), s["v"].float().transpose(1, 2)
    scores = torch.matmul(q, k.transpose(2, 3)) * scale
    valid = None
    if s["key_lengths"] is not None:
        valid = (torch.arange(tk, device="cuda") < s["key_lengths"].unsqueeze(1)).view(b, 1, 1, tk)
    if s["query_lengths"] is not None:
        rows_in = (torch.arange(tq, device="cuda") < s["query_lengths"].unsqueeze(1)).repeat(1, group).view(b, 1, rows, 1)
        valid = rows_in if valid is None else valid & rows_in
    if valid is not None:
        scores = scores.masked_fill(~valid, -math.inf)
    top = scores.amax(3, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = torch.exp(scores - top)
    total = p.sum(3, keepdim=True)
    p = p / torch.where(total > 0, total, torch.ones_like(total))
    o32 = torch.matmul(p, v)
    o = back(o32).to(dt)
    if case["form"] == "forward":
        return {"o": o}
    lse = (top + torch.log(total)).view(b, hk, group, tq).reshape(b, h, tq)
    do = by_kv_head(s["do"])
    dv = torch.matmul(p.transpose(2, 3), do)
    if valid is not None:                      # rows past the end take no part, whatever their gradient holds
        do = torch.where(rows_in, do, torch.zeros_like(do)) if s["query_lengths"] is not None else do
    ds = p * (torch.matmul(do, v.transpose(2, 3)) - (do * o32).sum(3, keepdim=True)) * scale
    dq, dk = torch.matmul(ds, k), torch.matmul(ds.transpose(2, 3), q)
    return {"o": o, "lse": lse, "dq": back(dq).to(dt), "dk": dk.transpose(1, 2).to(dt), "dv": dv.transpose(1, 2).to(dt)}


# ---- the package's calls -------------------------------------------------------------------------------------------


def _own_pass(s, case):
    from paper_1910_12308_b200 import operators as ops
    train = case["form"] == "train"
    if case["op"] == "dropout":
        got = {"out": ops.dropout(s["x"], case["rate"], s["seed"], s["event"], residual=s["residual"])}
        if train:
            got["dx"] = ops.dropout(s["dy"], case["rate"], s["seed"], s["event"])
        return got
    if case["op"] == "norm":
        how = {"eps": EPS, "rate": case["rate"], "seed": s["seed"], "event": s["event"]}
        if case["form"] == "8bit":
            codes, scales, total = ops.add_rms_norm(s["x"], s["weight"], residual=s["residual"], eight_bit=True, **how)
            return {"codes": codes, "scales": scales, "total": total}
        y, total = ops.add_rms_norm(s["x"], s["weight"], residual=s["residual"], **how)
        if not train:
            return {"y": y, "total": total}
        dx, dresidual, dweight = ops.add_rms_norm_backward(s["dy"], total, s["weight"], dtotal=s["dtotal"], **how)
        return {"y": y, "total": total, "dx": dx, "dresidual": dresidual, "dweight": dweight}
    ends = {"query_lengths": s["query_lengths"], "key_lengths": s["key_lengths"]}
    if not train:
        return {"o": ops.cross_attention(s["q"], s["k"], s["v"], **ends)}
    o, lse = ops.cross_attention(s["q"], s["k"], s["v"], need_lse=True, **ends)
    dq, dk, dv = ops.cross_attention_backward(s["do"], s["q"], s["k"], s["v"], o, lse, **ends)
    return {"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


def run(s):
    case = s["case"]
    if own:
        return _own_pass(s, case)
    dt = TYPES[case["type"]]
    return {"dropout": _plain_dropout_pass, "norm": _plain_norm_pass, "attention": _plain_attention_pass}[case["op"]](s, case, dt)


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------


def _exact_mask(rows, cols, rate, seed, event):
    """The factor of each element, 0 or 1 / (1 - p), with the generator in unsigned 64-bit arithmetic on the host."""
    groups = (cols + 7) // 8
    u = np.uint64
    word = [np.tile(np.arange(groups, dtype=u), rows), np.repeat(np.arange(rows, dtype=u), groups),
            np.full(rows * groups, event, dtype=u), np.full(rows * groups, STREAM, dtype=u)]
    key = [seed % 2 ** 32, seed // 2 ** 32]
    mask32, half = u(0xFFFFFFFF), u(32)
    for r in range(10):
        a, c = word[0] * u(0xD2511F53), word[2] * u(0xCD9E8D57)
        word = [(c >> half) ^ word[1] ^ u(key[0]), c & mask32, (a >> half) ^ word[3] ^ u(key[1]), a & mask32]
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    bits = np.stack(word, 1).astype(np.uint32).view(np.uint16).reshape(rows, groups * 8)[:, :cols]      # low half first
    drop = int(rate * 65536.0 + 0.5)
    return torch.from_numpy(np.where(bits < drop, 0.0, 65536.0 / (65536.0 - drop))).cuda()


def _exact_rows(case, s):
    dt = TYPES[case["type"]]
    mask = _exact_mask(case["rows"], case["cols"], case["rate"], s["seed"], s["event"]) if case["rate"] > 0 else 1.0
    total = s["x"].double() * mask
    if s["residual"] is not None:
        total = total + s["residual"].double()
    if case["op"] == "dropout":
        return {"out": total, "dx": s["dy"].double() * mask} if case["form"] == "train" else {"out": total}
    w = s["weight"].double()

    def norm(t, weight):
        return t / (t.square().sum(1, keepdim=True) / case["cols"] + EPS).sqrt() * weight

    y = norm(total, w)
    if case["form"] == "8bit":
        codes, scales = torch.zeros_like(y), []
        for at in range(0, case["cols"], 128):
            block = y[:, at:at + 128]
            scales.append(block.abs().max(1).values / E4M3_MAX)
            codes[:, at:at + 128] = block / scales[-1].unsqueeze(1)
        return {"codes": codes, "scales": torch.stack(scales, 1), "total": total}
    if case["form"] == "forward":
        return {"y": y, "total": total}
    kept, weight = total.to(dt).double().requires_grad_(), w.clone().requires_grad_()
    through, dweight = torch.autograd.grad(norm(kept, weight), (kept, weight), s["dy"].double())
    dtotal = through + s["dtotal"].double()
    return {"y": y, "total": total, "dx": dtotal * mask, "dresidual": dtotal, "dweight": dweight}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] != "attention":
        return _exact_rows(case, s)
    train = case["form"] == "train"
    group, scale = case["heads"] // case["kv_heads"], 1.0 / math.sqrt(case["dim"])
    got = {"o": torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")}
    if train:
        got["lse"] = torch.full((case["batch"], case["heads"], case["queries"]), -math.inf, dtype=torch.float64, device="cuda")
        got |= {"d" + n: torch.zeros(s[n].shape, dtype=torch.float64, device="cuda") for n in "qkv"}
    for b in range(case["batch"]):
        nq = int(s["query_lengths"][b]) if s["query_lengths"] is not None else case["queries"]
        nk = int(s["key_lengths"][b]) if s["key_lengths"] is not None else case["keys"]
        if not nq or not nk:
            continue
        for h in range(case["kv_heads"]):
            heads = slice(h * group, (h + 1) * group)
            q = s["q"][b, :nq, heads].double().requires_grad_(train)
            k, v = (s[n][b, :nk, h].double().requires_grad_(train) for n in "kv")
            logits = torch.einsum("tgd,sd->gts", q, k) * scale
            o = torch.einsum("gts,sd->tgd", torch.softmax(logits, -1), v)
            got["o"][b, :nq, heads] = o.detach()
            if train:
                got["lse"][b, heads, :nq] = torch.logsumexp(logits, -1).detach()
                dq, dk, dv = torch.autograd.grad(o, (q, k, v), s["do"][b, :nq, heads].double())
                got["dq"][b, :nq, heads], got["dk"][b, :nk, h], got["dv"][b, :nk, h] = dq, dk, dv
    return got
