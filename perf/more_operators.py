"""The operators with which a decoder answers, at sizes of real use: their cases, their inputs, their plain forms and
their definitions in 64 bits.

  append      new keys and values into a paged cache, the rotation by their position applied on the way, queries too
  attention   attention of a step's new tokens over that cache, whole or through a window beside the first tokens
  log_probs   log probabilities of given tokens, with entropy and the likeliest tokens; their gradient

`run` computes them with elementary tensor operations in 32 bits where `own` is false, and through the package's
calls where it is true. A "train" case is the forward and the backward pass of a training step.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SHORTEST = 8                    # ragged caches hold between an eighth of the longest and the longest


def _append(name, batch, heads, kv_heads, tokens, cached, dim, rotated, interleaved, page, kind, ragged, layout):
    return {"name": name, "op": "append", "batch": batch, "heads": heads, "kv_heads": kv_heads, "tokens": tokens,
            "cached": cached, "dim": dim, "rotated": rotated, "interleaved": interleaved, "page": page, "type": kind,
            "ragged": ragged, "layout": layout}


def _attention(name, batch, heads, kv_heads, tokens, keys, dim, window, sinks, page, kind, ragged, layout):
    return {"name": name, "op": "attention", "batch": batch, "heads": heads, "kv_heads": kv_heads, "tokens": tokens,
            "keys": keys, "dim": dim, "window": window, "sinks": sinks, "page": page, "type": kind, "ragged": ragged,
            "layout": layout}


def _log_probs(name, rows, vocabulary, kind, top, entropy, scale, masked, form):
    return {"name": name, "op": "log_probs", "rows": rows, "vocabulary": vocabulary, "type": kind, "top": top,
            "entropy": entropy, "scale": scale, "masked": masked, "form": form}


def listed():
    return [
        # one new token for each of 4 sentences: the smallest call of a decoding loop
        _append("append token small", 4, 8, 8, 1, 77, 64, 64, False, 16, "bf16", False, "tokens"),
        # drafts of up to 5 tokens for 96 sentences, half of each head rotated in neighbouring pairs, odd pages kept head by head
        _append("append drafts odd", 96, 12, 4, 5, 250, 80, 40, True, 24, "f16", True, "heads"),
        # the prompts of a batch at once, four query heads to each key head
        _append("append prompts", 16, 32, 8, 1024, 0, 128, 128, False, 64, "bf16", True, "tokens"),
        # one new token for each of 4 sentences over a short cache
        _attention("attention token small", 4, 8, 8, 1, 77, 64, 0, 0, 16, "bf16", False, "tokens"),
        # a decoding batch of 128 sentences of very unequal lengths, a key head for each query head
        _attention("attention token batch", 128, 16, 16, 1, 1024, 64, 0, 0, 16, "bf16", True, "tokens"),
        # few long documents, four query heads to each key head, pages kept head by head
        _attention("attention token long", 8, 32, 8, 1, 16384, 128, 0, 0, 64, "f16", False, "heads"),
        # a single document of an odd length, one key head for all
        _attention("attention token alone", 1, 8, 1, 1, 100001, 128, 0, 0, 32, "bf16", False, "tokens"),
        # drafts of four tokens checked at once, each seeing the last 1024 tokens and the first four
        _attention("attention drafts window", 64, 32, 8, 4, 4096, 128, 1024, 4, 32, "bf16", True, "tokens"),
        # one step of a beam over 8 sentences: the likeliest tokens of each
        _log_probs("log_probs step small", 8, 32000, "bf16", 4, False, 1.0, False, "forward"),
        # a decoding batch with a large vocabulary, a quarter of it ruled out, sampled at a temperature of 0.8
        _log_probs("log_probs step batch", 128, 131072, "bf16", 20, True, 1.25, True, "forward"),
        # a small training batch in fp32 over an odd vocabulary, with an entropy term
        _log_probs("log_probs train odd f32", 1500, 10007, "f32", 0, True, 1.0, False, "train"),
        # the loss of a training batch of 8192 target tokens, padded places among them
        _log_probs("log_probs train batch", 8192, 32000, "bf16", 0, False, 1.0, False, "train"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attention", "attention", "log_probs", "log_probs"])
    if op == "log_probs":
        form = rng.choice(["forward", "train"])
        vocabulary = _log(rng, 33, 200000)
        rows = _log(rng, 1, max(2, min(16384, 250 * 10 ** 6 // vocabulary // (2 if form == "forward" else 1))))
        kind = rng.choice(["bf16", "bf16", "f16", "f32"])
        if kind == "f32":
            rows = max(1, rows // 2)
        top = 0 if form == "train" else min(vocabulary, rng.choice([0, 1, 2, 5, 8, 20, 32]))
        if top:                                # the plain form sorts
            rows = max(1, min(rows, 2 ** 24 // vocabulary))
        c = _log_probs("", rows, vocabulary, kind, top, rng.random() < 0.5, rng.choice([1.0, 1.0, 1.25, 0.5]),
                       rng.random() < 0.3, form)
        del c["name"]
        return c
    kind, dim = rng.choice(["bf16", "bf16", "f16"]), rng.choice([32, 40, 64, 64, 80, 96, 128, 128])
    kv_heads, group = rng.choice([1, 2, 4, 6, 8, 16]), rng.choice([1, 1, 2, 3, 4, 8])
    heads, page = kv_heads * group, rng.choice([8, 16, 16, 24, 32, 64, 100, 128])
    ragged, layout = rng.random() < 0.5, rng.choice(["tokens", "heads"])
    if op == "append":
        tokens = rng.choice([1, 1, _log(rng, 2, 2048)])
        cached = _log(rng, 1, 2048) if rng.random() < 0.7 else 0
        new, held = 2 ** 26 // ((heads + 2 * kv_heads) * dim * tokens), 2 ** 26 // ((tokens + cached) * kv_heads * dim)
        batch = _log(rng, 1, max(1, min(256, new, held)))
        rotated = rng.choice([dim, dim, dim // 2, 0])
        c = _append("", batch, heads, kv_heads, tokens, cached, dim, rotated, rng.random() < 0.5, page, kind, ragged, layout)
    else:
        tokens = rng.choice([1, 1, 1, 2, 4, 8])
        keys = max(tokens, _log(rng, 1, 100000))
        while keys * kv_heads * dim > 2 ** 26:
            keys //= 2
        batch = _log(rng, 1, max(1, min(256, 2 ** 26 // (keys * kv_heads * dim))))
        window, sinks = (_log(rng, 1, max(2, keys)), rng.choice([0, 1, 4, 20])) if rng.random() < 0.3 else (0, 0)
        c = _attention("", batch, heads, kv_heads, tokens, keys, dim, window, sinks, page, kind, ragged, layout)
    del c["name"]
    return c


# ---- inputs --------------------------------------------------------------------------------------------------------


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = TYPES[case["type"]]

    def normal(*shape, std=1.0, dtype=dt):
        return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)

    s = {"case": case}
    if case["op"] == "log_probs":
        rows, vocabulary = case["rows"], case["vocabulary"]
        # scores of a trained model: most tokens far below the few that the place allows
        s["logits"] = normal(rows, vocabulary, std=2.5)
        s["logits"][torch.arange(rows, device="cuda"), torch.randint(vocabulary, (rows,), generator=g, device="cuda")] += 9.0
        s["tokens"] = torch.randint(vocabulary, (rows,), generator=g, device="cuda")
        if case["masked"]:                     # what a grammar or a word list rules out; the given tokens stay
            out = torch.rand(rows, vocabulary, generator=g, device="cuda") < 0.25
            out[torch.arange(rows, device="cuda"), s["tokens"]] = False
            s["logits"][out] = -math.inf
        if case["form"] == "train":
            s["tokens"][torch.rand(rows, generator=g, device="cuda") < 0.125] = -1         # padded places
            s["dlog_probs"] = normal(rows, dtype=torch.float32)
            s["dentropy"] = normal(rows, std=0.1, dtype=torch.float32) if case["entropy"] else None
        return s
    b, h, hk, t, d, page = (case[k] for k in ("batch", "heads", "kv_heads", "tokens", "dim", "page"))
    most = case["keys"] if case["op"] == "attention" else case["cached"] + t
    columns = -(-most // page) + 1             # the table has room for another page
    pages = b * columns + 1                    # the last page is in nobody's table, and holds zeros

    def cache():
        if case["layout"] == "tokens":
            x = normal(pages, page, hk, d)
        else:
            x = normal(pages, hk, page, d).transpose(1, 2)
        x[pages - 1] = 0
        return x

    def between(lo, hi):
        n = torch.randint(lo, hi + 1, (b,), generator=g, device="cuda", dtype=torch.int32)
        n[0] = hi
        return n

    s["k_pages"], s["v_pages"] = cache(), cache()
    if case["op"] == "append":
        s["counts"] = between(t - t // 2, t) if case["ragged"] else None
        s["lengths"] = between(-(-case["cached"] // SHORTEST), case["cached"]) if case["ragged"] else torch.full(
            (b,), case["cached"], dtype=torch.int32, device="cuda")
        s["lengths"] += s["counts"] if case["ragged"] else t
        s["q"], s["k"] = normal(b, t, h, d, std=1.5), normal(b, t, hk, d)
        s["v"] = normal(b, t, hk, d)
        half = case["rotated"] // 2
        s["frequencies"] = None
        if half:
            s["frequencies"] = (10000.0 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)).float()
    else:
        s["counts"] = None
        s["lengths"] = between(max(t, most // SHORTEST), most) if case["ragged"] else torch.full(
            (b,), most, dtype=torch.int32, device="cuda")
        s["q"] = normal(b, t, h, d, std=1.5)
    if case["ragged"] and b > 4:
        s["lengths"][b // 2] = 0               # a place of the batch without a sentence
    table = torch.randperm(pages - 1, generator=g, device="cuda").to(torch.int32).view(b, columns)
    used = torch.arange(columns, device="cuda") * page < s["lengths"].unsqueeze(1)
    s["table"] = torch.where(used, table, -1)  # pages are handed out as they are needed
    return s


def _visible(keys, case):
    """Tokens that one of the new ones sees in a cache of `keys`."""
    if not case["window"]:
        return keys
    return min(keys, min(keys, case["window"] + case["tokens"] - 1) + case["sinks"])


def work(case):
    size = 4 if case["type"] == "f32" else 2
    if case["op"] == "log_probs":
        n, rows = case["rows"] * case["vocabulary"], case["rows"]
        if case["form"] == "train":            # the rows are read for their sums, then once more for their gradient
            return {"bytes": 3 * n * size + rows * 40, "flops": 10 * n}
        return {"bytes": n * size + rows * (24 + 12 * case["top"]), "flops": 5 * n}
    b, h, hk, t, d = (case[k] for k in ("batch", "heads", "kv_heads", "tokens", "dim"))
    if case["op"] == "append":
        share = 0.75 if case["ragged"] and t > 1 else 1.0
        new = b * t * (h + 2 * hk) * d * share
        return {"bytes": 2 * new * size + b * 12, "flops": 3 * b * t * (h + hk) * case["rotated"] * share}
    longest = case["keys"]
    if case["ragged"]:                         # lengths are spread evenly
        some = [longest * (1 / SHORTEST + (1 - 1 / SHORTEST) * (i + 0.5) / 16) for i in range(16)]
        seen = sum(_visible(n, case) for n in some) / 16
    else:
        seen = _visible(longest, case)
    return {"bytes": 2 * b * hk * d * seen * size + 2 * b * t * h * d * size + 4 * b * seen / case["page"],
            "flops": 4 * b * h * t * d * seen}


# ---- plain forms ---------------------------------------------------------------------------------------------------


def _plain_rotate(x, cos, sin, case):
    r = case["rotated"]
    x = x.float()
    if not r:
        return x
    cos, sin = cos.unsqueeze(2), sin.unsqueeze(2)
    if case["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, x[..., r:]], -1)


def _plain_append_pass(s, case, dt):
    b, t, page = case["batch"], case["tokens"], case["page"]
    new = s["counts"] if s["counts"] is not None else torch.full_like(s["lengths"], t)
    new = torch.minimum(new, s["lengths"])
    place = torch.arange(t, device="cuda")
    live = place < new.unsqueeze(1)
    position = (s["lengths"] - new).unsqueeze(1) + place
    cos = sin = None
    if s["frequencies"] is not None:           # a float's place on a circle far from 0 needs more than a float
        angle = position.double().unsqueeze(2) * s["frequencies"].double()
        cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    q, k = (_plain_rotate(s[n], cos, sin, case) for n in "qk")
    keep = live.view(b, t, 1, 1)
    zero = torch.zeros((), device="cuda")
    column = torch.div(position, page, rounding_mode="floor").clamp(max=s["table"].shape[1] - 1)
    number = torch.gather(s["table"].long(), 1, column.long())
    number = torch.where(live, number, s["k_pages"].shape[0] - 1)                      # zeros onto the page of zeros
    slot = torch.where(live, position % page, 0).long()
    s["k_pages"][number, slot] = torch.where(keep, k, zero).to(dt)
    s["v_pages"][number, slot] = torch.where(keep, s["v"].float(), zero).to(dt)
    return {"q": torch.where(keep, q, zero).to(dt), "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _plain_attention_pass(s, case, dt):
    b, h, hk, t, d, page = (case[k] for k in ("batch", "heads", "kv_heads", "tokens", "dim", "page"))
    group, columns = h // hk, -(-case["keys"] // page)
    number = s["table"][:, :columns].clamp(min=0).long()
    k, v = (s[n][number].float().reshape(b, columns * page, hk, d).transpose(1, 2) for n in ("k_pages", "v_pages"))
    q = s["q"].float().view(b, t, hk, group, d).permute(0, 2, 1, 3, 4).reshape(b, hk, t * group, d)
    scores = torch.matmul(q, k.transpose(2, 3)) * d ** -0.5
    key = torch.arange(columns * page, device="cuda").view(1, 1, -1)
    own_place = (s["lengths"].view(b, 1, 1) - t + torch.arange(t, device="cuda").view(1, t, 1))
    seen = key <= own_place
    if case["window"]:
        seen = seen & ((key > own_place - case["window"]) | (key < case["sinks"]))
    seen = seen.repeat_interleave(group, 1).unsqueeze(1)
    scores = scores.masked_fill(~seen, -math.inf)
    top = scores.amax(3, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = torch.exp(scores - top)
    total = p.sum(3, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total > 0, total, torch.ones_like(total))
    return {"o": o.view(b, hk, t, group, d).permute(0, 2, 1, 3, 4).reshape(b, t, h, d).to(dt)}


def _plain_log_probs_pass(s, case, dt):
    x, given = s["logits"].float(), s["tokens"]
    held = given >= 0
    top = x.amax(1, keepdim=True)
    d = (x - top) * case["scale"]
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    log_total = torch.log(total)
    out = {"log_probs": torch.where(held, (d.gather(1, given.clamp(min=0).unsqueeze(1)) - log_total).squeeze(1), 0.0),
           "stats": torch.cat([top, log_total], 1)}
    entropy = None
    if case["entropy"]:
        entropy = log_total - torch.where(e > 0, e * d, torch.zeros_like(d)).sum(1, keepdim=True) / total
        out["entropy"] = entropy.squeeze(1)
    if case["top"]:                            # ties go to the lowest index
        order = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :case["top"]]
        out["top_tokens"], out["top_log_probs"] = order, d.gather(1, order) - log_total
    if case["form"] == "train":
        share = e / total
        given_share = torch.where(held, s["dlog_probs"], torch.zeros_like(s["dlog_probs"])).unsqueeze(1)
        dx = -given_share * share
        dx.scatter_add_(1, given.clamp(min=0).unsqueeze(1), given_share)
        if entropy is not None:
            dx = dx - s["dentropy"].unsqueeze(1) * torch.where(e > 0, share * (d - log_total + entropy), torch.zeros_like(d))
        out["dlogits"] = (dx * case["scale"]).to(dt)
    return out


# ---- the package's calls -------------------------------------------------------------------------------------------


def _own_pass(s, case):
    from paper_1910_12308_b200 import operators as ops
    if case["op"] == "append":
        q = ops.append_to_cache(s["k"], s["v"], s["k_pages"], s["v_pages"], s["table"], s["lengths"], counts=s["counts"],
                                q=s["q"], frequencies=s["frequencies"], interleaved=case["interleaved"])
        return {"q": q, "k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    if case["op"] == "attention":
        return {"o": ops.paged_attention(s["q"], s["k_pages"], s["v_pages"], s["table"], s["lengths"], counts=s["counts"],
                                         window=case["window"], sinks=case["sinks"])}
    got = ops.token_log_probs(s["logits"], s["tokens"], scale=case["scale"], top=case["top"], entropy=case["entropy"])
    out = {n: x for n, x in got._asdict().items() if x is not None}
    if case["form"] == "train":
        out["dlogits"] = ops.token_log_probs_backward(s["dlog_probs"], s["logits"], s["tokens"], got.stats,
                                                      entropy=got.entropy, dentropy=s["dentropy"], scale=case["scale"])
    return out


def run(s):
    case = s["case"]
    if own:
        return _own_pass(s, case)
    dt = TYPES[case["type"]]
    return {"append": _plain_append_pass, "attention": _plain_attention_pass, "log_probs": _plain_log_probs_pass}[case["op"]](s, case, dt)


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------


def _exact_append(case, s):
    got = {"q": torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda"),
           "k_pages": s["k_pages"].double(), "v_pages": s["v_pages"].double()}
    half, page = case["rotated"] // 2, case["page"]
    for b in range(case["batch"]):
        length = int(s["lengths"][b])
        n = min(length, case["tokens"] if s["counts"] is None else int(s["counts"][b]))
        if not n:
            continue
        at = torch.arange(length - n, length, device="cuda")
        number, slot = s["table"][b][at // page].long(), at % page

        def turn(x):
            x = x.double()
            if not half:
                return x
            spin = torch.polar(torch.ones(n, half, dtype=torch.float64, device="cuda"),
                               at.double().unsqueeze(1) * s["frequencies"].double()).unsqueeze(1)
            first, second = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if case["interleaved"] else (x[..., :half], x[..., half:2 * half])
            z = torch.complex(first.contiguous(), second.contiguous()) * spin
            x = x.clone()
            if case["interleaved"]:
                x[..., 0:2 * half:2], x[..., 1:2 * half:2] = z.real, z.imag
            else:
                x[..., :half], x[..., half:2 * half] = z.real, z.imag
            return x

        got["q"][b, :n] = turn(s["q"][b, :n])
        got["k_pages"][number, slot] = turn(s["k"][b, :n])
        got["v_pages"][number, slot] = s["v"][b, :n].double()
    return got


def _exact_attention(case, s):
    group, t, page = case["heads"] // case["kv_heads"], case["tokens"], case["page"]
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for b in range(case["batch"]):
        length = int(s["lengths"][b])
        if not length:
            continue
        at = torch.arange(length, device="cuda")
        number = s["table"][b][at // page].long()
        k, v = (s[n][number, at % page].double() for n in ("k_pages", "v_pages"))
        for i in range(t):
            here = length - t + i
            if here < 0:
                continue
            first = here - case["window"] + 1 if case["window"] else 0
            seen = (at <= here) & ((at >= first) | (at < case["sinks"]))
            q = s["q"][b, i].double().view(case["kv_heads"], group, -1)
            w = torch.softmax((torch.einsum("hgd,shd->hgs", q, k) / math.sqrt(case["dim"])).masked_fill(~seen, -math.inf), -1)
            o[b, i] = torch.einsum("hgs,shd->hgd", w, v).flatten(0, 1)
    return {"o": o}


def _exact_log_probs(case, s):
    names = ["log_probs", "stats"] + ["entropy"] * case["entropy"] + ["top_tokens", "top_log_probs"] * (case["top"] > 0)
    train = case["form"] == "train"
    got = {n: [] for n in names + ["dlogits"] * train}
    step = max(1, 2 ** 26 // case["vocabulary"])
    for at in range(0, case["rows"], step):
        raw, given = s["logits"][at:at + step].double(), s["tokens"][at:at + step]
        some = (given >= 0).double()
        x = raw * case["scale"]
        lse = torch.logsumexp(x, 1)
        logp = x - lse.unsqueeze(1)
        p = torch.exp(logp)
        here = torch.zeros_like(x)
        here[torch.arange(len(x), device="cuda"), given.clamp(min=0)] = some
        finite = torch.nan_to_num(logp, neginf=0.0)                # weighs nothing where p = 0
        got["log_probs"].append((finite * here).sum(1))
        most = raw.max(1).values
        got["stats"].append(torch.stack([most, lse - most * case["scale"]], 1))
        entropy = -(p * finite).sum(1)
        if case["entropy"]:
            got["entropy"].append(entropy)
        if case["top"]:
            order = torch.sort(raw, dim=1, descending=True, stable=True).indices[:, :case["top"]]
            got["top_tokens"].append(order)
            got["top_log_probs"].append(logp.gather(1, order))
        if train:
            dx = (s["dlog_probs"][at:at + step].double() * some).unsqueeze(1) * (here - p)
            if case["entropy"]:
                dx -= s["dentropy"][at:at + step].double().unsqueeze(1) * p * (finite + entropy.unsqueeze(1))
            got["dlogits"].append(dx * case["scale"])
    return {n: torch.cat(parts) for n, parts in got.items()}


def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attention": _exact_attention, "log_probs": _exact_log_probs}[case["op"]](case, s)
