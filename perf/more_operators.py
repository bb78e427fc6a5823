"""Attention over packed sequences and over a paged cache, the rows that fill the cache, and the linear layer with its addends.

A program that serves decoder or encoder layers of its own with ``op_linear``, ``op_qk_norm_rope`` and ``op_attention`` has several
requests at once.  These cases are what it calls then: the linear layer with bias and residual (``linear``), attention of sequences
that lie behind one another, each within itself, with masks, capped scores and a bias by distance (``packed``), new keys and values
on their way into the pages of a cache (``store``), and the attention of the new tokens over those pages (``paged``).

``run`` computes an operator from elementary torch operations, or, where ``own`` is set, calls the package.
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda:0"
GOLDEN = 0.6180339887498949


def _attention(op, seqs, new, keys, hq, hkv, hd, spread=0.0, causal=True, prefix=0, window=0, cap=0.0, slopes=False, page=0):
    return {"op": op, "seqs": seqs, "new": new, "keys": keys, "hq": hq, "hkv": hkv, "hd": hd, "spread": spread, "causal": causal, "prefix": prefix,
            "window": window, "cap": cap, "slopes": slopes, "page": page}


def listed():
    return [
        # The attention's output projection of a 7B decoder for a single token, added to the stream: one pass over 34 MB of weights.
        {"name": "linear_token", "op": "linear", "m": 1, "n": 4096, "k": 4096, "act": 0, "bias": False, "residual": "bf16", "bf16": True},
        # A vision encoder's second MLP layer over three views and a ragged rest, onto an fp32 stream.
        {"name": "linear_vision", "op": "linear", "m": 817, "n": 1152, "k": 4304, "act": 0, "bias": True, "residual": "f32", "bf16": False},
        # A batch through an encoder's first MLP layer: bias, GELU, throughput.
        {"name": "linear_batch", "op": "linear", "m": 8192, "n": 8192, "k": 2048, "act": 1, "bias": True, "residual": "none", "bf16": True},
        # Sixty short documents of 12 to 120 tokens side by side, bias by distance: nothing is long, everything is ragged.
        {"name": "packed_short", **_attention("packed", 60, 120, 0, 16, 16, 64, spread=0.9, slopes=True)},
        # Eight views of 1024 patches in a vision encoder: each sees itself, both ways.
        {"name": "packed_views", **_attention("packed", 8, 1024, 0, 12, 12, 64, causal=False)},
        # Four requests of a policy's image prefix, text and action tokens: the prefix sees itself both ways, the rest is causal.
        {"name": "packed_prefix", **_attention("packed", 4, 867, 0, 8, 1, 256, spread=0.1, prefix=816)},
        # Two long documents, capped scores: throughput.
        {"name": "packed_long", **_attention("packed", 2, 8192, 0, 16, 8, 128, spread=0.5, cap=50.0)},
        # New rows of a decoding step into the pages.
        {"name": "store_step", "op": "store", "seqs": 64, "new": 1, "keys": 8192, "spread": 0.8, "hkv": 8, "hd": 128, "page": 64},
        # The rows of a batch of prefixes into the pages.
        {"name": "store_batch", "op": "store", "seqs": 16, "new": 512, "keys": 512, "spread": 0.0, "hkv": 8, "hd": 128, "page": 16},
        # One token of one sequence over what it has in the cache: latency.
        {"name": "paged_token", **_attention("paged", 1, 1, 1500, 32, 8, 128, page=16)},
        # A decoding step of 64 sequences of 1700 to 8192 keys: one pass over their caches.
        {"name": "paged_step", **_attention("paged", 64, 1, 8192, 32, 8, 128, spread=0.8, page=64)},
        # Chunks of 512 new tokens of four sequences over long caches, a window over the last 4096.
        {"name": "paged_chunk", **_attention("paged", 4, 512, 16384, 32, 8, 128, spread=0.5, window=4096, page=32)},
    ]


# ---------------------------------------------------------------- further cases of the same ranges
def _log_int(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


def draw(rng):
    op = rng.choice(["linear", "linear", "packed", "packed", "store", "paged", "paged"])
    if op == "linear":
        return {"op": op, "m": _log_int(rng, 1, 8192), "n": _log_int(rng, 7, 8192), "k": _log_int(rng, 16, 2048, 8), "act": rng.randrange(3), "bias": rng.random() < 0.7,
                "residual": rng.choice(["none", "bf16", "f32"]), "bf16": rng.random() < 0.7}
    hkv = rng.choice([1, 2, 5, 8])
    hd = rng.choice([32, 64, 72, 128, 256])
    spread = round(rng.uniform(0.0, 0.9), 2)
    if op == "store":
        seqs = _log_int(rng, 1, 64)
        new = _log_int(rng, 1, 512)
        return {"op": op, "seqs": seqs, "new": new, "keys": _log_int(rng, new, 8192), "spread": spread, "hkv": hkv, "hd": min(hd, 128), "page": rng.choice([8, 16, 64, 256])}
    hq = hkv * rng.choice([1, 2, 3, 4])
    cap, slopes, causal = rng.choice([0.0, 0.0, 30.0, 50.0]), rng.random() < 0.25, rng.random() < 0.75
    window = _log_int(rng, 16, 4096) if causal and rng.random() < 0.3 else 0
    if op == "packed":
        new = _log_int(rng, 1, 4096)
        return _attention(op, _log_int(rng, 1, max(1, min(64, 8192 // new))), new, 0, hq, hkv, hd, spread, causal, rng.choice([0, 0, new // 2]) if causal else 0, window, cap, slopes)
    seqs = _log_int(rng, 1, 64)
    new = rng.choice([1, 1, _log_int(rng, 1, max(1, 1024 // seqs))])
    return _attention(op, seqs, new, _log_int(rng, max(new, 16), 8192), hq, hkv, hd, spread, causal, 0, window, cap, slopes, rng.choice([8, 16, 32, 64, 256]))


def _lengths(c):
    """New tokens and keys of each sequence: the longest first, the others shorter by up to `spread` of it, no two alike."""
    share = [1.0 - c["spread"] * ((s * GOLDEN) % 1.0) for s in range(c["seqs"])]
    if c["op"] == "packed":
        new = [max(1, int(c["new"] * x)) for x in share]
        return new, new
    return [c["new"]] * c["seqs"], [max(c["new"], int(c["keys"] * x)) for x in share]


# ---------------------------------------------------------------- inputs
def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed) * 7919 + 13)
    normal = lambda *s, dtype=torch.float32: torch.randn(*s, device=DEVICE, generator=gen, dtype=dtype)  # noqa: E731
    bf16 = torch.bfloat16
    s = {"case": dict(case)}
    if case["op"] == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        s["a"], s["w"] = normal(m, k).to(bf16), (normal(n, k) / math.sqrt(k)).to(bf16)
        s["bias"] = 0.5 * normal(n) if case["bias"] else None
        s["residual"] = None if case["residual"] == "none" else (2.0 * normal(m, n)).to(bf16 if case["residual"] == "bf16" else torch.float32)
        return s
    new, keys = _lengths(case)
    starts = lambda v: torch.tensor([sum(v[:i]) for i in range(len(v) + 1)], dtype=torch.int32, device=DEVICE)  # noqa: E731
    t, hkv, hd = sum(new), case["hkv"], case["hd"]
    s["offsets"], s["most_new"], s["most_keys"] = starts(new), max(new), max(keys)
    if case["op"] in ("packed", "paged"):
        hq = case["hq"]
        s["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)], device=DEVICE) if case["slopes"] else None
        s["prefix"] = torch.tensor([max(0, min(case["prefix"], x - 51)) if case["prefix"] else 0 for x in keys], dtype=torch.int32, device=DEVICE) if case["prefix"] else None
    if case["op"] == "packed":
        rows = normal(t, (hq + 2 * hkv) * hd, dtype=bf16)                    # the stacked projection: queries, keys, values
        rows[:, :hq * hd] *= 1.5
        s["q"], s["k"], s["v"] = rows[:, :hq * hd], rows[:, hq * hd:(hq + hkv) * hd], rows[:, (hq + hkv) * hd:]
        return s
    page = case["page"]
    need = [-(-x // page) for x in keys]
    pool = sum(need) + 7                                                     # (a few pages belong to nobody)
    order = torch.randperm(pool, generator=torch.Generator().manual_seed(int(seed) * 31 + 7)).to(torch.int32)
    table, at = torch.full((case["seqs"], max(need)), -1, dtype=torch.int32), 0
    for i, x in enumerate(need):
        table[i, :x] = order[at:at + x]
        at += x
    s["pages"], s["lengths"] = table.to(DEVICE), torch.tensor(keys, dtype=torch.int32, device=DEVICE)
    s["k_cache"], s["v_cache"] = normal(pool, page, hkv * hd, dtype=bf16), normal(pool, page, hkv * hd, dtype=bf16)
    if case["op"] == "store":
        rows = normal(t, 2 * hkv * hd, dtype=bf16)
        s["k"], s["v"] = rows[:, :hkv * hd], rows[:, hkv * hd:]
    else:
        s["q"] = (1.5 * normal(t, hq * hd)).to(bf16)
    return s


# ---------------------------------------------------------------- one pass
def _act(y, act):
    if act == 1:
        return 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y * y * y)))
    if act == 2:
        return y / (1.0 + torch.exp(-y))
    return y


def _places(starts, most, total):
    """Rows of each sequence as [seqs, most], and which of them there are."""
    lo, hi = starts[:-1].long(), starts[1:].long()
    at = lo[:, None] + torch.arange(most, device=lo.device)
    return at.clamp(max=max(total - 1, 0)), at < hi[:, None]


def _attend(s, q, k, v, rows, live, have):
    """Attention of padded sequences: q [seqs, new, hq, hd], k and v [seqs, keys, hkv, hd] in fp32, live rows, `have` keys each; the `rows` live ones back."""
    c = s["case"]
    n, new, hq, hd = q.shape
    most, hkv = k.shape[1], c["hkv"]
    there = torch.arange(most, device=q.device)[None] < have[:, None]                                  # [seqs, keys]
    v = torch.where(there[:, :, None, None], v, torch.zeros((), device=q.device))
    qg = q.permute(0, 2, 1, 3).reshape(n, hkv, hq // hkv * new, hd)
    score = (qg @ k.permute(0, 2, 3, 1)).view(n, hq, new, most) / math.sqrt(hd)
    if c["cap"]:
        score = c["cap"] * torch.tanh(score / c["cap"])
    count = live.sum(1)
    pos = (have - count)[:, None] + torch.arange(new, device=q.device)                                 # [seqs, new]
    far = pos[:, :, None] - torch.arange(most, device=q.device)                                        # [seqs, new, keys]
    if s["slopes"] is not None:
        score = score - s["slopes"][None, :, None, None] * far[:, None].abs().float()
    seen = there[:, None].expand(n, new, most)
    if c["causal"]:
        near = far >= 0
        if c["window"]:
            near = near & (far < c["window"])
        if s["prefix"] is not None:
            near = near | (torch.arange(most, device=q.device) < s["prefix"][:, None])[:, None]
        seen = seen & near
    score = torch.where(seen[:, None], score, torch.full((), -math.inf, device=q.device))
    top = score.amax(-1, keepdim=True).clamp(min=-1e30)
    p = torch.exp(score - top)
    p = p / p.sum(-1, keepdim=True).clamp(min=1e-30)
    y = (p.view(n, hkv, hq // hkv * new, most) @ v.permute(0, 2, 1, 3)).view(n, hq, new, hd).permute(0, 2, 1, 3).reshape(n * new, hq * hd)
    row = torch.arange(rows, device=q.device)
    seq = torch.searchsorted(s["offsets"][1:].long(), row, right=True)
    return y[seq * new + row - s["offsets"][seq].long()].to(torch.bfloat16)


def run(state):
    s, c = state, state["case"]
    op = c["op"]
    if own:
        from paper_2609_22335_b200 import api
        if op == "linear":
            return api.op_linear_bias(s["a"], s["w"], bias=s["bias"], residual=s["residual"], act=c["act"], out_bf16=c["bf16"])
        if op == "store":
            api.op_cache_store(s["k"], s["v"], s["k_cache"], s["v_cache"], s["pages"], s["lengths"], s["offsets"])
            return s["k_cache"], s["v_cache"]
        more = {"causal": c["causal"], "prefix": s["prefix"], "window": c["window"], "cap": c["cap"], "slopes": s["slopes"]}
        if op == "packed":
            return api.op_attention_packed(s["q"], s["k"], s["v"], s["offsets"], c["hq"], c["hkv"], c["hd"], **more)
        return api.op_attention_paged(s["q"], s["k_cache"], s["v_cache"], s["pages"], s["lengths"], s["offsets"], c["hq"], c["hkv"], c["hd"], **more)
    if op == "linear":
        y = s["a"].float() @ s["w"].float().T
        if s["bias"] is not None:
            y = y + s["bias"]
        y = _act(y, c["act"])
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return y.to(torch.bfloat16) if c["bf16"] else y
    hkv, hd = c["hkv"], c["hd"]
    if op == "store":
        t, page = s["k"].shape[0], c["page"]
        row = torch.arange(t, device=s["k"].device)
        seq = torch.searchsorted(s["offsets"][1:].long(), row, right=True)
        pos = s["lengths"][seq].long() - s["offsets"][seq + 1].long() + row
        at = s["pages"][seq, pos // page].long(), pos % page
        s["k_cache"][at], s["v_cache"][at] = s["k"], s["v"]
        return s["k_cache"], s["v_cache"]
    t, hq = s["q"].shape[0], c["hq"]
    at, live = _places(s["offsets"], s["most_new"], t)
    q = s["q"].float()[at].view(*at.shape, hq, hd)
    if op == "packed":
        k, v = (s[x].float()[at].view(*at.shape, hkv, hd) for x in ("k", "v"))
        return _attend(s, q, k, v, t, live, live.sum(1))
    pos = torch.arange(s["most_keys"], device=q.device)
    page = s["pages"].long()[:, pos // c["page"]].clamp(min=0)
    k, v = (s[x][page, pos % c["page"]].float().view(c["seqs"], -1, hkv, hd) for x in ("k_cache", "v_cache"))
    return _attend(s, q, k, v, t, live, s["lengths"].long())


# ---------------------------------------------------------------- what a pass cannot do without
def _pairs(c, new, keys):
    """Visible (row, key) pairs of a sequence."""
    if not c["causal"]:
        return new * keys
    prefix, window = (max(0, min(c["prefix"], keys - 51)) if c["prefix"] else 0), c["window"] or keys
    total = 0
    for i in range(new):
        p = keys - new + i
        lo = max(0, p - window + 1)
        total += p + 1 - lo + (prefix - (p + 1) + lo if prefix > p + 1 else min(prefix, lo))
    return total


def _keys_seen(c, new, keys):
    """Keys of a sequence that any of its rows sees."""
    if not c["causal"] or not c["window"]:
        return keys
    return min(keys, new + c["window"] - 1 + (c["prefix"] or 0))


def work(case):
    op = case["op"]
    if op == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        residual = {"none": 0, "bf16": 2, "f32": 4}[case["residual"]]
        return {"bytes": 2 * (m * k + n * k) + (4 * n if case["bias"] else 0) + m * n * (residual + (2 if case["bf16"] else 4)), "flops": 2 * m * n * k}
    new, keys = _lengths(case)
    t, row = sum(new), 2 * case["hkv"] * case["hd"]
    if op == "store":
        return {"bytes": 4 * t * row + 4 * (3 * case["seqs"]) + 4 * sum(-(-n // case["page"]) for n in new), "flops": 0}
    seen = sum(_keys_seen(case, n, k) for n, k in zip(new, keys))
    extra = 4 * (case["seqs"] + 1) + (4 * case["seqs"] + 4 * seen // case["page"] if op == "paged" else 0)
    return {"bytes": 4 * t * case["hq"] * case["hd"] + 2 * seen * row + extra, "flops": 4 * case["hq"] * case["hd"] * sum(_pairs(case, n, k) for n, k in zip(new, keys))}


# ---------------------------------------------------------------- the definitions, in 64 bits
def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "linear":
        y = s["a"].double() @ s["w"].double().T + (0.0 if s["bias"] is None else s["bias"].double())
        if case["act"] == 1:
            y = y * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3))
        elif case["act"] == 2:
            y = y * torch.sigmoid(y)
        return y if s["residual"] is None else y + s["residual"].double()
    new, keys = _lengths(case)
    hkv, hd, first = case["hkv"], case["hd"], 0
    if op == "store":
        for i, (n, have) in enumerate(zip(new, keys)):
            for j in range(n):
                p = have - n + j
                at = int(s["pages"][i, p // case["page"]]), p % case["page"]
                s["k_cache"][at], s["v_cache"][at] = s["k"][first + j], s["v"][first + j]
            first += n
        return s["k_cache"].double(), s["v_cache"].double()
    hq, out = case["hq"], []
    prefixes = None if s["prefix"] is None else s["prefix"].tolist()
    for i, (n, have) in enumerate(zip(new, keys)):
        if op == "packed":
            k, v = s["k"][first:first + n], s["v"][first:first + n]
        else:
            pages = s["pages"][i, :-(-have // case["page"])].long()
            k, v = (s[x][pages].reshape(-1, hkv * hd)[:have] for x in ("k_cache", "v_cache"))
        far = (have - n + torch.arange(n, device=DEVICE, dtype=torch.float64))[:, None] - torch.arange(have, device=DEVICE, dtype=torch.float64)
        hidden = torch.zeros(n, have, dtype=torch.bool, device=DEVICE)
        if case["causal"]:
            hidden = far < 0
            if case["window"]:
                hidden |= far >= case["window"]
            if prefixes is not None:
                hidden[:, :prefixes[i]] = False
        heads = []
        for h in range(hq):
            of = slice(h // (hq // hkv) * hd, (h // (hq // hkv) + 1) * hd)
            score = s["q"][first:first + n, h * hd:(h + 1) * hd].double() @ k[:, of].double().T * hd ** -0.5
            if case["cap"]:
                score = case["cap"] * torch.tanh(score / case["cap"])
            if s["slopes"] is not None:
                score -= s["slopes"][h].double() * far.abs()
            heads.append(torch.softmax(score.masked_fill_(hidden, -math.inf), -1) @ v[:, of].double())
        out.append(torch.cat(heads, 1))
        first += n
    return torch.cat(out)
