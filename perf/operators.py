"""The operators around the linear layer and the attention: 8-bit products with block scales, products grouped by expert, and
the norm and rotation of queries and keys.

A program that calls ``op_linear`` and ``op_attention`` on its own tensors runs decoder layers with them.  These cases are
what such a layer needs beside the two: activations and weights brought to 8 bits with a scale for each block of 128
(``quantize``), the product of two such matrices (``scaled``), products whose rows are sorted by expert, in bf16
(``grouped``) and in 8 bits (``grouped_scaled``), and the heads' RMS norm with the rotation by position between the
projection and the attention (``qk``).

``run`` computes an operator from elementary torch operations, or, where ``own`` is set, calls the package.
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda:0"
BLOCK = 128            # elements of K that share a scale
E4M3_MAX = 448.0
LEAST_SCALE = 2.0 ** -126


def listed():
    return [
        # One token's activations on their way into an 8-bit layer of a 7B decoder: a launch and a few KB.
        {"name": "quantize_token", "op": "quantize", "m": 1, "k": 4096, "rows": 1, "f32": False},
        # The activations of a batch of prefixes.
        {"name": "quantize_batch", "op": "quantize", "m": 8192, "k": 4096, "rows": 1, "f32": False},
        # The 7B decoder's gate projection for a single token: one pass over 45 MB of weights.
        {"name": "scaled_token", "op": "scaled", "m": 1, "n": 11008, "k": 4096, "act": 0, "bf16": True},
        # The same layer over one prefix, SiLU, fp32 result.
        {"name": "scaled_prefix", "op": "scaled", "m": 288, "n": 11008, "k": 4096, "act": 2, "bf16": False},
        # A vision encoder's MLP over three views and a ragged rest: no size is a multiple of a tile.
        {"name": "scaled_vision", "op": "scaled", "m": 817, "n": 4304, "k": 1152, "act": 1, "bf16": True},
        # A batch of prefixes through a decoder's MLP: throughput.
        {"name": "scaled_batch", "op": "scaled", "m": 8192, "n": 8192, "k": 2048, "act": 0, "bf16": True},
        # Eight rows (four tokens, two experts each) over sixteen experts: most experts idle, the rest have a row or two.
        {"name": "grouped_token", "op": "grouped", "t": 8, "g": 16, "n": 2048, "k": 2048, "skew": 0.5, "act": 0, "bf16": True},
        # A batch over eight experts, the busiest with several times the rows of the least busy one, fp32 result.
        {"name": "grouped_batch", "op": "grouped", "t": 8192, "g": 8, "n": 4096, "k": 2048, "skew": 1.0, "act": 0, "bf16": False},
        # 8-bit experts at decode: fifty tokens' rows over sixty-four experts.
        {"name": "grouped_scaled_step", "op": "grouped_scaled", "t": 100, "g": 64, "n": 2048, "k": 1024, "skew": 0.5, "act": 2, "bf16": True},
        # 8-bit experts over a batch, every expert with a ragged count.
        {"name": "grouped_scaled_batch", "op": "grouped_scaled", "t": 16384, "g": 32, "n": 4096, "k": 2048, "skew": 0.5, "act": 0, "bf16": True},
        # One decoded token far into its sequence: 16 query heads, 8 key heads.
        {"name": "qk_token", "op": "qk", "t": 1, "hq": 16, "hkv": 8, "hd": 128, "rot": 128, "interleaved": False, "f32": False, "pos0": 100000},
        # A batch of prefixes, read out of the stacked projection's rows.
        {"name": "qk_batch", "op": "qk", "t": 8192, "hq": 16, "hkv": 8, "hd": 128, "rot": 128, "interleaved": False, "f32": False, "pos0": 0},
    ]


# ---------------------------------------------------------------- further cases of the same ranges
def _log_int(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


def draw(rng):
    op = rng.choice(["quantize", "scaled", "scaled", "grouped", "grouped_scaled", "qk"])
    if op == "quantize":
        return {"op": op, "m": _log_int(rng, 1, 8192), "k": _log_int(rng, 16, 4096, 16), "rows": rng.choice([1, 1, BLOCK]), "f32": rng.random() < 0.3}
    if op == "scaled":
        return {"op": op, "m": _log_int(rng, 1, 8192), "n": _log_int(rng, 7, 8192), "k": _log_int(rng, 16, 2048, 16), "act": rng.randrange(3), "bf16": rng.random() < 0.7}
    if op == "qk":
        hd = rng.choice([16, 64, 80, 128, 256])
        hkv = rng.choice([1, 2, 5, 8])
        return {"op": op, "t": _log_int(rng, 1, 4096), "hq": hkv * rng.choice([1, 2, 3]), "hkv": hkv, "hd": hd, "rot": rng.choice([hd, hd, 16]),
                "interleaved": rng.random() < 0.3, "f32": rng.random() < 0.3, "pos0": rng.choice([0, 1000, 1000000])}
    step = 16 if op == "grouped_scaled" else 8
    return {"op": op, "t": _log_int(rng, 1, 8192), "g": _log_int(rng, 1, 32), "n": _log_int(rng, 7, 4096), "k": _log_int(rng, step, 2048, step),
            "skew": round(rng.uniform(0.0, 1.5), 2), "act": rng.randrange(3), "bf16": rng.random() < 0.7}


def _counts(c):
    """Rows of each expert, the busiest first: shares that fall with (1 + i) ** -skew, whole, `t` in all; empty ones among them where rows are few."""
    share = [(1.0 + i) ** -c["skew"] for i in range(c["g"])]
    ends = [0]
    total = 0.0
    for s in share:
        total += s
        ends.append(int(round(c["t"] * total / sum(share))))
    ends[-1] = c["t"]
    return [b - a for a, b in zip(ends, ends[1:])]


# ---------------------------------------------------------------- inputs
def _quantize(x, rows):
    """Values e4m3(x / s) and scales s = max(amax / 448, 2^-126) of each block of `rows` x 128, from elementary operations in fp32."""
    m, k = x.shape
    mb, kb = -(-m // rows), -(-k // BLOCK)
    padded = torch.zeros(mb * rows, kb * BLOCK, dtype=torch.float32, device=x.device)
    padded[:m, :k] = x
    blocks = padded.view(mb, rows, kb, BLOCK)
    amax = blocks.abs().amax(dim=(1, 3))
    scale = torch.maximum(amax / torch.full_like(amax, E4M3_MAX), torch.full_like(amax, LEAST_SCALE))     # (a tensor: a division, and no product with 1/448)
    q = (blocks / scale[:, None, :, None]).view(mb * rows, kb * BLOCK)[:m, :k]
    return q.to(torch.float8_e4m3fn).contiguous(), scale


def _spread(v, rows, m, k):
    """The scale of every element of an [m, k] matrix."""
    return v.repeat_interleave(rows, 0)[:m].repeat_interleave(BLOCK, 1)[:, :k]


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed) * 7919 + 13)
    normal = lambda *s: torch.randn(*s, device=DEVICE, generator=gen)  # noqa: E731
    op, s = case["op"], {"case": dict(case)}

    def activations(m, k):      # a few channels are ten times and more as large as the others, as behind a residual stream
        return normal(m, k) * torch.exp(0.8 * normal(1, k))

    if op == "quantize":
        if case["rows"] == 1:
            x = activations(case["m"], case["k"])
        else:
            x = 0.02 * normal(case["m"], case["k"])
        s["x"] = x if case["f32"] else x.to(torch.bfloat16)
    elif op == "scaled":
        s["a"], s["sa"] = _quantize(activations(case["m"], case["k"]).to(torch.bfloat16).float(), 1)
        s["w"], s["sw"] = _quantize(0.02 * normal(case["n"], case["k"]), BLOCK)
    elif op in ("grouped", "grouped_scaled"):
        t, g, n, k = (case[x] for x in ("t", "g", "n", "k"))
        counts = _counts(case)
        order = torch.randperm(g, generator=torch.Generator().manual_seed(int(seed) * 31 + 7)).tolist()
        ends = [0]
        for i in order:
            ends.append(ends[-1] + counts[i])
        s["offsets"] = torch.tensor(ends, dtype=torch.int32, device=DEVICE)       # where the router left its sorted rows
        s["most"] = max(counts)
        a = activations(t, k).to(torch.bfloat16)
        if op == "grouped":
            s["a"], s["w"] = a, torch.empty(g, n, k, dtype=torch.bfloat16, device=DEVICE)
            for i in range(g):
                s["w"][i] = 0.02 * normal(n, k)
        else:
            s["a"], s["sa"] = _quantize(a.float(), 1)
            s["w"] = torch.empty(g, n, k, dtype=torch.float8_e4m3fn, device=DEVICE)
            s["sw"] = torch.empty(g, -(-n // BLOCK), -(-k // BLOCK), device=DEVICE)
            for i in range(g):
                s["w"][i], s["sw"][i] = _quantize(0.02 * normal(n, k), BLOCK)
    else:
        t, hq, hkv, hd = (case[x] for x in ("t", "hq", "hkv", "hd"))
        rows = normal(t, (hq + 2 * hkv) * hd) * 3.0                                # the stacked projection: queries, keys, values
        s["qkv"] = rows if case["f32"] else rows.to(torch.bfloat16)
        s["q"], s["k"] = s["qkv"][:, :hq * hd], s["qkv"][:, hq * hd:(hq + hkv) * hd]
        s["gq"], s["gk"] = 1.0 + 0.1 * normal(hd), 1.0 + 0.1 * normal(hd)
        # several sequences side by side, each with positions of its own
        s["pos"] = (torch.arange(t, device=DEVICE) % 512 + case["pos0"] + int(seed) % 97).to(torch.int32)
    return s


# ---------------------------------------------------------------- one pass
def _act(y, act):
    if act == 1:
        return 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y * y * y)))
    if act == 2:
        return y / (1.0 + torch.exp(-y))
    return y


def _rotated(x, heads, gain, s):
    """RMS norm over each head, then the rotation by the row's position; fp32, angles in 64 bits, rounded once."""
    c = s["case"]
    hd, rot, eps = c["hd"], c["rot"], 1e-6
    x = x.float().view(-1, heads, hd)
    y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps) * gain
    freq = 10000.0 ** (-torch.arange(0, rot, 2, device=y.device, dtype=torch.float64) / rot)
    angle = s["pos"].double()[:, None] * freq
    cos, sin = torch.cos(angle).float()[:, None, :], torch.sin(angle).float()[:, None, :]
    if c["interleaved"]:
        u, v = y[..., 0:rot:2], y[..., 1:rot:2]
        turned = torch.stack([u * cos - v * sin, v * cos + u * sin], -1).flatten(-2)
    else:
        u, v = y[..., :rot // 2], y[..., rot // 2:rot]
        turned = torch.cat([u * cos - v * sin, v * cos + u * sin], -1)
    return torch.cat([turned, y[..., rot:]], -1).reshape(-1, heads * hd).to(torch.bfloat16)


def _grouped(a, w, s):
    """Each row times its expert's matrix: rows laid out expert by expert up to the busiest one's count, and taken back."""
    t, lo, hi = a.shape[0], s["offsets"][:-1].long(), s["offsets"][1:].long()
    at = lo[:, None] + torch.arange(s["most"], device=a.device)
    padded = torch.where((at < hi[:, None])[..., None], a[at.clamp(max=t - 1)], torch.zeros((), device=a.device))
    y = torch.bmm(padded, w.transpose(1, 2))
    row = torch.arange(t, device=a.device)
    expert = torch.searchsorted(hi, row, right=True)
    return y[expert, row - lo[expert]]


def run(state):
    s, c = state, state["case"]
    op = c["op"]
    if own:
        from paper_2609_22335_b200 import api
        if op == "quantize":
            return api.op_quantize(s["x"], block_rows=c["rows"])
        if op == "scaled":
            return api.op_linear_scaled(s["a"], s["sa"], s["w"], s["sw"], act=c["act"], out_bf16=c["bf16"])
        if op == "grouped":
            return api.op_linear_grouped(s["a"], s["w"], s["offsets"], act=c["act"], out_bf16=c["bf16"])
        if op == "grouped_scaled":
            return api.op_linear_grouped_scaled(s["a"], s["sa"], s["w"], s["sw"], s["offsets"], act=c["act"], out_bf16=c["bf16"])
        return api.op_qk_norm_rope(s["q"], s["k"], c["hq"], c["hkv"], c["hd"], gq=s["gq"], gk=s["gk"], eps=1e-6, pos=s["pos"], base=10000.0,
                                   rot=c["rot"], interleaved=c["interleaved"])
    if op == "quantize":
        return _quantize(s["x"].float(), c["rows"])
    if op == "qk":
        return _rotated(s["q"], c["hq"], s["gq"], s), _rotated(s["k"], c["hkv"], s["gk"], s)
    if op == "grouped":
        y = _grouped(s["a"].float(), s["w"].float(), s)
    else:
        a = s["a"].float() * _spread(s["sa"], 1, *s["a"].shape)
        if op == "scaled":
            y = a @ (s["w"].float() * _spread(s["sw"], BLOCK, *s["w"].shape)).T
        else:
            n, k = s["w"].shape[1:]
            scale = s["sw"].repeat_interleave(BLOCK, 1)[:, :n].repeat_interleave(BLOCK, 2)[:, :, :k]
            y = _grouped(a, s["w"].float() * scale, s)
    y = _act(y, c["act"])
    return y.to(torch.bfloat16) if c["bf16"] else y


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    op = case["op"]
    if op == "quantize":
        m, k = case["m"], case["k"]
        return {"bytes": m * k * (4 if case["f32"] else 2) + m * k + 4 * -(-m // case["rows"]) * -(-k // BLOCK), "flops": 3 * m * k}
    if op == "qk":
        heads = case["hq"] + case["hkv"]
        return {"bytes": case["t"] * heads * case["hd"] * ((4 if case["f32"] else 2) + 2) + 4 * case["t"] + 8 * case["hd"], "flops": case["t"] * heads * case["hd"] * 7}
    n, k, width = case["n"], case["k"], 2 if case["bf16"] else 4
    blocks = 4 * -(-k // BLOCK)
    if op == "scaled":
        m = case["m"]
        return {"bytes": m * k + n * k + m * blocks + -(-n // BLOCK) * blocks + m * n * width, "flops": 2 * m * n * k}
    t, busy = case["t"], sum(x > 0 for x in _counts(case))
    size = 2 if op == "grouped" else 1
    scales = 0 if op == "grouped" else t * blocks + busy * -(-n // BLOCK) * blocks
    return {"bytes": size * (t * k + busy * n * k) + scales + 4 * (case["g"] + 1) + t * n * width, "flops": 2 * t * n * k}


# ---------------------------------------------------------------- the definitions, in 64 bits
def _nearest_e4m3(v):
    """The nearest e4m3 value, ties to the even one: steps of 2^(e - 3) in [2^e, 2^(e + 1)), of 2^-9 below 2^-6."""
    exponent = torch.frexp(v.abs())[1].clamp(min=-5) - 1
    step = torch.ldexp(torch.ones_like(v), exponent - 3)
    return (torch.round(v / step) * step).clamp(-E4M3_MAX, E4M3_MAX)


def _block_of(n, rows):
    return torch.arange(n, device=DEVICE) // rows


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "quantize":
        x, r = s["x"].double(), case["rows"]
        bi, bj = _block_of(x.shape[0], r), _block_of(x.shape[1], BLOCK)
        cell = bi[:, None] * (int(bj[-1]) + 1) + bj[None, :]
        amax = torch.zeros((int(bi[-1]) + 1) * (int(bj[-1]) + 1), dtype=torch.float64, device=DEVICE)
        amax.scatter_reduce_(0, cell.flatten(), x.abs().flatten(), "amax")
        scale = (amax / E4M3_MAX).clamp(min=LEAST_SCALE)
        held = scale.float().double()                       # the scale is kept in fp32, and it is that one the values are taken relative to
        return _nearest_e4m3(x / held[cell]), scale.view(int(bi[-1]) + 1, -1)
    if op == "qk":
        t, hd, rot = case["t"], case["hd"], case["rot"]
        angle = torch.outer(s["pos"].double(), torch.exp(-math.log(10000.0) * torch.arange(rot // 2, device=DEVICE, dtype=torch.float64) * 2.0 / rot))
        turn = torch.complex(torch.cos(angle), torch.sin(angle))
        out = []
        for x, heads, gain in ((s["q"], case["hq"], s["gq"]), (s["k"], case["hkv"], s["gk"])):
            x = x.double().reshape(t, heads, hd)
            y = gain.double() * x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / hd + 1e-6)
            even, odd = (slice(0, rot, 2), slice(1, rot, 2)) if case["interleaved"] else (slice(0, rot // 2), slice(rot // 2, rot))
            z = torch.complex(y[..., even], y[..., odd]) * turn[:, None]
            y[..., even], y[..., odd] = z.real, z.imag
            out.append(y.reshape(t, heads * hd))
        return tuple(out)

    def dequantized(v, scales, rows):
        return v.double() * scales.double()[_block_of(v.shape[0], rows)][:, _block_of(v.shape[1], BLOCK)]

    if op == "scaled":
        y = dequantized(s["a"], s["sa"], 1) @ dequantized(s["w"], s["sw"], BLOCK).T
    else:
        a = s["a"].double() if op == "grouped" else dequantized(s["a"], s["sa"], 1)
        y = torch.zeros(case["t"], case["n"], dtype=torch.float64, device=DEVICE)
        ends = s["offsets"].tolist()
        for i, (lo, hi) in enumerate(zip(ends, ends[1:])):
            w = s["w"][i].double() if op == "grouped" else dequantized(s["w"][i], s["sw"][i], BLOCK)
            y[lo:hi] = a[lo:hi] @ w.T
    if case["act"] == 1:
        y = y * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3))
    elif case["act"] == 2:
        y = y * torch.sigmoid(y)
    return y
