"""Attention of several sequences from its definition, in 64 bits, and how far a result in bf16 may be from it.

Bound of a value o = sum_j p_j v_j, with A = sum_j p_j |v_j| and sums over visible keys: half a step of the result, 2^-8 |o|; half a step of each probability, which goes
into the second product as bf16 while the sum that divides it does not: 2^-8 A; the scores' errors d, which change every p_j by a factor of
1 + d and the sum with them: 2 d A; and the second product's sums, cut to 24 bits after each 16 keys: (n / 16 + 8) 2^-22 A (8: parts of split
keys).  d = (hd / 16 + 2) 2^-22 scale sum |q k| for the first product, 2^-20 for powers of two and their sums, 2^-20 of the row's largest score (its scaling,
rounded constants, the bias' product) and, of capped scores, 2^-19 cap (a power and a reciprocal good to 2^-22 each, and their product)."""
import math


def attend(q, k, v, hq, hkv, hd, causal=False, prefix=0, window=0, cap=0.0, slopes=None, scale=None):
    """One sequence: q [nq, hq*hd], k and v [nk, hkv*hd].  Returns (out, bound), 64 bits, [nq, hq*hd]."""
    import torch
    nq, nk, scale = q.shape[0], k.shape[0], hd ** -0.5 if scale is None else scale
    dev = q.device
    out = torch.zeros(nq, hq * hd, dtype=torch.float64, device=dev)
    tol = torch.zeros_like(out)
    if nq == 0 or nk == 0:
        return out, tol
    pos = torch.arange(nk - nq, nk, device=dev)
    far = pos[:, None] - torch.arange(nk, device=dev)[None]
    seen = torch.ones(nq, nk, dtype=torch.bool, device=dev)
    if causal:
        seen = far >= 0
        if window:
            seen &= far < window
        seen |= (torch.arange(nk, device=dev) < prefix)[None]
    for h in range(hq):
        g = h // (hq // hkv)
        qs, ks, vs = (x[:, i * hd:(i + 1) * hd].double() for x, i in ((q, h), (k, g), (v, g)))
        s = qs @ ks.T * scale
        d = (hd / 16 + 2) * 2.0 ** -22 * scale * (qs.abs() @ ks.abs().T)
        if cap:
            s = cap * torch.tanh(s / cap)
            d = d + 2.0 ** -19 * cap
        if slopes is not None:
            s = s - slopes[h].double() * far.abs()
        s = s.masked_fill(~seen, -math.inf)
        p = torch.softmax(s, -1)
        p = torch.where(seen, p, torch.zeros_like(p)).masked_fill(~seen.any(1, keepdim=True), 0.0)
        a = p @ vs.abs()
        o = p @ vs
        worst = torch.where(seen, d, torch.zeros_like(d)).amax(1, keepdim=True)
        top = torch.where(seen, s.abs(), torch.zeros_like(s)).amax(1, keepdim=True)
        delta = worst + 2.0 ** -20 + 2.0 ** -20 * top
        of = slice(h * hd, (h + 1) * hd)
        out[:, of] = o
        tol[:, of] = 2.0 ** -8 * o.abs() + (2.0 ** -8 + 2 * delta + (nk / 16 + 8) * 2.0 ** -22) * a
    return out, tol


def packed(q, k, v, ends_q, ends_k, hq, hkv, hd, prefix=None, **kw):
    """All sequences: [(first row, end, out, bound)]."""
    got = []
    for s, (a, b) in enumerate(zip(ends_q, ends_q[1:])):
        ka, kb = ends_k[s], ends_k[s + 1]
        got.append((a, b, *attend(q[a:b], k[ka:kb], v[ka:kb], hq, hkv, hd, prefix=prefix[s] if prefix else 0, **kw)))
    return got


def check(got, want):
    """`got`: the call's rows; `want`: packed()'s."""
    worst = 0.0
    for a, b, o, tol in want:
        x = got[a:b].double()
        assert bool(x.isfinite().all())
        off = (x - o).abs()
        if off.numel():
            worst = max(worst, float((off / tol.clamp(min=1e-30)).max()) if bool((off > 0).any()) else 0.0)
            assert bool((off <= tol).all()), (a, b, worst)
    return worst
