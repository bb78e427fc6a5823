"""Head norms and rotation against the formula in 64 bits.

Tolerance: the bf16 result is off by half a step, 2^-8 |y|.  In front of that, fp32: the sum of squares 21 additions deep and the root of its
mean less than 2^-20, sines of an angle good to 2^-26 turns plus 2^-24 relative rounding 2^-21, products and their sum 2^-22, so
less than 2^-18 of the two values that are turned into each other."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def formula(x, heads, hd, gain, eps, pos, base, rot, interleaved):
    """float64 numpy; returns (y, the size of what was summed up in each value)."""
    t = x.shape[0]
    x = x.astype(np.float64).reshape(t, heads, hd)
    with np.errstate(all="ignore"):
        y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * (1.0 if gain is None else gain.astype(np.float64))
    size = np.abs(y)
    if rot:
        angle = np.asarray(pos, np.float64)[:, None] * base ** (-2.0 * np.arange(rot // 2) / rot)
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        a, b = (np.s_[..., 0:rot:2], np.s_[..., 1:rot:2]) if interleaved else (np.s_[..., :rot // 2], np.s_[..., rot // 2:rot])
        u, v = y[a].copy(), y[b].copy()
        y[a], y[b] = u * c - v * s, v * c + u * s
        size[a] = size[b] = np.abs(u) + np.abs(v)
    return y.reshape(t, -1), size.reshape(t, -1)


def near(got, want):
    y, size = want
    got = got.float().cpu().numpy().astype(np.float64)
    assert np.array_equal(np.isnan(got), np.isnan(y))
    ok = ~np.isnan(y)
    assert np.all(np.abs(got - y)[ok] <= (2.0 ** -8 * np.abs(y) + 2.0 ** -18 * size + 1e-38)[ok])


def inputs(t, hq, hkv, hd, f32, seed):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rows = 3 * torch.randn(t, (hq + 2 * hkv) * hd, device="cuda", generator=gen)
    rows = rows if f32 else rows.to(torch.bfloat16)
    return rows[:, :hq * hd], rows[:, hq * hd:(hq + hkv) * hd], 1 + 0.3 * torch.randn(hd, device="cuda", generator=gen), 1 + 0.3 * torch.randn(hd, device="cuda", generator=gen)


def numpy_of(x):
    return x.float().cpu().numpy()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("t,hq,hkv,hd,rot,f32", [
    (1, 1, 1, 16, 16, False), (1, 16, 8, 128, 128, False), (3, 32, 32, 128, 128, True), (51, 8, 1, 256, 256, False), (7, 15, 5, 64, 64, False),
    (130, 4, 2, 80, 80, True), (33, 3, 1, 80, 32, False), (5, 6, 2, 48, 16, True), (2, 5, 5, 240, 240, False), (100, 2, 1, 32, 0, False), (1000, 9, 3, 64, 48, False)])
def test_matches_the_formula(t, hq, hkv, hd, rot, f32, interleaved):
    import torch
    from paper_2609_22335_b200 import api
    q, k, gq, gk = inputs(t, hq, hkv, hd, f32, t + hd)
    pos = torch.randint(0, 5000, (t,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(torch.int32)
    oq, ok = api.op_qk_norm_rope(q, k, hq, hkv, hd, gq=gq, gk=gk, eps=1e-5, pos=pos, rot=rot, interleaved=interleaved)
    p = pos.cpu().numpy()
    near(oq, formula(numpy_of(q), hq, hd, gq.cpu().numpy(), 1e-5, p, 10000.0, rot, interleaved))
    near(ok, formula(numpy_of(k), hkv, hd, gk.cpu().numpy(), 1e-5, p, 10000.0, rot, interleaved))


@pytest.mark.parametrize("base", [10000.0, 500000.0, 2.0])
def test_far_and_negative_positions(base):
    """2^31 - 1 is 3.4e8 turns of the first pair.  (The formula's own angle is good to 2^-53 of that: 2^-22.)"""
    import torch
    from paper_2609_22335_b200 import api
    places = [0, 1, -1, 131071, 10 ** 7, 2 ** 31 - 1, -2 ** 31, 123456789]
    q, k, gq, _ = inputs(len(places), 2, 1, 128, True, 3)
    pos = torch.tensor(places, dtype=torch.int32, device="cuda")
    oq, ok = api.op_qk_norm_rope(q, k, 2, 1, 128, gq=gq, pos=pos, base=base)
    near(oq, formula(numpy_of(q), 2, 128, gq.cpu().numpy(), 1e-6, places, base, 128, False))
    near(ok, formula(numpy_of(k), 1, 128, None, 1e-6, places, base, 128, False))


def test_positions_that_count_on_from_a_start_and_queries_alone():
    import torch
    from paper_2609_22335_b200 import api
    q, k, _, gk = inputs(70, 4, 2, 64, False, 8)
    oq, none = api.op_qk_norm_rope(q, None, 4, 0, 64, pos0=1000)
    assert none is None
    near(oq, formula(numpy_of(q), 4, 64, None, 1e-6, np.arange(70) + 1000, 10000.0, 64, False))
    both, ok = api.op_qk_norm_rope(q, k, 4, 2, 64, gk=gk, pos0=1000)
    assert torch.equal(both, oq)
    near(ok, formula(numpy_of(k), 2, 64, gk.cpu().numpy(), 1e-6, np.arange(70) + 1000, 10000.0, 64, False))


def test_a_row_alone_gives_what_it_gives_in_a_batch():
    import torch
    from paper_2609_22335_b200 import api
    q, k, gq, gk = inputs(20000, 6, 2, 64, False, 8)
    oq, ok = api.op_qk_norm_rope(q, k, 6, 2, 64, gq=gq, gk=gk)
    for i in (0, 1, 777, 19999):
        a, b = api.op_qk_norm_rope(q[i:i + 1], k[i:i + 1], 6, 2, 64, gq=gq, gk=gk, pos0=i)
        assert torch.equal(a, oq[i:i + 1]) and torch.equal(b, ok[i:i + 1])


@pytest.mark.parametrize("interleaved", [False, True])
def test_in_place_and_into_a_caches_rows(interleaved):
    import torch
    from paper_2609_22335_b200 import api
    t, hq, hkv, hd = 90, 8, 2, 64
    q, k, gq, gk = inputs(t, hq, hkv, hd, False, 4)
    want = api.op_qk_norm_rope(q, k, hq, hkv, hd, gq=gq, gk=gk, interleaved=interleaved)
    cache = torch.full((200, hkv * hd + 64), 7.0, dtype=torch.bfloat16, device="cuda")
    whole = q._base.clone()
    api.op_qk_norm_rope(q, k, hq, hkv, hd, gq=gq, gk=gk, interleaved=interleaved, out_q=q, out_k=cache[40:40 + t, :hkv * hd])
    torch.cuda.synchronize()
    assert torch.equal(q, want[0]) and torch.equal(cache[40:40 + t, :hkv * hd], want[1])
    assert torch.equal(q._base[:, hq * hd:], whole[:, hq * hd:])                     # keys and values as they were
    assert (cache[:40] == 7).all() and (cache[40 + t:] == 7).all() and (cache[:, hkv * hd:] == 7).all()


def test_zero_heads_and_heads_with_a_nan():
    import torch
    from paper_2609_22335_b200 import api
    q, k, gq, gk = inputs(6, 4, 2, 64, True, 4)
    q[1, 64:128] = 0.0
    q[2, 70] = float("nan")
    k[3, 5] = float("inf")
    oq, ok = api.op_qk_norm_rope(q, k, 4, 2, 64, gq=gq, gk=gk)
    torch.cuda.synchronize()
    assert (oq[1, 64:128] == 0).all() and torch.isnan(oq[2, 64:128]).all() and not torch.isnan(oq[2, :64]).any() and not torch.isnan(oq[2, 128:]).any()
    want = formula(numpy_of(k), 2, 64, gk.cpu().numpy(), 1e-6, np.arange(6), 10000.0, 64, False)[0]
    assert np.array_equal(np.isnan(numpy_of(ok)), np.isnan(want))
