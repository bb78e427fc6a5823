"""Capped scores: each is a function of itself alone, whatever else its block, its tile or its page holds."""
import math

import pytest

from test_gpu_packed_attention import ends, ints, make, run
from test_gpu_paged_attention import Cache, run as run_paged

pytestmark = pytest.mark.gpu

# heads of which a tile's rows are all taken, and those that leave two, three or eight over; tiles of one and of two, and of wide heads
HEADS = [(8, 2, 64), (3, 1, 64), (6, 2, 128), (5, 1, 72), (12, 1, 32), (3, 1, 256)]
LENGTHS = [[90, 60], [1010, 300], [2600, 1700]]


@pytest.mark.parametrize("hq,hkv,hd", HEADS)
@pytest.mark.parametrize("lengths", LENGTHS, ids=str)
@pytest.mark.parametrize("cap", [4.0, 10.0])
def test_neighbours_change_no_bit(hq, hkv, hd, lengths, cap):
    """Scores on both sides of half the cap beside none that are: the next sequence's queries and keys, hidden keys, what another call left in shared memory."""
    import torch
    e = ends(lengths)
    n = e[1]
    q, k, v = make(e[-1], hq, hkv, hd, seed=n + hd)
    for size in (0.3, 1.0, 3.0):
        mine = q.clone()
        mine[:n] *= size
        want = run(mine, k, v, e, hq, hkv, hd, causal=True, cap=cap)[:n]
        for factor in (0.0, 100.0):
            other = mine.clone()
            other[n:] *= factor
            assert torch.equal(run(other, k, v, e, hq, hkv, hd, causal=True, cap=cap)[:n], want)
            keys = k.clone()
            keys[n - 7:] *= factor
            assert torch.equal(run(mine, keys, v, e, hq, hkv, hd, causal=True, cap=cap)[:n - 7], want[:n - 7])
            four = make(600, 4, 1, hd, seed=1)
            run(factor * four[0], *four[1:], [0, 600], 4, 1, hd, cap=cap)
            assert torch.equal(run(mine, k, v, e, hq, hkv, hd, causal=True, cap=cap)[:n], want)


@pytest.mark.parametrize("hq,hkv,hd", HEADS)
@pytest.mark.parametrize("cap", [50.0, 1e4, 1e20])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan, 3e38])
def test_hidden_keys_of_any_value_change_no_bit(hq, hkv, hd, cap, value):
    import torch
    for lengths in ([300, 40], [2600]):
        e = ends(lengths)
        q, k, v = make(e[-1], hq, hkv, hd, seed=hd)
        hurt = e[1] - 5
        keys = k.clone()
        keys[hurt, ::2] = value
        for how in (dict(causal=True), dict(causal=True, window=20)):
            want, got = (run(q, x, v, e, hq, hkv, hd, cap=cap, **how) for x in (k, keys))
            assert torch.equal(got[:hurt], want[:hurt]) and torch.equal(got[e[1]:], want[e[1]:])


@pytest.mark.parametrize("hq,hkv,hd", [(8, 2, 64), (3, 1, 128), (5, 1, 256)])
@pytest.mark.parametrize("cap", [20.0, 1e4])
def test_rows_of_a_page_behind_the_length_change_no_bit(hq, hkv, hd, cap):
    import torch
    keys, new = [1001, 37], [40, 1]
    eq, ek = ends(new), ends(keys)
    q, k, v = make(eq[-1], hq, hkv, hd, seed=3, keys=ek[-1])
    got = []
    for value in (0.0, 1e30, math.inf, math.nan):
        c = Cache(keys, hkv, hd, 32, seed=4)
        for x in (c.k, c.v):
            x.fill_(value)
        c.fill_fast(k, v)
        got.append(run_paged(c, q, eq, hq, hkv, hd, cap=cap))
    assert bool(got[0].isfinite().all()) and all(torch.equal(x, got[0]) for x in got[1:])


@pytest.mark.parametrize("hd", [64, 128, 256])
def test_a_score_beyond_half_the_cap_leaves_the_others_as_they_are(hd):
    """A key that no row gives any weight, at -0.6 and at -0.4 of the cap: the other scores are the same numbers."""
    import torch
    for n in (200, 2500):
        e = [0, n]
        q, k, v = make(n, 2, 1, hd, seed=6)
        q[:, 0::hd] = 1.0
        got = []
        for at in (-4000.0, -6000.0):
            keys = k.clone()
            keys[:, 0] = 0
            keys[n // 2] = 0
            keys[n // 2, 0] = at
            got.append(run(q, keys, v, e, 2, 1, hd, cap=1e4, scale=1.0))
        assert torch.equal(*got)


@pytest.mark.parametrize("n,hd", [(200, 64), (6000, 64), (6000, 128), (2000, 256)])
def test_scores_below_zero_are_as_good_as_those_above(n, hd):
    """tanh is odd: two keys whose scores change sign change places, bit for bit.  (A cap times log2 e that rounds to 2^20, so that nothing else rounds; the scores lie a few
    units of the last place of the capped ones apart.)"""
    import numpy as np
    import torch
    c = np.float32(2.0 ** 20 / np.log2(np.e))
    cap = next(float(x) for x in (c, np.nextafter(c, np.float32(0)), np.nextafter(c, np.float32(1e9))) if x * np.float32(1.44269504) == np.float32(2 ** 20))
    g = torch.Generator(device="cuda").manual_seed(n)
    q, k, v = (torch.zeros(m, hd, dtype=torch.bfloat16, device="cuda") for m in (n, 2, 2))
    q[:, 0] = 0.05 + 3 * torch.rand(n, device="cuda", generator=g)
    q[:, 1] = torch.randint(1, 9, (n,), device="cuda", generator=g).bfloat16()
    k[:, 0], k[1, 1], v[1] = 1, 2.0 ** -19, 1
    up, down = (run(q, s * k, w, [0, n], 1, 1, hd, ends_k=[0, 2], scale=cap, cap=cap) for s, w in ((1, v), (-1, 1 - v)))
    assert bool(((up > 0.5) & (up < 0.999)).any()) and torch.equal(up, down)


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("hd", [8, 256])
def test_a_capped_score_is_off_by_what_is_stated(sign, hd):
    """One capped score beside one that is 0, with a bias by distance that makes up for it, so that the weight tells the score to a fraction of the cap's last places.  Units of 2^-23 of
    the cap: tanh 2.2, the bias' and the score's roundings 0.5 each, half a step of a result between 0.1 and 0.9 0.4 -- below 4, which the header promises, in all."""
    import torch
    from paper_2609_22335_b200 import api
    cap, heads = 2.0 ** 20, 512
    for seed in range(8):
        g = torch.Generator(device="cuda").manual_seed(seed)
        x = (sign * cap * (0.02 + 3.5 * torch.rand(heads, device="cuda", generator=g))).bfloat16()
        exact = cap * torch.tanh(x.double() / cap)
        slopes = (exact - (2 * torch.rand(heads, device="cuda", generator=g) - 1)).float()
        q, k, v = (torch.zeros(n, hd, dtype=torch.bfloat16, device="cuda") for n in (heads, 2, 2))
        q[:, 0], k[0, 0], v[0] = x, 1, 1
        y = api.op_attention_packed(q.view(1, -1), k, v, ints([0, 1]), heads, 1, hd, offsets_k=ints([0, 2]), scale=1.0, cap=cap, slopes=slopes).view(heads, hd)[:, 0].double()
        assert bool(((y > 0.1) & (y < 0.9)).all())
        off = (torch.log(y) - torch.log1p(-y) - (exact - slopes.double())).abs()
        assert float(off.max()) <= 3.6 * 2.0 ** -23 * cap, float(off.max()) / cap * 2 ** 23
