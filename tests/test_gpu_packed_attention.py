"""Attention of packed sequences against the definition in 64 bits (tests/sequences_reference.py has the tolerance)."""
import math

import pytest

import sequences_reference as ref

pytestmark = pytest.mark.gpu


def make(rows, hq, hkv, hd, seed, keys=None):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda n, w: torch.randn(n, w, device="cuda", generator=g).bfloat16()      # noqa: E731
    keys = rows if keys is None else keys
    return 1.5 * r(rows, hq * hd), r(keys, hkv * hd), r(keys, hkv * hd)


def ends(lengths, first=0):
    out = [first]
    for n in lengths:
        out.append(out[-1] + n)
    return out


def ints(x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def run(q, k, v, ends_q, hq, hkv, hd, ends_k=None, prefix=None, **kw):
    import torch
    from paper_2609_22335_b200 import api
    scratch = torch.empty(api.op_attention_sequences_scratch_bytes(hd), dtype=torch.uint8, device="cuda")
    got = api.op_attention_packed(q, k, v, ints(ends_q), hq, hkv, hd, offsets_k=None if ends_k is None else ints(ends_k), prefix=None if prefix is None else ints(prefix),
                                  scratch=scratch, **kw)
    assert api.op_status(api.OP_ATTENTION_PACKED, scratch) == api.VLA_OK
    return got


def slopes_of(hq):
    import torch
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)], device="cuda")


LENGTHS = [[1], [5], [128], [129], [300], [1, 1, 1], [7, 0, 64, 65, 130], [1000], [40] * 30, [513, 2, 255, 256], [2500, 700]]
HEADS = [(1, 1, 64), (4, 4, 128), (8, 2, 64), (6, 2, 128), (8, 1, 256), (5, 1, 72), (3, 3, 8), (2, 1, 136), (15, 5, 64), (70, 1, 32)]


@pytest.mark.parametrize("lengths", LENGTHS, ids=str)
@pytest.mark.parametrize("hq,hkv,hd", HEADS)
@pytest.mark.parametrize("causal", [False, True])
def test_against_64_bits(lengths, hq, hkv, hd, causal):
    e = ends(lengths)
    q, k, v = make(e[-1], hq, hkv, hd, seed=e[-1] + hd)
    ref.check(run(q, k, v, e, hq, hkv, hd, causal=causal), ref.packed(q, k, v, e, e, hq, hkv, hd, causal=causal))


@pytest.mark.parametrize("lengths", [[1], [37], [300], [7, 0, 64, 65, 130], [1000, 129]], ids=str)
@pytest.mark.parametrize("hq,hkv,hd", [(8, 2, 64), (4, 4, 128), (8, 1, 256)])
@pytest.mark.parametrize("how", [dict(cap=5.0), dict(slopes=True), dict(cap=30.0, slopes=True, causal=True), dict(causal=True, window=1), dict(causal=True, window=33),
                                 dict(causal=True, window=200, prefix=20), dict(causal=True, prefix=10), dict(causal=True, prefix=150, cap=50.0), dict(scale=0.02),
                                 dict(causal=True, window=128, slopes=True)], ids=str)
def test_masks_caps_and_distances(lengths, hq, hkv, hd, how):
    e = ends(lengths)
    how = dict(how)
    q, k, v = make(e[-1], hq, hkv, hd, seed=e[-1] + hd)
    if how.get("slopes"):
        how["slopes"] = slopes_of(hq)
    if "prefix" in how:
        how["prefix"] = [min(how["prefix"], max(n - 2, 0)) for n in lengths]
    ref.check(run(q, k, v, e, hq, hkv, hd, **how), ref.packed(q, k, v, e, e, hq, hkv, hd, **how))


@pytest.mark.parametrize("nq,nk", [([3, 200, 1], [500, 0, 40]), ([300], [100]), ([50, 50], [1, 129]), ([1] * 9, [2000, 1, 64, 128, 129, 0, 3, 700, 256]), ([20], [6000])], ids=str)
@pytest.mark.parametrize("hq,hkv,hd", [(8, 2, 64), (4, 1, 128), (2, 1, 256)])
@pytest.mark.parametrize("how", [dict(), dict(causal=True), dict(causal=True, window=50, prefix=3), dict(causal=True, cap=20.0)], ids=str)
def test_keys_of_their_own(nq, nk, hq, hkv, hd, how):
    """Fewer or more keys than rows, none among them: rows in front of the first key see nothing and become zeros."""
    eq, ek, how = ends(nq), ends(nk), dict(how)
    q, k, v = make(eq[-1], hq, hkv, hd, seed=1, keys=ek[-1])
    if "prefix" in how:
        how["prefix"] = [how["prefix"]] * len(nq)
    want = ref.packed(q, k, v, eq, ek, hq, hkv, hd, **({**how, "prefix": [min(how["prefix"][0], n) for n in nk]} if "prefix" in how else how))
    ref.check(run(q, k, v, eq, hq, hkv, hd, ends_k=ek, **how), want)


@pytest.mark.parametrize("hq,hkv,hd", [(8, 2, 64), (4, 2, 128), (2, 1, 256), (5, 1, 72)])
def test_views_of_a_stacked_projection_and_rows_of_no_sequence(hq, hkv, hd):
    """Rows in front of the first sequence, between (none: they ascend) and behind the last one stay as they were, and what lies there may be NaN."""
    import torch
    e = [5, 80, 80, 333]
    q, k, v = make(360, hq, hkv, hd, seed=3)
    rows = torch.full((360, (hq + 2 * hkv) * hd + 16), math.nan, dtype=torch.bfloat16, device="cuda")
    at = [hq * hd, (hq + hkv) * hd, (hq + 2 * hkv) * hd]
    for x, a, b in ((q, 0, at[0]), (k, at[0], at[1]), (v, at[1], at[2])):
        rows[5:333, a:b] = x[5:333]
    wide = torch.full((360, hq * hd + 24), 7.0, dtype=torch.bfloat16, device="cuda")
    out = wide[:, 8:8 + hq * hd]
    for how in (dict(), dict(causal=True), dict(cap=9.0)):
        assert run(rows[:, :at[0]], rows[:, at[0]:at[1]], rows[:, at[1]:at[2]], e, hq, hkv, hd, out=out, **how) is out
        ref.check(out, ref.packed(q, k, v, e, e, hq, hkv, hd, **how))
        assert bool((wide[:, :8] == 7).all() and (wide[:, 8 + hq * hd:] == 7).all() and (out[:5] == 7).all() and (out[333:] == 7).all())


@pytest.mark.parametrize("hq,hkv,hd", [(4, 2, 64), (2, 2, 128), (2, 1, 256)])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("lengths", [[300, 140], [40] * 4, [1500]], ids=str)
def test_what_a_row_does_not_see_has_no_part_in_it(hq, hkv, hd, value, lengths):
    """A key and a value that are not finite reach the rows that see them and no other one."""
    import torch
    e = ends(lengths)
    q, k, v = make(e[-1], hq, hkv, hd, seed=4)
    hurt = lengths[0] * 2 // 3
    for how in (dict(causal=True), dict(causal=True, window=20)):
        want = ref.packed(q, k, v, e, e, hq, hkv, hd, **how)
        for x in (k, v):
            y = x.clone()
            y[hurt, hd // 2] = value
            got = run(q, y if x is k else k, y if x is v else v, e, hq, hkv, hd, **how)
            sees = torch.zeros(e[-1], dtype=torch.bool, device="cuda")
            sees[hurt:min(hurt + how.get("window", e[1]), e[1])] = True
            clean = [(a, b, o, t) for a, b, o, t in want]
            for a, b, o, t in clean:
                free = ~sees[a:b]
                assert bool(((got[a:b].double() - o).abs() <= t)[free].all())
            heads = got.view(e[-1], hq, hd)[sees][:, :hq // hkv]
            if x is v:
                assert not bool(heads[:, :, hd // 2].isfinite().any())
            elif math.isnan(value):
                assert bool(heads.isnan().all())


def test_rows_whose_scores_are_far_apart():
    """Scores of many hundreds: the running maximum moves in every block, and all but a few probabilities vanish."""
    q, k, v = make(700, 4, 2, 64, seed=5)
    e = [0, 700]
    for causal in (False, True):
        ref.check(run(30 * q, 10 * k, v, e, 4, 2, 64, causal=causal), ref.packed(30 * q, 10 * k, v, e, e, 4, 2, 64, causal=causal))


def test_a_query_that_is_nan_is_its_rows_alone():
    import torch
    e = [0, 200, 333]
    for hd in (64, 256):
        q, k, v = make(333, 4, 2, hd, seed=15)
        want = ref.packed(q, k, v, e, e, 4, 2, hd, causal=True)
        q[77, 2 * hd + 3] = math.nan
        got = run(q, k, v, e, 4, 2, hd, causal=True)
        assert bool(got[77, 2 * hd:3 * hd].isnan().all())
        got[77, 2 * hd:3 * hd] = want[0][2][77, 2 * hd:3 * hd].bfloat16()
        ref.check(got, want)


def test_thousands_of_sequences_none_at_all_and_windows_without_end():
    import torch
    lengths = [(7 * s) % 4 for s in range(3000)]
    e = ends(lengths)
    q, k, v = make(e[-1], 2, 1, 64, seed=16)
    got, off = run(q, k, v, e, 2, 1, 64, causal=True), torch.tensor(e[:-1], device="cuda")
    # (rows of up to three: the first of each is its own value, the second weighs two)
    for n in range(1, 4):
        first = off[torch.tensor([x == n for x in lengths], device="cuda")]
        assert bool((got[first].view(-1, 2, 64) == v[first][:, None]).all())
    picked = [s for s in range(0, 3000, 61)]
    ref.check(got, [(e[s], e[s + 1], *ref.attend(q[e[s]:e[s + 1]], k[e[s]:e[s + 1]], v[e[s]:e[s + 1]], 2, 1, 64, causal=True)) for s in picked])
    out = torch.full_like(q, 3.0)
    assert bool((run(q, k, v, [0] * 5, 2, 1, 64, out=out) == 3).all())
    for n, keys in ((50, 20), (300, 10)):                # more rows than keys: positions in front of the first one
        q, k, v = make(n, 2, 1, 64, seed=17, keys=keys)
        ref.check(run(q, k, v, [0, n], 2, 1, 64, ends_k=[0, keys], causal=True, window=(1 << 31) - 1, prefix=[3]), ref.packed(q, k, v, [0, n], [0, keys], 2, 1, 64, causal=True, prefix=[3]))


def test_caps_from_tiny_to_none_to_speak_of():
    e = [0, 150, 400]
    q, k, v = make(400, 4, 2, 64, seed=18)
    for cap in (1e-3, 0.5, 2.0, 5.0, 69.0, 70.0, 1e4, 1e20):
        # (from 1e4 on the cap changes nothing that 32 bits show, and its share of the tolerance would hide everything)
        ref.check(run(q, k, v, e, 4, 2, 64, causal=True, cap=cap), ref.packed(q, k, v, e, e, 4, 2, 64, causal=True, cap=0.0 if cap >= 1e4 else cap))


def test_the_same_call_gives_the_same_bits_and_two_calls_at_once_do_not_meet():
    import torch
    from paper_2609_22335_b200 import api
    e = ends([900, 33, 411])
    made = [make(e[-1], 8, 2, 128, seed=s) for s in (6, 7)]
    off = ints(e)
    want = [run(*x, e, 8, 2, 128, causal=True) for x in made]
    streams = [torch.cuda.Stream() for _ in made]
    torch.cuda.synchronize()
    for _ in range(5):
        got = [api.op_attention_packed(*x, off, 8, 2, 128, causal=True, stream=s) for x, s in zip(made, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_captured_first_and_replayed_on_new_lengths():
    """The graph reads lengths when it runs: one captured call serves any sequences that fit."""
    import torch
    from paper_2609_22335_b200 import api
    q, k, v = make(600, 4, 2, 96, seed=8)
    off = ints([0, 100, 600])
    side = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        got = api.op_attention_packed(q, k, v, off, 4, 2, 96, causal=True, stream=side)
    for e in ([0, 100, 600], [0, 600, 600], [0, 1, 2], [0, 0, 599]):
        off.copy_(ints(e))
        got.zero_()
        g.replay()
        torch.cuda.synchronize()
        ref.check(got, ref.packed(q, k, v, e, e, 4, 2, 96, causal=True))
        assert not bool(got[e[-1]:].any())


def test_a_wait_that_runs_out_is_reported():
    import torch
    from paper_2609_22335_b200 import api
    for lengths, heads in (([300, 400], (8, 2, 64)), ([1] * 5, (8, 2, 128)), ([200], (2, 1, 256))):
        e = ends(lengths)
        q, k, v = make(e[-1], *heads, seed=9)
        scratch = torch.empty(api.op_attention_sequences_scratch_bytes(heads[2]), dtype=torch.uint8, device="cuda")
        api.debug_op_fault(True, wait_limit_ns=1_000_000)
        try:
            api.op_attention_packed(q, k, v, ints(e), *heads, scratch=scratch)
            assert api.op_status(api.OP_ATTENTION_PACKED, scratch) == api.VLA_ERR_TIMEOUT
        finally:
            api.debug_op_fault(False)
        ref.check(run(q, k, v, e, *heads), ref.packed(q, k, v, e, e, *heads))


@pytest.mark.parametrize("heads", [(8, 2, 64), (4, 4, 128), (2, 1, 256)])
def test_short_sequences_need_no_scratch_memory(heads):
    """Up to 512 keys the bits are those of the call with it; what went wrong is in a word of the library then."""
    import torch
    from paper_2609_22335_b200 import api
    for lengths in ([512], [1, 200, 0, 311], [3] * 100):
        e = ends(lengths)
        q, k, v = make(e[-1], *heads, seed=19)
        off = ints(e)
        got = api.op_attention_packed(q, k, v, off, *heads, causal=True)
        assert api.op_status(api.OP_ATTENTION_SHORT) == api.VLA_OK
        assert torch.equal(got, run(q, k, v, e, *heads, causal=True))
        ref.check(got, ref.packed(q, k, v, e, e, *heads, causal=True))
        api.debug_op_fault(True, wait_limit_ns=1_000_000)
        try:
            api.op_attention_packed(q, k, v, off, *heads)
            assert api.op_status(api.OP_ATTENTION_SHORT) == api.VLA_ERR_TIMEOUT
        finally:
            api.debug_op_fault(False)
        api.op_attention_packed(q, k, v, off, *heads)
        assert api.op_status(api.OP_ATTENTION_SHORT) == api.VLA_OK
