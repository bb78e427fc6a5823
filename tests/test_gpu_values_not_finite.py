"""Values that are infinite or NaN where some rows of a tile see them and others do not: rows done again, and who waits for them."""
import math

import pytest

import sequences_reference as ref
from test_gpu_packed_attention import ends, ints, make, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hkv,hd", [(4, 2, 64), (2, 1, 128), (2, 1, 256)])
@pytest.mark.parametrize("lengths", [[3000, 500, 400], [3000] + [30] * 60], ids=["long", "short"])
def test_rows_done_again_let_no_wait_run_out(hq, hkv, hd, lengths):
    """A sequence of which all rows have to be done again, for longer than a wait may take: its partners go on afterwards, and other sequences get their rows."""
    import torch
    from paper_2609_22335_b200 import api
    e = ends(lengths)
    q, k, v = make(e[-1], hq, hkv, hd, seed=1)
    want = run(q, k, v, e, hq, hkv, hd, causal=True)
    w = v.clone()
    w[:e[1], 3] = math.inf
    scratch = torch.empty(api.op_attention_sequences_scratch_bytes(hd), dtype=torch.uint8, device="cuda")
    api.debug_op_fault(False, wait_limit_ns=1_000_000)
    try:
        got = api.op_attention_packed(q, k, w, ints(e), hq, hkv, hd, causal=True, scratch=scratch)
        assert api.op_status(api.OP_ATTENTION_PACKED, scratch) == api.VLA_OK
    finally:
        api.debug_op_fault(False)
    assert torch.equal(got[e[1]:], want[e[1]:])
    heads = got[:e[1]].view(-1, hq, hd)[:, :hq // hkv]
    assert bool((heads[:, :, 3] == math.inf).all())
    heads[:, :, 3] = 0
    assert bool(heads.isfinite().all())


def want_of(q, k, v, hq, hkv, hd, how, prefix=0):
    """(finite part, its tolerance, NaN seen, +inf seen, -inf seen) of one sequence, 64 bits, each [nq, hq*hd].  Every probability is above 0 here."""
    import torch
    o, tol = ref.attend(q, k, torch.where(v.isfinite(), v, torch.zeros_like(v)), hq, hkv, hd, prefix=prefix, **how)
    nq, nk = q.shape[0], k.shape[0]
    far = torch.arange(nk - nq, nk, device=q.device)[:, None] - torch.arange(nk, device=q.device)[None]
    seen = torch.ones(nq, nk, dtype=torch.bool, device=q.device)
    if how.get("causal"):
        seen = far >= 0
        if how.get("window"):
            seen &= far < how["window"]
        seen |= (torch.arange(nk, device=q.device) < prefix)[None]
    kinds = [(seen.float() @ x.float() > 0).view(nq, hkv, 1, hd).expand(nq, hkv, hq // hkv, hd).reshape(nq, hq * hd) for x in (v.isnan(), v == math.inf, v == -math.inf)]
    return o, tol, *kinds


def check_kinds(got, want):
    o, tol, nan, up, down = want
    bad = nan | (up & down)
    assert bool(got[bad].isnan().all())
    assert bool((got[up & ~bad] == math.inf).all() and (got[down & ~bad] == -math.inf).all())
    fine = ~(nan | up | down)
    assert bool(got[fine].isfinite().all()) and bool(((got.double() - o).abs() <= tol)[fine].all())


def spoil(v, seed, share):
    """A share of the values becomes NaN, inf or -inf."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    hit, kind = torch.rand(v.shape, device="cuda", generator=g) < share, torch.randint(0, 3, v.shape, device="cuda", generator=g)
    kinds = torch.tensor([math.nan, math.inf, -math.inf], device="cuda").bfloat16()
    return torch.where(hit, kinds[kind], v)


HOW = [dict(), dict(causal=True), dict(causal=True, window=40), dict(causal=True, window=200, prefix=100), dict(causal=True, cap=8.0), dict(causal=True, prefix=300)]


@pytest.mark.parametrize("lengths", [[37], [300, 140], [40] * 20, [1800, 1100], [3000, 7]], ids=str)
@pytest.mark.parametrize("hq,hkv,hd", [(8, 2, 64), (2, 2, 128), (3, 1, 72), (2, 1, 256), (4, 2, 8), (1, 1, 136)])
@pytest.mark.parametrize("how", HOW, ids=str)
@pytest.mark.parametrize("share", [1e-4, 1e-2, 1.0])
def test_each_column_is_what_its_rows_see(lengths, hq, hkv, hd, how, share):
    e, how = ends(lengths), dict(how)
    prefix = how.pop("prefix", 0)
    q, k, v = make(e[-1], hq, hkv, hd, seed=e[-1] + hd)
    v = spoil(v, e[-1], share)
    got = run(0.3 * q, k, v, e, hq, hkv, hd, prefix=[min(prefix, n) for n in lengths] if prefix else None, **how)
    for a, b in zip(e, e[1:]):
        check_kinds(got[a:b], want_of(0.3 * q[a:b], k[a:b], v[a:b], hq, hkv, hd, how, min(prefix, b - a)))


@pytest.mark.parametrize("new,keys", [([1], [2000]), ([3, 1, 30], [700, 1, 5000]), ([200], [3000]), ([1] * 40, [333] * 40)], ids=str)
@pytest.mark.parametrize("hq,hkv,hd", [(8, 2, 128), (4, 1, 256), (6, 2, 64)])
@pytest.mark.parametrize("share", [1e-4, 1e-2, 1.0])
def test_over_pages(new, keys, hq, hkv, hd, share):
    from test_gpu_paged_attention import Cache, run as run_paged
    eq, ek = ends(new), ends(keys)
    q, k, v = make(eq[-1], hq, hkv, hd, seed=hd, keys=ek[-1])
    q, v = 0.3 * q, spoil(v, 3, share)
    c = Cache(keys, hkv, hd, 24, seed=1)
    c.fill_fast(k, v)
    for how in (dict(causal=True), dict(causal=True, window=90)):
        got = run_paged(c, q, eq, hq, hkv, hd, **how)
        for s in range(len(new)):
            rows, at = slice(eq[s], eq[s + 1]), slice(ek[s], ek[s + 1])
            check_kinds(got[rows], want_of(q[rows], k[at], v[at], hq, hkv, hd, how))


@pytest.mark.parametrize("value,everywhere", [(math.nan, False), (math.nan, True), (math.inf, False)])
@pytest.mark.parametrize("hq,hkv,hd", [(8, 4, 128), (4, 2, 64), (4, 1, 256)])
def test_a_value_that_rows_see_costs_a_look_at_the_values(hq, hkv, hd, value, everywhere):
    """A value that rightly makes thousands of rows NaN or infinite: no row has to be worked out key by key for it (a thousand times as long as the call itself)."""
    import torch
    from paper_2609_22335_b200 import api
    n = 4096
    q, k, v = make(n, hq, hkv, hd, seed=2)
    off, scratch, w = ints([0, n]), torch.empty(api.op_attention_sequences_scratch_bytes(hd), dtype=torch.uint8, device="cuda"), v.clone()
    w[slice(None) if everywhere else 0, hd // 2] = value
    for causal in (False, True):
        took = []
        for x in (v, w):
            best = math.inf
            for _ in range(4):
                a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
                a.record()
                api.op_attention_packed(q, k, x, off, hq, hkv, hd, causal=causal, scratch=scratch)
                b.record()
                torch.cuda.synchronize()
                best = min(best, a.elapsed_time(b))
            took.append(best)
        assert took[1] < 40 * took[0], took


@pytest.mark.parametrize("new,keys", [(1, 700), (1, 3000), (1, 20000), (40, 3000), (600, 6000)])
@pytest.mark.parametrize("hq,hkv,hd", [(8, 2, 64), (4, 1, 256)])
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_a_key_without_any_weight_is_seen_all_the_same(new, keys, hq, hkv, hd, value):
    """Its probability underflows, and 0 times a value that is not finite is NaN, whichever part of the keys it lies in."""
    import torch
    q, k, v = make(new, hq, hkv, hd, seed=5, keys=keys)
    q[:, 0::hd], k[:, 0::hd] = 1.0, -400.0
    k[:keys // 5, 0::hd] = 400.0
    v[keys - 3, 5] = value
    got = run(q, k, v, [0, new], hq, hkv, hd, ends_k=[0, keys], scale=1.0).view(new, hq, hd)[:, :hq // hkv]
    assert not bool(got[:, :, 5].isfinite().any()) and bool(got[:, :, :5].isfinite().all()) and bool(got[:, :, 6:].isfinite().all())
