"""Attention over a paged cache, and the rows that fill it, against the definition in 64 bits (tests/sequences_reference.py has the tolerance)."""
import math

import pytest

import sequences_reference as ref
from test_gpu_packed_attention import ends, ints, make, run as run_packed, slopes_of

pytestmark = pytest.mark.gpu


class Cache:
    """Pages in a random order; rows that belong to nobody, and pages too, are NaN."""

    def __init__(self, keys, hkv, hd, page, seed, joined=False, spare=3):
        import torch
        g = torch.Generator().manual_seed(seed)
        need = [-(-n // page) for n in keys]
        self.n, width = sum(need) + spare, hkv * hd
        order = torch.randperm(self.n, generator=g).tolist()
        self.table = torch.full((len(keys), max(need + [1])), -1, dtype=torch.int32)
        for i, x in enumerate(need):
            self.table[i, :x] = torch.tensor(order[:x], dtype=torch.int32)
            del order[:x]
        if joined:                              # keys and values of a page side by side in one tensor, with a gap behind each row
            both = torch.full((self.n, 2, page, width + 8), math.nan, dtype=torch.bfloat16, device="cuda")
            self.k, self.v = both[:, 0, :, :width], both[:, 1, :, :width]
        else:
            self.k, self.v = (torch.full((self.n, page, width), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.keys, self.page, self.pages, self.lengths = keys, page, self.table.cuda(), ints(keys)

    def fill(self, k, v):
        """The rows of all sequences, one behind another."""
        at = 0
        for s, n in enumerate(self.keys):
            for j in range(n):
                where = int(self.table[s, j // self.page]), j % self.page
                self.k[where], self.v[where] = k[at + j], v[at + j]
            at += n

    def fill_fast(self, k, v):
        import torch
        seq = torch.cat([torch.full((n,), s) for s, n in enumerate(self.keys)]).long()
        pos = torch.cat([torch.arange(n) for n in self.keys])
        where = self.table[seq, pos // self.page].long().cuda(), (pos % self.page).cuda()
        self.k[where], self.v[where] = k, v


def run(c, q, ends_q, hq, hkv, hd, prefix=None, **kw):
    import torch
    from paper_2609_22335_b200 import api
    scratch = torch.empty(api.op_attention_sequences_scratch_bytes(hd), dtype=torch.uint8, device="cuda")
    got = api.op_attention_paged(q, c.k, c.v, c.pages, c.lengths, ints(ends_q), hq, hkv, hd, prefix=None if prefix is None else ints(prefix), scratch=scratch, **kw)
    assert api.op_status(api.OP_ATTENTION_PAGED, scratch) == api.VLA_OK
    return got


CASES = [([1], [1]), ([1], [2000]), ([1] * 8, [1, 7, 64, 65, 128, 129, 1000, 3]), ([1] * 40, [200] * 40), ([5, 0, 130], [5, 40, 900]), ([300], [1300]), ([2, 3], [5000, 64]), ([64] * 4, [64, 80, 256, 700])]


@pytest.mark.parametrize("new,keys", CASES, ids=lambda x: str(x)[:40])
@pytest.mark.parametrize("hq,hkv,hd", [(8, 2, 64), (8, 2, 128), (8, 1, 256), (15, 5, 72), (4, 4, 32)])
@pytest.mark.parametrize("page", [8, 16, 24, 64, 256])
def test_against_64_bits(new, keys, hq, hkv, hd, page):
    import torch
    eq, ek = ends(new), ends(keys)
    q, k, v = make(eq[-1], hq, hkv, hd, seed=page + hd, keys=ek[-1])
    c = Cache(keys, hkv, hd, page, seed=page, joined=page == 16)
    c.fill_fast(k, v)
    ref.check(run(c, q, eq, hq, hkv, hd), ref.packed(q, k, v, eq, ek, hq, hkv, hd, causal=True))
    ref.check(run(c, q, eq, hq, hkv, hd, causal=False), ref.packed(q, k, v, eq, ek, hq, hkv, hd))


@pytest.mark.parametrize("new,keys", [([1] * 3, [1500, 10, 260]), ([70, 3], [400, 1000])], ids=str)
@pytest.mark.parametrize("hq,hkv,hd", [(8, 2, 128), (4, 1, 256)])
@pytest.mark.parametrize("how", [dict(window=100), dict(window=100, prefix=30, cap=20.0), dict(slopes=True), dict(prefix=200, slopes=True, cap=50.0), dict(scale=0.5)], ids=str)
def test_masks_caps_and_distances(new, keys, hq, hkv, hd, how):
    eq, ek, how = ends(new), ends(keys), dict(how)
    if how.get("slopes"):
        how["slopes"] = slopes_of(hq)
    if "prefix" in how:
        how["prefix"] = [min(how["prefix"], n - 2) for n in keys]
    q, k, v = make(eq[-1], hq, hkv, hd, seed=2, keys=ek[-1])
    c = Cache(keys, hkv, hd, 16, seed=1)
    c.fill_fast(k, v)
    ref.check(run(c, q, eq, hq, hkv, hd, **how), ref.packed(q, k, v, eq, ek, hq, hkv, hd, causal=True, **how))


def test_pages_that_do_not_exist_are_zeros_and_long_lengths_are_the_tables():
    import torch
    hq, hkv, hd, page, keys = 4, 2, 64, 16, [100, 64]
    eq, ek = [0, 1, 4], ends(keys)
    q, k, v = make(4, hq, hkv, hd, seed=3, keys=ek[-1])
    c = Cache(keys, hkv, hd, page, seed=2)
    c.fill_fast(k, v)
    want = [k.clone(), v.clone()]
    for s, slot, entry in ((0, 2, -1), (1, 1, c.n), (0, 0, -2147483648), (1, 3, 2147483647)):
        c.pages[s, slot] = entry
        for x in want:
            x[ek[s] + slot * page:ek[s] + slot * page + page] = 0
    c.pages[1, 4:] = 0
    ref.check(run(c, q, eq, hq, hkv, hd), ref.packed(q, *want, eq, ek, hq, hkv, hd, causal=True))
    # lengths beyond the table, and below 0
    c = Cache([112, 112], hkv, hd, page, seed=2)
    k, v = make(1, hq, hkv, hd, seed=4, keys=224)[1:]
    c.fill_fast(k, v)
    c.lengths.copy_(ints([1 << 30, -5]))
    ref.check(run(c, q, eq, hq, hkv, hd), ref.packed(q, k, v, eq, [0, 112, 112], hq, hkv, hd, causal=True))


@pytest.mark.parametrize("page", [1, 8, 17, 64])
@pytest.mark.parametrize("hkv,hd", [(1, 8), (2, 64), (8, 128), (40, 72)])
@pytest.mark.parametrize("new,keys", [([1], [1]), ([1] * 70, [90] * 70), ([3, 0, 200, 1], [3, 50, 333, 64])], ids=lambda x: str(x)[:30])
def test_rows_into_pages(page, hkv, hd, new, keys):
    """Each row to its place, bit for bit (NaN and all), and nothing else touched."""
    import torch
    from paper_2609_22335_b200 import api
    e = ends(new, first=2)
    rows = torch.randint(-32768, 32768, (e[-1] + 3, 2 * hkv * hd + 8), dtype=torch.int16, device="cuda").view(torch.bfloat16)
    k, v = rows[:, :hkv * hd], rows[:, hkv * hd:2 * hkv * hd]
    c, want = (Cache(keys, hkv, hd, page, seed=5, joined=True) for _ in range(2))
    api.op_cache_store(k, v, c.k, c.v, c.pages, c.lengths, ints(e))
    for s, n in enumerate(new):
        for j in range(n):
            p = keys[s] - n + j
            at = int(want.table[s, p // page]), p % page
            want.k[at], want.v[at] = k[e[s] + j], v[e[s] + j]
    bits = lambda x: x.contiguous().view(torch.int16)      # noqa: E731
    assert torch.equal(bits(c.k), bits(want.k)) and torch.equal(bits(c.v), bits(want.v))


def test_rows_without_a_place_are_left_out():
    import torch
    from paper_2609_22335_b200 import api
    k = torch.ones(6, 16, dtype=torch.bfloat16, device="cuda")
    kc, vc = (torch.zeros(4, 8, 16, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    # two rows of a sequence of one token; a length behind the table; a page of -1; a page beyond the cache
    api.op_cache_store(k, 2 * k, kc, vc, ints([[0, 1], [0, 1], [-1, 1], [4, 2]]), ints([1, 17, 3, 8]), ints([0, 2, 3, 4, 6]))
    want = torch.zeros_like(kc)
    want[0, 0] = 1
    assert torch.equal(kc, want) and torch.equal(vc, 2 * want)


def test_a_layer_step_by_step_and_all_at_once():
    """Projection, head norms with rotation, rows into pages, attention over them, output projection onto the stream: a prefix, then chunk and tokens, against
    the whole sequences at once through the packed attention."""
    import torch
    from paper_2609_22335_b200 import api
    d, hq, hkv, hd, page = 512, 8, 2, 64, 16
    lengths, cuts = [150, 37, 260], [(100, 30, 200), (149, 36, 203), (150, 37, 260)]
    g = torch.Generator(device="cuda").manual_seed(11)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)      # noqa: E731
    x = [r(n, d).bfloat16() for n in lengths]
    w, b = (r((hq + 2 * hkv) * hd, d) / d ** 0.5).bfloat16(), 0.1 * r((hq + 2 * hkv) * hd)
    wo, bo, gain = (r(d, hq * hd) / (hq * hd) ** 0.5).bfloat16(), 0.1 * r(d), 1 + 0.1 * r(hd)

    def project(rows, pos):
        y = api.op_linear_bias(rows, w, bias=b, out_bf16=True)
        q, k = api.op_qk_norm_rope(y[:, :hq * hd], y[:, hq * hd:(hq + hkv) * hd], hq, hkv, hd, gq=gain, gk=gain, pos=pos)
        return q, k, y[:, (hq + hkv) * hd:]

    rows = torch.cat(x)
    e = ends(lengths)
    q, k, v = project(rows, torch.cat([torch.arange(n, dtype=torch.int32, device="cuda") for n in lengths]))
    whole = api.op_linear_bias(api.op_attention_packed(q, k, v, ints(e), hq, hkv, hd, causal=True), wo, bias=bo, residual=rows, out_bf16=True)
    ref.check(api.op_attention_packed(q, k, v, ints(e), hq, hkv, hd, causal=True), ref.packed(q, k, v, e, e, hq, hkv, hd, causal=True))
    c = Cache(lengths, hkv, hd, page, seed=6)
    got, done = [torch.zeros_like(y) for y in x], (0, 0, 0)
    for cut in cuts:
        new = [b_ - a_ for a_, b_ in zip(done, cut)]
        part = torch.cat([y[a_:b_] for y, a_, b_ in zip(x, done, cut)])
        q, k, v = project(part, torch.cat([torch.arange(a_, b_, dtype=torch.int32, device="cuda") for a_, b_ in zip(done, cut)]))
        off, have = ints(ends(new)), ints(list(cut))
        api.op_cache_store(k, v, c.k, c.v, c.pages, have, off)
        y = api.op_attention_paged(q, c.k, c.v, c.pages, have, off, hq, hkv, hd)
        y = api.op_linear_bias(y, wo, bias=bo, residual=part, out_bf16=True)
        for s, (a_, b_) in enumerate(zip(done, cut)):
            got[s][a_:b_] = y[ends(new)[s]:ends(new)[s + 1]]
        done = cut
    # The attention's rows may differ by what each may be off, 2^-7 (|o| + A), A some times |o|; the projection averages over 512 of them.
    off = (torch.cat(got).double() - whole.double()).norm() / whole.double().norm()
    assert float(off) < 4 * 2.0 ** -8


def test_one_captured_step_serves_growing_sequences():
    """Store and attention in one graph: lengths, offsets and pages are read when it runs."""
    import torch
    from paper_2609_22335_b200 import api
    hq, hkv, hd, page = 8, 2, 128, 16
    keys = [40, 100, 1]
    c = Cache([64, 128, 16], hkv, hd, page, seed=7)
    total = ends([64, 128, 16])
    _, k, v = make(1, hq, hkv, hd, seed=12, keys=total[-1])
    q = make(3, hq, hkv, hd, seed=13)[0]
    c.fill_fast(k, v)
    off, have = ints([0, 1, 2, 3]), ints(keys)
    new_k, new_v = k[:3].clone(), v[:3].clone()
    side = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        api.op_cache_store(new_k, new_v, c.k, c.v, c.pages, have, off, stream=side)
        got = api.op_attention_paged(q, c.k, c.v, c.pages, have, off, hq, hkv, hd, stream=side)
    for step in range(4):
        now = [n + step for n in keys]
        have.copy_(ints(now))
        new_k.copy_(make(1, hq, hkv, hd, seed=20 + step, keys=3)[1])
        for s, n in enumerate(now):
            k[total[s] + n - 1], v[total[s] + n - 1] = new_k[s], new_v[s]
        g.replay()
        torch.cuda.synchronize()
        rows = lambda x: torch.cat([x[total[s]:total[s] + n] for s, n in enumerate(now)])      # noqa: E731
        ref.check(got, ref.packed(q, rows(k), rows(v), [0, 1, 2, 3], ends(now), hq, hkv, hd, causal=True))


def test_places_far_into_a_large_cache():
    """Elements of the cache beyond 2^31 and bytes beyond 2^32: pages at its end are written and read."""
    import torch
    from paper_2609_22335_b200 import api
    hq, hkv, hd, page = 8, 8, 128, 64
    n = 2 ** 31 // (page * hkv * hd) + 40
    kc, vc = (torch.zeros(n, page, hkv * hd, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q, k, v = make(2, hq, hkv, hd, seed=14, keys=150)
    pages = ints([[n - 1, n - 3, n - 2], [n - 9, 0, 0]])
    off, have = ints([0, 140, 150]), ints([140, 10])
    api.op_cache_store(k, v, kc, vc, pages, have, off)
    got = api.op_attention_paged(q, kc, vc, pages, have, ints([0, 1, 2]), hq, hkv, hd)
    ref.check(got, ref.packed(q, k, v, [0, 1, 2], [0, 140, 150], hq, hkv, hd, causal=True))
