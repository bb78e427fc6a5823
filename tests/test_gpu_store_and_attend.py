"""Rows into pages and the attention over them agree on which token a row is."""
import pytest

import sequences_reference as ref
from test_gpu_packed_attention import ends, ints, make
from test_gpu_paged_attention import Cache, run as run_paged

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("offsets,rows", [([0, 3, 9], [3, 2]), ([0, 3, 5], [3, 2]), ([-4, 3, 5], [3, 2]), ([0, 5, 7], [5, 0]), ([0, 9, 9], [5, 0]), ([0, 5, 2 ** 31 - 1], [5, 0])], ids=str)
def test_offsets_beyond_the_rows_are_their_end(offsets, rows):
    """Five new rows: an offset in front of the first or behind the last counts as the nearer end to both."""
    from paper_2609_22335_b200 import api
    hq, hkv, hd, page, keys = 4, 2, 64, 16, [50, 33]
    ek, eq = ends(keys), ends(rows)
    q, k, v = make(5, hq, hkv, hd, seed=1, keys=ek[-1])
    c = Cache(keys, hkv, hd, page, seed=2)
    c.fill_fast(k, v)
    new = [ek[s] + keys[s] - n + i for s, n in enumerate(rows) for i in range(n)]
    for s, n in enumerate(rows):
        for p in range(keys[s] - n, keys[s]):
            c.k[int(c.table[s, p // page]), p % page] = c.v[int(c.table[s, p // page]), p % page] = 0
    api.op_cache_store(k[new], v[new], c.k, c.v, c.pages, c.lengths, ints(offsets))
    ref.check(run_paged(c, q, offsets, hq, hkv, hd), ref.packed(q, k, v, eq, ek, hq, hkv, hd, causal=True))
