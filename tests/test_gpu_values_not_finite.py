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
