"""Where attention of several sequences says that a wait ran out."""
import pytest

import test_sequences_refusals as refusals
from test_sequences_refusals import lib, mem      # noqa: F401  (fixtures)

from paper_2609_22335_b200 import api


@pytest.mark.parametrize("paged", [False, True])
def test_whose_word_is_one_of_two(lib, mem, paged):      # noqa: F811
    name = "vla_op_attention_paged" if paged else "vla_op_attention_packed"
    fine = refusals.good(mem[0], paged)
    for status in (-1, 1, 2, api.OP_ATTENTION_PACKED, api.OP_ATTENTION_PAGED, 10, 1 << 30):
        assert refusals.call(lib, name, {**fine, "reserved": status}) == api.VLA_ERR_INVALID
    for status in (0, api.OP_ATTENTION_SHORT):           # (past all other questions: scratch that is too small)
        assert refusals.call(lib, name, {**fine, "scratch_bytes": 1000, "reserved": status}) == api.VLA_ERR_NOMEM


@pytest.mark.gpu
@pytest.mark.parametrize("keys", [300, 700, 5000])
def test_a_call_that_makes_its_own_scratch_can_be_asked(keys):
    """Its scratch is gone when it returns; a call with scratch of the caller's own leaves the device's word alone."""
    import torch
    r = lambda *s: torch.randn(*s, device="cuda").bfloat16()      # noqa: E731
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")      # noqa: E731
    q, k, v = r(keys, 128), r(keys, 64), r(keys, 64)
    pages = -(-keys // 8)
    kc, vc, table = r(pages, 8, 64), r(pages, 8, 64), torch.arange(pages, dtype=torch.int32, device="cuda")[None].contiguous()
    own = torch.empty(api.op_attention_sequences_scratch_bytes(64), dtype=torch.uint8, device="cuda")
    calls = [lambda **kw: api.op_attention_packed(q, k, v, ints([0, keys]), 2, 1, 64, **kw), lambda **kw: api.op_attention_paged(q[:1], kc, vc, table, ints([keys]), ints([0, 1]), 2, 1, 64, **kw)]
    for call, op in zip(calls, (api.OP_ATTENTION_PACKED, api.OP_ATTENTION_PAGED)):
        want = call()
        assert api.op_status(api.OP_ATTENTION_SHORT) == api.VLA_OK
        api.debug_op_fault(True, wait_limit_ns=1_000_000)
        try:
            call(scratch=own)
            assert api.op_status(op, own) == api.VLA_ERR_TIMEOUT and api.op_status(api.OP_ATTENTION_SHORT) == api.VLA_OK
            call()
            assert api.op_status(api.OP_ATTENTION_SHORT) == api.VLA_ERR_TIMEOUT
        finally:
            api.debug_op_fault(False)
        assert torch.equal(call(scratch=own), want)
        assert api.op_status(op, own) == api.VLA_OK and api.op_status(api.OP_ATTENTION_SHORT) == api.VLA_ERR_TIMEOUT
        assert torch.equal(call(), want) and api.op_status(api.OP_ATTENTION_SHORT) == api.VLA_OK
