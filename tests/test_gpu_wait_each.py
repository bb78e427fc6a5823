"""The operators' limit is one of each wait, not of the call: calls that run several times as long as a wait may take succeed."""
import pytest

pytestmark = pytest.mark.gpu

LIMIT_US = 500                                  # a wait for operands or sums takes some microseconds


@pytest.fixture(autouse=True)
def memory_back():
    yield
    import torch
    torch.cuda.empty_cache()


def runs_longer_than_a_wait_may(call, status):
    import torch
    from paper_2609_22335_b200 import api
    want = call()
    assert status() == api.VLA_OK
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    api.debug_op_fault(False, wait_limit_ns=LIMIT_US * 1000)
    try:
        e0.record()
        got = call()
        e1.record()
        assert status() == api.VLA_OK
    finally:
        api.debug_op_fault(False)
    torch.cuda.synchronize()
    assert e0.elapsed_time(e1) * 1e3 > 2 * LIMIT_US and torch.equal(got, want)


def test_linear():
    import torch
    from paper_2609_22335_b200 import api
    a, w = (torch.randn(16384, 8192, device="cuda").to(torch.bfloat16) for _ in range(2))
    runs_longer_than_a_wait_may(lambda: api.op_linear(a, w, out_bf16=True), lambda: api.op_status(api.OP_LINEAR))
    narrow = torch.randn(2 ** 20, 8192, device="cuda").to(torch.bfloat16)            # (a CTA a tile of few rows: 17 GB of weights)
    runs_longer_than_a_wait_may(lambda: api.op_linear(a[:16], narrow, out_bf16=True), lambda: api.op_status(api.OP_LINEAR))


def test_attention():
    """1024 queries of 32 heads: a tile a CTA, over 131072 keys."""
    import torch
    from paper_2609_22335_b200 import api
    q, k, v = (torch.randn(t, h * 128, device="cuda").to(torch.bfloat16) for t, h in ((1024, 32), (131072, 8), (131072, 8)))
    scratch = torch.empty(api.op_attention_scratch_bytes(131072, 8, 128), dtype=torch.uint8, device="cuda")
    runs_longer_than_a_wait_may(lambda: api.op_attention(q, k, v, 32, 8, 128, scratch=scratch), lambda: api.op_status(api.OP_ATTENTION, scratch))


@pytest.mark.parametrize("rows,n,k,experts", [(16384, 16384, 16384, 0), (16384, 16384, 8192, 4), (16, 2 ** 20, 8192, 0), (64, 2 ** 18, 8192, 4)])
def test_layers_by_blocks(rows, n, k, experts):
    """Pairs and operands exchanged, of one matrix and by expert."""
    import torch
    from paper_2609_22335_b200 import api
    lead, kb = (experts,) if experts else (), k // 128
    a = torch.randn(rows, k, device="cuda").to(torch.float8_e4m3fn)
    w = torch.empty(*lead, n, k, device="cuda", dtype=torch.float8_e4m3fn)
    for part in w.view(-1, 2 ** 14, k):
        part.copy_(torch.randn(2 ** 14, k, device="cuda"))
    sa, sw = torch.rand(rows, kb, device="cuda"), torch.rand(*lead, n // 128, kb, device="cuda")
    if not experts:
        runs_longer_than_a_wait_may(lambda: api.op_linear_scaled(a, sa, w, sw, out_bf16=True), lambda: api.op_status(api.OP_LINEAR_SCALED))
        return
    offsets = torch.arange(experts + 1, dtype=torch.int32, device="cuda") * (rows // experts)
    runs_longer_than_a_wait_may(lambda: api.op_linear_grouped_scaled(a, sa, w, sw, offsets, out_bf16=True), lambda: api.op_status(api.OP_LINEAR_GROUPED_SCALED))
    b, x = a.to(torch.bfloat16), w.to(torch.bfloat16)
    runs_longer_than_a_wait_may(lambda: api.op_linear_grouped(b, x, offsets, out_bf16=True), lambda: api.op_status(api.OP_LINEAR_GROUPED))
