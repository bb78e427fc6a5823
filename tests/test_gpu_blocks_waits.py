"""Waits that run out in every kernel of the linear layers by blocks (which shapes take which: test_blocks_reach.py): the call returns, its status says so,
and the next call is right.  A wait is made to run out by loads that are never issued."""
import pytest

from test_gpu_linear_blocks import eight_bit, gen, near, scaled, sort_of

pytestmark = pytest.mark.gpu

# (m, n, k): operands exchanged at every height, alone and with a shared K; narrow tiles with K shared by 1, 2 and 4; middle, wide, pairs
SCALED = [(1, 64, 128), (1, 64, 1024), (1, 64, 2048), (1, 64, 4096), (160, 4000, 128), (20, 11008, 1024), (33, 2000, 8192), (33, 18000, 256), (33, 11008, 2048), (64, 6000, 4096),
          (257, 64, 128), (257, 64, 2048), (257, 64, 4096), (257, 96, 128), (130, 11008, 128), (520, 4000, 1024)]
# (rows of each expert, n, k): the same by expert, in bf16 and in 8 bits
GROUPED = [([1], 64, 128), ([1], 64, 512), ([1], 64, 1024), ([1], 64, 2048), ([1], 64, 4096), ([33], 8000, 128), ([160], 3000, 128), ([200, 0, 300, 100], 400, 1024), ([200, 0, 300, 100], 400, 512),
           ([16], 11008, 4096), ([10, 10], 11008, 8192), ([40, 0, 9, 31], 8000, 128), ([80], 4000, 512), ([80], 4000, 1024), ([100, 0, 57, 100], 1000, 1024), ([100, 0, 57, 100], 1000, 2048),
           ([257], 64, 128), ([257], 64, 1024), ([257], 64, 2048), ([257], 64, 4096), ([80], 4000, 128), ([257], 96, 128), ([16, 17], 11008, 128), ([60, 0, 30, 40], 6000, 128),
           ([80], 11008, 512), ([80], 11008, 1024)]


def runs_out(call, status, right):
    import torch
    from paper_2609_22335_b200 import api
    for how in (1, 2):
        api.debug_op_fault(how, wait_limit_ns=1_000_000)          # 1 ms
        try:
            for _ in range(3):
                call()
                assert status() == api.VLA_ERR_TIMEOUT
        finally:
            api.debug_op_fault(0)
        got = call()
        assert status() == api.VLA_OK
        right(got)
    torch.cuda.synchronize()


@pytest.mark.parametrize("m,n,k", SCALED)
def test_scaled(m, n, k):
    from paper_2609_22335_b200 import api
    a, sa = eight_bit(1, m, k, 1)
    w, sw = eight_bit(128, n, k, 2)
    runs_out(lambda: api.op_linear_scaled(a, sa, w, sw), lambda: api.op_status(api.OP_LINEAR_SCALED), lambda y: near(y, scaled(a, sa, 1), scaled(w, sw, 128), 0, True))


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("counts,n,k", GROUPED)
def test_grouped(counts, n, k, f8):
    import torch
    from paper_2609_22335_b200 import api
    offsets, t = sort_of(counts)
    ends, e = offsets.tolist(), len(counts)
    if f8:
        a, sa = eight_bit(1, t, k, 1)
        w, sw = eight_bit(128, n, k, 2, groups=e)
        call, op = (lambda: api.op_linear_grouped_scaled(a, sa, w, sw, offsets)), api.OP_LINEAR_GROUPED_SCALED
        of = lambda i, lo, hi: (scaled(a[lo:hi], sa[lo:hi], 1), scaled(w[i], sw[i], 128))     # noqa: E731
    else:
        a = torch.randn(t, k, device="cuda", generator=gen(1)).to(torch.bfloat16)
        w = (0.1 * torch.randn(e, n, k, device="cuda", generator=gen(2))).to(torch.bfloat16)
        call, op = (lambda: api.op_linear_grouped(a, w, offsets)), api.OP_LINEAR_GROUPED
        of = lambda i, lo, hi: (a[lo:hi].double(), w[i].double())                              # noqa: E731

    def right(y):
        for i, (lo, hi) in enumerate(zip(ends, ends[1:])):
            near(y[lo:hi], *of(i, lo, hi), 0, f8)
    runs_out(call, lambda: api.op_status(op), right)
