"""What the linear layers by blocks promise whatever kernel a shape takes (test_blocks_reach.py: these shapes take all of them): results at any alignment, nothing
of another expert's or of nobody's rows, and the error of sums that are cut as they are.

Tolerance of bf16 operands, relative to sum_k |a| |w|: an MMA of 16 products that truncates each and the running sum to 24 bits is off by less than
17 * 2^-23; a sum is cut after two blocks of 64 at most, eight MMAs, 136 * 2^-23; adding up at most ceil(k / 64) parts, and those of two sets
and eight CTAs, rounds by 2^-24 each."""
import pytest

from test_gpu_blocks_waits import GROUPED, SCALED
from test_gpu_linear_blocks import eight_bit, gen, near, scaled, sort_of

pytestmark = pytest.mark.gpu

LEAD, REST = 1, 2                               # rows of nobody in front and behind
LONG = [([1], 64, 4096), ([80], 6000, 2048), ([200], 800, 4096), ([800], 1504, 2048), ([257], 64, 8192), ([512], 400, 2048), ([33], 2000, 8192), ([80], 4000, 4096), ([500, 0, 300], 4000, 2048),
        ([800], 3000, 2048), ([300, 0, 212], 4096, 4096)]


def grouped_case(counts, n, k, f8, lead=0, rest=0):
    """(a, its scales, w, its scales, offsets, call(out32 pointer, out16 pointer))"""
    import torch
    from paper_2609_22335_b200 import api
    offsets, t = sort_of(counts, lead, rest)
    e, lib = len(counts), api.load_library()
    if f8:
        a, sa = eight_bit(1, t, k, 1)
        w, sw = eight_bit(128, n, k, 2, groups=e)
        call = lambda p32, p16: lib.vla_op_linear_grouped_scaled(a.data_ptr(), sa.data_ptr(), w.data_ptr(), sw.data_ptr(), offsets.data_ptr(), p32, p16, t, n, k, e, 0, None)  # noqa: E731
        return a, sa, w, sw, offsets, call
    a = torch.randn(t, k, device="cuda", generator=gen(1)).to(torch.bfloat16)
    w = (0.1 * torch.randn(e, n, k, device="cuda", generator=gen(2))).to(torch.bfloat16)
    return a, None, w, None, offsets, lambda p32, p16: lib.vla_op_linear_grouped(a.data_ptr(), w.data_ptr(), offsets.data_ptr(), p32, p16, t, n, k, e, 0, None)


def at_any_alignment(m, n, call):
    """Both results from addresses of which one, both or none allow wide stores, against those from aligned ones; nothing around them is touched."""
    import torch
    from paper_2609_22335_b200 import api
    want = None
    for off32, off16 in ((0, 0), (1, 0), (0, 1), (2, 2), (4, 4), (3, 2)):
        b32, b16 = torch.full((m * n + 8,), 7.0, device="cuda"), torch.full((m * n + 8,), 7.0, device="cuda", dtype=torch.bfloat16)
        o32, o16 = b32[off32:off32 + m * n], b16[off16:off16 + m * n]
        assert call(o32.data_ptr(), o16.data_ptr()) == api.VLA_OK
        torch.cuda.synchronize()
        if want is None:
            want = o32.clone()
            assert bool(torch.isfinite(want).all())
        assert torch.equal(o32, want) and torch.equal(o16, want.to(torch.bfloat16))
        assert all(bool((b[:o] == 7).all()) and bool((b[o + m * n:] == 7).all()) for b, o in ((b32, off32), (b16, off16)))


@pytest.mark.parametrize("m,n,k", SCALED)
def test_scaled_results_at_any_alignment(m, n, k):
    from paper_2609_22335_b200 import api
    a, sa = eight_bit(1, m, k, 1)
    w, sw = eight_bit(128, n, k, 2)
    lib = api.load_library()
    at_any_alignment(m, n, lambda p32, p16: lib.vla_op_linear_scaled(a.data_ptr(), sa.data_ptr(), w.data_ptr(), sw.data_ptr(), p32, p16, m, n, k, 0, None))


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("counts,n,k", GROUPED)
def test_grouped_results_at_any_alignment(counts, n, k, f8):
    *held, call = grouped_case(counts, n, k, f8)
    at_any_alignment(sum(counts), n, call)


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("counts,n,k", GROUPED)
def test_nothing_leaks_from_other_experts_or_from_nobodys_rows(counts, n, k, f8):
    """NaN in nobody's rows, and in every second expert's rows and weights with rows or without."""
    import torch
    from paper_2609_22335_b200 import api
    a, sa, w, sw, offsets, call = grouped_case(counts, n, k, f8, LEAD, REST)
    ends, bad = offsets.tolist(), [e for e in range(len(counts)) if e % 2 == 1]
    A = scaled(a, sa, 1) if f8 else a.double()
    nans = (a.view(torch.uint8), w.view(torch.uint8), 0x7F) if f8 else (a, w, float("nan"))
    for rows in [slice(0, LEAD), slice(ends[-1], None)] + [slice(ends[e], ends[e + 1]) for e in bad]:
        nans[0][rows] = nans[2]
    for e in bad:
        nans[1][e] = nans[2]
    out = torch.full((ends[-1] + REST, n), 7.0, device="cuda")
    assert call(out.data_ptr(), None) == api.VLA_OK
    torch.cuda.synchronize()
    assert bool((out[:LEAD] == 7).all()) and bool((out[ends[-1]:] == 7).all())
    for e, (lo, hi) in enumerate(zip(ends, ends[1:])):
        if e in bad:
            assert bool(torch.isnan(out[lo:hi]).all())
        else:
            near(out[lo:hi], A[lo:hi], scaled(w[e], sw[e], 128) if f8 else w[e].double(), 0, f8)


@pytest.mark.parametrize("positive", [False, True])
@pytest.mark.parametrize("counts,n,k", LONG)
def test_the_error_of_bf16_sums_is_that_of_short_ones(counts, n, k, positive):
    """Positive numbers add up every truncation in the same direction."""
    import torch
    from paper_2609_22335_b200 import api
    offsets, t = sort_of(counts)
    a = torch.randn(t, k, device="cuda", generator=gen(1)).to(torch.bfloat16)
    w = (0.1 * torch.randn(len(counts), n, k, device="cuda", generator=gen(2))).to(torch.bfloat16)
    if positive:
        a, w = a.abs(), w.abs()
    got, ends = api.op_linear_grouped(a, w, offsets), offsets.tolist()
    for e, (lo, hi) in enumerate(zip(ends, ends[1:])):
        x, v = a[lo:hi].double(), w[e].double()
        d = (got[lo:hi].double() - x @ v.T).abs()
        assert bool((d <= (136 + (-(-k // 64) + 9) / 2) * 2.0 ** -23 * (x.abs() @ v.abs().T)).all())
