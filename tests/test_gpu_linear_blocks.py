"""Linear layers on 8-bit operands with block scales and linear layers grouped by expert, against the formulas in 64 bits.

Tolerances, relative to sum_k |A_ik| |W_jk| of the scaled matrices: an MMA of 32 products (16 in bf16) that truncates each of them and the running sum to
24 bits is off by less than 33 * 2^-23 of that; sums are cut every 128 bytes (512 in bf16) of K, four (16) MMAs, so the tensor core adds less
than 132 (272) * 2^-23; adding the parts up and scaling adds a rounding each, 2^-24 per part and 2^-23 for the scale.  A bf16 result is off by another
half step, 2^-8 |y|.  The activations are 1.1-Lipschitz (1.13 and 1.10) and their own arithmetic is good to 2^-19 |y| + 2^-20 (ex2, rcp)."""
import math

import pytest

pytestmark = pytest.mark.gpu


def gen(seed):
    import torch
    return torch.Generator(device="cuda").manual_seed(seed)


def eight_bit(rows, n, k, seed, groups=None):
    """Random e4m3 values over their whole range and scales that differ by block."""
    import torch
    lead = () if groups is None else (groups,)
    g = gen(seed)
    v = (torch.randn(*lead, n, k, device="cuda", generator=g) * torch.exp(torch.randn(*lead, n, k, device="cuda", generator=g))).clamp(-448, 448).to(torch.float8_e4m3fn)
    s = torch.exp(torch.randn(*lead, -(-n // rows), -(-k // 128), device="cuda", generator=g)) * 0.01
    return v, s


def scaled(v, s, rows):
    n, k = v.shape[-2:]
    return v.double() * s.double().repeat_interleave(rows, -2)[..., :n, :].repeat_interleave(128, -1)[..., :k]


def act64(y, act):
    import torch
    if act == 1:
        return 0.5 * y * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)))
    return y / (1 + torch.exp(-y)) if act == 2 else y


def near(got, a, w, act, f8):
    """a [m,k], w [n,k] double."""
    import torch
    y, size = a @ w.T, a.abs() @ w.abs().T
    k = a.shape[1]
    parts = -(-k // (128 if f8 else 256))
    tol = ((132 if f8 else 272) + parts / 2 + 2) * 2.0 ** -23 * size
    if act:
        y = act64(y, act)
        tol = 1.13 * tol + 2.0 ** -19 * y.abs() + 2.0 ** -20
    if got.dtype == torch.bfloat16:
        tol = tol * (1 + 2.0 ** -7) + 2.0 ** -8 * y.abs()
    d = (got.double() - y).abs()
    assert bool(torch.isfinite(got).all()) and bool((d <= tol + 1e-30).all()), float((d / (tol + 1e-30)).max())


# (between them they reach every kernel, width, height and split there is: test_blocks_plan.py)
SCALED = [(1, 1, 16), (1, 7, 128), (1, 2048, 1024), (3, 33, 144), (16, 64, 256), (17, 130, 400), (33, 128, 1040), (64, 257, 512), (100, 520, 128),
          (128, 256, 2048), (129, 96, 64), (300, 1000, 384), (513, 2050, 272), (1000, 4304, 1152), (40, 11008, 512),
          (20, 16000, 256), (20, 11008, 1024), (20, 11008, 512), (33, 8000, 512), (33, 11008, 2048), (33, 2000, 8192), (33, 4000, 8192), (51, 6000, 8192),
          (200, 11008, 256), (200, 11008, 1024)]


@pytest.mark.parametrize("m,n,k", SCALED)
@pytest.mark.parametrize("act,bf16", [(0, False), (1, False), (2, True)])
def test_scaled_matches_the_formula(m, n, k, act, bf16):
    import torch
    from paper_2609_22335_b200 import api
    a, sa = eight_bit(1, m, k, m + k)
    w, sw = eight_bit(128, n, k, n + k + 1)
    got = api.op_linear_scaled(a, sa, w, sw, act=act, out_bf16=bf16)
    assert api.op_status(api.OP_LINEAR_SCALED) == api.VLA_OK
    near(got, scaled(a, sa, 1), scaled(w, sw, 128), act, True)


# Several 256-wide tiles a CTA: whole blocks of rows go out as boxes of 64 (bf16) or 32 (fp32) columns, of which the last tile has none, some or a part.
BOXES = [(2600, 4360, 256), (2600, 4384, 144), (2600, 4396, 256), (2600, 4424, 128), (4100, 4352, 400), (2600, 4363, 256)]


@pytest.mark.parametrize("m,n,k", BOXES)
@pytest.mark.parametrize("act", [0, 2])
def test_rows_that_go_out_as_boxes(m, n, k, act):
    """Both results at once, between guard values; then by expert, where rows end inside of boxes."""
    import torch
    from paper_2609_22335_b200 import api
    a, sa = eight_bit(1, m, k, m + k)
    w, sw = eight_bit(128, n, k, n + k + 1)
    want = scaled(a, sa, 1), scaled(w, sw, 128)
    buf32, buf16 = torch.full((m * n + 64,), 7.0, device="cuda"), torch.full((m * n + 64,), 7.0, device="cuda", dtype=torch.bfloat16)
    o32, o16 = buf32[32:32 + m * n].view(m, n), buf16[32:32 + m * n].view(m, n)
    for p32, p16 in ((o32, o16), (o32, None), (None, o16)):
        o32.fill_(float("nan"))
        o16.fill_(float("nan"))
        rc = api.load_library().vla_op_linear_scaled(a.data_ptr(), sa.data_ptr(), w.data_ptr(), sw.data_ptr(), p32.data_ptr() if p32 is not None else None,
                                                     p16.data_ptr() if p16 is not None else None, m, n, k, act, torch.cuda.current_stream().cuda_stream)
        assert rc == api.VLA_OK and api.op_status(api.OP_LINEAR_SCALED) == api.VLA_OK
        for o in (p32, p16):
            if o is not None:
                near(o, *want, act, True)
        for b in (buf32, buf16):
            assert bool((b[:32] == 7).all()) and bool((b[-32:] == 7).all())
    if k % 8 == 0:
        offsets, t = sort_of([m // 2 + 7, 0, m - m // 2 - 40], rest=33)
        x = torch.randn(t, k, device="cuda", generator=gen(1)).to(torch.bfloat16)
        v = (0.1 * torch.randn(3, n, k, device="cuda", generator=gen(2))).to(torch.bfloat16)
        for bf16 in (False, True):
            out = torch.full((t, n), 7.0, device="cuda", dtype=torch.bfloat16 if bf16 else torch.float32)
            api.op_linear_grouped(x, v, offsets, act=act, out_bf16=bf16, out=out)
            ends = offsets.tolist()
            for e in (0, 2):
                near(out[ends[e]:ends[e + 1]], x[ends[e]:ends[e + 1]].double(), v[e].double(), act, False)
            assert bool((out[ends[-1]:] == 7).all())


def test_scaled_takes_what_quantize_gives():
    import torch
    from paper_2609_22335_b200 import api
    x = torch.randn(70, 600, device="cuda", generator=gen(1))
    x = x[:, :592].contiguous()
    w = 0.05 * torch.randn(200, 592, device="cuda", generator=gen(2))
    a, sa = api.op_quantize(x)
    q, sq = api.op_quantize(w, block_rows=128)
    got = api.op_linear_scaled(a, sa, q, sq)
    near(got, scaled(a, sa, 1), scaled(q, sq, 128), 0, True)
    # ... and is as near to the product itself as eight bits are: an operand is off by half a step, 2^-4 of its value, with random signs
    ref = x.double() @ w.double().T
    assert float((got.double() - ref).norm() / ref.norm()) < 2.0 ** -4


def sort_of(counts, lead=0, rest=0):
    """offsets of groups with these row counts behind `lead` rows, and the rows in all."""
    import torch
    ends = [lead]
    for c in counts:
        ends.append(ends[-1] + c)
    return torch.tensor(ends, dtype=torch.int32, device="cuda"), ends[-1] + rest


COUNTS = [[1], [5], [300], [0, 0, 1], [1, 0, 0], [0, 130, 0, 0, 17, 128, 1], [16] * 9, [1] * 40, [0] * 30 + [3] + [0] * 33 + [2], [700, 3, 129], [64, 65, 63, 0, 200]]


@pytest.mark.parametrize("counts", COUNTS)
@pytest.mark.parametrize("n,k,act,bf16", [(96, 136, 0, False), (257, 1040, 1, True), (2048, 64, 2, False)])
def test_grouped_matches_the_formula(counts, n, k, act, bf16):
    import torch
    from paper_2609_22335_b200 import api
    offsets, t = sort_of(counts)
    a = torch.randn(t, k, device="cuda", generator=gen(t + k)).to(torch.bfloat16)
    w = (0.1 * torch.randn(len(counts), n, k, device="cuda", generator=gen(n))).to(torch.bfloat16)
    got = api.op_linear_grouped(a, w, offsets, act=act, out_bf16=bf16)
    assert api.op_status(api.OP_LINEAR_GROUPED) == api.VLA_OK
    ends = offsets.tolist()
    for e, (lo, hi) in enumerate(zip(ends, ends[1:])):
        near(got[lo:hi], a[lo:hi].double(), w[e].double(), act, False)


@pytest.mark.parametrize("counts", COUNTS)
@pytest.mark.parametrize("n,k,act,bf16", [(96, 144, 0, False), (257, 1040, 1, True), (2048, 64, 2, False)])
def test_grouped_scaled_matches_the_formula(counts, n, k, act, bf16):
    import torch
    from paper_2609_22335_b200 import api
    offsets, t = sort_of(counts)
    a, sa = eight_bit(1, t, k, t + k)
    w, sw = eight_bit(128, n, k, n + k, groups=len(counts))
    got = api.op_linear_grouped_scaled(a, sa, w, sw, offsets, act=act, out_bf16=bf16)
    assert api.op_status(api.OP_LINEAR_GROUPED_SCALED) == api.VLA_OK
    ends = offsets.tolist()
    for e, (lo, hi) in enumerate(zip(ends, ends[1:])):
        near(got[lo:hi], scaled(a[lo:hi], sa[lo:hi], 1), scaled(w[e], sw[e], 128), act, True)


EVERY = [([32], 8000, 128), ([150, 0, 200, 250], 130, 4224), ([10, 10], 8000, 1024), ([150, 0, 200, 250], 130, 2112), ([17, 16], 16000, 128), ([80], 4000, 512), ([80], 2000, 4096), ([80], 11008, 512), ([16], 11008, 256),
         ([80], 11008, 256), ([16], 11008, 4160), ([16], 11008, 4096), ([16], 1500, 4096), ([51], 6000, 8192), ([33], 11008, 2048), ([20], 11008, 1024)]


@pytest.mark.parametrize("counts,n,k", EVERY)
def test_grouped_by_every_kernel(counts, n, k):
    test_grouped_matches_the_formula(counts, n, k, 0, True)
    test_grouped_scaled_matches_the_formula(counts, n, k, 0, False)


def test_grouped_over_many_experts():
    """1024 experts, most of them without rows."""
    import torch
    from paper_2609_22335_b200 import api
    counts = [0] * 1024
    for i, c in ((0, 2), (31, 1), (32, 5), (33, 40), (500, 1), (1023, 3)):
        counts[i] = c
    offsets, t = sort_of(counts)
    a = torch.randn(t, 64, device="cuda", generator=gen(5)).to(torch.bfloat16)
    w = torch.randn(1024, 72, 64, device="cuda", generator=gen(6)).to(torch.bfloat16)
    got = api.op_linear_grouped(a, w, offsets)
    ends = offsets.tolist()
    for e in range(1024):
        if counts[e]:
            near(got[ends[e]:ends[e + 1]], a[ends[e]:ends[e + 1]].double(), w[e].double(), 0, False)


@pytest.mark.parametrize("f8", [False, True])
def test_rows_of_no_expert_stay_and_nothing_leaks_between_experts(f8):
    """Rows in front of the first and behind the last expert are left as they were; NaN there, in rows of another expert or in another expert's
    weights (which the same boxes load) reaches no result."""
    import torch
    from paper_2609_22335_b200 import api
    n, k, counts = 100, 144, [40, 0, 9, 150]
    offsets, t = sort_of(counts, lead=5, rest=60)
    ends = offsets.tolist()
    if f8:
        a, sa = eight_bit(1, t, k, 1)
        w, sw = eight_bit(128, n, k, 2, groups=4)
        bad = torch.full((), 0x7F, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
        raw_a, raw_w = a.view(torch.uint8), w.view(torch.uint8)
        raw_a[:5], raw_a[ends[-1]:], raw_a[ends[2]:ends[3]], raw_w[1], raw_w[2] = 0x7F, 0x7F, 0x7F, 0x7F, 0x7F
        call = lambda out: api.op_linear_grouped_scaled(a, sa, w, sw, offsets, out=out)     # noqa: E731
        A, W = scaled(a, sa, 1), scaled(w, sw, 128)
    else:
        a = torch.randn(t, k, device="cuda", generator=gen(1)).to(torch.bfloat16)
        w = torch.randn(4, n, k, device="cuda", generator=gen(2)).to(torch.bfloat16)
        a[:5] = a[ends[-1]:] = a[ends[2]:ends[3]] = w[1] = w[2] = float("nan")
        call = lambda out: api.op_linear_grouped(a, w, offsets, out=out)                    # noqa: E731
        A, W = a.double(), w.double()
    out = torch.full((t, n), 7.0, device="cuda")
    call(out)
    torch.cuda.synchronize()
    assert (out[:5] == 7).all() and (out[ends[-1]:] == 7).all() and torch.isnan(out[ends[2]:ends[3]]).all()
    for e in (0, 3):
        near(out[ends[e]:ends[e + 1]], A[ends[e]:ends[e + 1]], W[e], 0, f8)


def test_offsets_out_of_order_or_range_stay_inside():
    """An offset below the one before counts as that one, one above t as t, one below 0 as 0."""
    import torch
    from paper_2609_22335_b200 import api
    t, n, k = 60, 40, 64
    a = torch.randn(t, k, device="cuda", generator=gen(1)).to(torch.bfloat16)
    w = torch.randn(5, n, k, device="cuda", generator=gen(2)).to(torch.bfloat16)
    raw = torch.tensor([-9, 20, 10, 30, 2 ** 31 - 1, 5], dtype=torch.int32, device="cuda")
    out = api.op_linear_grouped(a, w, raw, out=torch.zeros(t, n, device="cuda"))
    for e, (lo, hi) in enumerate([(0, 20), (20, 20), (20, 30), (30, 60), (60, 60)]):
        near(out[lo:hi], a[lo:hi].double(), w[e].double(), 0, False)
    nothing = torch.full((6,), 60, dtype=torch.int32, device="cuda")
    out = api.op_linear_grouped(a, w, nothing, out=torch.full((t, n), 3.0, device="cuda"))
    assert api.op_status(api.OP_LINEAR_GROUPED) == api.VLA_OK and (out == 3).all()


@pytest.mark.parametrize("odd", [1, 2, 4])
def test_outputs_at_any_alignment(odd):
    """out32 and out16 through the C entry, both at once, at addresses that allow no wide stores."""
    import torch
    from paper_2609_22335_b200 import api
    m, n, k = 37, 48, 256
    a, sa = eight_bit(1, m, k, 1)
    w, sw = eight_bit(128, n, k, 2)
    o32 = torch.full((m * n + 8,), 7.0, device="cuda")
    o16 = torch.full((m * n + 8,), 7.0, device="cuda", dtype=torch.bfloat16)
    lib = api.load_library()
    assert lib.vla_op_linear_scaled(a.data_ptr(), sa.data_ptr(), w.data_ptr(), sw.data_ptr(), o32[odd:].data_ptr(), o16[odd:].data_ptr(), m, n, k, 0, None) == api.VLA_OK
    torch.cuda.synchronize()
    want = api.op_linear_scaled(a, sa, w, sw)
    assert torch.equal(o32[odd:odd + m * n].view(m, n), want) and torch.equal(o16[odd:odd + m * n].view(m, n), want.to(torch.bfloat16))
    assert (o32[:odd] == 7).all() and (o32[odd + m * n:] == 7).all() and (o16[:odd] == 7).all() and (o16[odd + m * n:] == 7).all()


def test_a_wait_that_runs_out_is_reported_and_a_captured_call_works_again():
    import torch
    from paper_2609_22335_b200 import api
    a, sa = eight_bit(1, 50, 256, 1)
    w, sw = eight_bit(128, 300, 256, 2)
    b = torch.randn(50, 256, device="cuda", generator=gen(3)).to(torch.bfloat16)
    x = torch.randn(3, 300, 256, device="cuda", generator=gen(4)).to(torch.bfloat16)
    x8, sx8 = eight_bit(128, 300, 256, 5, groups=3)
    offsets, _ = sort_of([20, 0, 30])

    def calls(stream=None):
        return (api.op_linear_scaled(a, sa, w, sw, stream=stream), api.op_linear_grouped(b, x, offsets, stream=stream),
                api.op_linear_grouped_scaled(a, sa, x8, sx8, offsets, stream=stream))

    def status():
        return [api.op_status(o) for o in (api.OP_LINEAR_SCALED, api.OP_LINEAR_GROUPED, api.OP_LINEAR_GROUPED_SCALED)]

    want = calls()
    assert status() == [api.VLA_OK] * 3
    side = torch.cuda.Stream()
    graphs = []
    try:
        for drop in (False, True):
            api.debug_op_fault(drop, wait_limit_ns=1_000_000 if drop else 0)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                out = calls(side)
            graphs.append((g, out))
    finally:
        api.debug_op_fault(False)
    for _ in range(2):
        graphs[1][0].replay()
        assert status() == [api.VLA_ERR_TIMEOUT] * 3
        graphs[0][0].replay()
        assert status() == [api.VLA_OK] * 3
        assert all(torch.equal(p, q) for p, q in zip(graphs[0][1], want))


FIRST = """
import torch
from paper_2609_22335_b200 import api
x, w = torch.randn(70, 512, device="cuda").to(torch.bfloat16), torch.randn(2, 128, 512, device="cuda").to(torch.bfloat16)
at = torch.tensor([0, 30, 70], dtype=torch.int32, device="cuda")
g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
with torch.cuda.graph(g, stream=side):
    out = api.op_linear_grouped(x, w, at, stream=side)
    q, s = api.op_quantize(x, stream=side)
out.fill_(3)
s.fill_(3)
g.replay()
torch.cuda.synchronize()
assert torch.equal(out, api.op_linear_grouped(x, w, at)) and torch.equal(s, api.op_quantize(x)[1]) and api.op_status(api.OP_LINEAR_GROUPED) == api.VLA_OK
"""


def test_the_first_call_of_a_process_can_be_captured():
    import os
    import subprocess
    import sys
    subprocess.run([sys.executable, "-c", FIRST], check=True, timeout=300, cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))


LONG_K = [(1, 64), (128, 64), (128, 9500), (128, 19000), (300, 19000), (700, 12900)]


@pytest.mark.parametrize("m,n", LONG_K)
def test_long_rows_of_k(m, n):
    """Every ring of the kernels goes round many times, at every tile width: a k-block's hand-overs must not run into the next round's."""
    import torch
    from paper_2609_22335_b200 import api
    k = 8208
    a, sa = eight_bit(1, m, k, 1)
    w, sw = eight_bit(128, n, k, 2)
    got = api.op_linear_scaled(a, sa, w, sw)
    assert api.op_status(api.OP_LINEAR_SCALED) == api.VLA_OK
    near(got, scaled(a, sa, 1), scaled(w, sw, 128), 0, True)
    offsets, _ = sort_of([m // 2, m - m // 2])
    x = torch.randn(m, k, device="cuda", generator=gen(3)).to(torch.bfloat16)
    y = (0.1 * torch.randn(2, n // 2, k, device="cuda", generator=gen(4))).to(torch.bfloat16)
    got = api.op_linear_grouped(x, y, offsets)
    assert api.op_status(api.OP_LINEAR_GROUPED) == api.VLA_OK
    for e, (lo, hi) in enumerate([(0, m // 2), (m // 2, m)]):
        near(got[lo:hi], x[lo:hi].double(), y[e].double(), 0, False)


def test_results_do_not_depend_on_the_run():
    import torch
    from paper_2609_22335_b200 import api
    a, sa = eight_bit(1, 400, 1024, 1)
    w, sw = eight_bit(128, 1500, 1024, 2)
    first = api.op_linear_scaled(a, sa, w, sw)
    one = api.op_linear_scaled(a[:1].contiguous(), sa[:1].contiguous(), w, sw)
    for _ in range(5):
        assert torch.equal(api.op_linear_scaled(a, sa, w, sw), first)
        assert torch.equal(api.op_linear_scaled(a[:1].contiguous(), sa[:1].contiguous(), w, sw), one)


def test_a_decoder_layer_of_them():
    """quantize -> q|k|v projection -> head norms and rotation -> attention -> output projection -> quantize -> experts, as a program would chain them, against
    the same chain in fp64 on the operands each step was given (each step's own tolerance is the other tests' matter: 3e-2 for a whole chain of bf16 steps)."""
    import torch
    from paper_2609_22335_b200 import api
    t, d, hq, hkv, hd, experts, n = 130, 512, 8, 2, 64, 4, 384
    x = torch.randn(t, d, device="cuda", generator=gen(1)).to(torch.bfloat16)
    wqkv = 0.05 * torch.randn((hq + 2 * hkv) * hd, d, device="cuda", generator=gen(2))
    wo = (0.05 * torch.randn(d, hq * hd, device="cuda", generator=gen(3))).to(torch.bfloat16)
    we = 0.05 * torch.randn(experts * n, d, device="cuda", generator=gen(4))
    w8, s8 = api.op_quantize(wqkv, block_rows=128)
    e8, es8 = api.op_quantize(we, block_rows=128)
    offsets, _ = sort_of([70, 0, 10, 50])

    def layer(stream=None):
        a8, sa8 = api.op_quantize(x, stream=stream)
        qkv = api.op_linear_scaled(a8, sa8, w8, s8, out_bf16=True, stream=stream)
        q, k, v = qkv[:, :hq * hd], qkv[:, hq * hd:(hq + hkv) * hd], qkv[:, (hq + hkv) * hd:]
        q, k = api.op_qk_norm_rope(q, k, hq, hkv, hd, stream=stream)
        with torch.cuda.stream(stream or torch.cuda.default_stream()):
            v = v.contiguous()
        o = api.op_attention(q, k, v, hq, hkv, hd, causal=True, stream=stream)
        y = api.op_linear(o, wo, stream=stream)
        y8, sy8 = api.op_quantize(y, stream=stream)
        return api.op_linear_grouped_scaled(y8, sy8, e8.view(experts, n, d), es8.view(experts, n // 128, d // 128), offsets, act=2, out_bf16=True, stream=stream), (a8, sa8, y8, sy8)

    got, (a8, sa8, y8, sy8) = layer()
    qkv = scaled(a8, sa8, 1) @ scaled(w8, s8, 128).T
    q, k, v = (z.reshape(t, -1, hd) for z in (qkv[:, :hq * hd], qkv[:, hq * hd:(hq + hkv) * hd], qkv[:, (hq + hkv) * hd:]))
    angle = torch.arange(t, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(hd // 2, device="cuda", dtype=torch.float64) * 2 / hd)
    c, s = angle.cos()[:, None], angle.sin()[:, None]

    def turned(z):
        z = z / (z.square().mean(-1, keepdim=True) + 1e-6).sqrt()
        u, w = z[..., :hd // 2], z[..., hd // 2:]
        return torch.cat([u * c - w * s, w * c + u * s], -1)
    q, k = turned(q), turned(k).repeat_interleave(hq // hkv, 1)
    p = torch.einsum("ihd,jhd->hij", q, k) / math.sqrt(hd)
    p = p.masked_fill(torch.ones(t, t, device="cuda", dtype=torch.bool).triu(1), float("-inf")).softmax(-1)
    o = torch.einsum("hij,jhd->ihd", p, v.repeat_interleave(hq // hkv, 1)).reshape(t, -1)
    y = o @ wo.double().T
    back = scaled(y8, sy8, 1)
    assert float((back - y).norm() / y.norm()) < 2.0 ** -4 + 3e-2        # (half an e4m3 step, and bf16 in front of it)
    ends = offsets.tolist()
    e64 = scaled(e8, es8, 128).view(experts, n, d)
    ref = torch.cat([act64(back[lo:hi] @ e64[e].T, 2) for e, (lo, hi) in enumerate(zip(ends, ends[1:]))])
    assert float((got.double() - ref).norm() / ref.norm()) < 1e-2
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again, _ = layer(side)
    torch.cuda.synchronize()
    assert torch.equal(again, got)


def test_calls_on_two_streams_at_once():
    """Calls of every kind from two streams, interleaved, with nothing between them but the order of each stream."""
    import torch
    from paper_2609_22335_b200 import api
    a, sa = eight_bit(1, 300, 1024, 1)
    w, sw = eight_bit(128, 1000, 1024, 2, groups=3)
    x = torch.randn(300, 1024, device="cuda", generator=gen(3)).to(torch.bfloat16)
    v = (0.1 * torch.randn(3, 1000, 1024, device="cuda", generator=gen(4))).to(torch.bfloat16)
    offsets, _ = sort_of([100, 7, 193])
    few, _ = sort_of([2, 0, 9])

    def calls(s):
        return [api.op_linear_scaled(a, sa, w[0], sw[0], stream=s), api.op_linear_grouped(x, v, offsets, act=2, stream=s), api.op_linear_grouped_scaled(a, sa, w, sw, offsets, act=1, stream=s),
                api.op_linear_grouped(x[:11], v, few, out_bf16=True, stream=s), api.op_linear_scaled(a[:1], sa[:1], w[1], sw[1], stream=s), *api.op_quantize(x, stream=s)]

    want = calls(None)
    torch.cuda.synchronize()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    got = [calls(streams[i & 1]) for i in range(20)]
    torch.cuda.synchronize()
    for each in got:
        assert all(torch.equal(p.view(torch.uint8), q.view(torch.uint8)) for p, q in zip(each, want))
    assert [api.op_status(o) for o in (api.OP_LINEAR_SCALED, api.OP_LINEAR_GROUPED, api.OP_LINEAR_GROUPED_SCALED)] == [api.VLA_OK] * 3
