"""Values to 8 bits with block scales: the bytes and scales of the formula, computed with numpy in IEEE fp32."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def e4m3_values(v):
    """Nearest e4m3 values, ties to even (steps of 2^(e - 3), 2^-9 below 2^-6); every |v| here is at most 448."""
    v = v.astype(np.float64)
    e = np.maximum(np.frexp(np.abs(np.where(np.isfinite(v), v, 0)))[1] - 1, -6)
    step = np.ldexp(1.0, e - 3)
    return np.round(v / step) * step


def formula(x, rows):
    """x fp32 [m,k] -> (values q stands for, scales)."""
    m, k = x.shape
    mb, kb = -(-m // rows), -(-k // 128)
    p = np.zeros((mb * rows, kb * 128), np.float32)
    p[:m, :k] = x
    p = p.reshape(mb, rows, kb, 128)
    with np.errstate(all="ignore"):
        s = np.maximum(np.abs(p).max(axis=(1, 3)) / np.float32(448), np.float32(2.0 ** -126))
        q = e4m3_values(p / s[:, None, :, None])
    return q.reshape(mb * rows, kb * 128)[:m, :k], s


def check(x, rows, api, view=None):
    import torch
    t = torch.from_numpy(x).cuda() if view is None else view
    q, s = api.op_quantize(t, block_rows=rows)
    torch.cuda.synchronize()
    want_q, want_s = formula(x, rows)
    assert q.shape == x.shape and s.shape == want_s.shape
    assert np.array_equal(s.cpu().numpy(), want_s, equal_nan=True)
    got = q.float().cpu().numpy()
    assert np.array_equal(got, want_q, equal_nan=True)
    return q, s


@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("m,k", [(1, 16), (1, 4096), (3, 128), (7, 144), (127, 112), (128, 256), (129, 1040), (300, 640), (2000, 528)])
def test_bytes_and_scales_are_the_formulas(m, k, f32, rows):
    import torch
    from paper_2609_22335_b200 import api
    rng = np.random.default_rng(m * 100 + k)
    x = (rng.standard_normal((m, k)) * np.exp(2 * rng.standard_normal((1, k)))).astype(np.float32)
    if not f32:
        x = torch.from_numpy(x).to(torch.bfloat16).float().numpy()
    view = torch.from_numpy(x).cuda()
    check(x, rows, api, view if f32 else view.to(torch.bfloat16))


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("seed", range(4))
def test_quotients_round_as_a_division_does(f32, seed):
    """Millions of quotients, many of them near ties of e4m3 (bf16 values over bf16 maxima), scales of every fraction, ones of nothing but ones among them."""
    import torch
    from paper_2609_22335_b200 import api
    rng = np.random.default_rng(seed)
    x = (rng.standard_normal((8192, 512)) * np.exp2(rng.integers(-60, 60, (8192, 1)))).astype(np.float32)
    ones = np.float32(np.uint32(0x3FFFFFFF).view(np.float32)) * np.float32(448)          # amax / 448 has a fraction of ones, or nearly
    x[:64, ::128] = ones * np.exp2(rng.integers(-20, 20, (64, 4))).astype(np.float32)
    if not f32:
        x = torch.from_numpy(x).to(torch.bfloat16).float().numpy()
    view = torch.from_numpy(x).cuda()
    check(x, 1, api, view if f32 else view.to(torch.bfloat16))


def test_many_rows_take_the_same_values_as_few():
    """More blocks than the chip takes one by one: several a turn, with a ragged last turn."""
    import torch
    from paper_2609_22335_b200 import api
    x = torch.randn(4099, 1168, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)).to(torch.bfloat16)
    q, s = api.op_quantize(x)
    for at in range(0, 4099, 1000):
        qq, ss = api.op_quantize(x[at:at + 9].contiguous())
        assert torch.equal(qq.view(torch.uint8), q[at:at + 9].view(torch.uint8)) and torch.equal(ss, s[at:at + 9])


@pytest.mark.parametrize("rows", [1, 128])
def test_rows_that_lie_apart(rows):
    import torch
    from paper_2609_22335_b200 import api
    big = torch.randn(200, 400, device="cuda", generator=torch.Generator(device="cuda").manual_seed(4)).to(torch.bfloat16)
    view = big[:, 64:64 + 272]
    check(view.float().cpu().numpy(), rows, api, view)


@pytest.mark.parametrize("rows", [1, 128])
def test_values_at_the_ends_of_the_range(rows):
    """Zeros, subnormal numbers, the largest ones, ties; an infinity or NaN poisons its own block and no other."""
    import torch
    from paper_2609_22335_b200 import api
    rng = np.random.default_rng(9)
    x = rng.standard_normal((256, 1024)).astype(np.float32)
    x[:, :128] = 0.0
    x[:, 128:256] *= np.float32(1e-40)
    x[:, 256:384] *= np.float32(3e37)
    x[:, 384:512] *= np.float32(2.0 ** -117)
    x[:, 512:640] = np.where(rng.random((256, 128)) < 0.5, 448, rng.integers(1, 4000, (256, 128)) / 8).astype(np.float32)      # ties between two values
    x[5, 700], x[200, 710], x[6, 800], x[201, 900] = np.inf, -np.inf, np.nan, np.nan
    q, s = check(x, rows, api)
    back = q.float().cpu().numpy() * np.repeat(np.repeat(s.cpu().numpy(), rows, 0), 128, 1)
    assert np.isnan(back[5, 640:768]).all() and np.isnan(back[6, 768:896]).all() and np.isfinite(back[7, :640]).all()
    if rows == 1:
        assert np.isfinite(back[7]).all()


def test_captured_into_a_graph_and_on_a_side_stream():
    import torch
    from paper_2609_22335_b200 import api
    x = torch.randn(50, 256, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    api.op_quantize(x, stream=side)
    with torch.cuda.graph(g, stream=side):
        q, s = api.op_quantize(x, stream=side)
    x.mul_(3.0)
    torch.cuda.synchronize()
    g.replay()
    torch.cuda.synchronize()
    want, scales = formula(x.cpu().numpy(), 1)
    assert np.array_equal(q.float().cpu().numpy(), want) and np.array_equal(s.cpu().numpy(), scales)
