"""Quotients and bytes of the quantiser where a shortened division could differ from IEEE's: values next to e4m3's ties over scales next to a power of two,
down to where remainders are subnormal; zeros of both signs, beside blocks of every kind."""
import numpy as np
import pytest

from test_gpu_quantize import formula

pytestmark = pytest.mark.gpu

TIES = np.array([(2 * j + 1) * 2.0 ** -10 for j in range(8)] + [(17 + 2 * j) * 2.0 ** (e - 4) for e in (-6, -3, 0, 5) for j in range(8)])


def bytes_of(x, rows):
    """The formula's bytes and scales; a NaN is 0x7F."""
    q, s = formula(x, rows)
    a = np.abs(np.where(np.isnan(q), 0, q))
    e = np.maximum(np.frexp(np.where(a > 0, a, 1))[1] - 1, -6)
    m = np.ldexp(a, 3 - e).astype(np.int64)                      # 8 .. 15, below 8 for subnormal values
    b = np.where(m >= 8, (e + 7) * 8 + m - 8, m) | np.where(np.signbit(x), 0x80, 0)
    return np.where(np.isnan(q), 0x7F, b).astype(np.uint8), s


def same(x, rows, bf16=False):
    import torch
    from paper_2609_22335_b200 import api
    t = torch.from_numpy(x).cuda()
    q, s = api.op_quantize(t.to(torch.bfloat16) if bf16 else t, block_rows=rows)
    want, scales = bytes_of(x, rows)
    got = q.view(torch.uint8).cpu().numpy()
    assert np.array_equal(s.cpu().numpy(), scales, equal_nan=True)
    nan = want == 0x7F
    assert np.array_equal(got & 0x7F, want & 0x7F)
    assert np.array_equal(got[~nan], want[~nan])


@pytest.mark.parametrize("rows", [1, 128])
def test_quotients_next_to_ties_over_small_scales(rows):
    """A quotient of a scale's neighbours above a tie is the next fp32 number above it, if the division is exact to the last bit."""
    blocks = []
    for exponent in range(-100, -60):
        for last in list(range(1, 40)) + [1000, 123456]:
            s = np.float32(np.ldexp(2.0 - last * 2.0 ** -23, exponent))
            x = (TIES.astype(np.float64) * np.float64(s)).astype(np.float32)
            x = np.concatenate([[s * np.float32(448)], x, np.nextafter(x, np.float32(1)), np.nextafter(x, np.float32(0))]).astype(np.float32)
            blocks.append(np.pad(x, (0, 128 - x.size)))
    x = np.stack(blocks)
    if rows == 128:                                              # (a block of 128 x 128 for each)
        x = np.concatenate([np.pad(b[None], ((0, 127), (0, 0))) for b in x])
    same(x, rows)


@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("k", [128, 384, 1152, 2048])
def test_zeros_keep_their_sign_whatever_is_beside_them(k, bf16, rows):
    """Zeros of both signs, and values that become zero, in blocks of every kind: ordinary, all zero, tiny, with an infinity or a NaN."""
    import torch
    rng = np.random.default_rng(k)
    x = rng.standard_normal((1500, k)).astype(np.float32)
    x[rng.random(x.shape) < 0.2] = 0.0
    x[rng.random(x.shape) < 0.1] *= np.float32(1e-5)
    kinds = rng.integers(0, 8, (1500 if rows == 1 else -(-1500 // 128), k // 128)).repeat(rows, 0)[:1500].repeat(128, 1)
    x[kinds == 0] = 0.0
    x[kinds == 1] *= np.float32(1e-33)
    x[(kinds == 2) & (rng.random(x.shape) < 0.01)] = np.inf
    x[(kinds == 3) & (rng.random(x.shape) < 0.01)] = np.nan
    x = np.where(rng.random(x.shape) < 0.5, -x, x)
    if bf16:
        x = torch.from_numpy(x).to(torch.bfloat16).float().numpy()
    same(x, rows, bf16)
