"""Sizes and positions that the C interface's 32-bit arguments cannot hold are refused; they must not arrive as something smaller."""
import pytest

pytestmark = pytest.mark.gpu


def refused(call):
    from paper_2609_22335_b200 import api
    with pytest.raises(api.VlaError) as e:
        call()
    assert e.value.code == api.VLA_ERR_INVALID


@pytest.mark.parametrize("pos0", [2 ** 31, -2 ** 31 - 1, 2 ** 32 + 5])
def test_positions(pos0):
    import torch
    from paper_2609_22335_b200 import api
    refused(lambda: api.op_qk_norm_rope(torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda"), None, 1, 0, 64, pos0=pos0))


def test_the_last_positions_count_on():
    """Rows behind the largest start are at positions that need more than 32 bits."""
    import torch
    from paper_2609_22335_b200 import api
    from test_gpu_qk_norm_rope import formula, near, numpy_of
    q = torch.randn(3, 64, device="cuda")
    got, _ = api.op_qk_norm_rope(q, None, 1, 0, 64, pos0=2 ** 31 - 1)
    near(got, formula(numpy_of(q), 1, 64, None, 1e-6, [2 ** 31 - 1, 2 ** 31, 2 ** 31 + 1], 10000.0, 64, False))


def test_long_rows():
    import torch
    from paper_2609_22335_b200 import api
    k = 2 ** 32 + 128
    refused(lambda: api.op_quantize(torch.empty(1, k, dtype=torch.bfloat16, device="cuda")))
    a, s = torch.empty(1, k, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(1, k // 128, device="cuda")
    refused(lambda: api.op_linear_scaled(a, s, a, s))
    offsets = torch.zeros(2, dtype=torch.int32, device="cuda")
    refused(lambda: api.op_linear_grouped_scaled(a, s, a[None], s[None], offsets))
    del a
    b = torch.empty(1, k, dtype=torch.bfloat16, device="cuda")
    refused(lambda: api.op_linear_grouped(b, b[None], offsets))
    del b
    torch.cuda.empty_cache()
