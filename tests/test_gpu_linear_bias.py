"""The linear layer with bias and residual against the formula in 64 bits.

Tolerance, element by element: half a step of the result's type; the tensor core's sums, cut (not rounded) to 24 bits after each 16 of K, so at most 2^-22 of
S = sum |a w| for each of K / 16 additions and two more where parts of K meet, times 1.2 (the activations' steepest slope is 1.13); 2^-22 of bias, residual and
result for the 32-bit additions; and of an activation of x (2 |x| + 8) 2^-22 of its value, since e^x is taken from x log2(e) rounded to 24 bits, with
a power and a reciprocal good to 2^-22 each."""
import math

import pytest

pytestmark = pytest.mark.gpu


def _make(m, n, k, bias, residual, seed, ld=None):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)      # noqa: E731
    a, w = r(m, k).bfloat16(), (r(n, k) / math.sqrt(k)).bfloat16()
    b = 0.5 * r(n) if bias else None
    x = None
    if residual:
        x = (2.0 * r(m, ld or n)).to({"bf16": torch.bfloat16, "f32": torch.float32}[residual])[:, :n]
    return a, w, b, x


def _act(y, act):
    import torch
    if act == 1:
        return y * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3))
    return y * torch.sigmoid(y) if act == 2 else y


def _check(got, a, w, b, x, act):
    import torch
    a, w = a.double(), w.double()
    z = a @ w.T
    sums = a.abs() @ w.abs().T
    if b is not None:
        z = z + b.double()
    y = _act(z, act)
    of_act = (2 * z.abs() + 8) * 2.0 ** -22 * y.abs() if act else 0.0
    want = y if x is None else y + x.double()
    tol = want.abs() * torch.finfo(got.dtype).eps / 2 + 1.2 * (a.shape[1] / 16 + 2) * 2.0 ** -22 * sums + of_act
    tol = tol + 2.0 ** -22 * (y.abs() + want.abs() + (0.0 if b is None else b.double().abs()) + (0.0 if x is None else x.double().abs()))
    off = (got.double() - want).abs()
    assert bool((off <= tol).all()), float((off / tol).max())


SHAPES = [(1, 1, 8), (1, 4096, 4096), (3, 7, 24), (16, 33, 72), (50, 720, 2048), (97, 2050, 136), (128, 256, 8192), (129, 113, 64), (200, 130, 4096), (288, 11008, 256),
          (817, 1152, 4304), (1000, 1001, 96), (2048, 2048, 2048), (4100, 520, 1040)]


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("out_bf16", [False, True])
@pytest.mark.parametrize("bias,residual,act", [(True, "f32", 0), (True, "bf16", 1), (False, "bf16", 2), (True, None, 1), (False, "f32", 1), (False, None, 2)])
def test_against_64_bits(m, n, k, out_bf16, bias, residual, act):
    from paper_2609_22335_b200 import api
    a, w, b, x = _make(m, n, k, bias, residual, seed=m + n + k)
    got = api.op_linear_bias(a, w, bias=b, residual=x, act=act, out_bf16=out_bf16)
    assert api.op_status(api.OP_LINEAR_BIAS) == api.VLA_OK
    _check(got, a, w, b, x, act)


@pytest.mark.parametrize("residual", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k,ld,skip", [(40, 64, 128, 96, 0), (40, 64, 128, 67, 0), (300, 256, 192, 258, 2), (300, 256, 192, 264, 1), (300, 256, 192, 272, 8)])
def test_rows_that_lie_apart_and_begin_anywhere(residual, m, n, k, ld, skip):
    """Strides and starts that allow sixteen bytes at a time, four, and single elements; what lies between the rows is NaN."""
    import torch
    from paper_2609_22335_b200 import api
    a, w, b, x = _make(m, n, k, True, residual, 5)
    flat = torch.full((m * ld + skip,), math.nan, dtype=x.dtype, device="cuda")
    view = flat[skip:].view(m, ld)[:, :n]
    view.copy_(x)
    bias = torch.full((n + 3,), math.nan, device="cuda")[3:]
    bias.copy_(b)
    for out_bf16 in (False, True):
        _check(api.op_linear_bias(a, w, bias=bias, residual=view, out_bf16=out_bf16), a, w, b, x, 0)


@pytest.mark.parametrize("m,n,k", [(1, 4096, 512), (77, 130, 64), (200, 99, 64), (817, 1152, 520), (2048, 1024, 256)])
@pytest.mark.parametrize("residual", ["bf16", "f32"])
def test_the_result_takes_the_residuals_place(m, n, k, residual):
    from paper_2609_22335_b200 import api
    a, w, b, x = _make(m, n, k, True, residual, 6)
    want = api.op_linear_bias(a, w, bias=b, residual=x, act=2, out_bf16=residual == "bf16")
    stream = x.clone()
    assert api.op_linear_bias(a, w, bias=b, residual=stream, act=2, out_bf16=residual == "bf16", out=stream) is stream
    assert (stream == want).all()


def test_without_addends_it_is_the_plain_layer():
    """Same kernels, same sums: without an activation the bits are those of op_linear."""
    from paper_2609_22335_b200 import api
    for m, n, k in ((1, 512, 512), (300, 1000, 264), (2048, 2048, 512)):
        a, w, _, _ = _make(m, n, k, False, None, 7)
        assert (api.op_linear_bias(a, w) == api.op_linear(a, w)).all()


def test_infinities_and_nan_go_where_they_are():
    import torch
    from paper_2609_22335_b200 import api
    a, w, b, x = _make(130, 96, 64, True, "f32", 8)
    x[3, 5], x[4, 6], b[7] = math.inf, math.nan, -math.inf
    got = api.op_linear_bias(a, w, bias=b, residual=x)
    bad = torch.zeros_like(got, dtype=torch.bool)
    bad[3, 5] = bad[4, 6] = True
    bad[:, 7] = True
    assert bool((~got.isfinite() == bad).all()) and got[3, 5] == math.inf and bool(got[4, 6].isnan()) and bool((got[:, 7] == -math.inf).all())


def test_captured_first_and_on_another_stream():
    import torch
    from paper_2609_22335_b200 import api
    a, w, b, x = _make(60, 256, 320, True, "bf16", 9)
    want = api.op_linear_bias(a, w, bias=b, residual=x, out_bf16=True)
    side = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        got = api.op_linear_bias(a, w, bias=b, residual=x, out_bf16=True, stream=side)
    got.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert (got == want).all()


def test_a_wait_that_runs_out_is_reported():
    from paper_2609_22335_b200 import api
    for m, n, k in ((60, 256, 320), (2048, 2048, 512)):
        a, w, b, x = _make(m, n, k, True, "bf16", 9)
        api.debug_op_fault(True, wait_limit_ns=1_000_000)
        try:
            api.op_linear_bias(a, w, bias=b, residual=x)
            assert api.op_status(api.OP_LINEAR_BIAS) == api.VLA_ERR_TIMEOUT
        finally:
            api.debug_op_fault(False)
        api.op_linear_bias(a, w, bias=b, residual=x)
        assert api.op_status(api.OP_LINEAR_BIAS) == api.VLA_OK
