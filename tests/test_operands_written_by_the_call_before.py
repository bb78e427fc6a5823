"""A kernel starts while the one in front of it, which may write its bias or its slopes, still runs."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_22335_b200", "csrc")


def test_no_operator_reads_operands_as_constant_memory():
    """__ldg and ld.global.nc ask for memory that nobody writes while the kernel runs."""
    for f in sorted(os.listdir(CSRC)):
        if f.startswith("op"):
            code = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, f)).read())
            assert not re.search(r"__ldg|ld\.global(\.\w+)*\.nc", code), f


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(3, 512, 256), (300, 512, 1024), (2500, 1024, 512)])
def test_a_bias_and_slopes_of_the_call_before(m, n, k):
    import torch
    from paper_2609_22335_b200 import api
    g = torch.Generator(device="cuda").manual_seed(m)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()      # noqa: E731
    a, w, one, u = r(m, k), r(n, k), r(1, 64), r(8, n, 64)
    q, kv, off = r(m, 8 * 64), r(m, 64), torch.tensor([0, m], dtype=torch.int32, device="cuda")
    bias, slopes = torch.empty(1, n, device="cuda"), torch.empty(1, 8, device="cuda")

    def chain(wait):
        got = []
        for i in range(8):
            api.op_linear_bias(one, u[i], out=bias)
            wait()
            got.append(api.op_linear_bias(a, w, bias=bias[0]))
            wait()
            api.op_linear_bias(one, u[i, :8], out=slopes, act=0)
            wait()
            got.append(api.op_attention_packed(q, kv, kv, off, 8, 1, 64, causal=True, slopes=slopes[0]))
            wait()
        return got

    want = chain(torch.cuda.synchronize)
    for _ in range(3):
        assert all(torch.equal(x, y) for x, y in zip(chain(lambda: None), want))
