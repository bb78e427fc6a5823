"""Addresses that a kernel could not read or write are refused before anything reaches a GPU."""
import pytest

from paper_2609_22335_b200 import api
from test_op_refusals import changed, lib, mem  # noqa: F401  (fixtures)


@pytest.mark.parametrize("bad", ["gq", "gk", "pos"])
@pytest.mark.parametrize("off", [1, 2])
def test_qk_norm_rope(lib, mem, bad, off):  # noqa: F811
    p = mem[0]
    good = dict(q=p, k=p + 1024, f32=0, ldq=128, ldk=64, oq=p + 2048, ok=p + 4096, ldoq=128, ldok=64, t=2, hq=2, hkv=1, hd=64, gq=p + 8192, gk=p + 9216, eps=1e-6, pos=p + 10240,
                pos0=0, rot=64, base=10000.0, inter=0, stream=None)
    assert lib.vla_op_qk_norm_rope(*changed(good, **{bad: good[bad] + off})) == api.VLA_ERR_INVALID


def test_linear(lib, mem):  # noqa: F811
    p = mem[0]
    good = dict(a=p, w=p + 2048, o32=p + 4096, o16=p + 8192, m=4, n=16, k=32, act=0, stream=None)
    for bad in (dict(a=p + 8), dict(w=p + 2050), dict(o32=p + 4098), dict(o16=p + 8193)):
        assert lib.vla_op_linear(*changed(good, **bad)) == api.VLA_ERR_INVALID, bad


def test_attention(lib, mem):  # noqa: F811
    p = mem[0]
    good = dict(q=p, k=p + 4096, v=p + 8192, out=p + 12288, tq=4, tkv=4, hq=1, hkv=1, hd=64, causal=0)
    for bad in (dict(q=p + 8), dict(k=p + 4098), dict(v=p + 8200), dict(out=p + 12296), dict(out=p + 12290)):
        assert lib.vla_op_attention(*changed(good, **bad), p + 16384, 1 << 15, None) == api.VLA_ERR_INVALID, bad
        assert lib.vla_op_attention_static(*changed(good, **bad), None) == api.VLA_ERR_INVALID, bad
