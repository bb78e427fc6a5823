"""Numbers that no 32-bit float holds are refused like any other that an attention does not take."""
import math

import pytest

from paper_2609_22335_b200 import api


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [dict(cap=1e39), dict(cap=-1e39), dict(cap=1e308), dict(cap=1e30), dict(cap=math.inf), dict(cap=math.nan), dict(scale=1e39), dict(scale=-1e39), dict(scale=1e30),
                                 dict(scale=math.inf), dict(scale=math.nan), dict(scale=1e-320, cap=1e39), dict(cap=10 ** 400)], ids=str)
def test_refused(bad):
    import torch
    z = lambda *s, t=torch.bfloat16: torch.zeros(*s, dtype=t, device="cuda")     # noqa: E731
    q, k, off = z(4, 128), z(4, 64), z(3, t=torch.int32)
    for call in (lambda: api.op_attention_packed(q, k, k, off, 2, 1, 64, **bad),
                 lambda: api.op_attention_paged(q, z(4, 8, 64), z(4, 8, 64), z(2, 3, t=torch.int32), z(2, t=torch.int32), off, 2, 1, 64, **bad)):
        with pytest.raises(api.VlaError) as e:
            call()
        assert e.value.code == api.VLA_ERR_INVALID
