"""What the operators refuse, before anything reaches a GPU: the C entries by their status, the Python ones by VlaError."""
import ctypes as C

import pytest

from paper_2609_22335_b200 import api, build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return api.load_library()


@pytest.fixture(scope="module")
def mem():
    raw = C.create_string_buffer(1 << 16)
    return (C.addressof(raw) + 255) // 256 * 256, raw


def changed(good, **new):
    return list({**good, **new}.values())


def test_quantize(lib, mem):
    p = mem[0]
    good = dict(x=p, f32=0, ld=64, q=p + 4096, s=p + 8192, m=4, k=64, rows=1, stream=None)
    for bad in (dict(x=None), dict(q=None), dict(s=None), dict(m=0), dict(k=0), dict(k=60), dict(k=8), dict(rows=2), dict(rows=0), dict(ld=48), dict(ld=65),
                dict(x=p + 2), dict(q=p + 4104), dict(s=p + 8194), dict(f32=1, ld=66), dict(m=-1)):
        assert lib.vla_op_quantize(*changed(good, **bad)) == api.VLA_ERR_INVALID, bad


def test_linear_scaled(lib, mem):
    p = mem[0]
    good = dict(a=p, sa=p + 1024, w=p + 2048, sw=p + 4096, o32=p + 8192, o16=None, m=4, n=4, k=32, act=0, stream=None)
    for bad in (dict(a=None), dict(sa=None), dict(w=None), dict(sw=None), dict(o32=None), dict(m=0), dict(n=0), dict(k=0), dict(k=8), dict(k=40), dict(act=3), dict(act=-1),
                dict(a=p + 8), dict(w=p + 2056), dict(sa=p + 1025), dict(o32=p + 8193), dict(o16=p + 1), dict(m=(1 << 30) + 1), dict(n=(1 << 30) + 1)):
        assert lib.vla_op_linear_scaled(*changed(good, **bad)) == api.VLA_ERR_INVALID, bad


@pytest.mark.parametrize("f8", [False, True])
def test_linear_grouped(lib, mem, f8):
    p = mem[0]
    good = dict(a=p, w=p + 2048, off=p + 4096, o32=p + 8192, o16=None, t=4, n=4, k=32, experts=2, act=0, stream=None)
    call = lib.vla_op_linear_grouped
    bads = [dict(a=None), dict(w=None), dict(off=None), dict(o32=None), dict(t=0), dict(n=0), dict(k=0), dict(k=36), dict(experts=0), dict(experts=1025),
            dict(experts=1024, n=1 << 21), dict(act=3), dict(a=p + 8), dict(w=p + 2056), dict(off=p + 4097), dict(t=(1 << 30) + 1)]
    if f8:
        good = dict(a=p, sa=p + 1024, w=p + 2048, sw=p + 4096, **{k: v for k, v in good.items() if k not in ("a", "w")})
        call = lib.vla_op_linear_grouped_scaled
        bads += [dict(sa=None), dict(sw=None), dict(k=40), dict(sw=p + 3073)]
    for bad in bads:
        assert call(*changed(good, **bad)) == api.VLA_ERR_INVALID, bad


def test_qk_norm_rope(lib, mem):
    p = mem[0]
    good = dict(q=p, k=p + 1024, f32=0, ldq=128, ldk=64, oq=p + 2048, ok=p + 4096, ldoq=128, ldok=64, t=2, hq=2, hkv=1, hd=64, gq=None, gk=None, eps=1e-6, pos=None, pos0=0,
                rot=64, base=10000.0, inter=0, stream=None)
    for bad in (dict(q=None), dict(oq=None), dict(k=None), dict(ok=None), dict(t=0), dict(hq=0), dict(hkv=-1), dict(hd=8), dict(hd=72), dict(hd=272), dict(rot=-16), dict(rot=80),
                dict(rot=8), dict(eps=-1.0), dict(eps=float("nan")), dict(base=1.0), dict(base=float("nan")), dict(base=float("inf")), dict(ldq=120), dict(ldq=132), dict(ldk=48),
                dict(ldoq=64), dict(ldok=60), dict(q=p + 8), dict(oq=p + 2050), dict(f32=1, ldq=130)):
        assert lib.vla_op_qk_norm_rope(*changed(good, **bad)) == api.VLA_ERR_INVALID, bad


def test_the_python_entries_want_tensors_of_the_current_device():
    import torch
    b = torch.zeros(4, 64, dtype=torch.bfloat16)
    f8 = torch.zeros(4, 64, dtype=torch.float8_e4m3fn)
    s = torch.ones(4, 1)
    off = torch.zeros(2, dtype=torch.int32)
    for call in (lambda: api.op_quantize(b), lambda: api.op_linear_scaled(f8, s, f8, s[:1]), lambda: api.op_linear_grouped(b, b[None], off),
                 lambda: api.op_linear_grouped_scaled(f8, s, f8[None], s[None, :1], off), lambda: api.op_qk_norm_rope(b, None, 1, 0, 64)):
        with pytest.raises(api.VlaError) as e:
            call()
        assert e.value.code == api.VLA_ERR_INVALID


@pytest.mark.gpu
def test_the_python_entries_look_at_shapes_types_and_strides():
    import torch
    z = lambda *s, t=torch.bfloat16: torch.zeros(*s, dtype=t, device="cuda")     # noqa: E731
    f8, i32, f32 = torch.float8_e4m3fn, torch.int32, torch.float32
    a, w, sa, sw = z(4, 128, t=f8), z(32, 128, t=f8), z(4, 1, t=f32), z(1, 1, t=f32)
    b, x, off = z(4, 128), z(2, 32, 128), z(3, t=i32)
    refused = [
        lambda: api.op_quantize(z(4, 128).half()), lambda: api.op_quantize(z(128, 4).T), lambda: api.op_quantize(z(4, 120)), lambda: api.op_quantize(z(0, 128)),
        lambda: api.op_quantize(b, block_rows=64), lambda: api.op_quantize(z(128)),
        lambda: api.op_linear_scaled(b, sa, w, sw), lambda: api.op_linear_scaled(a, sa, z(32, 112, t=f8), sw), lambda: api.op_linear_scaled(a, z(1, 4, t=f32), w, sw),
        lambda: api.op_linear_scaled(a, sa, w, z(32, 1, t=f32)), lambda: api.op_linear_scaled(a, sa.double(), w, sw), lambda: api.op_linear_scaled(a[:, :64], sa, w[:, :64], sw),
        lambda: api.op_linear_scaled(a, sa, w, sw, act=3),
        lambda: api.op_linear_grouped(b, x, z(2, t=i32)), lambda: api.op_linear_grouped(b, x, off.long()), lambda: api.op_linear_grouped(b, x[0], off),
        lambda: api.op_linear_grouped(b, x, off, out=z(4, 32)), lambda: api.op_linear_grouped(b, x, off, out=z(5, 32, t=f32)), lambda: api.op_linear_grouped(z(0, 128), x, off),
        lambda: api.op_linear_grouped_scaled(a, sa, z(2, 32, 128, t=f8), sw, off),
        lambda: api.op_qk_norm_rope(z(4, 128), z(4, 64), 2, 1, 60), lambda: api.op_qk_norm_rope(z(4, 128), z(4, 64).float(), 2, 1, 64), lambda: api.op_qk_norm_rope(z(4, 128), None, 2, 1, 64),
        lambda: api.op_qk_norm_rope(z(4, 128), z(4, 64), 2, 1, 64, gq=z(64)), lambda: api.op_qk_norm_rope(z(4, 128), z(4, 64), 2, 1, 64, pos=z(4, t=torch.int64)),
        lambda: api.op_qk_norm_rope(z(4, 128), z(3, 64), 2, 1, 64), lambda: api.op_qk_norm_rope(z(4, 128), z(4, 64), 2, 1, 64, out_q=z(4, 128, t=f32)),
        lambda: api.op_qk_norm_rope(z(4, 136)[:, 8:], None, 2, 0, 64, rot=24)]
    for i, call in enumerate(refused):
        with pytest.raises(api.VlaError) as e:
            call()
        assert e.value.code == api.VLA_ERR_INVALID, i
