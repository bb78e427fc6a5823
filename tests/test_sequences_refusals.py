"""What the operators for several sequences and the layer with addends refuse, before anything reaches a GPU."""
import ctypes as C
import math

import pytest

from paper_2609_22335_b200 import api, build

ATTENTION = ("q k v out ld_q ld_k ld_v ld_out page_k page_v offsets_q offsets_k lengths pages prefix slopes scratch scratch_bytes seqs tq tk n_pages page_size max_pages hq hkv hd "
             "causal window scale cap reserved").split()
STORE = "k v k_cache v_cache ld_k ld_v row_k page_k row_v page_v pages lengths offsets seqs t n_pages page_size max_pages width".split()


@pytest.fixture(scope="module")
def lib():
    build.build()
    return api.load_library()


@pytest.fixture(scope="module")
def mem():
    raw = C.create_string_buffer(1 << 16)
    return (C.addressof(raw) + 255) // 256 * 256, raw


def good(p, paged):
    d = dict.fromkeys(ATTENTION, 0)
    d.update(q=p, k=p + 4096, v=p + 8192, out=p + 12288, ld_q=128, ld_k=64, ld_v=64, ld_out=128, offsets_q=p, scratch=p, scratch_bytes=1 << 40, seqs=2, tq=4, hq=2, hkv=1, hd=64,
             causal=1, scale=0.125)
    if paged:
        d.update(page_k=512, page_v=512, lengths=p, pages=p, n_pages=4, page_size=8, max_pages=2)
    else:
        d.update(offsets_k=p, tk=4)
    return d


def call(lib, name, d):
    return getattr(lib, name)(api._ATTENTION_ARGS.pack(*(d[k] for k in ATTENTION)), None)


BOTH = [dict(q=0), dict(k=0), dict(v=0), dict(out=0), dict(offsets_q=0), dict(seqs=0), dict(seqs=-1), dict(seqs=(1 << 20) + 1), dict(tq=0), dict(tq=(1 << 30) + 1), dict(hq=0), dict(hkv=0),
        dict(hq=3, hkv=2, ld_q=192, ld_out=192, ld_k=128, ld_v=128), dict(hq=65538, ld_q=1 << 23, ld_out=1 << 23), dict(hd=0), dict(hd=4), dict(hd=60), dict(hd=264, ld_q=528, ld_out=528, ld_k=264, ld_v=264),
        dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(cap=-1.0), dict(cap=math.nan), dict(cap=math.inf), dict(cap=1e-40), dict(window=-1), dict(causal=0, window=4),
        dict(causal=0, prefix=4096), dict(reserved=1), dict(ld_q=120), dict(ld_q=132), dict(ld_out=64), dict(ld_out=129), dict(ld_k=56), dict(ld_v=68), dict(ld_v=1 << 38)]


@pytest.mark.parametrize("paged", [False, True])
def test_attention(lib, mem, paged):
    p, name = mem[0], "vla_op_attention_paged" if paged else "vla_op_attention_packed"
    bads = BOTH + [dict(q=p + 8), dict(k=p + 2), dict(v=p + 4), dict(out=p + 8), dict(offsets_q=p + 2), dict(prefix=p + 2), dict(slopes=p + 1)]
    if paged:
        bads += [dict(page_k=56), dict(page_k=516), dict(page_v=0), dict(lengths=0), dict(pages=0), dict(lengths=p + 1), dict(pages=p + 2), dict(n_pages=0), dict(n_pages=(1 << 30) + 1), dict(page_size=0),
                 dict(page_size=4), dict(page_size=12), dict(page_size=(1 << 20) + 8), dict(max_pages=0), dict(max_pages=1 << 28)]
    else:
        bads += [dict(offsets_k=0), dict(offsets_k=p + 2), dict(tk=0), dict(tk=(1 << 30) + 1)]
    for bad in bads:
        assert call(lib, name, {**good(p, paged), **bad}) == api.VLA_ERR_INVALID, bad
    # (none at all is for calls of at most 512 keys a sequence)
    for bad in (dict(scratch=0, tk=1000, max_pages=200), dict(scratch=p + 128), dict(scratch_bytes=1000)):
        assert call(lib, name, {**good(p, paged), **bad}) == api.VLA_ERR_NOMEM, bad
    assert getattr(lib, name)(None, None) == api.VLA_ERR_INVALID
    # more key blocks of a head than are counted
    big = dict(tq=1 << 30, tk=1 << 30) if not paged else dict(tq=1 << 30, page_size=1 << 10, max_pages=1 << 20)
    assert call(lib, name, {**good(p, paged), **big}) == api.VLA_ERR_INVALID


def test_scratch_bytes(lib):
    out = C.c_size_t(0)
    for hd in (0, 4, 12, 257, 264, -8):
        assert lib.vla_op_attention_sequences_scratch_bytes(hd, C.byref(out)) == api.VLA_ERR_INVALID
    assert lib.vla_op_attention_sequences_scratch_bytes(64, None) == api.VLA_ERR_INVALID
    assert lib.vla_op_attention_sequences_scratch_bytes(64, C.byref(out)) == api.VLA_OK and 1 << 20 < out.value < 1 << 26


def test_cache_store(lib, mem):
    p = mem[0]
    fine = dict(k=p, v=p + 4096, k_cache=p + 8192, v_cache=p + 12288, ld_k=64, ld_v=64, row_k=64, page_k=512, row_v=64, page_v=512, pages=p, lengths=p, offsets=p, seqs=2, t=4, n_pages=4,
                page_size=8, max_pages=2, width=64)
    for bad in (dict(k=0), dict(v=0), dict(k_cache=0), dict(v_cache=0), dict(pages=0), dict(lengths=0), dict(offsets=0), dict(k=p + 8), dict(v_cache=p + 2), dict(pages=p + 2), dict(offsets=p + 1),
                dict(ld_k=56), dict(ld_v=66), dict(row_k=60), dict(row_v=0), dict(page_k=56), dict(page_v=65), dict(seqs=0), dict(t=0), dict(t=-1), dict(n_pages=0), dict(page_size=0),
                dict(max_pages=0), dict(max_pages=1 << 28), dict(width=0), dict(width=4), dict(width=60), dict(width=(1 << 24) + 8)):
        assert lib.vla_op_cache_store(api._CACHE_STORE_ARGS.pack(*({**fine, **bad}[k] for k in STORE)), None) == api.VLA_ERR_INVALID, bad
    assert lib.vla_op_cache_store(None, None) == api.VLA_ERR_INVALID


def test_linear_bias(lib, mem):
    p = mem[0]
    fine = dict(a=p, w=p + 2048, bias=p + 4096, res=p + 5120, f32=1, ld=4, o32=p + 8192, o16=None, m=4, n=4, k=32, act=0, stream=None)
    for bad in (dict(a=None), dict(w=None), dict(o32=None), dict(m=0), dict(n=0), dict(k=0), dict(k=12), dict(act=3), dict(act=-1), dict(a=p + 8), dict(w=p + 2050), dict(bias=p + 2), dict(res=p + 2),
                dict(res=p + 1, f32=0), dict(o32=p + 2), dict(o16=p + 1), dict(ld=3), dict(ld=-4), dict(m=(1 << 30) + 1), dict(n=(1 << 30) + 1, ld=1 << 31)):
        assert lib.vla_op_linear_bias(*{**fine, **bad}.values()) == api.VLA_ERR_INVALID, bad


def test_the_python_entries_want_tensors_of_the_current_device():
    import torch
    b, off = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    cache, pages = torch.zeros(2, 8, 64, dtype=torch.bfloat16), torch.zeros(1, 2, dtype=torch.int32)
    for call_ in (lambda: api.op_linear_bias(b, b), lambda: api.op_attention_packed(b, b, b, off, 1, 1, 64), lambda: api.op_attention_paged(b, cache, cache, pages, off[:1], off, 1, 1, 64),
                  lambda: api.op_cache_store(b, b, cache, cache, pages, off[:1], off)):
        with pytest.raises(api.VlaError) as e:
            call_()
        assert e.value.code == api.VLA_ERR_INVALID


@pytest.mark.gpu
def test_the_python_entries_look_at_shapes_types_and_strides():
    import torch
    z = lambda *s, t=torch.bfloat16: torch.zeros(*s, dtype=t, device="cuda")     # noqa: E731
    i32, f32 = torch.int32, torch.float32
    a, w, b, x = z(4, 128), z(32, 128), z(32, t=f32), z(4, 32)
    q, k, off = z(4, 128), z(4, 64), z(3, t=i32)
    kc, pages, have = z(4, 8, 64), z(2, 3, t=i32), z(2, t=i32)
    lin, packed, paged, store = api.op_linear_bias, api.op_attention_packed, api.op_attention_paged, api.op_cache_store
    refused = [
        lambda: lin(a.half(), w), lambda: lin(a, w[:, :64]), lambda: lin(a[:, :64], w), lambda: lin(a[0], w), lambda: lin(a, w, bias=b.bfloat16()), lambda: lin(a, w, bias=b[:31]),
        lambda: lin(a, w, bias=z(64, t=f32)[::2]), lambda: lin(a, w, residual=x.half()), lambda: lin(a, w, residual=x[:3]), lambda: lin(a, w, residual=z(32, 4).T), lambda: lin(a, w, out=x),
        lambda: lin(a, w, out_bf16=True, out=z(4, 64)[:, :32]), lambda: lin(a, w, act=3), lambda: lin(z(0, 128), w), lambda: lin(z(4, 12), z(32, 12)),
        lambda: packed(q.float(), k, k, off, 2, 1, 64), lambda: packed(q, k, k, off.long(), 2, 1, 64), lambda: packed(q, k, k, off[:1], 2, 1, 64), lambda: packed(q, k[:3], k[:3], off, 2, 1, 64),
        lambda: packed(q, k, k[:3], off, 2, 1, 64), lambda: packed(q, k, k, off, 2, 1, 60), lambda: packed(q, k, k, off, 1, 1, 64), lambda: packed(q, k, k, off, 2, 1, 64, offsets_k=off[:2]),
        lambda: packed(q, k, k, off, 2, 1, 64, causal=True, prefix=have.long()), lambda: packed(q, k, k, off, 2, 1, 64, prefix=have), lambda: packed(q, k, k, off, 2, 1, 64, window=4),
        lambda: packed(q, k, k, off, 2, 1, 64, causal=True, window=-1), lambda: packed(q, k, k, off, 2, 1, 64, causal=True, window=1 << 31), lambda: packed(q, k, k, off, 2, 1, 64, slopes=z(1, t=f32)),
        lambda: packed(q, k, k, off, 2, 1, 64, out=z(4, 128, t=f32)), lambda: packed(q, k, k, off, 2, 1, 64, out=z(128, 4).T), lambda: packed(q, k, k, off, 2, 1, 64, scale=0.0),
        lambda: packed(q, k, k, off, 2, 1, 64, cap=-1.0), lambda: packed(z(4, 132)[:, 4:], k, k, off, 2, 1, 64), lambda: packed(z(0, 128), z(0, 64), z(0, 64), off, 2, 1, 64),
        lambda: paged(q, kc, kc[:, :4], pages, have, off, 2, 1, 64), lambda: paged(q, kc.float(), kc.float(), pages, have, off, 2, 1, 64), lambda: paged(q, kc[0], kc[0], pages, have, off, 2, 1, 64),
        lambda: paged(q, kc, kc, pages[:1], have, off, 2, 1, 64), lambda: paged(q, kc, kc, pages.long(), have, off, 2, 1, 64), lambda: paged(q, kc, kc, pages.T, have, off, 2, 1, 64),
        lambda: paged(q, kc, kc, pages, have[:1], off, 2, 1, 64), lambda: paged(q, z(4, 12, 64), z(4, 12, 64), pages, have, off, 2, 1, 64), lambda: paged(q, kc, kc, pages, have, off, 2, 2, 64),
        lambda: store(k, k, z(4, 8, 32), z(4, 8, 32), pages, have, off), lambda: store(k, k[:3], kc, kc, pages, have, off), lambda: store(k.float(), k, kc, kc, pages, have, off),
        lambda: store(z(64, 4).T, k, kc, kc, pages, have, off), lambda: store(z(4, 4), z(4, 4), z(4, 8, 4), z(4, 8, 4), pages, have, off), lambda: store(k[:0], k[:0], kc, kc, pages, have, off)]
    for i, call_ in enumerate(refused):
        with pytest.raises(api.VlaError) as e:
            call_()
        assert e.value.code == api.VLA_ERR_INVALID, i
    for small in (torch.empty(1000, dtype=torch.uint8, device="cuda"), torch.empty(1 << 27, dtype=torch.uint8, device="cuda")[1:]):
        with pytest.raises(api.VlaError) as e:
            packed(q, k, k, off, 2, 1, 64, scratch=small)
        assert e.value.code == api.VLA_ERR_NOMEM


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["linear_bias", "packed", "paged", "store"])
def test_on_the_current_stream(name):
    """Behind the work that makes their inputs, into memory of that stream."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()          # noqa: E731
    q, k, v, w = r(70, 256), r(70, 128), r(70, 128), r(96, 256)
    off, pages, have = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 20, 70], [[0, 1, 2, 3, 4, 5, 6], [7, 8, 9, 10, 11, 12, 13]], [20, 50]))
    kc, vc = r(14, 8, 128), r(14, 8, 128)
    calls = {"linear_bias": ([q], lambda: api.op_linear_bias(q, w, residual=q[:, :96])), "packed": ([q, k], lambda: api.op_attention_packed(q, k, v, off, 4, 2, 64)),
             "paged": ([q, kc], lambda: api.op_attention_paged(q, kc, vc, pages, have, off, 4, 2, 64)), "store": ([k, v], lambda: (api.op_cache_store(k, v, kc, vc, pages, have, off), kc, vc)[1:])}
    inputs, call_ = calls[name]
    copies = lambda y: [t.clone() for t in (y if isinstance(y, tuple) else (y,))]      # noqa: E731
    values = [t.clone() for t in inputs]
    want = copies(call_())
    for t in inputs:
        t.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        for t, x in zip(inputs, values):
            t.copy_(x)
        got = copies(call_())
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
