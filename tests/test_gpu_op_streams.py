"""The Python entries of the operators run on torch's current stream where they are given none: behind the work that makes their inputs, into memory of
that stream, and into a capture that is under way."""
import pytest

pytestmark = pytest.mark.gpu

NAMES = ["quantize", "linear_scaled", "linear_grouped", "linear_grouped_scaled", "qk_norm_rope", "linear", "attention", "attention_static"]


def case(name):
    """(inputs that are filled late, the call on them)"""
    import torch
    from paper_2609_22335_b200 import api
    gen = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s: torch.randn(*s, device="cuda", generator=gen)                   # noqa: E731
    f8 = torch.float8_e4m3fn
    offsets = torch.tensor([0, 20, 70], dtype=torch.int32, device="cuda")
    x, w3 = r(70, 256).to(torch.bfloat16), r(2, 96, 256).to(torch.bfloat16)
    a8, w8, sa, sw = r(70, 256).to(f8), r(2, 96, 256).to(f8), r(70, 2).abs(), r(2, 1, 2).abs()
    q, k, out = r(70, 256).to(torch.bfloat16), r(70, 128).to(torch.bfloat16), torch.empty(70, 256, device="cuda", dtype=torch.bfloat16)
    return {"quantize": ([x], lambda: api.op_quantize(x)),
            "linear_scaled": ([a8, sa], lambda: api.op_linear_scaled(a8, sa, w8[0], sw[0])),
            "linear_grouped": ([x], lambda: api.op_linear_grouped(x, w3, offsets)),
            "linear_grouped_scaled": ([a8, sa], lambda: api.op_linear_grouped_scaled(a8, sa, w8, sw, offsets)),
            "qk_norm_rope": ([q, k], lambda: api.op_qk_norm_rope(q, k, 4, 2, 64)),
            "linear": ([x], lambda: api.op_linear(x, w3[0])),
            "attention": ([q, k], lambda: api.op_attention(q, k, k, 4, 2, 64)),
            "attention_static": ([q, k], lambda: api.op_attention_static(q, k, k, out, 4, 2, 64))}[name]


def copies(got):
    import torch
    return [t.clone().view(torch.uint8) for t in (got if isinstance(got, tuple) else (got,))]


def late(inputs, values, stream):
    """Fills the inputs on `stream` some milliseconds from now."""
    import torch
    torch.cuda._sleep(20_000_000)
    for t, v in zip(inputs, values):
        t.copy_(v)


@pytest.mark.parametrize("name", NAMES)
def test_on_the_current_stream(name):
    import torch
    inputs, call = case(name)
    values = [t.clone() for t in inputs]
    want = copies(call())
    for t in inputs:
        t.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        late(inputs, values, side)
        got = copies(call())
    torch.cuda.synchronize()
    assert all(torch.equal(g, w) for g, w in zip(got, want))


@pytest.mark.parametrize("name", NAMES)
def test_in_a_capture(name):
    import torch
    inputs, call = case(name)
    want = copies(call())
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = call()
    for t in got if isinstance(got, tuple) else (got,):
        t.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(copies(got), want))


def test_status_waits_for_the_current_stream():
    import torch
    from paper_2609_22335_b200 import api
    inputs, call = case("linear_scaled")
    values = [t.clone() for t in inputs]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        late(inputs, values, side)
        call()
        assert api.op_status(api.OP_LINEAR_SCALED) == api.VLA_OK and side.query()


def test_attentions_own_scratch_is_memory_of_its_stream():
    """What the call allocates for itself goes back when it returns; it must not be handed to another stream before the kernel has written it."""
    import torch
    from paper_2609_22335_b200 import api
    q, k = torch.randn(70, 256, device="cuda").to(torch.bfloat16), torch.randn(70, 128, device="cuda").to(torch.bfloat16)
    n = api.op_attention_scratch_bytes(70, 2, 64)
    api.op_attention(q, k, k, 4, 2, 64)
    torch.full((n,), 7, dtype=torch.uint8, device="cuda")        # (kernels are loaded on their first call, which takes a while)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)
    got = api.op_attention(q, k, k, 4, 2, 64, stream=side)
    mine = [torch.full((n,), 7, dtype=torch.uint8, device="cuda") for _ in range(8)]
    torch.cuda.synchronize()
    assert all(bool((m == 7).all()) for m in mine) and got.shape == q.shape


@pytest.mark.parametrize("name", ["linear", "attention", "quantize", "linear_scaled", "linear_grouped", "linear_grouped_scaled", "qk_norm_rope"])
def test_results_are_memory_of_the_stream_that_writes_them(name):
    """A result that is dropped before its kernel has run must not be written into what the current stream has made of its memory."""
    import torch
    from paper_2609_22335_b200 import api
    entry, side = getattr(api, "op_" + name), torch.cuda.Stream()
    inputs, call = case(name)
    shapes = [t.shape for t in copies(call())]
    [torch.full(s, 7, dtype=torch.uint8, device="cuda") for s in shapes]
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)
    try:
        setattr(api, "op_" + name, lambda *a, **k: entry(*a, stream=side, **k))
        call()
    finally:
        setattr(api, "op_" + name, entry)
    mine = [torch.full(s, 7, dtype=torch.uint8, device="cuda") for _ in range(8) for s in shapes]
    torch.cuda.synchronize()
    assert all(bool((m == 7).all()) for m in mine)
