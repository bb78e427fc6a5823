"""Times the stand-alone operators (linear layers, fused attention and what stands around them, on caller-owned tensors).

    python -m paper_2609_22335_b200.opbench linear M N K [--act 0|1|2] [--f32] [--iters 20]
    python -m paper_2609_22335_b200.opbench attention TQ TKV HQ HKV HD [--causal] [--iters 20]
    python -m paper_2609_22335_b200.opbench quantize M K [--block-rows 1|128] [--f32] [--iters 20]
    python -m paper_2609_22335_b200.opbench linear_scaled M N K [--act 0|1|2] [--f32] [--iters 20]
    python -m paper_2609_22335_b200.opbench linear_grouped T N K EXPERTS [--act 0|1|2] [--f32] [--iters 20]
    python -m paper_2609_22335_b200.opbench linear_grouped_scaled T N K EXPERTS [--act 0|1|2] [--f32] [--iters 20]
    python -m paper_2609_22335_b200.opbench qk_norm_rope T HQ HKV HD [--interleaved] [--f32] [--iters 20]

Prints one JSON line: microseconds per call (CUDA events around `iters` back-to-back calls after three
warm-up calls) and the achieved TFLOP/s (2 M N K, or 4 TQ TKV HQ HD) or, of quantize and qk_norm_rope, GB/s.  Experts
get equally many rows, or one more.  Also the command to put under ncu
when an operator is profiled.
"""
from __future__ import annotations

import argparse
import json


def _time(fn, iters):
    import torch
    for _ in range(3):
        fn()
    torch.cuda.synchronize()
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    e0.record()
    for _ in range(iters):
        fn()
    e1.record()
    torch.cuda.synchronize()
    return e0.elapsed_time(e1) / iters * 1e3


def main(argv=None):
    import torch
    from . import api
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("op", choices=["linear", "attention", "quantize", "linear_scaled", "linear_grouped", "linear_grouped_scaled", "qk_norm_rope"])
    ap.add_argument("dims", type=int, nargs="+")
    ap.add_argument("--act", type=int, default=0)
    ap.add_argument("--f32", action="store_true", help="linear layers: fp32 output instead of bf16; quantize, qk_norm_rope: fp32 input")
    ap.add_argument("--causal", action="store_true")
    ap.add_argument("--block-rows", type=int, default=1, help="quantize: rows that share a scale")
    ap.add_argument("--interleaved", action="store_true", help="qk_norm_rope: pairs of neighbours")
    ap.add_argument("--iters", type=int, default=20)
    a = ap.parse_args(argv)
    g = torch.Generator(device="cuda").manual_seed(0)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g).to(torch.bfloat16)  # noqa: E731
    if a.op == "linear":
        m, n, k = a.dims
        x, w = rnd(m, k), (0.05 * torch.randn(n, k, device="cuda", generator=g)).to(torch.bfloat16)
        us = _time(lambda: api.op_linear(x, w, act=a.act, out_bf16=not a.f32), a.iters)
        status = api.op_status(api.OP_LINEAR)
        flops = 2.0 * m * n * k
        out = {"op": "linear", "m": m, "n": n, "k": k, "act": a.act, "out": "f32" if a.f32 else "bf16"}
    elif a.op == "quantize":
        m, k = a.dims
        x = rnd(m, k).float() if a.f32 else rnd(m, k)
        us = _time(lambda: api.op_quantize(x, block_rows=a.block_rows), a.iters)
        status, flops, moved = api.VLA_OK, None, m * k * (x.element_size() + 1.0) + 4.0 * -(-m // a.block_rows) * -(-k // 128)
        out = {"op": a.op, "m": m, "k": k, "block_rows": a.block_rows, "in": "f32" if a.f32 else "bf16"}
    elif a.op.startswith("linear_"):
        m, n, k, experts = (a.dims + [0])[:4]
        x, w = rnd(m, k), 0.05 * rnd(max(experts, 1), n, k)
        offsets = torch.tensor([m * e // max(experts, 1) for e in range(experts + 1)], dtype=torch.int32, device="cuda")
        kw = {"act": a.act, "out_bf16": not a.f32}
        if a.op != "linear_grouped":
            xq, sx = api.op_quantize(x)
            each = [api.op_quantize(e, block_rows=128) for e in w]
            wq, sw = torch.stack([e[0].view(torch.uint8) for e in each]).view(torch.float8_e4m3fn), torch.stack([e[1] for e in each])
        if a.op == "linear_scaled":
            us = _time(lambda: api.op_linear_scaled(xq, sx, wq[0], sw[0], **kw), a.iters)
        elif a.op == "linear_grouped":
            us = _time(lambda: api.op_linear_grouped(x, w, offsets, **kw), a.iters)
        else:
            us = _time(lambda: api.op_linear_grouped_scaled(xq, sx, wq, sw, offsets, **kw), a.iters)
        status = api.op_status({"linear_scaled": api.OP_LINEAR_SCALED, "linear_grouped": api.OP_LINEAR_GROUPED}.get(a.op, api.OP_LINEAR_GROUPED_SCALED))
        flops = 2.0 * m * n * k
        out = {"op": a.op, "m": m, "n": n, "k": k, "experts": experts, "act": a.act, "out": "f32" if a.f32 else "bf16"}
    elif a.op == "qk_norm_rope":
        t, hq, hkv, hd = a.dims
        x = rnd(t, (hq + hkv) * hd).float() if a.f32 else rnd(t, (hq + hkv) * hd)
        us = _time(lambda: api.op_qk_norm_rope(x[:, :hq * hd], x[:, hq * hd:], hq, hkv, hd, rot=hd, interleaved=a.interleaved), a.iters)
        status, flops, moved = api.VLA_OK, None, x.numel() * (x.element_size() + 2.0)
        out = {"op": a.op, "t": t, "hq": hq, "hkv": hkv, "hd": hd, "interleaved": a.interleaved, "in": "f32" if a.f32 else "bf16"}
    else:
        tq, tkv, hq, hkv, hd = a.dims
        q, kk, v = rnd(tq, hq * hd), rnd(tkv, hkv * hd), rnd(tkv, hkv * hd)
        scratch = torch.empty(api.op_attention_scratch_bytes(tkv, hkv, hd), dtype=torch.uint8, device="cuda")
        us = _time(lambda: api.op_attention(q, kk, v, hq, hkv, hd, causal=a.causal, scratch=scratch), a.iters)
        status = api.op_status(api.OP_ATTENTION, scratch)
        flops = 4.0 * tq * tkv * hq * hd
        out = {"op": "attention", "tq": tq, "tkv": tkv, "hq": hq, "hkv": hkv, "hd": hd, "causal": a.causal}
    out.update({"us_per_call": round(us, 2), "status": status, **({"gbs": round(moved / us / 1e3, 1)} if flops is None else {"tflops": round(flops / us / 1e6, 1)})})
    print(json.dumps(out))


if __name__ == "__main__":
    main()
