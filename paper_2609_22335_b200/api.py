"""ctypes binding of libvla_b200.so: the same entry points as include/vla.h.

Argument marshalling only -- every step of the forward pass runs inside the
CUDA library.  PyTorch supplies the device arena and the CUDA streams.  There
is no CPU fallback: importing this module without the built library, or
creating an engine without a CUDA device, raises.
"""
from __future__ import annotations

import ctypes as C
import os
import struct

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libvla_b200.so")

VLA_OK, VLA_ERR_INVALID, VLA_ERR_STATE, VLA_ERR_BUSY, VLA_ERR_NOT_READY, VLA_ERR_TIMEOUT, VLA_ERR_CUDA, VLA_ERR_NOMEM = range(8)
MODE_COSCHED, MODE_TWO_STREAM, MODE_SERIAL, MODE_MULTI_STREAM = 0, 1, 2, 3
MODES = {"cosched": MODE_COSCHED, "two_stream": MODE_TWO_STREAM, "serial": MODE_SERIAL, "multi_stream": MODE_MULTI_STREAM}
_MLP = {"gelu": 0, "swiglu": 1, "geglu": 2}
_HANDOFF = {"kv_last": 0, "kv_all": 1, "features": 2, "cog": 3}
_HEAD = {"A": 0, "B": 1, "C": 2, "D": 3}
_SOLVER = {"euler": 0, "ddim": 1}

EXPORTS = ["vla_required_arena_bytes", "vla_init", "vla_load_weights", "vla_submit_frame", "vla_submit_frame_device",
           "vla_poll_actions", "vla_hold_launches", "vla_wait_idle", "vla_get_trace", "vla_reset_trace", "vla_program_info", "vla_debug_fetch",
           "vla_get_counters", "vla_set_class_tags", "vla_get_class_tags", "vla_policy_probe", "vla_policy_probe_ex", "vla_debug_bump_dependency", "vla_debug_guards", "vla_last_error",
           "vla_destroy", "vla_op_status", "vla_debug_op_fault", "vla_debug_tile_linear", "vla_debug_tile_addends", "vla_debug_tile_attention",
           "vla_op_attention_scratch_bytes", "vla_op_attention", "vla_op_linear", "vla_op_linear_bias",
           "vla_op_attention_static_capacity", "vla_op_attention_static", "vla_op_quantize", "vla_op_linear_scaled",
           "vla_op_linear_grouped", "vla_op_linear_grouped_scaled", "vla_op_qk_norm_rope",
           "vla_op_attention_sequences_scratch_bytes", "vla_op_attention_packed", "vla_op_attention_paged", "vla_op_cache_store"]


class vla_model_desc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in (
        "n_cam", "img", "patch", "vis_layers", "vis_d", "vis_heads", "vis_hd", "vis_mlp", "shuffle", "connector",
        "n_text", "vocab", "llm_layers", "d", "hq", "hkv", "hd", "mlp", "mlp_kind", "rope", "causal", "handoff",
        "head", "act_layers", "act_d", "act_heads", "act_mlp", "act_mlp_kind", "state_dim", "horizon", "act_dim",
        "n_steps", "solver")] + [("guidance", C.c_float), ("suffix_mask", C.c_int32), ("vis_layernorm", C.c_int32)]


class vla_runtime_opts(C.Structure):
    _fields_ = [("arena", C.c_void_p), ("arena_bytes", C.c_size_t), ("stream_a", C.c_void_p), ("stream_b", C.c_void_p),
                ("mode", C.c_int32), ("n_streams", C.c_int32), ("ring_depth", C.c_int32), ("policy", C.c_int32),
                ("wait_limit_ns", C.c_uint64), ("trace_capacity", C.c_uint32), ("workers_per_sm", C.c_int32),
                ("u_max", C.c_int32), ("head_passes", C.c_int32), ("reserved_", C.c_int32)]


class vla_tensor(C.Structure):
    _fields_ = [("name", C.c_char_p), ("host_ptr", C.c_void_p), ("dtype", C.c_int32), ("rank", C.c_int32),
                ("shape", C.c_int64 * 4)]


class vla_trace_rec(C.Structure):
    _fields_ = [("inst", C.c_uint32), ("node", C.c_uint32), ("tile", C.c_uint32), ("sm", C.c_uint16), ("worker", C.c_uint8),
                ("cls", C.c_uint8), ("frame", C.c_uint64), ("t_start", C.c_uint64), ("t_end", C.c_uint64)]


class vla_node_info(C.Structure):
    _fields_ = [("op", C.c_int32), ("cls", C.c_int32), ("n_tiles", C.c_int32), ("n_pred", C.c_int32), ("phase", C.c_int32),
                ("step", C.c_int32), ("succ_begin", C.c_int32), ("succ_count", C.c_int32), ("smem_bytes", C.c_int32), ("tmem_cols", C.c_int32),
                ("name", C.c_char * 48), ("flops", C.c_double), ("weight_bytes", C.c_double)]


TRACE_DTYPE = np.dtype([("inst", "<u4"), ("node", "<u4"), ("tile", "<u4"), ("sm", "<u2"), ("worker", "u1"), ("cls", "u1"),
                        ("frame", "<u8"), ("t_start", "<u8"), ("t_end", "<u8")])

_lib = None


def load_library() -> C.CDLL:
    """Loads the in-tree shared library; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_2609_22335_b200.build` (there is no CPU fallback)")
    lib = C.CDLL(LIB_PATH)
    P = C.POINTER
    lib.vla_required_arena_bytes.argtypes = [P(vla_model_desc), P(vla_runtime_opts), P(C.c_size_t)]
    lib.vla_init.argtypes = [P(vla_model_desc), P(vla_runtime_opts), P(C.c_void_p)]
    lib.vla_load_weights.argtypes = [C.c_void_p, P(vla_tensor), C.c_size_t, C.c_int32]
    for fn in (lib.vla_submit_frame, lib.vla_submit_frame_device):
        fn.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, P(C.c_uint64)]
    lib.vla_poll_actions.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, P(C.c_uint64)]
    lib.vla_wait_idle.argtypes = [C.c_void_p, C.c_uint32]
    lib.vla_hold_launches.argtypes = [C.c_void_p, C.c_int32]
    lib.vla_get_trace.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t, P(C.c_size_t)]
    lib.vla_reset_trace.argtypes = [C.c_void_p]
    lib.vla_program_info.argtypes = [C.c_void_p, P(vla_node_info), C.c_size_t, P(C.c_size_t), P(C.c_int32), C.c_size_t,
                                     P(C.c_size_t)]
    lib.vla_debug_fetch.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_char_p, C.c_void_p, C.c_size_t, P(C.c_size_t)]
    lib.vla_get_counters.argtypes = [C.c_void_p, P(C.c_uint64), P(C.c_uint64), P(C.c_uint64)]
    lib.vla_policy_probe.argtypes = [C.c_int32, P(C.c_int32), P(C.c_int32), P(C.c_int32), P(C.c_int32), P(C.c_int32),
                                     C.c_int32, C.c_int32, P(C.c_int32), P(C.c_int32)]
    lib.vla_policy_probe_ex.argtypes = [C.c_int32, P(C.c_int32), P(C.c_int32), P(C.c_int32), P(C.c_int32), P(C.c_int32),
                                        C.c_int32, C.c_int32, C.c_int32, P(C.c_int32), P(C.c_int32), P(C.c_int32), P(C.c_int32)]
    lib.vla_set_class_tags.argtypes = [C.c_void_p, P(C.c_int32)]
    lib.vla_get_class_tags.argtypes = [C.c_void_p, P(C.c_int32)]
    lib.vla_debug_guards.argtypes = [C.c_void_p, C.c_int32, P(C.c_size_t)]
    lib.vla_debug_bump_dependency.argtypes = [C.c_void_p] + [C.c_int32] * 4
    lib.vla_op_status.argtypes = [C.c_int32, C.c_void_p, C.c_void_p]
    lib.vla_debug_op_fault.argtypes = [C.c_int32, C.c_uint64]
    lib.vla_debug_tile_linear.argtypes = [C.c_void_p] * 5 + [C.c_int32] * 6
    lib.vla_debug_tile_addends.argtypes = [C.c_void_p] * 10 + [C.c_int32] * 4
    lib.vla_debug_tile_attention.argtypes = [C.c_void_p] * 6 + [C.c_int32] * 8
    lib.vla_op_attention_scratch_bytes.argtypes = [C.c_int32, C.c_int32, C.c_int32, P(C.c_size_t)]
    lib.vla_op_attention.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p] + [C.c_int32] * 6 + [C.c_void_p, C.c_size_t, C.c_void_p]
    lib.vla_op_linear.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p] + [C.c_int32] * 4 + [C.c_void_p]
    lib.vla_op_linear_bias.argtypes = [C.c_void_p] * 4 + [C.c_int32, C.c_int64] + [C.c_void_p] * 2 + [C.c_int32] * 4 + [C.c_void_p]
    lib.vla_op_attention_static_capacity.argtypes = [P(C.c_size_t)]
    lib.vla_op_attention_static.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p] + [C.c_int32] * 6 + [C.c_void_p]
    lib.vla_op_quantize.argtypes = [C.c_void_p, C.c_int32, C.c_int64, C.c_void_p, C.c_void_p] + [C.c_int32] * 3 + [C.c_void_p]
    lib.vla_op_linear_scaled.argtypes = [C.c_void_p] * 6 + [C.c_int32] * 4 + [C.c_void_p]
    lib.vla_op_linear_grouped.argtypes = [C.c_void_p] * 5 + [C.c_int32] * 5 + [C.c_void_p]
    lib.vla_op_linear_grouped_scaled.argtypes = [C.c_void_p] * 7 + [C.c_int32] * 5 + [C.c_void_p]
    lib.vla_op_qk_norm_rope.argtypes = ([C.c_void_p] * 2 + [C.c_int32] + [C.c_int64] * 2 + [C.c_void_p] * 2 + [C.c_int64] * 2 + [C.c_int32] * 4 +
                                        [C.c_void_p] * 2 + [C.c_float, C.c_void_p] + [C.c_int32] * 2 + [C.c_float, C.c_int32, C.c_void_p])
    lib.vla_op_attention_sequences_scratch_bytes.argtypes = [C.c_int32, P(C.c_size_t)]
    for fn in (lib.vla_op_attention_packed, lib.vla_op_attention_paged, lib.vla_op_cache_store):
        fn.argtypes = [C.c_char_p, C.c_void_p]                                  # (a struct's bytes: thirty arguments one by one took 3 us more)
    lib.vla_last_error.argtypes = [C.c_void_p]
    lib.vla_last_error.restype = C.c_char_p
    lib.vla_destroy.argtypes = [C.c_void_p]
    for name in EXPORTS:
        if name != "vla_last_error":
            getattr(lib, name).restype = C.c_int
    _lib = lib
    return lib


def make_desc(m) -> vla_model_desc:
    """vla_synth ModelDesc (or any object with the same fields) -> C struct."""
    d = vla_model_desc()
    for name, _ in vla_model_desc._fields_:
        v = getattr(m, name, 0)
        if name in ("mlp_kind", "act_mlp_kind"):
            v = _MLP[v]
        elif name == "handoff":
            v = _HANDOFF[v]
        elif name == "head":
            v = _HEAD[v]
        elif name == "solver":
            v = _SOLVER[v]
        setattr(d, name, float(v) if name == "guidance" else int(v))
    return d


class VlaError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"vla error {code}: {msg}")
        self.code = code


def vla_required_arena_bytes(desc: vla_model_desc, opts: vla_runtime_opts) -> int:
    out = C.c_size_t(0)
    rc = load_library().vla_required_arena_bytes(C.byref(desc), C.byref(opts), C.byref(out))
    if rc != VLA_OK:
        raise VlaError(rc, "invalid model description or options")
    return out.value


class Engine:
    """One library context plus the torch-owned arena and streams it runs on."""

    def __init__(self, model, mode="cosched", n_streams=None, ring_depth=2, policy=0, trace_capacity=0,
                 wait_limit_ns=0, workers_per_sm=0, u_max=0, head_passes=1, device="cuda:0"):
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("a CUDA device is required (there is no CPU fallback)")
        self.lib = load_library()
        self.torch = torch
        self.model = model
        self.device = torch.device(device)
        torch.cuda.set_device(self.device)
        self.desc = make_desc(model)
        self.n_streams = int(n_streams if n_streams is not None else model.n_streams)
        self.ring_depth = ring_depth
        self.mode = MODES[mode] if isinstance(mode, str) else int(mode)
        self.opts = vla_runtime_opts()
        self.opts.mode = self.mode
        self.opts.n_streams = self.n_streams
        self.opts.ring_depth = ring_depth
        self.opts.policy = policy
        self.opts.wait_limit_ns = wait_limit_ns
        self.opts.trace_capacity = trace_capacity
        self.opts.workers_per_sm = workers_per_sm
        self.opts.u_max = u_max
        self.opts.head_passes = head_passes
        self.arena_bytes = vla_required_arena_bytes(self.desc, self.opts)
        self.arena = torch.empty(self.arena_bytes + 256, dtype=torch.uint8, device=self.device)
        base = self.arena.data_ptr()
        self.opts.arena = (base + 255) // 256 * 256
        self.opts.arena_bytes = self.arena_bytes
        self.stream_a = torch.cuda.Stream(device=self.device)
        self.stream_b = torch.cuda.Stream(device=self.device)
        self.opts.stream_a = self.stream_a.cuda_stream
        self.opts.stream_b = self.stream_b.cuda_stream
        self.ctx = C.c_void_p(None)
        rc = self.lib.vla_init(C.byref(self.desc), C.byref(self.opts), C.byref(self.ctx))
        if rc != VLA_OK:
            msg = self.last_error() if self.ctx else "vla_init failed"
            if self.ctx:
                self.lib.vla_destroy(self.ctx)
                self.ctx = C.c_void_p(None)
            raise VlaError(rc, msg)
        self.head_passes = max(1, int(head_passes))
        self._frames_done = [0] * self.n_streams     # frames of each stream whose chunk has been polled
        self.chunk_shape = (model.horizon, model.act_dim) if self.head_passes == 1 else (self.head_passes, model.horizon, model.act_dim)

    # ---- thin wrappers -------------------------------------------------------------
    def last_error(self) -> str:
        return (self.lib.vla_last_error(self.ctx) or b"").decode()

    def _check(self, rc):
        if rc != VLA_OK:
            raise VlaError(rc, self.last_error())

    def load_weights(self, weights, batch_bytes=1 << 30):
        """weights: mapping name -> fp32 ndarray of bf16-representable values (vla_synth.gen.Weights)."""
        from vla_synth.gen import bf16_bits
        from vla_synth.configs import is_vector
        names = list(weights.names())
        batch, keep, size = [], [], 0

        def flush(final):
            arr = (vla_tensor * len(batch))(*batch)
            self._check(self.lib.vla_load_weights(self.ctx, arr, len(batch), 1 if final else 0))
            batch.clear(); keep.clear()

        for i, name in enumerate(names):
            w = weights[name]
            fp32 = is_vector(name) or name in ("vis.pos", "llm.pos", "act.pos")
            a = np.ascontiguousarray(w, dtype=np.float32) if fp32 else bf16_bits(w)
            keep.append(a)
            t = vla_tensor()
            t.name = name.encode()
            t.host_ptr = a.ctypes.data
            t.dtype = 0 if fp32 else 1
            t.rank = a.ndim
            for k, s in enumerate(a.shape):
                t.shape[k] = s
            batch.append(t)
            size += a.nbytes
            if size >= batch_bytes and i + 1 < len(names):
                flush(False)
                size = 0
        flush(True)

    def submit(self, stream, frame) -> int:
        """frame: dict image/text/state/noise of host numpy arrays. Returns VLA_OK or VLA_ERR_BUSY; raises otherwise."""
        img = np.ascontiguousarray(frame["image"], dtype=np.float32)
        txt = np.ascontiguousarray(frame["text"], dtype=np.int32)
        st = None if frame.get("state") is None else np.ascontiguousarray(frame["state"], dtype=np.float32)
        nz = np.ascontiguousarray(frame["noise"], dtype=np.float32)
        rc = self.lib.vla_submit_frame(self.ctx, stream, img.ctypes.data, txt.ctypes.data,
                                       None if st is None else st.ctypes.data, nz.ctypes.data, None)
        if rc not in (VLA_OK, VLA_ERR_BUSY):
            self._check(rc)
        return rc

    def submit_ptrs(self, stream, image_ptr, text_ptr, state_ptr, noise_ptr, device=False) -> int:
        fn = self.lib.vla_submit_frame_device if device else self.lib.vla_submit_frame
        rc = fn(self.ctx, stream, image_ptr, text_ptr, state_ptr, noise_ptr, None)
        if rc not in (VLA_OK, VLA_ERR_BUSY):
            self._check(rc)
        return rc

    def poll(self, stream, out=None):
        """Returns (chunk ndarray, frame id) or None when nothing is ready."""
        if out is None:
            out = np.empty(self.chunk_shape, dtype=np.float32)
        fid = C.c_uint64(0)
        rc = self.lib.vla_poll_actions(self.ctx, stream, out.ctypes.data, C.byref(fid))
        if rc == VLA_ERR_NOT_READY:
            return None
        self._check(rc)
        self._frames_done[stream] = fid.value + 1
        return out, fid.value

    def hold_launches(self, on):
        """While on, submitted frames are queued but the persistent kernel is not launched (see vla_hold_launches)."""
        self._check(self.lib.vla_hold_launches(self.ctx, int(bool(on))))

    def wait_idle(self, timeout_ms=60000):
        self._check(self.lib.vla_wait_idle(self.ctx, timeout_ms))

    def run(self, frames, timeout_s=600.0):
        """frames[r][n] -> chunks[r][n]; submits as fast as the rings accept and polls in frame order.

        The calling thread polls without a pause until nothing has come for 0.1 s (a chunk is usually milliseconds away, and a
        sleep would add its 60 us and more): it keeps one host core busy while frames are in flight.  A program that cannot
        spare the core calls ``submit`` and ``poll`` in its own rhythm.
        """
        import time
        R = len(frames)
        base = list(self._frames_done)
        nxt = [0] * R
        got = [[None] * len(frames[r]) for r in range(R)]
        remaining = sum(len(f) for f in frames)
        t0 = last = time.time()
        while remaining:
            progressed = False
            for r in range(R):
                while nxt[r] < len(frames[r]):
                    if self.submit(r, frames[r][nxt[r]]) == VLA_ERR_BUSY:
                        break
                    nxt[r] += 1
                    progressed = True
            for r in range(R):
                while True:
                    res = self.poll(r)
                    if res is None:
                        break
                    chunk, fid = res
                    got[r][fid - base[r]] = chunk
                    remaining -= 1
                    progressed = True
            now = time.time()
            if progressed:
                last = now
            elif now - t0 > timeout_s:
                raise TimeoutError("no progress")
            elif now - last > 0.1:
                time.sleep(0.0002)
        return got

    def trace(self):
        n = C.c_size_t(0)
        self._check(self.lib.vla_get_trace(self.ctx, None, 0, C.byref(n)))
        cap = min(n.value, self.opts.trace_capacity)
        arr = np.zeros(cap, dtype=TRACE_DTYPE)
        if cap:
            self._check(self.lib.vla_get_trace(self.ctx, arr.ctypes.data, cap, C.byref(n)))
        return arr, n.value

    def reset_trace(self):
        self._check(self.lib.vla_reset_trace(self.ctx))

    def program_info(self):
        nn, ns = C.c_size_t(0), C.c_size_t(0)
        self._check(self.lib.vla_program_info(self.ctx, None, 0, C.byref(nn), None, 0, C.byref(ns)))
        nodes = (vla_node_info * nn.value)()
        succ = (C.c_int32 * max(ns.value, 1))()
        self._check(self.lib.vla_program_info(self.ctx, nodes, nn.value, C.byref(nn), succ, ns.value, C.byref(ns)))
        out = [dict(op=n.op, cls=n.cls, n_tiles=n.n_tiles, n_pred=n.n_pred, phase=n.phase, step=n.step,
                    smem_bytes=n.smem_bytes, tmem_cols=n.tmem_cols, flops=n.flops, weight_bytes=n.weight_bytes,
                    succ=[succ[n.succ_begin + i] for i in range(n.succ_count)], name=n.name.decode()) for n in nodes]
        return out

    def debug_fetch(self, stream, slot, name):
        n = C.c_size_t(0)
        self._check(self.lib.vla_debug_fetch(self.ctx, stream, slot, name.encode(), None, 0, C.byref(n)))
        out = np.empty(n.value, dtype=np.float32)
        self._check(self.lib.vla_debug_fetch(self.ctx, stream, slot, name.encode(), out.ctypes.data, n.value, C.byref(n)))
        return out

    def counters(self):
        a, b, c = C.c_uint64(0), C.c_uint64(0), C.c_uint64(0)
        self._check(self.lib.vla_get_counters(self.ctx, C.byref(a), C.byref(b), C.byref(c)))
        return dict(tiles=a.value, kernel_launches=b.value, persistent_launches=c.value)

    def class_tags(self):
        """The eight tile classes' (tau_TC, tau_ALU, tau_MEM) tags."""
        t = (C.c_int32 * 24)()
        self._check(self.lib.vla_get_class_tags(self.ctx, t))
        return [[t[3 * k + x] for x in range(3)] for k in range(8)]

    def set_class_tags(self, tags):
        """tags[8][3]; entries that are None keep their current value."""
        cur = self.class_tags()
        flat = [int((tags[k] or cur[k])[x]) for k in range(8) for x in range(3)]
        self._check(self.lib.vla_set_class_tags(self.ctx, (C.c_int32 * 24)(*flat)))

    def fill_guards(self):
        """Writes the guard pattern behind every buffer (see vla_debug_guards)."""
        self._check(self.lib.vla_debug_guards(self.ctx, 1, None))

    def overwritten_guards(self) -> int:
        """How many guards no longer hold the pattern (0 = no tile wrote outside its buffers)."""
        n = C.c_size_t(0)
        self._check(self.lib.vla_debug_guards(self.ctx, 0, C.byref(n)))
        return n.value

    def bump_dependency(self, stream, slot, node, delta):
        """Test hook: adds ``delta`` to one node's dependency counter (see vla_debug_bump_dependency)."""
        self._check(self.lib.vla_debug_bump_dependency(self.ctx, stream, slot, node, delta))

    def close(self):
        if self.ctx:
            self.lib.vla_destroy(self.ctx)
            self.ctx = C.c_void_p(None)
        self.arena = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


POLICIES = {"two_phase": 0, "class_order": 1, "round_robin": 2, "two_phase_g": 3, "two_phase_r": 4}
OP_LINEAR, OP_ATTENTION, OP_ATTENTION_STATIC, OP_LINEAR_SCALED, OP_LINEAR_GROUPED, OP_LINEAR_GROUPED_SCALED, OP_LINEAR_BIAS, OP_ATTENTION_PACKED, OP_ATTENTION_PAGED, OP_ATTENTION_SHORT = range(10)


def policy_probe(taus, pending, feasible, cta_count, u, rr_start=0, u_max=0, policy=0, grid=None, res=None):
    """Runs the device pick once on the GPU; returns (picked, phase, cta_count, u)."""
    lib = load_library()
    n = len(taus)
    flat = (C.c_int32 * (3 * n))(*[int(x) for t in taus for x in t])
    pend = (C.c_int32 * n)(*[int(bool(x)) for x in pending])
    feas = (C.c_int32 * n)(*[int(bool(x)) for x in feasible])
    cc = (C.c_int32 * n)(*[int(x) for x in cta_count])
    uu = (C.c_int32 * 3)(*[int(x) for x in u])
    picked, phase = C.c_int32(-1), C.c_int32(0)
    gg = None if grid is None else (C.c_int32 * n)(*[int(x) for x in grid])
    rs = None if res is None else (C.c_int32 * n)(*[int(x) for x in res])
    if policy == 0 and grid is None and res is None:
        rc = lib.vla_policy_probe(n, flat, pend, feas, cc, uu, rr_start, u_max, C.byref(picked), C.byref(phase))
    else:
        rc = lib.vla_policy_probe_ex(n, flat, pend, feas, cc, uu, rr_start, u_max, policy, gg, rs, C.byref(picked),
                                     C.byref(phase))
    if rc != VLA_OK:
        raise VlaError(rc, "policy probe failed")
    return picked.value, phase.value, list(cc), list(uu)


_current_stream = None


def _look_up_current_stream():
    """A function that asks torch for the current stream's handle.  (torch.cuda.current_stream() makes an object: a tenth of a small call's time.)"""
    global _current_stream
    import torch
    torch.cuda.init()
    of, device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
    _current_stream = lambda: of(device())                                       # noqa: E731
    return _current_stream


def _stream_ptr(stream):
    """The stream a call runs on: the one given or, for None, torch's current one (of the current device), behind the work that made the call's inputs."""
    return (_current_stream or _look_up_current_stream())() if stream is None else stream.cuda_stream


def op_attention_scratch_bytes(tkv, hkv, hd) -> int:
    out = C.c_size_t(0)
    rc = load_library().vla_op_attention_scratch_bytes(tkv, hkv, hd, C.byref(out))
    if rc != VLA_OK:
        raise VlaError(rc, "bad attention shape")
    return out.value


def op_attention(q, k, v, hq, hkv, hd, causal=False, scratch=None, stream=None):
    """q [tq, hq*hd], k/v [tkv, hkv*hd]: CUDA bf16 torch tensors.  Returns out [tq, hq*hd] bf16.  (Like every op_* below: on ``stream``, a
    torch.cuda.Stream, or on torch's current one.)"""
    import torch
    tq, tkv = q.shape[0], k.shape[0]
    out = _new(stream, q.shape, q.dtype, q)
    if scratch is None:
        scratch = _new(stream, (op_attention_scratch_bytes(tkv, hkv, hd),), torch.uint8, q)       # (goes back to its stream's memory when this returns)
    rc = load_library().vla_op_attention(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), tq, tkv, hq, hkv, hd,
                                         int(causal), scratch.data_ptr(), scratch.numel(), _stream_ptr(stream))
    if rc != VLA_OK:
        raise VlaError(rc, "vla_op_attention failed")
    return out


def op_linear(a, w, act=0, out_bf16=False, stream=None):
    """a [m,k], w [n,k]: CUDA bf16 torch tensors.  Returns act(a w^T) as fp32 (or bf16) [m,n]."""
    import torch                               # (the call's host time is what a small layer costs: nothing is looked up twice)
    m, k = a.shape
    n = w.shape[0]
    if out_bf16:
        out = _new(stream, (m, n), torch.bfloat16, a)
        p32, p16 = None, out.data_ptr()
    else:
        out = _new(stream, (m, n), torch.float32, a)
        p32, p16 = out.data_ptr(), None
    rc = (_lib or load_library()).vla_op_linear(a.data_ptr(), w.data_ptr(), p32, p16, m, n, k, act,
                                                _stream_ptr(stream))
    if rc != VLA_OK:
        raise VlaError(rc, "vla_op_linear failed")
    return out


def op_attention_static(q, k, v, out, hq, hkv, hd, causal=False, stream=None):
    """Attention for callers that may not allocate: scratch lives in a fixed device array inside the library.

    Unlike ``op_attention`` this wrapper creates nothing either: the caller supplies ``out``.  Shapes whose
    scratch need exceeds the fixed array raise with VLA_ERR_NOMEM.  Calls share the array, so do not overlap them.
    """
    tq, tkv = q.shape[0], k.shape[0]
    rc = load_library().vla_op_attention_static(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), tq, tkv, hq, hkv, hd,
                                                int(causal), _stream_ptr(stream))
    if rc == VLA_ERR_NOMEM:
        raise VlaError(rc, "attention shape needs more scratch than the library's fixed array holds")
    if rc != VLA_OK:
        raise VlaError(rc, "vla_op_attention_static failed")
    return out


def _refuse(name, why):
    raise VlaError(VLA_ERR_INVALID, f"{name}: {why}")


def _elsewhere(first, *others):
    """Whether any of the tensors (None: not given) is not on the current CUDA device.  (The calls below cost their host time: one question each.)"""
    import torch
    dev = first.get_device()
    if dev < 0 or dev != torch.cuda.current_device():
        return True
    for t in others:
        if t is not None and t.get_device() != dev:
            return True
    return False


def _new(stream, shape, dtype, like):
    """A result: memory of the stream that writes it (None: the current one), so that it is not handed out again while that one still runs."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    import torch
    with torch.cuda.stream(stream):
        return like.new_empty(shape, dtype=dtype)


def op_quantize(x, block_rows=1, stream=None):
    """x [m,k]: CUDA bf16 or fp32, rows may lie apart.  Returns (q [m,k] float8_e4m3fn, scales fp32 [ceil(m / block_rows), ceil(k / 128)]) with
    x ~ q * scale of its block of block_rows x 128 (see vla_op_quantize); block_rows 1 (activations) or 128 (weights)."""
    import torch
    f32 = x.dtype == torch.float32
    if x.dim() != 2 or not (f32 or x.dtype == torch.bfloat16) or _elsewhere(x):
        _refuse("op_quantize", "x is a bf16 or fp32 matrix on the current CUDA device")
    m, k = x.shape
    ld, step = x.stride()
    if m < 1 or k < 16 or k % 16 or step != 1 or (block_rows != 1 and block_rows != 128) or (m | k) >> 31:
        _refuse("op_quantize", "rows in one piece, at least one, k a multiple of 16, below 2^31 of either, block_rows 1 or 128")
    q = _new(stream, (m, k), torch.float8_e4m3fn, x)
    s = _new(stream, (m if block_rows == 1 else (m + 127) // 128, (k + 127) // 128), torch.float32, x)
    rc = (_lib or load_library()).vla_op_quantize(x.data_ptr(), int(f32), ld if m > 1 else k, q.data_ptr(), s.data_ptr(), m, k, block_rows,
                                                  _stream_ptr(stream))
    if rc != VLA_OK:
        raise VlaError(rc, "vla_op_quantize failed")
    return q, s


def _blocks(name, a, scale_a, w, scale_w, offsets, out, act, out_bf16, stream):
    """What the linear layers below have in common: their arguments looked at, the result made, and the C arguments in front of the sizes."""
    import torch
    dtype = torch.bfloat16 if scale_a is None else torch.float8_e4m3fn
    grouped = offsets is not None
    if a.dtype != dtype or w.dtype != dtype or a.dim() != 2 or w.dim() != (3 if grouped else 2) or _elsewhere(a, w, scale_a, scale_w, offsets, out):
        _refuse(name, f"a [rows,k] and w [{'experts,' if grouped else ''}n,k] are {dtype} on the current CUDA device")
    m, k = a.shape
    shape = w.shape
    n = shape[-2]
    if shape[-1] != k or not a.is_contiguous() or not w.is_contiguous() or (m | n | k | shape[0]) >> 31:
        _refuse(name, "a and w are contiguous, rows of the same k, all sizes below 2^31")
    if scale_a is not None:
        kb, nb = (k + 127) // 128, (n + 127) // 128
        if (scale_a.shape != (m, kb) or scale_w.shape != ((shape[0], nb, kb) if grouped else (nb, kb)) or scale_a.dtype != torch.float32 or
                scale_w.dtype != torch.float32 or not scale_a.is_contiguous() or not scale_w.is_contiguous()):
            _refuse(name, "scales are contiguous fp32, one for each row (of a) or 128 rows (of w) and 128 columns")
    if grouped and (offsets.shape != (shape[0] + 1,) or offsets.dtype != torch.int32 or not offsets.is_contiguous()):
        _refuse(name, "offsets is contiguous int32, [experts + 1]")
    result = torch.bfloat16 if out_bf16 else torch.float32
    if out is None:
        out = _new(stream, (m, n), result, a)
    elif out.shape != (m, n) or out.dtype != result or not out.is_contiguous():
        _refuse(name, "out is contiguous, [rows,n], fp32 or, with out_bf16, bf16")
    return m, n, k, out, (None, out.data_ptr()) if out_bf16 else (out.data_ptr(), None), _stream_ptr(stream)


def op_linear_bias(a, w, bias=None, residual=None, act=0, out_bf16=False, out=None, stream=None):
    """a [m,k], w [n,k]: CUDA bf16, contiguous; bias fp32 [n]; residual bf16 or fp32 [m,n], rows may lie apart.  Returns act(a w^T + bias) + residual as
    fp32 (or bf16) [m,n], in ``out`` where it is given, which may be the residual itself (see vla_op_linear_bias)."""
    if _bf16 is None:
        _look_up_types()
    name, sa, sw, dev = "op_linear_bias", a.shape, w.shape, a.get_device()
    elsewhere = dev < 0 or dev != _device_now() or w.get_device() != dev
    for t in (bias, residual, out):
        if t is not None and t.get_device() != dev:
            elsewhere = True
    if elsewhere or a.dtype != _bf16 or w.dtype != _bf16 or len(sa) != 2 or len(sw) != 2:
        _refuse(name, "a [m,k] and w [n,k] are bf16 on the current CUDA device, like all else")
    m, k = sa
    n = sw[0]
    if sw[1] != k or not a.is_contiguous() or not w.is_contiguous() or (m | n | k) >> 31:
        _refuse(name, "a and w are contiguous, rows of the same k, all sizes below 2^31")
    if bias is not None and (bias.shape != (n,) or bias.dtype != _f32 or not bias.is_contiguous()):
        _refuse(name, "bias is contiguous fp32, [n]")
    f32, ld, res = False, 0, None
    if residual is not None:
        f32 = residual.dtype == _f32
        if not (f32 or residual.dtype == _bf16) or residual.shape != (m, n) or (n > 1 and residual.stride(1) != 1):
            _refuse(name, "residual is bf16 or fp32 [m,n], rows in one piece")
        ld, res = residual.stride(0) if m > 1 else n, residual.data_ptr()
    result = _bf16 if out_bf16 else _f32
    if out is None:
        out = _new(stream, (m, n), result, a)
    elif out.shape != (m, n) or out.dtype != result or not out.is_contiguous():
        _refuse(name, "out is contiguous, [m,n], fp32 or, with out_bf16, bf16")
    p32, p16 = (None, out.data_ptr()) if out_bf16 else (out.data_ptr(), None)
    rc = (_lib or load_library()).vla_op_linear_bias(a.data_ptr(), w.data_ptr(), None if bias is None else bias.data_ptr(), res, int(f32), ld, p32, p16, m, n, k, act,
                                                     _stream_ptr(stream))
    if rc != VLA_OK:
        raise VlaError(rc, "vla_op_linear_bias failed")
    return out


def op_linear_scaled(a, scale_a, w, scale_w, act=0, out_bf16=False, stream=None):
    """a [m,k], w [n,k]: float8_e4m3fn with the scales ``op_quantize`` gives (block_rows 1 and 128).  Returns act(A W^T) of the scaled matrices as
    fp32 (or bf16) [m,n]."""
    m, n, k, out, (p32, p16), s = _blocks("op_linear_scaled", a, scale_a, w, scale_w, None, None, act, out_bf16, stream)
    rc = (_lib or load_library()).vla_op_linear_scaled(a.data_ptr(), scale_a.data_ptr(), w.data_ptr(), scale_w.data_ptr(), p32, p16, m, n, k, act, s)
    if rc != VLA_OK:
        raise VlaError(rc, "vla_op_linear_scaled failed")
    return out


def op_linear_grouped(a, w, offsets, act=0, out_bf16=False, out=None, stream=None):
    """a [t,k] bf16, rows sorted by expert; w [experts,n,k] bf16; offsets int32 [experts + 1] on the GPU: rows offsets[e] .. offsets[e + 1] go through
    expert e.  Returns act(a W_e^T) as fp32 (or bf16) [t,n]; rows outside of all experts are left as they were in ``out`` (without one: undefined)."""
    m, n, k, out, (p32, p16), s = _blocks("op_linear_grouped", a, None, w, None, offsets, out, act, out_bf16, stream)
    rc = (_lib or load_library()).vla_op_linear_grouped(a.data_ptr(), w.data_ptr(), offsets.data_ptr(), p32, p16, m, n, k, w.shape[0], act, s)
    if rc != VLA_OK:
        raise VlaError(rc, "vla_op_linear_grouped failed")
    return out


def op_linear_grouped_scaled(a, scale_a, w, scale_w, offsets, act=0, out_bf16=False, out=None, stream=None):
    """``op_linear_grouped`` on float8_e4m3fn operands: scale_a [t, ceil(k/128)], scale_w [experts, ceil(n/128), ceil(k/128)]."""
    m, n, k, out, (p32, p16), s = _blocks("op_linear_grouped_scaled", a, scale_a, w, scale_w, offsets, out, act, out_bf16, stream)
    rc = (_lib or load_library()).vla_op_linear_grouped_scaled(a.data_ptr(), scale_a.data_ptr(), w.data_ptr(), scale_w.data_ptr(), offsets.data_ptr(), p32, p16,
                                                               m, n, k, w.shape[0], act, s)
    if rc != VLA_OK:
        raise VlaError(rc, "vla_op_linear_grouped_scaled failed")
    return out


def op_qk_norm_rope(q, k, hq, hkv, hd, gq=None, gk=None, eps=1e-6, pos=None, pos0=0, base=10000.0, rot=None, interleaved=False,
                    out_q=None, out_k=None, stream=None):
    """RMS norm of each head of q [t, hq*hd] and k [t, hkv*hd] (CUDA bf16 or fp32, rows may lie apart; k None with hkv 0) and the rotation of the
    first ``rot`` values of each (None: all) by position: ``pos`` int32 [t], or pos0 + row.  gq, gk: fp32 gains [hd] or None.  Returns (out_q, out_k),
    bf16, new ones without gaps where none are given (see vla_op_qk_norm_rope)."""
    import torch
    name, f32, bf16 = "op_qk_norm_rope", torch.float32, torch.bfloat16
    dt = q.dtype
    if (dt != bf16 and dt != f32) or q.dim() != 2 or hq < 1 or hkv < 0 or (k is None) != (hkv == 0) or _elsewhere(q, k, gq, gk, pos, out_q, out_k):
        _refuse(name, "q, and k where there are key heads, are bf16 or fp32 matrices on the current CUDA device, like all else")
    t, wq = q.shape
    ld_q, step = q.stride()
    wk, ld_k, ptr_k, ld_ok, ptr_ok = hkv * hd, 0, None, 0, None
    if wq != hq * hd or step != 1 or t < 1 or (t | wq) >> 31:
        _refuse(name, "q is [t, hq*hd], rows in one piece, at least one, below 2^31 of either")
    if pos0 >> 31 not in (0, -1):
        _refuse(name, "pos0 is a 32-bit number")
    if k is not None:
        if k.dtype != dt or k.shape != (t, wk) or k.stride(1) != 1:
            _refuse(name, "k is [t, hkv*hd], of q's type, rows in one piece")
        ld_k, ptr_k = k.stride(0), k.data_ptr()
    for x in (gq, gk):
        if x is not None and (x.shape != (hd,) or x.dtype != f32 or not x.is_contiguous()):
            _refuse(name, "gains are contiguous fp32, [hd]")
    if pos is not None and (pos.shape != (t,) or pos.dtype != torch.int32 or not pos.is_contiguous()):
        _refuse(name, "pos is contiguous int32, [t]")
    if out_q is None:
        out_q, ld_oq = _new(stream, (t, wq), bf16, q), wq
    else:
        if out_q.dtype != bf16 or out_q.shape != (t, wq) or out_q.stride(1) != 1:
            _refuse(name, "out_q is bf16 [t, hq*hd], rows in one piece")
        ld_oq = out_q.stride(0)
    if hkv == 0:
        if out_k is not None:
            _refuse(name, "out_k goes with k")
    elif out_k is None:
        out_k, ld_ok = _new(stream, (t, wk), bf16, q), wk
    else:
        if out_k.dtype != bf16 or out_k.shape != (t, wk) or out_k.stride(1) != 1:
            _refuse(name, "out_k is bf16 [t, hkv*hd], rows in one piece")
        ld_ok = out_k.stride(0)
    if out_k is not None:
        ptr_ok = out_k.data_ptr()
    if t == 1:                                 # (the stride of one row says nothing)
        ld_q = ld_oq = wq
        ld_k = ld_ok = wk
    rc = (_lib or load_library()).vla_op_qk_norm_rope(q.data_ptr(), ptr_k, int(dt == f32), ld_q, ld_k, out_q.data_ptr(), ptr_ok, ld_oq, ld_ok, t, hq, hkv, hd,
                                                      None if gq is None else gq.data_ptr(), None if gk is None else gk.data_ptr(), eps,
                                                      None if pos is None else pos.data_ptr(), pos0, hd if rot is None else rot, base, int(interleaved),
                                                      _stream_ptr(stream))
    if rc != VLA_OK:
        raise VlaError(rc, "vla_op_qk_norm_rope failed")
    return out_q, out_k


def op_attention_sequences_scratch_bytes(hd) -> int:
    """Scratch memory of ``op_attention_packed`` and ``op_attention_paged`` at this head width."""
    out = C.c_size_t(0)
    rc = load_library().vla_op_attention_sequences_scratch_bytes(hd, C.byref(out))
    if rc != VLA_OK:
        raise VlaError(rc, "bad head width")
    return out.value


_bf16 = _f32 = _i32 = _u8 = _device_now = _empty_like = None


def _look_up_types():
    """torch's types as names of this module.  (The calls below ask some twenty questions each, and a statement that imports takes as long as two of them.)"""
    global _bf16, _f32, _i32, _u8, _device_now, _empty_like
    import torch
    _f32, _i32, _u8, _device_now, _empty_like, _bf16 = torch.float32, torch.int32, torch.uint8, torch._C._cuda_getDevice, torch.empty_like, torch.bfloat16


def _offsets(name, offsets, others):
    """The number of sequences, with the devices of all tensors looked at."""
    if _bf16 is None:
        _look_up_types()
    shape, dev = offsets.shape, offsets.get_device()
    bad = len(shape) != 1 or shape[0] < 2 or shape[0] >> 31 or offsets.dtype != _i32 or not offsets.is_contiguous() or dev < 0 or dev != _device_now()
    for t in others:
        if t is not None and t.get_device() != dev:
            bad = True
    if bad:
        _refuse(name, "offsets is contiguous int32 [seqs + 1], on the current CUDA device like all else")
    return shape[0] - 1


def _row_step(name, what, x, rows, width):
    """Elements from one row of x [rows, width] (bf16) to the next."""
    if x.dtype != _bf16 or x.shape != (rows, width):
        _refuse(name, what)
    ld, one = x.stride()
    if one != 1:
        _refuse(name, what + ", rows in one piece")
    return ld if rows > 1 else width                                # (the stride of one row says nothing)


def _sequences(name, q, seqs, keys, hq, hkv, hd, prefix, window, cap, slopes, scale, out, scratch, stream):
    """What the two attentions below have in common, ``keys`` being the most that a sequence may have: (tq, ld_q, out, ld_out, scratch, its pointer and bytes, pointers of
    prefix and slopes, scale, whose status word)."""
    if q.dim() != 2 or hq < 1 or hkv < 1 or hd < 8 or hd > 256 or hd % 8:
        _refuse(name, "q is a matrix; hd a multiple of 8, at most 256")
    tq, width = q.shape[0], hq * hd
    if tq < 1 or (tq | width | hkv * hd) >> 31 or window >> 31:
        _refuse(name, "at least one row, below 2^31 of them, window a number from 0 to 2^31 - 1")
    if scale is None:
        scale = hd ** -0.5
    if not (0.0 <= cap < 1e30 and 0.0 < scale < 1e30):
        _refuse(name, "cap a number from 0, scale one above 0, both below 1e30")
    ld_q = _row_step(name, "q is bf16 [tq, hq*hd]", q, tq, width)
    p_prefix = p_slopes = 0
    if prefix is not None:
        if prefix.shape != (seqs,) or prefix.dtype != _i32 or not prefix.is_contiguous():
            _refuse(name, "prefix is contiguous int32, [seqs]")
        p_prefix = prefix.data_ptr()
    if slopes is not None:
        if slopes.shape != (hq,) or slopes.dtype != _f32 or not slopes.is_contiguous():
            _refuse(name, "slopes is contiguous fp32, [hq]")
        p_slopes = slopes.data_ptr()
    if out is None:
        out, ld_out = _empty_like(q) if stream is None else _new(stream, (tq, width), _bf16, q), width      # (contiguous, whatever lies between q's rows)
    else:
        ld_out = _row_step(name, "out is bf16 [tq, hq*hd]", out, tq, width)
    status = 0
    if scratch is None:
        size, at, status = 0, 0, OP_ATTENTION_SHORT
        if keys > 512:                                              # (shorter calls need none; goes back to its stream's memory when the call returns, so the status lies elsewhere)
            size = _scratch_sizes.get(hd)
            if size is None:
                size = _scratch_sizes[hd] = op_attention_sequences_scratch_bytes(hd)
            scratch = _new(stream, (size,), _u8, q)
            at = scratch.data_ptr()
    elif scratch.dtype != _u8 or not scratch.is_contiguous():
        _refuse(name, "scratch is contiguous uint8")
    else:
        size, at = scratch.numel(), scratch.data_ptr()
    return tq, ld_q, out, ld_out, scratch, at, size, p_prefix, p_slopes, scale, status


_scratch_sizes = {}


_ATTENTION_ARGS = struct.Struct("=18Q11i2fi")                        # vla_attention_args
_CACHE_STORE_ARGS = struct.Struct("=13Q6i")                          # vla_cache_store_args


def op_attention_packed(q, k, v, offsets, hq, hkv, hd, offsets_k=None, causal=False, prefix=None, window=0, cap=0.0, slopes=None, scale=None, out=None,
                        scratch=None, stream=None):
    """Attention of sequences that lie behind one another, each within itself: rows offsets[s] .. offsets[s + 1] of q [tq, hq*hd], and of k and v
    [tk, hkv*hd] (or offsets_k[s] .. offsets_k[s + 1] of them), are sequence s.  CUDA bf16, rows may lie apart; offsets int32 [seqs + 1] on the GPU.
    causal: row i of nq sees the keys up to nk - nq + i, the last ``window`` of them (0: all), and the first prefix[s] whatever their place.  cap: scores become
    cap tanh(s / cap); slopes fp32 [hq]: a score loses slopes[h] times the distance.  scale None: 1 / sqrt(hd).  Returns out [tq, hq*hd] bf16; rows that no
    sequence has are left as they were in ``out`` (without one: undefined), rows that see no key are zeros (see vla_op_attention_packed)."""
    name = "op_attention_packed"
    seqs = _offsets(name, offsets, (q, k, v, offsets_k, prefix, slopes, out, scratch))
    tk = k.shape[0]
    tq, ld_q, out, ld_out, scratch, at, size, p_prefix, p_slopes, scale, status = _sequences(name, q, seqs, tk, hq, hkv, hd, prefix, window, cap, slopes, scale, out, scratch, stream)
    if offsets_k is None:
        offsets_k = offsets
        if tk != tq:
            _refuse(name, "without offsets_k, k and v have q's rows")
    elif offsets_k.shape != (seqs + 1,) or offsets_k.dtype != offsets.dtype or not offsets_k.is_contiguous():
        _refuse(name, "offsets_k is contiguous int32, [seqs + 1]")
    if tk < 1 or tk >> 31:
        _refuse(name, "k and v have at least one row, below 2^31 of them")
    ld_k, ld_v = _row_step(name, "k is bf16 [tk, hkv*hd]", k, tk, hkv * hd), _row_step(name, "v is bf16 [tk, hkv*hd]", v, tk, hkv * hd)
    args = _ATTENTION_ARGS.pack(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), ld_q, ld_k, ld_v, ld_out, 0, 0, offsets.data_ptr(), offsets_k.data_ptr(), 0, 0,
                                p_prefix, p_slopes, at, size, seqs, tq, tk, 0, 0, 0, hq, hkv, hd, 1 if causal else 0, window, scale, cap, status)
    rc = (_lib or load_library()).vla_op_attention_packed(args, _stream_ptr(stream))
    if rc != VLA_OK:
        raise VlaError(rc, "vla_op_attention_packed failed")
    return out


def _cache(name, k_cache, v_cache, pages, lengths, seqs, width):
    """Sizes and strides of a cache's two tensors: (n_pages, page_size, max_pages, row_k, page_k, row_v, page_v)."""
    shape = k_cache.shape
    if len(shape) != 3 or shape[2] != width or v_cache.shape != shape or k_cache.dtype != _bf16 or v_cache.dtype != _bf16:
        _refuse(name, "k_cache and v_cache are bf16 [n_pages, page_size, hkv*hd]")
    n, size, _ = shape
    (page_k, row_k, one_k), (page_v, row_v, one_v) = k_cache.stride(), v_cache.stride()
    if one_k != 1 or one_v != 1 or n < 1 or size < 1 or (n | size) >> 31:
        _refuse(name, "the caches' rows are in one piece, at least one page of at least one row, below 2^31 of either")
    if size == 1:                                                   # (the stride of a single row or page says nothing)
        row_k = row_v = width
    if n == 1:
        page_k, page_v = size * row_k, size * row_v
    table = pages.shape
    if len(table) != 2 or pages.dtype != _i32 or not pages.is_contiguous() or lengths.shape != (seqs,) or lengths.dtype != _i32 or not lengths.is_contiguous():
        _refuse(name, "pages [seqs, max_pages] and lengths [seqs] are contiguous int32")
    rows, most = table
    if rows != seqs or most < 1 or most >> 31:
        _refuse(name, "pages has a row of at least one entry for each sequence")
    return n, size, most, row_k, page_k, row_v, page_v


def op_attention_paged(q, k_cache, v_cache, pages, lengths, offsets, hq, hkv, hd, causal=True, prefix=None, window=0, cap=0.0, slopes=None, scale=None, out=None,
                       scratch=None, stream=None):
    """``op_attention_packed`` of the new tokens over keys and values that lie in pages: rows offsets[s] .. offsets[s + 1] of q are the last ones of
    lengths[s] tokens, of which token j is row j % page_size of page pages[s, j // page_size] of k_cache and v_cache [n_pages, page_size, hkv*hd].
    page_size a multiple of 8; pages int32 [seqs, max_pages], lengths int32 [seqs], offsets int32 [seqs + 1], all on the GPU; entries of ``pages`` behind a
    sequence's length are not looked at (see vla_op_attention_paged)."""
    name = "op_attention_paged"
    seqs = _offsets(name, offsets, (q, k_cache, v_cache, pages, lengths, prefix, slopes, out, scratch))
    n, page, most, row_k, page_k, row_v, page_v = _cache(name, k_cache, v_cache, pages, lengths, seqs, hkv * hd)
    tq, ld_q, out, ld_out, scratch, at, size, p_prefix, p_slopes, scale, status = _sequences(name, q, seqs, most * page, hq, hkv, hd, prefix, window, cap, slopes, scale, out, scratch, stream)
    args = _ATTENTION_ARGS.pack(q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), out.data_ptr(), ld_q, row_k, row_v, ld_out, page_k, page_v, offsets.data_ptr(), 0,
                                lengths.data_ptr(), pages.data_ptr(), p_prefix, p_slopes, at, size, seqs, tq, 0, n, page, most, hq, hkv, hd, 1 if causal else 0,
                                window, scale, cap, status)
    rc = (_lib or load_library()).vla_op_attention_paged(args, _stream_ptr(stream))
    if rc != VLA_OK:
        raise VlaError(rc, "vla_op_attention_paged failed")
    return out


def op_cache_store(k, v, k_cache, v_cache, pages, lengths, offsets, stream=None):
    """New keys and values into the pages that ``op_attention_paged`` reads: rows offsets[s] .. offsets[s + 1] of k and v [t, hkv*hd] (CUDA bf16, rows may lie
    apart) become the last ones of lengths[s] tokens.  Rows whose place is in front of the first token, behind the table or on a page that does not exist
    are left out (see vla_op_cache_store)."""
    name = "op_cache_store"
    seqs = _offsets(name, offsets, (k, v, k_cache, v_cache, pages, lengths))
    if k.dim() != 2:
        _refuse(name, "k and v are matrices")
    t, width = k.shape
    if t < 1 or (t | width) >> 31:
        _refuse(name, "at least one row, below 2^31 of them")
    ld_k, ld_v = _row_step(name, "k is bf16 [t, hkv*hd]", k, t, width), _row_step(name, "v is bf16 [t, hkv*hd]", v, t, width)
    n, size, most, row_k, page_k, row_v, page_v = _cache(name, k_cache, v_cache, pages, lengths, seqs, width)
    args = _CACHE_STORE_ARGS.pack(k.data_ptr(), v.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), ld_k, ld_v, row_k, page_k, row_v, page_v, pages.data_ptr(), lengths.data_ptr(),
                                  offsets.data_ptr(), seqs, t, n, size, most, width)
    rc = (_lib or load_library()).vla_op_cache_store(args, _stream_ptr(stream))
    if rc != VLA_OK:
        raise VlaError(rc, "vla_op_cache_store failed")


def op_status(op, scratch=None, stream=None) -> int:
    """Waits for ``stream`` (None: torch's current one) and returns the operator's status word as a VLA_* code (VLA_OK or VLA_ERR_TIMEOUT).
    Operators with ``scratch`` have it there: pass the same.  OP_ATTENTION_SHORT: of calls of ``op_attention_packed`` and ``op_attention_paged`` that were given
    none (a word per device: ask before another such call is made)."""
    return load_library().vla_op_status(op, None if scratch is None else scratch.data_ptr(), _stream_ptr(stream))


def debug_op_fault(drop_operand_loads, wait_limit_ns=0):
    """Test hook: make the operators' bounded waits run out (see vla_debug_op_fault; True is 1)."""
    rc = load_library().vla_debug_op_fault(int(drop_operand_loads), int(wait_limit_ns))
    if rc != VLA_OK:
        raise VlaError(rc, "vla_debug_op_fault failed")


def debug_tile_linear(a, w, n, x=None, act=0, gated=False, fast=False, out32=True, out16=False):
    """Test hook: the engine's GEMM tile body (see vla_debug_tile_linear).  Returns (fp32 [m,n] or None, bf16 [m,n] or None)."""
    import torch
    m, k = a.shape
    o32 = a.new_empty((m, n), dtype=torch.float32) if out32 else None
    o16 = a.new_empty((m, n), dtype=torch.bfloat16) if out16 else None
    ptr = lambda t: None if t is None else t.data_ptr()
    rc = load_library().vla_debug_tile_linear(a.data_ptr(), w.data_ptr(), ptr(x), ptr(o32), ptr(o16), m, n, k, act, int(gated), int(fast))
    if rc != VLA_OK:
        raise VlaError(rc, "vla_debug_tile_linear failed")
    return o32, o16


def debug_tile_addends(a, w, n, x=None, bias=None, vec=None, tab=None, tab2=None, act=0, out32=True, out16=False, ss=False, in_place=False):
    """Test hook: the GEMM tile body with addends (see vla_debug_tile_addends).  Returns (fp32 [m,n], bf16 [m,n], sums of squares), None
    where not asked for; ``in_place``: the fp32 rows take the place of ``x``."""
    import torch
    m, k = a.shape
    o32 = x if in_place else a.new_empty((m, n), dtype=torch.float32) if out32 else None
    o16 = a.new_empty((m, n), dtype=torch.bfloat16) if out16 else None
    sums = a.new_empty((m, (n + 127) // 128), dtype=torch.float32) if ss else None
    ptr = lambda t: None if t is None else t.data_ptr()
    rc = load_library().vla_debug_tile_addends(a.data_ptr(), w.data_ptr(), ptr(x), ptr(bias), ptr(vec), ptr(tab), ptr(tab2), ptr(o32), ptr(o16),
                                               ptr(sums), m, n, k, act)
    if rc != VLA_OK:
        raise VlaError(rc, "vla_debug_tile_addends failed")
    return o32, o16, sums


def debug_tile_attention(q, k0, v0, hq, hkv, hd, k1=None, v1=None, causal=False, sfx=0):
    """Test hook: the engine's attention tile body (see vla_debug_tile_attention); v0, v1 [t, hkv*hd] as they lie."""
    import torch

    def transposed(v):
        t = v.new_zeros((v.shape[1], (v.shape[0] + 63) // 64 * 64))
        t[:, :v.shape[0]] = v.T
        return t
    vt0, vt1 = transposed(v0), None if v1 is None else transposed(v1)
    out = torch.empty_like(q)
    rc = load_library().vla_debug_tile_attention(q.data_ptr(), k0.data_ptr(), vt0.data_ptr(), None if k1 is None else k1.data_ptr(),
                                                 None if vt1 is None else vt1.data_ptr(), out.data_ptr(), q.shape[0], k0.shape[0],
                                                 0 if k1 is None else k1.shape[0], hq, hkv, hd, int(causal), sfx)
    if rc != VLA_OK:
        raise VlaError(rc, "vla_debug_tile_attention failed")
    return out
