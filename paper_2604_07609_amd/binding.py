"""ctypes binding of include/blink.h. Same names as the C ABI, numpy arrays in and out."""
import ctypes as C
import os
import struct
import sys

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))

FLAG_TRACE, FLAG_EXIT_WHEN_IDLE, FLAG_KEEP_LOGITS, FLAG_NO_GRAPH, FLAG_CHUNKED_PREFILL, FLAG_PREEMPTION, FLAG_PREFIX_CACHE, FLAG_SPECULATIVE = 1, 2, 8, 16, 32, 64, 128, 256
FLAG_HOST_STEP = 512
ERR_INVAL, ERR_TOO_LARGE, ERR_FULL, ERR_DEVICE, ERR_STATE = -1, -2, -3, -4, -5
EVENT_FIRST, EVENT_LAST = 1, 2

EXPORTS = ["blink_init", "blink_init_attention", "blink_submit", "blink_run", "blink_set_exit_when_idle", "blink_wait", "blink_stop", "blink_poll_outputs", "blink_shutdown",
           "blink_get_trace", "blink_get_stats", "blink_debug_read", "blink_time_phase", "blink_get_phase_times", "blink_calibration_copy",
           "blink_calibration_rates", "blink_clock_sync", "blink_sample_rows", "blink_sample_rows_static", "blink_kv_cache_bytes", "blink_qk_norm_rope",
           "blink_kv_cache_read", "blink_paged_attention", "blink_attention_workspace_bytes", "blink_last_error"]


class DBG:
    LOGITS, FREE_STACK, INPUT_IDS, POSITIONS, SLOT_MAPPING, SEQ_BATCH_SLOT, BLOCK_TABLES, SEQ_LENS, CU_SEQLENS, \
        SLOT_STATES, HIDDEN, ROUTING, ATTN_ITEMS = range(1, 14)


class Config(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("n_layers", "d_model", "n_q_heads", "n_kv_heads", "head_dim", "d_ffn", "vocab", "dtype")] + [
        ("rms_eps", C.c_float), ("rope_theta", C.c_float), ("weights", C.c_void_p), ("weights_bytes", C.c_uint64),
        ("kv_block_size", C.c_uint32), ("kv_num_blocks", C.c_uint32), ("max_batch", C.c_uint32), ("max_seq_len", C.c_uint32),
        ("max_prefill_tokens", C.c_uint32), ("ring_slots", C.c_uint32), ("eos_token_id", C.c_int32), ("device", C.c_int32),
        ("flags", C.c_uint32), ("trace_capacity", C.c_uint32), ("idle_poll_us", C.c_uint32), ("pump_depth", C.c_uint32),
        ("tune", C.c_uint32), ("n_experts", C.c_uint32), ("n_active", C.c_uint32), ("spec_tokens", C.c_uint32)]


class AttentionOptions(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("qk_norm", "window", "sinks", "kv_bits")]


class Sampling(C.Structure):
    _fields_ = [("temperature", C.c_float), ("top_k", C.c_uint32), ("top_p", C.c_float), ("seed", C.c_uint64)]


class CacheDesc(C.Structure):
    _fields_ = [("data", C.c_void_p), ("n_blocks", C.c_uint32), ("n_kv_heads", C.c_uint32), ("head_dim", C.c_uint32), ("bits", C.c_uint32)]


class QkNormRopeArgs(C.Structure):
    _fields_ = [("cache", CacheDesc)] + [(n, C.c_uint32) for n in ("n_q_heads", "n_tokens", "in_type", "rope_rows")] + [
        (n, C.c_void_p) for n in ("q", "k", "v")] + [(n, C.c_uint64) for n in ("q_stride", "k_stride", "v_stride")] + [
        (n, C.c_void_p) for n in ("q_gain", "k_gain", "positions", "slots", "rope_table", "q_out")] + [
        ("q_out_stride", C.c_uint64), ("eps", C.c_float), ("q_scale", C.c_float)]


class PagedAttentionArgs(C.Structure):
    _fields_ = [("cache", CacheDesc)] + [(n, C.c_uint32) for n in ("n_q_heads", "n_seqs", "n_tokens", "max_q", "max_blocks", "window", "sinks")] + [
        ("scale", C.c_float), ("q", C.c_void_p), ("out", C.c_void_p), ("q_stride", C.c_uint64), ("out_stride", C.c_uint64)] + [
        (n, C.c_void_p) for n in ("cu_seqlens", "seq_lens", "block_tables", "workspace")] + [("workspace_bytes", C.c_uint64)]


# the same three as `struct` packs them (fields in order, native alignment)
_CACHE, _QK_NORM_ROPE, _PAGED_ATTENTION = struct.Struct("@P4I"), struct.Struct("@P4I4I3P3Q6PQ2f"), struct.Struct("@P4I7If2P2Q4PQ")


class Stats(C.Structure):
    _fields_ = [("iterations", C.c_uint64), ("prefill_iterations", C.c_uint64), ("tokens_out", C.c_uint64),
                ("tokens_prefilled", C.c_uint64), ("next_ticket", C.c_uint64), ("n_running", C.c_uint32),
                ("free_blocks", C.c_uint32), ("committed_blocks", C.c_uint32), ("device_error", C.c_uint32),
                ("running", C.c_uint32), ("windows", C.c_uint32), ("kv_bytes", C.c_uint64), ("weight_bytes", C.c_uint64),
                ("ring_bytes", C.c_uint64), ("prefix_hit_blocks", C.c_uint64), ("prefix_evictions", C.c_uint64),
                ("pinned_blocks", C.c_uint32), ("pad1", C.c_uint32), ("spec_drafted", C.c_uint64), ("spec_accepted", C.c_uint64)]


EVENT_DTYPE = np.dtype([("request_id", "<u8"), ("index", "<u4"), ("token", "<i4"), ("flags", "<u4"), ("iteration", "<u4"),
                        ("device_ns", "<u8")], align=True)
TRACE_DTYPE = np.dtype([("iteration", "<u4"), ("kind", "<u4"), ("tail", "<u8"), ("n_admitted", "<u4"), ("n_seqs", "<u4"),
                        ("n_tokens", "<u4"), ("free_blocks", "<u4"), ("first_admitted", "<u8"), ("t_sched_begin_ns", "<u8"),
                        ("t_sched_end_ns", "<u8"), ("t_forward_end_ns", "<u8"), ("t_publish_end_ns", "<u8"), ("ctx_tokens", "<u8"),
                        ("chain", "<u8"), ("n_resumed", "<u4"), ("n_preempted", "<u4")],
                       align=True)


class BlinkError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"blink error {code}: {msg}")
        self.code = code


def lib_path():
    return os.path.join(HERE, "libblink.so")


_lib = None


def load_library():
    """Loads libblink.so; raises if it has not been built (there is no fallback path)."""
    global _lib
    if _lib is not None:
        return _lib
    p = lib_path()
    if not os.path.exists(p):
        raise ImportError(f"{p} is missing: build it with `python -m paper_2604_07609_amd.build`")
    lib = C.CDLL(p)
    vp, u32, u64 = C.c_void_p, C.c_uint32, C.c_uint64
    lib.blink_init.argtypes = [C.POINTER(Config), C.POINTER(vp)]
    lib.blink_init_attention.argtypes = [C.POINTER(Config), C.POINTER(AttentionOptions), C.POINTER(vp)]
    lib.blink_submit.argtypes = [vp, vp, u32, u32, C.POINTER(Sampling), C.POINTER(u64)]
    lib.blink_run.argtypes = [vp, u64]
    lib.blink_wait.argtypes = [vp]
    lib.blink_set_exit_when_idle.argtypes = [vp, u32]
    lib.blink_stop.argtypes = [vp]
    lib.blink_poll_outputs.argtypes = [vp, vp, u32, C.POINTER(u32)]
    lib.blink_shutdown.argtypes = [vp]
    lib.blink_get_trace.argtypes = [vp, vp, u64, C.POINTER(u64)]
    lib.blink_get_stats.argtypes = [vp, C.POINTER(Stats)]
    lib.blink_debug_read.argtypes = [vp, u32, vp, u64, C.POINTER(u64)]
    lib.blink_time_phase.argtypes = [vp, C.c_int32]
    lib.blink_calibration_copy.argtypes = [vp, u64]
    lib.blink_calibration_rates.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(C.c_double), C.POINTER(C.c_double)]
    lib.blink_get_phase_times.argtypes = [vp, vp, u64, C.POINTER(u64)]
    lib.blink_clock_sync.argtypes = [vp, C.POINTER(u64), C.POINTER(u64), C.POINTER(u64)]
    lib.blink_sample_rows.argtypes = [C.c_int32, vp, u32, u32, vp, vp, vp]
    lib.blink_sample_rows_static.argtypes = [C.c_int32, vp, u32, u32, vp, vp, vp]
    lib.blink_kv_cache_bytes.argtypes = [u32, u32, u32, u32, C.POINTER(u64)]
    lib.blink_qk_norm_rope.argtypes = [C.c_int32, vp, vp]
    lib.blink_kv_cache_read.argtypes = [C.c_int32, vp, vp, u32, vp, vp, vp]
    lib.blink_paged_attention.argtypes = [C.c_int32, vp, vp]
    lib.blink_attention_workspace_bytes.argtypes = [C.c_int32, vp, u32, u32, u32, C.POINTER(u64)]
    lib.blink_last_error.restype = C.c_char_p
    for n in EXPORTS[:-1]:
        getattr(lib, n).restype = C.c_int
    _lib = lib
    return lib


def _check(lib, rc):
    if rc != 0:
        raise BlinkError(rc, lib.blink_last_error().decode())


def _sample_rows(fn_name, logits, params, token_index, device=0):
    lib = load_library()
    logits = np.ascontiguousarray(logits, dtype=np.float32)
    n, v = logits.shape
    ps = (Sampling * n)(*[Sampling(float(p["temperature"]), int(p["top_k"]), float(p["top_p"]), int(p["seed"]) & 0xFFFFFFFFFFFFFFFF) for p in params])
    ti = np.ascontiguousarray(token_index, dtype=np.uint32)
    assert ti.size == n
    out = np.zeros(n, dtype=np.int32)
    _check(lib, getattr(lib, fn_name)(int(device), logits.ctypes.data, n, v, C.cast(ps, C.c_void_p), ti.ctypes.data, out.ctypes.data))
    return out


def sample_rows(logits, params, token_index, device=0):
    """blink_sample_rows: logits float32 [n][vocab], params: list of dicts (temperature, top_k, top_p, seed),
    token_index: output index per row. Returns int32 [n]."""
    return _sample_rows("blink_sample_rows", logits, params, token_index, device)


def sample_rows_static(logits, params, token_index, device=0):
    """blink_sample_rows_static: as sample_rows, staging in the library's static device array (no allocation)."""
    return _sample_rows("blink_sample_rows_static", logits, params, token_index, device)


# ---- operators on device memory: any tensors with data_ptr(), get_device(), shape, stride(), dtype and is_contiguous() as torch's have them ----
# A call on a few tokens is over in microseconds, so what it asks of every tensor is kept short, and its arguments are packed at once.
_FLOAT, _HALF, _BF16, _INT, _OTHER = range(5)          # the first three: BLINK_TYPE_*
_KINDS = {"torch.float32": _FLOAT, "torch.float16": _HALF, "torch.bfloat16": _BF16, "torch.int32": _INT}
_kind_of = {}                                          # the same by dtype object, as they come


def _kind(t):
    k = _kind_of.get(t.dtype)
    if k is None:
        k = _kind_of[t.dtype] = _KINDS.get(str(t.dtype), _OTHER)
    return k


def _dense(name, t, kind, shape, device):
    """Address of a contiguous tensor."""
    if t.get_device() != device or _kind(t) != kind or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {[n for n, k in _KINDS.items() if k == kind][0]} of the shape {tuple(shape)} on device {device}; "
                         f"it is {t.dtype}, {tuple(t.shape)}, strides {tuple(t.stride())}, on device {t.get_device()}")
    return t.data_ptr()


def _rows(name, t, shape, device):
    """Address of a tensor [tokens, heads, hd] whose rows [heads, hd] are contiguous, and the elements from one row to the next."""
    st, width = t.stride(), shape[1] * shape[2]
    if t.get_device() != device or t.shape != shape or (st[2] != 1 and shape[2] != 1) or (st[1] != shape[2] and shape[1] != 1) or (shape[0] > 1 and st[0] < width):
        raise ValueError(f"{name} must have the shape {tuple(shape)} with contiguous rows, on device {device}; it has {tuple(t.shape)}, strides {tuple(st)}, on device {t.get_device()}")
    return t.data_ptr(), st[0] if shape[0] > 1 else width


def _stream(stream, t, device):
    """Handle of the stream that a call goes to. None: the one its tensors are used on, torch's current one of the device (the null stream for
    other libraries' tensors)."""
    if stream is None:
        torch = sys.modules.get("torch")
        return torch.cuda.current_stream(device).cuda_stream if torch and isinstance(t, torch.Tensor) else 0
    return stream


def kv_cache_bytes(n_blocks, n_kv_heads, head_dim, bits=16):
    """Bytes of one layer of a paged cache with `n_blocks` blocks of 16 tokens."""
    lib, n = load_library(), C.c_uint64()
    _check(lib, lib.blink_kv_cache_bytes(n_blocks, n_kv_heads, head_dim, bits, C.byref(n)))
    return n.value


class KVCache:
    """One layer of a paged cache in a contiguous device tensor `data` of kv_cache_bytes(...) bytes, of any type (blink_kv_cache)."""

    def __init__(self, data, n_blocks, n_kv_heads, head_dim, bits=16):
        need = kv_cache_bytes(n_blocks, n_kv_heads, head_dim, bits)
        if data.get_device() < 0:
            raise ValueError(f"data is on {data.device}")
        if not data.is_contiguous() or data.numel() * data.element_size() != need:
            raise ValueError(f"data must be contiguous and have {need} bytes; it has {data.numel() * data.element_size()}, strides {tuple(data.stride())}")
        self.data, self.device = data, data.get_device()
        self.desc = CacheDesc(data.data_ptr(), n_blocks, n_kv_heads, head_dim, bits)
        self.n_kv_heads, self.head_dim, self._packed = n_kv_heads, head_dim, (data.data_ptr(), n_blocks, n_kv_heads, head_dim, bits)


def qk_norm_rope(q, k, v, positions, slots, rope_table, cache, q_out, q_gain=None, k_gain=None, eps=1e-6, q_scale=1.0, stream=None):
    """blink_qk_norm_rope: q [tokens, q heads, hd], k and v [tokens, kv heads, hd] (float32, float16 or bfloat16, rows may be parts
    of wider ones), int32 positions and slots [tokens], float32 rope_table [rows, hd / 2, 2] -> q_out float16 like q, keys and
    values into `cache`. Gains: float32 [hd] or None. stream: a stream's handle, None: torch's current stream."""
    lib, dev, hd, nkv = _lib or load_library(), cache.device, cache.head_dim, cache.n_kv_heads
    if len(q.shape) != 3:
        raise ValueError(f"q must have three dimensions; it has {tuple(q.shape)}")
    T, nq, kind = q.shape[0], q.shape[1], _kind(q)
    if kind > _BF16 or _kind(k) != kind or _kind(v) != kind or _kind(q_out) != _HALF:
        raise ValueError(f"q, k and v must be of one type, float32, float16 or bfloat16, and q_out float16; they are {q.dtype}, {k.dtype}, {v.dtype}, {q_out.dtype}")
    qp, qs = _rows("q", q, (T, nq, hd), dev)
    kp, ks = _rows("k", k, (T, nkv, hd), dev)
    vp, vs = _rows("v", v, (T, nkv, hd), dev)
    op, os_ = _rows("q_out", q_out, (T, nq, hd), dev)
    rows = rope_table.shape[0]
    a = _QK_NORM_ROPE.pack(*cache._packed, nq, T, kind, rows, qp, kp, vp, qs, ks, vs,
                           0 if q_gain is None else _dense("q_gain", q_gain, _FLOAT, (hd,), dev), 0 if k_gain is None else _dense("k_gain", k_gain, _FLOAT, (hd,), dev),
                           _dense("positions", positions, _INT, (T,), dev), _dense("slots", slots, _INT, (T,), dev),
                           _dense("rope_table", rope_table, _FLOAT, (rows, hd // 2, 2), dev), op, os_, eps, q_scale)
    rc = lib.blink_qk_norm_rope(dev, a, _stream(stream, q, dev))
    if rc:
        _check(lib, rc)


def kv_cache_read(cache, slots, k_out, v_out, stream=None):
    """blink_kv_cache_read: the tokens at int32 slots [tokens] into k_out, v_out, contiguous float16 [tokens, kv heads, hd].
    stream: as for qk_norm_rope."""
    lib, dev = _lib or load_library(), cache.device
    shape = (slots.shape[0], cache.n_kv_heads, cache.head_dim)
    _check(lib, lib.blink_kv_cache_read(dev, _CACHE.pack(*cache._packed), _dense("slots", slots, _INT, shape[:1], dev), shape[0],
                                        _dense("k_out", k_out, _HALF, shape, dev), _dense("v_out", v_out, _HALF, shape, dev), _stream(stream, slots, dev)))


def attention_workspace_bytes(n_q_heads, cache, n_seqs, max_q=1):
    """Bytes of the workspace of paged_attention for up to n_seqs sequences of up to max_q queries. Its first 8 KiB hold zeros
    before its first call; calls of any shapes may share one in turn."""
    lib, n = load_library(), C.c_uint64()
    _check(lib, lib.blink_attention_workspace_bytes(cache.device, C.byref(cache.desc), n_q_heads, n_seqs, max_q, C.byref(n)))
    return n.value


def paged_attention(q, cache, block_tables, seq_lens, cu_seqlens, out, workspace, max_q=1, window=0, sinks=0, scale=1.0, stream=None):
    """blink_paged_attention: q, out float16 [tokens, q heads, hd]; int32 block_tables [seqs, blocks], seq_lens [seqs], cu_seqlens
    [seqs + 1]; workspace: a contiguous tensor of attention_workspace_bytes(...) bytes. stream: as for qk_norm_rope."""
    lib, dev, hd = _lib or load_library(), cache.device, cache.head_dim
    if len(q.shape) != 3 or len(block_tables.shape) != 2:
        raise ValueError(f"q must have three dimensions and block_tables two; they have {tuple(q.shape)} and {tuple(block_tables.shape)}")
    T, nq = q.shape[0], q.shape[1]
    S, width = block_tables.shape
    if _kind(q) != _HALF or _kind(out) != _HALF:
        raise ValueError(f"q and out must be float16; they are {q.dtype} and {out.dtype}")
    qp, qs = _rows("q", q, (T, nq, hd), dev)
    op, os_ = _rows("out", out, (T, nq, hd), dev)
    if workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError(f"workspace must be contiguous and on device {dev}; it is on device {workspace.get_device()}")
    a = _PAGED_ATTENTION.pack(*cache._packed, nq, S, T, max_q, width, window, sinks, scale, qp, op, qs, os_, _dense("cu_seqlens", cu_seqlens, _INT, (S + 1,), dev),
                              _dense("seq_lens", seq_lens, _INT, (S,), dev), _dense("block_tables", block_tables, _INT, (S, width), dev), workspace.data_ptr(),
                              workspace.numel() * workspace.element_size())
    rc = lib.blink_paged_attention(dev, a, _stream(stream, q, dev))
    if rc:
        _check(lib, rc)


class Engine:
    """One serving engine on one GPU. model/engine: dicts as in synth.configs (model: also qk_norm, window, sinks, kv_bits of
    blink_attention_options); blob: uint8 array (synth.pack_blob)."""

    def __init__(self, model, engine, blob, flags=0, device=0, trace_capacity=0, idle_poll_us=0, pump_depth=0, tune=0):
        self.lib = load_library()
        self.model, self.engine = dict(model), dict(engine)
        blob = np.ascontiguousarray(blob, dtype=np.uint8)
        cfg = Config()
        for k in ("n_layers", "d_model", "n_q_heads", "n_kv_heads", "head_dim", "d_ffn", "vocab", "dtype", "rms_eps", "rope_theta"):
            setattr(cfg, k, model[k])
        for k in ("kv_block_size", "kv_num_blocks", "max_batch", "max_seq_len", "max_prefill_tokens", "ring_slots", "eos_token_id"):
            setattr(cfg, k, engine[k])
        cfg.weights = blob.ctypes.data
        cfg.weights_bytes = blob.nbytes
        if engine.get("chunked_prefill"):
            flags |= FLAG_CHUNKED_PREFILL
        if engine.get("preemption"):
            flags |= FLAG_PREEMPTION
        if engine.get("prefix_cache"):
            flags |= FLAG_PREFIX_CACHE
        if engine.get("speculative"):
            flags |= FLAG_SPECULATIVE
            cfg.spec_tokens = int(engine["speculative"])
        cfg.device, cfg.flags, cfg.trace_capacity, cfg.idle_poll_us = device, flags, trace_capacity, idle_poll_us
        cfg.pump_depth, cfg.tune = pump_depth, tune
        cfg.n_experts, cfg.n_active = model.get("n_experts", 0), model.get("n_active", 0)
        self.h = C.c_void_p()
        opt = AttentionOptions(*(int(model.get(k, 0)) for k in ("qk_norm", "window", "sinks", "kv_bits")))
        _check(self.lib, self.lib.blink_init_attention(C.byref(cfg), C.byref(opt), C.byref(self.h)))

    def submit(self, prompt, max_new_tokens, temperature=0.0, top_k=0, top_p=1.0, seed=0):
        p = np.ascontiguousarray(prompt, dtype=np.int32)
        s = Sampling(float(temperature), int(top_k), float(top_p), int(seed) & 0xFFFFFFFFFFFFFFFF)
        rid = C.c_uint64()
        _check(self.lib, self.lib.blink_submit(self.h, p.ctypes.data, p.size, int(max_new_tokens), C.byref(s), C.byref(rid)))
        return rid.value

    def submit_request(self, r):
        return self.submit(r["prompt"], r["max_new_tokens"], r["temperature"], r["top_k"], r["top_p"], r["seed"])

    def run(self, max_iterations=0):
        _check(self.lib, self.lib.blink_run(self.h, int(max_iterations)))

    def set_exit_when_idle(self, on):
        _check(self.lib, self.lib.blink_set_exit_when_idle(self.h, 1 if on else 0))

    def wait(self):
        _check(self.lib, self.lib.blink_wait(self.h))

    def stop(self):
        _check(self.lib, self.lib.blink_stop(self.h))

    def poll(self, cap=4096):
        buf = np.empty(cap, dtype=EVENT_DTYPE)
        n = C.c_uint32()
        _check(self.lib, self.lib.blink_poll_outputs(self.h, buf.ctypes.data, cap, C.byref(n)))
        return buf[: n.value]

    def drain(self, cap=4096):
        """Polls until a poll returns nothing. Returns all events as one array."""
        out = []
        while True:
            ev = self.poll(cap)
            if ev.size == 0:
                break
            out.append(ev.copy())
        return np.concatenate(out) if out else np.zeros(0, dtype=EVENT_DTYPE)

    def trace(self, cap=1 << 16):
        buf = np.zeros(cap, dtype=TRACE_DTYPE)
        n = C.c_uint64()
        _check(self.lib, self.lib.blink_get_trace(self.h, buf.ctypes.data, cap, C.byref(n)))
        return buf[: n.value]

    def stats(self):
        s = Stats()
        _check(self.lib, self.lib.blink_get_stats(self.h, C.byref(s)))
        return {k: getattr(s, k) for k, _ in Stats._fields_}

    def debug_read(self, what, dtype, max_bytes=None):
        if max_bytes is None:
            m, e = self.model, self.engine
            max_t = max(e["max_prefill_tokens"], e["max_seq_len"], e["max_batch"])
            max_bytes = 8 + 4 * max(e["max_batch"] * (1 + int(e.get("speculative", 0))) * m["vocab"], e["kv_num_blocks"] + 1, max_t * m["d_model"],
                                    m["n_layers"] * max_t * m.get("n_active", 0),
                                    e["max_batch"] * ((e["max_seq_len"] + 15) // 16), e["ring_slots"])
        buf = np.empty(max_bytes, dtype=np.uint8)
        n = C.c_uint64()
        _check(self.lib, self.lib.blink_debug_read(self.h, int(what), buf.ctypes.data, buf.nbytes, C.byref(n)))
        out = buf[: n.value].view(dtype)
        return out if 2 * n.value > max_bytes else out.copy()      # (a copy only where it frees most of the buffer)

    def time_phase(self, phase):
        _check(self.lib, self.lib.blink_time_phase(self.h, int(phase)))

    def calibration_copy(self, nbytes):
        _check(self.lib, self.lib.blink_calibration_copy(self.h, int(nbytes)))

    def calibration_rates(self):
        """(GB/s of a plain 1 GiB copy kernel, read + written; TFLOP/s of a register-only bf16 MFMA loop; GB/s of a plain
        read of 1 GiB) on this device."""
        c, m, r = C.c_double(), C.c_double(), C.c_double()
        _check(self.lib, self.lib.blink_calibration_rates(self.h, C.byref(c), C.byref(m), C.byref(r)))
        return c.value, m.value, r.value

    def clock_sync(self):
        """(device_ns, host_ns on CLOCK_MONOTONIC, uncertainty_ns): the device clock read no later than host_ns."""
        d, h, u = C.c_uint64(), C.c_uint64(), C.c_uint64()
        _check(self.lib, self.lib.blink_clock_sync(self.h, C.byref(d), C.byref(h), C.byref(u)))
        return d.value, h.value, u.value

    def phase_times_ms(self, cap=1 << 20):
        buf = np.zeros(cap, dtype=np.float32)
        n = C.c_uint64()
        _check(self.lib, self.lib.blink_get_phase_times(self.h, buf.ctypes.data, cap, C.byref(n)))
        return buf[: n.value].copy()

    def shutdown(self):
        if self.h:
            _check(self.lib, self.lib.blink_shutdown(self.h))
            self.h = C.c_void_p()

    def __enter__(self):
        return self

    def __exit__(self, *a):
        self.shutdown()
