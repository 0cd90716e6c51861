"""ctypes binding of libcmoe.so; the names are those of include/cmoe.h.

Argument marshalling only: every step of the decode path runs in the HIP
kernels behind the C ABI.  ``Engine`` is a convenience owner of the buffers the
library asks for (allocated with PyTorch, which serves here only as the device
memory and stream provider).
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Optional

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcmoe.so")

CMOE_OK = 0
CMOE_ERR_INVALID_ARG = -1
CMOE_ERR_UNSUPPORTED = -2
CMOE_ERR_HIP = -3
CMOE_ERR_STATE = -4

CMOE_MODE_TEMPORAL = 0
CMOE_MODE_SPATIO_TEMPORAL = 1
CMOE_MODE_SPATIO_ONLY = 2
CMOE_POLICY_ROUTER = 0
CMOE_POLICY_LRU = 1
CMOE_POLICY_LFU = 2
CMOE_POLICY_LRFU = 3
CMOE_F32 = 0
CMOE_BF16 = 1
CMOE_POOL_DEVICE = 0
CMOE_POOL_HOST_PINNED = 1
CMOE_FLAG_FILL_ON_MAIN = 0x1
CMOE_FLAG_FFN_GROUPED = 0x2
CMOE_FLAG_FFN_SINGLE = 0x4
CMOE_FLAG_FILL_ON_SIDE = 0x8

CMOE_FORMAT_DTYPE = 0
CMOE_FORMAT_MX8 = 1

CMOE_VIEW_LOGITS = 0
CMOE_VIEW_SELECTED = 1
CMOE_VIEW_GATES = 2
CMOE_VIEW_CACHE = 3
CMOE_VIEW_COUNTERS = 4
CMOE_VIEW_PHYS = 5
CMOE_VIEW_SLOTS = 6
CMOE_VIEW_EVENTS = 7
CMOE_VIEW_FILLS = 8
CMOE_VIEW_ACTIVE = 9
CMOE_VIEW_PRIORITY = 10
CMOE_VIEW_SELCOUNT = 11
CMOE_KERNEL_COUNT = 6
KERNEL_NAMES = ("router", "cache_step", "fill", "ffn_up", "ffn_down", "combine")

EXPORTED = ("cmoe_query", "cmoe_init", "cmoe_step", "cmoe_step_noalloc", "cmoe_step_logits", "cmoe_stats", "cmoe_get_cache",
            "cmoe_set_cache", "cmoe_set_R", "cmoe_reset", "cmoe_destroy", "cmoe_view_bytes", "cmoe_read",
            "cmoe_profile_begin", "cmoe_profile_end", "cmoe_concentration", "cmoe_read_probe", "cmoe_add_norm", "cmoe_quantize",
            "cmoe_moe_query", "cmoe_moe_init", "cmoe_moe_layer", "cmoe_moe_block", "cmoe_moe_destroy", "cmoe_last_error")


class cmoe_config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("L", "N", "K", "d", "F", "C", "R", "S", "mode", "dtype",
                                              "pool_kind", "warmup_tokens")] + \
        [("flags", ctypes.c_uint32), ("policy", ctypes.c_int32), ("lrfu_lambda", ctypes.c_float),
         ("arena_slots", ctypes.c_int32)]


class cmoe_weights(ctypes.Structure):
    _fields_ = [("w_router", ctypes.c_void_p), ("w_temporal", ctypes.c_void_p), ("w_spatio", ctypes.c_void_p),
                ("logit_bias", ctypes.c_void_p), ("cold_pool", ctypes.c_void_p)]


class cmoe_sizes(ctypes.Structure):
    _fields_ = [("arena_bytes", ctypes.c_size_t), ("state_bytes", ctypes.c_size_t),
                ("workspace_bytes", ctypes.c_size_t)]


class cmoe_buffers(ctypes.Structure):
    _fields_ = [("arena", ctypes.c_void_p), ("state", ctypes.c_void_p), ("workspace", ctypes.c_void_p)]


class cmoe_stats_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("accesses", "hits", "demand_misses", "proactive_loads", "tokens",
                                              "traffic_bytes", "phys_fills", "phys_bytes")]

    def as_dict(self):
        return {n: int(getattr(self, n)) for n, _ in self._fields_}


class cmoe_norm(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("rows", "d", "dtype", "delta_dtype")] + [("eps", ctypes.c_float)] + \
        [f for n in ("residual", "delta", "residual_out") for f in ((n, ctypes.c_void_p), (n + "_stride", ctypes.c_int64))] + \
        [("weight", ctypes.c_void_p)] + \
        [f for n in ("h", "h8", "h8_scale") for f in ((n, ctypes.c_void_p), (n + "_stride", ctypes.c_int64))] + \
        [("n_rows", ctypes.c_void_p)]


class cmoe_moe_config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("L", "N", "K", "d", "F", "T", "dtype", "weights", "activations")]


class cmoe_moe_weights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("w_router", "logit_bias", "experts", "expert_scales")]


class cmoe_moe_call(ctypes.Structure):
    _fields_ = [("layer", ctypes.c_int32), ("T", ctypes.c_int32)] + \
        [f for n in ("h", "h8", "h8_scale", "y") for f in ((n, ctypes.c_void_p), (n + "_stride", ctypes.c_int64))] + \
        [(n, ctypes.c_void_p) for n in ("n_tokens", "selected", "gates")]


class CmoeError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"cmoe status {status}: {msg}")
        self.status = status


_lib = None


def lib():
    """Loads libcmoe.so; raises if it has not been built (there is no fallback)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with paper_2609_04895_amd.build.build()")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, i64p = ctypes.c_void_p, ctypes.c_int32, ctypes.POINTER(ctypes.c_int64)
        L.cmoe_query.argtypes = [ctypes.POINTER(cmoe_config), ctypes.POINTER(cmoe_sizes)]
        L.cmoe_init.argtypes = [ctypes.POINTER(cmoe_config), ctypes.POINTER(cmoe_weights),
                                ctypes.POINTER(cmoe_buffers), vp, vp, ctypes.POINTER(vp)]
        L.cmoe_step.argtypes = [vp, vp, vp]
        L.cmoe_step_noalloc.argtypes = [vp, vp, vp]
        L.cmoe_step_logits.argtypes = [vp, vp, vp, vp]
        L.cmoe_stats.argtypes = [vp, ctypes.POINTER(cmoe_stats_t), i64p, i64p]
        L.cmoe_get_cache.argtypes = [vp, i32, i32, ctypes.POINTER(i32), ctypes.POINTER(i32)]
        L.cmoe_set_cache.argtypes = [vp, i32, i32, ctypes.POINTER(i32), i32]
        L.cmoe_set_R.argtypes = [vp, i32]
        L.cmoe_reset.argtypes = [vp]
        L.cmoe_destroy.argtypes = [vp]
        L.cmoe_view_bytes.argtypes = [vp, i32]
        L.cmoe_view_bytes.restype = ctypes.c_size_t
        L.cmoe_read.argtypes = [vp, i32, vp, ctypes.c_size_t]
        L.cmoe_profile_begin.argtypes = [vp, i32, ctypes.c_uint32]
        L.cmoe_profile_end.argtypes = [vp, ctypes.POINTER(ctypes.c_double), i64p]
        L.cmoe_concentration.argtypes = [vp, i32, ctypes.POINTER(ctypes.c_double)]
        L.cmoe_read_probe.argtypes = [vp, ctypes.c_int64, i32, ctypes.POINTER(ctypes.c_double)]
        i64, ref = ctypes.c_int64, ctypes.POINTER
        L.cmoe_add_norm.argtypes = [vp, vp]  # cmoe_norm, as a structure or its bytes
        L.cmoe_quantize.argtypes = [vp, i32, i64, i64, i64, vp, i64, vp, i64, vp]
        L.cmoe_moe_query.argtypes = [ref(cmoe_moe_config), ref(ctypes.c_size_t)]
        L.cmoe_moe_init.argtypes = [ref(cmoe_moe_config), ref(cmoe_moe_weights), vp, vp, ref(vp)]
        L.cmoe_moe_layer.argtypes = [vp, vp]
        L.cmoe_moe_block.argtypes = [vp, vp, vp]
        L.cmoe_moe_destroy.argtypes = [vp]
        L.cmoe_last_error.argtypes = []
        L.cmoe_last_error.restype = ctypes.c_char_p
        for n in EXPORTED:
            if n not in ("cmoe_view_bytes", "cmoe_last_error"):
                getattr(L, n).restype = ctypes.c_int
        _lib = L
    return _lib


def _check(status: int):
    if status != CMOE_OK:
        raise CmoeError(status, lib().cmoe_last_error().decode())


def make_config(L, N, K, d, F, C, R, S, mode, dtype, pool_kind=CMOE_POOL_DEVICE, warmup_tokens=0, flags=0,
                policy=CMOE_POLICY_ROUTER, lrfu_lambda=0.5, arena_slots=0):
    return cmoe_config(L, N, K, d, F, C, R, S, mode, dtype, pool_kind, warmup_tokens, flags, policy, lrfu_lambda,
                       arena_slots)


def router_slots(cfg: cmoe_config):
    """Names of the router slots of the logits view, in order."""
    names = ["native"]
    if cfg.policy == CMOE_POLICY_ROUTER:
        names.append("temporal")
    if cfg.mode in (CMOE_MODE_SPATIO_TEMPORAL, CMOE_MODE_SPATIO_ONLY):
        names.append("spatio")
    return names


def cmoe_query(cfg: cmoe_config) -> cmoe_sizes:
    out = cmoe_sizes()
    _check(lib().cmoe_query(ctypes.byref(cfg), ctypes.byref(out)))
    return out


def cmoe_read_probe(buf, reps: int = 5) -> float:
    """GB/s of the device's streaming read of the device tensor buf (at
    least 64 MiB) with the expert weight loads' access pattern."""
    rate = ctypes.c_double()
    _check(lib().cmoe_read_probe(ctypes.c_void_p(buf.data_ptr()), buf.numel() * buf.element_size(), reps,
                                 ctypes.byref(rate)))
    return rate.value


def _ptr(t) -> Optional[int]:
    return None if t is None else int(t.data_ptr())


class Engine:
    """One handle plus the caller-owned buffers (torch tensors on cuda:0)."""

    def __init__(self, cfg: cmoe_config, w_router, w_temporal, w_spatio, logit_bias, cold_pool,
                 main_stream=None, side_stream=None, workspace=True):
        """workspace=False binds no workspace: every token then goes through
        cmoe_step_noalloc."""
        import torch
        self.torch = torch
        self.cfg = cfg
        sizes = cmoe_query(cfg)
        dev = torch.device("cuda", torch.cuda.current_device())

        def buf(n):
            # 256-byte aligned (the caching allocator aligns blocks to >= 512 bytes)
            return torch.empty(max(int(n), 256), dtype=torch.uint8, device=dev)

        self.arena = buf(sizes.arena_bytes)
        self.state = buf(sizes.state_bytes)
        self.workspace = buf(sizes.workspace_bytes) if workspace else None
        self._keep = (w_router, w_temporal, w_spatio, logit_bias, cold_pool)
        self.main_stream = main_stream if main_stream is not None else torch.cuda.current_stream()
        self.side_stream = side_stream
        wts = cmoe_weights(_ptr(w_router), _ptr(w_temporal), _ptr(w_spatio), _ptr(logit_bias), _ptr(cold_pool))
        bufs = cmoe_buffers(_ptr(self.arena), _ptr(self.state), _ptr(self.workspace) if workspace else None)
        h = ctypes.c_void_p()
        _check(lib().cmoe_init(ctypes.byref(cfg), ctypes.byref(wts), ctypes.byref(bufs),
                               ctypes.c_void_p(self.main_stream.cuda_stream),
                               ctypes.c_void_p(side_stream.cuda_stream if side_stream is not None else None),
                               ctypes.byref(h)))
        self.handle = h

    # -- the decode path
    def cmoe_step(self, h, y):
        _check(lib().cmoe_step(self.handle, ctypes.c_void_p(h.data_ptr()), ctypes.c_void_p(y.data_ptr())))

    def cmoe_step_noalloc(self, h, y):
        _check(lib().cmoe_step_noalloc(self.handle, ctypes.c_void_p(h.data_ptr()), ctypes.c_void_p(y.data_ptr())))

    def cmoe_step_logits(self, zR, zT=None, zS=None):
        _check(lib().cmoe_step_logits(self.handle, ctypes.c_void_p(zR.data_ptr()), ctypes.c_void_p(_ptr(zT)),
                                      ctypes.c_void_p(_ptr(zS))))

    # -- counters and state
    def cmoe_stats(self):
        c = self.cfg
        total = cmoe_stats_t()
        per = np.zeros((c.S, c.L, 5), np.int64)
        phys = np.zeros((c.L, 2), np.int64)
        _check(lib().cmoe_stats(self.handle, ctypes.byref(total), per.ctypes.data_as(ctypes.POINTER(ctypes.c_int64)),
                                phys.ctypes.data_as(ctypes.POINTER(ctypes.c_int64))))
        return total.as_dict(), per, phys

    def cmoe_get_cache(self, stream: int, layer: int):
        out = (ctypes.c_int32 * self.cfg.C)()
        n = ctypes.c_int32()
        _check(lib().cmoe_get_cache(self.handle, stream, layer, out, ctypes.byref(n)))
        return [int(out[i]) for i in range(n.value)]

    def cmoe_set_cache(self, stream: int, layer: int, experts):
        arr = (ctypes.c_int32 * max(1, len(experts)))(*experts)
        _check(lib().cmoe_set_cache(self.handle, stream, layer, arr, len(experts)))

    def cmoe_set_R(self, R: int):
        _check(lib().cmoe_set_R(self.handle, R))

    def cmoe_reset(self):
        _check(lib().cmoe_reset(self.handle))

    def cmoe_read(self, view: int) -> np.ndarray:
        c = self.cfg
        n = lib().cmoe_view_bytes(self.handle, view)
        raw = np.empty(n, np.uint8)
        _check(lib().cmoe_read(self.handle, view, raw.ctypes.data_as(ctypes.c_void_p), n))
        n_r = len(router_slots(c))
        NW = (c.N + 63) // 64
        shapes = {
            CMOE_VIEW_LOGITS: (np.float32, (c.L, c.S, n_r, c.N)),
            CMOE_VIEW_SELECTED: (np.int32, (c.L, c.S, c.K)),
            CMOE_VIEW_GATES: (np.float32, (c.L, c.S, c.K)),
            CMOE_VIEW_CACHE: (np.uint64, (c.S, c.L, NW)),
            CMOE_VIEW_COUNTERS: (np.int64, (c.S, c.L, 5)),
            CMOE_VIEW_PHYS: (np.int64, (c.L, 2)),
            CMOE_VIEW_SLOTS: (np.int32, (c.L, c.N)),
            CMOE_VIEW_EVENTS: (np.int32, (c.L, c.S, 4)),
            CMOE_VIEW_FILLS: (np.int32, (c.L, 2)),
            CMOE_VIEW_ACTIVE: (np.int64, (c.L,)),
            CMOE_VIEW_PRIORITY: (np.float32, (c.S, c.L, c.N)),
            CMOE_VIEW_SELCOUNT: (np.uint64, (c.L, c.N)),
        }
        dt, shape = shapes[view]
        return raw.view(dt).reshape(shape)

    def cmoe_concentration(self, top_m: int = 8):
        """(effective experts, entropy in nats, max frequency, top-m mass),
        layer means of the native selection frequencies."""
        out = (ctypes.c_double * 4)()
        _check(lib().cmoe_concentration(self.handle, int(top_m), out))
        return tuple(float(v) for v in out)

    def cache_sets(self) -> np.ndarray:
        """Cache membership as a bool array [S][L][N]."""
        w = self.cmoe_read(CMOE_VIEW_CACHE)
        c = self.cfg
        bits = np.unpackbits(w.view(np.uint8).reshape(c.S, c.L, -1), axis=-1, bitorder="little")
        return bits[:, :, :c.N].astype(bool)

    # -- timing
    def cmoe_profile_begin(self, max_tokens: int, kernels=None):
        mask = 0 if kernels is None else sum(1 << KERNEL_NAMES.index(k) for k in kernels)
        _check(lib().cmoe_profile_begin(self.handle, max_tokens, mask))

    def cmoe_profile_end(self):
        ms = (ctypes.c_double * CMOE_KERNEL_COUNT)()
        n = (ctypes.c_int64 * CMOE_KERNEL_COUNT)()
        _check(lib().cmoe_profile_end(self.handle, ms, n))
        return {KERNEL_NAMES[i]: (float(ms[i]), int(n[i])) for i in range(CMOE_KERNEL_COUNT)}

    def cmoe_destroy(self):
        if self.handle is not None:
            _check(lib().cmoe_destroy(self.handle))
            self.handle = None

    def __del__(self):
        try:
            self.cmoe_destroy()
        except Exception:
            pass


# ------------------------------------------------------------ operators without a cache
# A call of these takes as little as a few microseconds of the device, so their
# arguments are checked and packed with as few Python steps as it takes: one
# structure as bytes, addresses and the current stream as plain integers.
_NORM = struct.Struct("iiiif4x" + "q" * 14)  # cmoe_norm
_CALL = struct.Struct("ii" + "q" * 11)       # cmoe_moe_call


def _torch():
    """torch, and the cmoe_dtype of its types (torch is imported on first use)."""
    global _torch_types
    if _torch_types is None:
        import torch
        _torch_types = (torch, {torch.float32: CMOE_F32, torch.bfloat16: CMOE_BF16})
    return _torch_types


_torch_types = None


def _invalid(msg):
    raise CmoeError(CMOE_ERR_INVALID_ARG, msg)


def _pack(fields, *values):
    try:
        return fields.pack(*values)
    except struct.error as e:  # a number that is not a whole one or that its field cannot hold
        _invalid(f"an argument is out of range: {e}")


def _rows(t, name, dtype, shape, dev):
    """Address and row stride of a tensor [rows][cols] of device `dev` whose rows
    are contiguous; raises on any other tensor."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev:
        _invalid(f"{name} must be a {list(shape)} tensor of {dtype} on the other tensors' device")
    if t.is_contiguous():
        return t.data_ptr(), shape[1]
    row, col = t.stride()
    if col != 1 and shape[1] > 1:
        _invalid(f"the rows of {name} must be contiguous")
    return t.data_ptr(), (row if shape[0] > 1 else shape[1])


def _flat(t, name, dtype, numel, dev):
    if t.dtype is not dtype or t.numel() != numel or not t.is_contiguous() or t.get_device() != dev:
        _invalid(f"{name} must be a contiguous tensor of {numel} values of {dtype} on the other tensors' device")
    return t.data_ptr()


def _on_current(torch, dev):
    """The work goes to the current device, so the tensors have to be there."""
    if dev < 0 or dev != torch._C._cuda_getDevice():
        _invalid("the tensors must be on the current device")


def _stream_of(torch, stream, dev):
    """hipStream_t of `stream`, or of the current stream."""
    _on_current(torch, dev)
    return stream.cuda_stream if stream is not None else torch._C._cuda_getCurrentRawStream(dev)


def _norm_args(residual, delta, weight, eps, residual_out, h, h8, h8_scale, n_rows):
    torch, types = _torch()
    dt, shape, dev = residual.dtype, residual.shape, residual.get_device()
    if dt not in types or len(shape) != 2:
        _invalid("residual must be a [rows][d] tensor of float32 or bfloat16")
    rows, d = shape
    p, ps = _rows(residual, "residual", dt, shape, dev)
    delta_dtype = pd = pds = po = pos = pw = ph = phs = p8 = p8s = pc = pcs = pn = 0
    if delta is not None:
        delta_dtype = types.get(delta.dtype, -1)
        if delta_dtype < 0:
            _invalid("delta must be float32 or bfloat16")
        pd, pds = _rows(delta, "delta", delta.dtype, shape, dev)
    if residual_out is not None:
        po, pos = _rows(residual_out, "residual_out", dt, shape, dev)
    if weight is not None:
        pw = _flat(weight, "weight", dt, d, dev)
    if h is not None:
        ph, phs = _rows(h, "h", dt, shape, dev)
    if h8 is not None:
        p8, p8s = _rows(h8, "h8", torch.uint8, shape, dev)
    if h8_scale is not None:
        pc, pcs = _rows(h8_scale, "h8_scale", torch.uint8, (rows, d // 32), dev)
    if n_rows is not None:
        pn = _flat(n_rows, "n_rows", torch.int32, 1, dev)
    return _pack(_NORM, rows, d, types[dt], delta_dtype, eps, p, ps, pd, pds, po, pos, pw, ph, phs, p8, p8s, pc, pcs, pn)


def cmoe_add_norm(residual, delta=None, weight=None, eps=1e-6, residual_out=None, h=None, h8=None, h8_scale=None,
                  n_rows=None, stream=None):
    """The residual's addition and RMS norm (see the header) of [rows][d]
    tensors into the outputs given, on `stream` or the current one.  residual_out
    may be residual."""
    a = _norm_args(residual, delta, weight, eps, residual_out, h, h8, h8_scale, n_rows)
    st = lib().cmoe_add_norm(a, _stream_of(_torch()[0], stream, residual.get_device()))
    if st:
        _check(st)


def cmoe_quantize(src, q, scale, stream=None):
    """[rows][cols] values of float32 or bfloat16 into 8 bits: q [rows][cols]
    and scale [rows][cols / 32], both uint8."""
    torch, types = _torch()
    dt, shape, dev = src.dtype, src.shape, src.get_device()
    if dt not in types or len(shape) != 2:
        _invalid("src must be a [rows][cols] tensor of float32 or bfloat16")
    rows, cols = shape
    p, stride = _rows(src, "src", dt, shape, dev)
    pq, q_stride = _rows(q, "q", torch.uint8, shape, dev)
    ps, s_stride = _rows(scale, "scale", torch.uint8, (rows, cols // 32), dev)
    st = lib().cmoe_quantize(p, types[dt], rows, cols, stride, pq, q_stride, ps, s_stride, _stream_of(torch, stream, dev))
    if st:
        _check(st)


def quantize_experts(experts):
    """A pool [L][N][3 d F] in 8 bits: (values, scales) [L][N][3 d F] and
    [L][N][3 d F / 32], for MoeLayers with CMOE_FORMAT_MX8."""
    torch, _ = _torch()
    if experts.dim() != 3 or not experts.is_contiguous() or experts.shape[2] % 32:
        _invalid("experts must be a contiguous [L][N][3 d F] tensor")
    L, N, n = experts.shape
    q = torch.empty((L, N, n), dtype=torch.uint8, device=experts.device)
    scale = torch.empty((L, N, n // 32), dtype=torch.uint8, device=experts.device)
    # one long row of whole blocks, in calls of 2^34 values, the most that one takes
    total, step = experts.numel(), 1 << 34
    src, qs, ss = experts.view(1, total), q.view(1, total), scale.view(1, total // 32)
    for at in range(0, total, step):
        end = min(at + step, total)
        cmoe_quantize(src[:, at:end], qs[:, at:end], ss[:, at // 32:end // 32])
    return q, scale


def make_moe_config(L, N, K, d, F, T, dtype, weights=CMOE_FORMAT_DTYPE, activations=CMOE_FORMAT_DTYPE):
    return cmoe_moe_config(L, N, K, d, F, T, dtype, weights, activations)


def cmoe_moe_query(cfg: cmoe_moe_config) -> int:
    out = ctypes.c_size_t()
    _check(lib().cmoe_moe_query(ctypes.byref(cfg), ctypes.byref(out)))
    return out.value


class MoeLayers:
    """L MoE layers without caches: one handle plus its workspace.  The weights
    are the caller's tensors: w_router [L][N][d], logit_bias [L][N] fp32 or
    None, experts [L][N][3 d F] (expert_scales [L][N][3 d F / 32] with 8-bit
    ones), norm_weight [L][d] or None (ones) for cmoe_moe_block.  All calls run
    on `stream` (default: the stream that is current here).  Where a call's
    tensors belong to another stream, the caller lets the two wait for each other
    and keeps the tensors until the call is done (or calls their record_stream)."""

    def __init__(self, cfg: cmoe_moe_config, w_router, logit_bias, experts, expert_scales=None, norm_weight=None,
                 norm_eps=1e-6, stream=None):
        self.handle = None
        torch, _ = _torch()
        size = cmoe_moe_query(cfg)
        self.cfg, self.K, self.d, self.L = cfg, cfg.K, cfg.d, cfg.L
        self.device = torch.cuda.current_device()
        self.dtype = torch.bfloat16 if cfg.dtype == CMOE_BF16 else torch.float32
        n = cfg.L * cfg.N * 3 * cfg.d * cfg.F
        mx8 = cfg.weights == CMOE_FORMAT_MX8
        w = cmoe_moe_weights(
            _flat(w_router, "w_router", self.dtype, cfg.L * cfg.N * cfg.d, self.device),
            None if logit_bias is None else _flat(logit_bias, "logit_bias", torch.float32, cfg.L * cfg.N, self.device),
            _flat(experts, "experts", torch.uint8 if mx8 else self.dtype, n, self.device), None)
        if mx8:
            if expert_scales is None:
                _invalid("8-bit experts need expert_scales")
            w.expert_scales = _flat(expert_scales, "expert_scales", torch.uint8, n // 32, self.device)
        if norm_weight is not None:
            _flat(norm_weight, "norm_weight", self.dtype, cfg.L * cfg.d, self.device)
            norm_weight = list(norm_weight.view(cfg.L, cfg.d))
        self.norm_weight, self.norm_eps = norm_weight, norm_eps
        self._keep = (w_router, logit_bias, experts, expert_scales)
        self.stream = stream if stream is not None else torch.cuda.current_stream()
        with torch.cuda.stream(self.stream):  # the allocator's owner of the memory: the stream that uses it
            self.workspace = torch.empty(size, dtype=torch.uint8, device="cuda")
        for t in (w_router, logit_bias, experts, expert_scales, None if norm_weight is None else norm_weight[0]):
            if t is not None:  # once dropped, memory of the weights waits for the calls in flight
                t.record_stream(self.stream)
        h = ctypes.c_void_p()
        _check(lib().cmoe_moe_init(ctypes.byref(cfg), ctypes.byref(w), self.workspace.data_ptr(),
                                   self.stream.cuda_stream, ctypes.byref(h)))
        self.handle = h

    def _call(self, layer, rows, h, h8, h8_scale, y, n_tokens, selected, gates):
        torch, _ = _torch()
        dev, d = self.device, self.d
        shape = (rows, d)
        ph = phs = p8 = p8s = pc = pcs = pn = psel = pg = 0
        if h is not None:
            ph, phs = _rows(h, "h", self.dtype, shape, dev)
        if h8 is not None:
            p8, p8s = _rows(h8, "h8", torch.uint8, shape, dev)
        if h8_scale is not None:
            pc, pcs = _rows(h8_scale, "h8_scale", torch.uint8, (rows, d // 32), dev)
        py, pys = _rows(y, "y", torch.float32, shape, dev)
        if n_tokens is not None:
            pn = _flat(n_tokens, "n_tokens", torch.int32, 1, dev)
        if selected is not None:
            psel = _flat(selected, "selected", torch.int32, rows * self.K, dev)
        if gates is not None:
            pg = _flat(gates, "gates", torch.float32, rows * self.K, dev)
        return _pack(_CALL, layer, rows, ph, phs, p8, p8s, pc, pcs, py, pys, pn, psel, pg)

    def cmoe_moe_layer(self, layer, h, y, h8=None, h8_scale=None, n_tokens=None, selected=None, gates=None):
        """y [T][d] = the layer's output for the hidden states h [T][d]; the
        rows of both may be apart.  h8 and h8_scale: the experts' input with
        8-bit activations.  selected, gates: [T][K]."""
        c = self._call(layer, h.shape[0], h, h8, h8_scale, y, n_tokens, selected, gates)
        st = lib().cmoe_moe_layer(self.handle, c)
        if st:
            _check(st)

    def cmoe_moe_block(self, layer, residual, delta, y, residual_out=None, n_tokens=None, selected=None, gates=None):
        """Norm of residual + delta (None: of the residual), then the layer."""
        if not 0 <= layer < self.L:
            _invalid("layer must be in [0, L)")
        w = None if self.norm_weight is None else self.norm_weight[layer]
        n = _norm_args(residual, delta, w, self.norm_eps, residual_out, None, None, None, None)
        if residual.get_device() != self.device:
            _invalid("residual must be on the handle's device")
        c = self._call(layer, residual.shape[0], None, None, None, y, n_tokens, selected, gates)
        st = lib().cmoe_moe_block(self.handle, n, c)
        if st:
            _check(st)

    def cmoe_moe_destroy(self):
        if self.handle is not None:
            _check(lib().cmoe_moe_destroy(self.handle))
            self.handle = None

    def __del__(self):
        try:
            self.cmoe_moe_destroy()
        except Exception:
            pass
