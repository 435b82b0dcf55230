"""Thin ctypes binding of the GLIDE C ABI (include/glide.h): argument marshalling only.

Every step of the path runs in the CUDA kernels of libglide.so.  torch is used for
device memory and streams.  There is no fallback: if the library has not been built
(python -m paper_2607_24788_b200.build) loading raises.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Optional, Sequence

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libglide.so")

GLIDE_F32, GLIDE_BF16, GLIDE_BF16_CACHE4 = 0, 1, 4
GLIDE_PHI_SOFTMAX, GLIDE_PHI_PROJ_SOFTMAX2 = 0, 1
GLIDE_MERGE_SHARED, GLIDE_MERGE_SUM_EVICTED, GLIDE_MERGE_SUM_ALL = 0, 1, 2
GLIDE_DECODE_AUTO, GLIDE_DECODE_MMA, GLIDE_DECODE_FMA, GLIDE_DECODE_STREAM = 0, 1, 2, 3
GLIDE_PREFILL_AUTO, GLIDE_PREFILL_MMA_SYNC, GLIDE_PREFILL_TCGEN05, GLIDE_PREFILL_FMA = 0, 1, 2, 3

GLIDE_OK = 0
GLIDE_ERR_INVALID_ARG = 1
GLIDE_ERR_UNSUPPORTED = 2
GLIDE_ERR_WORKSPACE_TOO_SMALL = 3
GLIDE_ERR_CAPACITY = 4
GLIDE_ERR_STATE = 5
GLIDE_ERR_CUDA = 6
GLIDE_ERR_SCRATCH_LIMIT = 7


class GlideError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {strerror(code)} (status {code})")


class glide_config(ctypes.Structure):
    _fields_ = [
        ("n_layers", ctypes.c_int32), ("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
        ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("io_dtype", ctypes.c_int32),
        ("phi", ctypes.c_int32), ("merge", ctypes.c_int32),
        ("windows", ctypes.POINTER(ctypes.c_int64)), ("q_to_kv", ctypes.POINTER(ctypes.c_int32)),
        ("max_tokens", ctypes.c_int64), ("softmax_scale", ctypes.c_float), ("prefill_chunk", ctypes.c_int32),
        ("decode_chunk", ctypes.c_int32), ("decode_state_splits", ctypes.c_int32), ("decode_impl", ctypes.c_int32),
        ("prefill_impl", ctypes.c_int32),
        ("phi_wq", ctypes.c_void_p), ("phi_wk", ctypes.c_void_p), ("gated", ctypes.c_int32), ("reserved_", ctypes.c_int32),
    ]


class glide_paged_config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_layers", "n_q_heads", "n_kv_heads", "head_dim", "io_dtype", "page_size", "n_pages", "max_batch")] + \
               [(n, ctypes.c_int64) for n in ("max_tokens", "layer_stride", "page_stride", "head_stride", "row_stride")] + \
               [("softmax_scale", ctypes.c_float), ("weights", ctypes.c_int32)]


class glide_paged_call(ctypes.Structure):
    _fields_ = [("layer", ctypes.c_int32), ("batch", ctypes.c_int32), ("dev_table", ctypes.c_void_p), ("table_cols", ctypes.c_int32),
                ("n_sink", ctypes.c_int32), ("table_stride", ctypes.c_int64), ("dev_lens", ctypes.c_void_p), ("dev_starts", ctypes.c_void_p)] + \
               [(n, ctypes.c_int64) for n in ("n_tokens", "q_stride", "kv_stride", "out_stride", "window")] + \
               [(n, ctypes.c_void_p) for n in ("dev_weight", "dev_pos", "dev_seen")] + [("track_stride", ctypes.c_int64)]


class glide_rotation(ctypes.Structure):
    _fields_ = [("dev_cos", ctypes.c_void_p), ("dev_sin", ctypes.c_void_p), ("n_positions", ctypes.c_int64), ("stride", ctypes.c_int64),
                ("rot_dim", ctypes.c_int32), ("neighbours", ctypes.c_int32)]


class glide_layer_info_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("window", "capacity", "n", "count", "head_slot", "n_evicted")]


_lib = None


def load_library() -> ctypes.CDLL:
    """dlopen libglide.so and declare the prototypes. Raises if the library is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} not built: run `python -m paper_2607_24788_b200.build` "
                           "(there is no CPU or PyTorch fallback for the GLIDE kernels)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    cfgp = ctypes.POINTER(glide_config)
    lib.glide_workspace_bytes.argtypes = [cfgp, ctypes.POINTER(ctypes.c_size_t)]
    lib.glide_create.argtypes = [cfgp, vp, ctypes.c_size_t, vp, ctypes.POINTER(vp)]
    lib.glide_prefill.argtypes = [vp, i32, i32, i64, vp, vp, vp, vp, vp]
    lib.glide_decode_step.argtypes = [vp, vp, vp, vp, vp, vp]
    lib.glide_decode_step_noalloc.argtypes = [vp, vp, vp, vp, vp, vp]
    lib.glide_prefill_gated.argtypes = [vp, i32, i32, i64, vp, vp, vp, vp, vp, vp]
    lib.glide_decode_step_gated.argtypes = [vp, vp, vp, vp, vp, vp, vp]
    lib.glide_export_gates.argtypes = [vp, i32, vp, vp]
    lib.glide_import_gates.argtypes = [vp, i32, vp, vp]
    lib.glide_decode_step_layers.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp]
    lib.glide_reset_seq.argtypes = [vp, i32, vp]
    lib.glide_park_seq.argtypes = [vp, i32, vp]
    lib.glide_prefill_seq.argtypes = [vp, i32, i64, vp, vp, vp, vp, vp]
    lib.glide_seq_tokens.argtypes = [vp, i32, ctypes.POINTER(i64)]
    lib.glide_seq_layer_info.argtypes = [vp, i32, i32, vp, ctypes.POINTER(glide_layer_info_t)]
    lib.glide_destroy.argtypes = [vp]
    lib.glide_layer_info.argtypes = [vp, i32, vp, ctypes.POINTER(glide_layer_info_t)]
    lib.glide_export_state.argtypes = [vp, i32, vp, vp, vp, vp, vp]
    lib.glide_import_state.argtypes = [vp, i32, i64, vp, vp, vp, vp, vp]
    lib.glide_reset.argtypes = [vp, vp]
    lib.glide_device_status.argtypes = [vp, vp, ctypes.POINTER(i32)]
    lib.glide_decode_launch_info.argtypes = [vp, ctypes.POINTER(i32), ctypes.POINTER(i32), ctypes.POINTER(i32)]
    lib.glide_stream_schedule.argtypes = [cfgp, i32, i64, ctypes.POINTER(i32), i32, ctypes.POINTER(i32)]
    lib.glide_stream_schedule.restype = ctypes.c_int
    pagedp, callp = ctypes.POINTER(glide_paged_config), ctypes.POINTER(glide_paged_call)
    lib.glide_paged_workspace_bytes.argtypes = [pagedp, ctypes.POINTER(ctypes.c_size_t)]
    lib.glide_paged_create.argtypes = [pagedp, vp, vp, vp, ctypes.c_size_t, vp, ctypes.POINTER(vp)]
    lib.glide_paged_destroy.argtypes = [vp]
    lib.glide_paged_prefill.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp]
    lib.glide_paged_decode.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp]
    lib.glide_paged_weights.argtypes = [vp, vp, vp, vp, vp]
    lib.glide_paged_evict.argtypes = [vp, vp, i64, i64, vp, vp, vp, vp]
    lib.glide_paged_append.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp]
    lib.glide_paged_read.argtypes = [vp, vp, vp, vp, vp]
    lib.glide_paged_bounds.argtypes = [vp, vp, vp, vp]
    lib.glide_paged_decode_sparse.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp]
    lib.glide_paged_check_call.argtypes = [pagedp, callp]
    lib.glide_paged_device_status.argtypes = [vp, vp, ctypes.POINTER(i32)]
    lib.glide_strerror.argtypes = [ctypes.c_int]
    lib.glide_strerror.restype = ctypes.c_char_p
    for name in ("glide_workspace_bytes", "glide_create", "glide_prefill", "glide_decode_step", "glide_destroy",
                 "glide_decode_step_noalloc", "glide_decode_step_layers", "glide_prefill_gated",
                 "glide_decode_step_gated", "glide_export_gates", "glide_import_gates",
                 "glide_layer_info", "glide_export_state", "glide_import_state", "glide_reset",
                 "glide_device_status", "glide_decode_launch_info", "glide_paged_workspace_bytes", "glide_paged_create",
                 "glide_paged_destroy", "glide_paged_prefill", "glide_paged_decode", "glide_paged_weights", "glide_paged_evict",
                 "glide_paged_append", "glide_paged_read", "glide_paged_bounds", "glide_paged_decode_sparse",
                 "glide_paged_check_call", "glide_paged_device_status"):
        getattr(lib, name).restype = ctypes.c_int
    _lib = lib
    return lib


def strerror(code: int) -> str:
    return load_library().glide_strerror(int(code)).decode()


def glide_stream_schedule(cfg, n_sms: int = 148, smem_limit: int = 232448):
    """The streaming decode kernel's all-layer schedule for `cfg` (host only): an int32 array [segments][12], see
    include/glide.h."""
    import numpy as np
    lib = load_library()
    n = ctypes.c_int32(0)
    _check(lib.glide_stream_schedule(ctypes.byref(cfg), n_sms, smem_limit, None, 0, ctypes.byref(n)), "glide_stream_schedule")
    rows = np.zeros((n.value, 12), dtype=np.int32)
    if n.value:
        _check(lib.glide_stream_schedule(ctypes.byref(cfg), n_sms, smem_limit,
                                         rows.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)), n.value, ctypes.byref(n)),
               "glide_stream_schedule")
    return rows


def _check(code: int, where: str):
    if code != GLIDE_OK:
        raise GlideError(code, where)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "device buffers must be contiguous CUDA tensors"
    return t.data_ptr()


def _stream(stream: Optional[torch.cuda.Stream]) -> Optional[int]:
    if stream is None:   # the raw handle of the current device's current stream, without a Stream object around it
        return _raw_stream(_current_device()) or None
    return stream.cuda_stream or None


# torch.cuda.current_stream() builds an object per call (2.5 us of a step's host time); these are what it asks
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda dev: torch.cuda.current_stream(dev).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def make_config(windows: Sequence[int], batch: int, n_q_heads: int, n_kv_heads: int, head_dim: int, max_tokens: int,
                dtype: torch.dtype = torch.bfloat16, q_to_kv: Optional[Sequence[int]] = None,
                softmax_scale: float = 0.0, prefill_chunk: int = 0, decode_chunk: int = 0,
                decode_state_splits: int = 0, decode_impl: int = 0, prefill_impl: int = 0, merge: int = 0,
                phi: int = GLIDE_PHI_SOFTMAX, phi_wq: Optional[torch.Tensor] = None,
                phi_wk: Optional[torch.Tensor] = None, gated: bool = False):
    """Returns (glide_config, keepalive) -- keepalive holds the host arrays the struct points to.
    phi = GLIDE_PHI_PROJ_SOFTMAX2 takes the projections phi_wq [L][H][d][d], phi_wk [L][Hkv][d][d] (device tensors of
    the I/O dtype; the library borrows them)."""
    win = (ctypes.c_int64 * len(windows))(*[int(w) for w in windows])
    qmap = (ctypes.c_int32 * len(q_to_kv))(*[int(x) for x in q_to_kv]) if q_to_kv is not None else None
    cfg = glide_config()
    cfg.n_layers, cfg.batch, cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim = len(windows), batch, n_q_heads, n_kv_heads, head_dim
    cfg.io_dtype = {torch.float32: GLIDE_F32, torch.bfloat16: GLIDE_BF16}[dtype]
    cfg.phi, cfg.merge = int(phi), int(merge)
    if phi_wq is not None or phi_wk is not None:
        L = len(windows)
        assert phi_wq.shape == (L, n_q_heads, head_dim, head_dim) and phi_wk.shape == (L, n_kv_heads, head_dim, head_dim)
        assert phi_wq.dtype == dtype and phi_wk.dtype == dtype
    cfg.phi_wq, cfg.phi_wk = _ptr(phi_wq), _ptr(phi_wk)
    cfg.gated, cfg.reserved_ = int(bool(gated)), 0
    cfg.windows = ctypes.cast(win, ctypes.POINTER(ctypes.c_int64))
    cfg.q_to_kv = ctypes.cast(qmap, ctypes.POINTER(ctypes.c_int32)) if qmap is not None else None
    cfg.max_tokens = int(max_tokens)
    cfg.softmax_scale = float(softmax_scale)
    cfg.prefill_chunk, cfg.decode_chunk, cfg.decode_state_splits = int(prefill_chunk), int(decode_chunk), int(decode_state_splits)
    cfg.decode_impl = int(decode_impl)
    cfg.prefill_impl = int(prefill_impl)
    return cfg, (win, qmap, phi_wq, phi_wk)


def glide_workspace_bytes(cfg: glide_config) -> int:
    out = ctypes.c_size_t(0)
    _check(load_library().glide_workspace_bytes(ctypes.byref(cfg), ctypes.byref(out)), "glide_workspace_bytes")
    return int(out.value)


class Glide:
    """Owns a torch workspace and a glide_ctx; methods carry the C ABI's names."""

    def __init__(self, windows: Sequence[int], batch: int, n_q_heads: int, n_kv_heads: int, head_dim: int,
                 max_tokens: int, dtype: torch.dtype = torch.bfloat16, device="cuda", **kw):
        self.lib = load_library()
        self.device = torch.device(device)
        self.dtype = dtype
        self.L, self.B, self.H, self.Hkv, self.d = len(windows), batch, n_q_heads, n_kv_heads, head_dim
        self.windows = [int(w) for w in windows]
        self.max_tokens = int(max_tokens)
        self.dp = 2 * head_dim if kw.get("phi", GLIDE_PHI_SOFTMAX) == GLIDE_PHI_PROJ_SOFTMAX2 else head_dim
        self.gated = bool(kw.get("gated", False))
        self.cfg, self._keep = make_config(windows, batch, n_q_heads, n_kv_heads, head_dim, max_tokens, dtype, **kw)
        self.workspace_bytes = glide_workspace_bytes(self.cfg)
        with torch.cuda.device(self.device):
            # 256-byte alignment is required; 2 MiB keeps the library's own 2 MiB-aligned offsets of the streamed
            # arrays aligned in device memory as well
            align = 2 << 20
            self.workspace = torch.empty(self.workspace_bytes + align, dtype=torch.uint8, device=self.device)
            base = self.workspace.data_ptr()
            self._ws_ptr = (base + align - 1) // align * align
            handle = ctypes.c_void_p()
            _check(self.lib.glide_create(ctypes.byref(self.cfg), self._ws_ptr, self.workspace_bytes, _stream(None),
                                         ctypes.byref(handle)), "glide_create")
        self._h = handle
        self._q_row, self._kv_row = (batch, n_q_heads, head_dim), (batch, n_kv_heads, head_dim)   # a layer's tensors

    def _step_args(self, q, k, v, out, layer_count: int):
        """Checks of a decode step's tensors (layer_count layers); their addresses."""
        q_shape, kv_shape = (layer_count, *self._q_row), (layer_count, *self._kv_row)
        assert q.shape == q_shape and out.shape == q_shape and k.shape == kv_shape and v.shape == kv_shape
        dt = self.dtype
        assert q.dtype is dt and k.dtype is dt and v.dtype is dt and out.dtype is dt
        assert (q.is_cuda and k.is_cuda and v.is_cuda and out.is_cuda and q.is_contiguous() and k.is_contiguous()
                and v.is_contiguous() and out.is_contiguous()), "device buffers must be contiguous CUDA tensors"
        return q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr()

    # -- the four calls of the hot path ---------------------------------------------------------
    def glide_prefill(self, q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor,
                      out: Optional[torch.Tensor] = None, layer_begin: int = 0, layer_count: Optional[int] = None,
                      stream=None) -> None:
        lc = self.L - layer_begin if layer_count is None else layer_count
        T = k.shape[2]
        assert k.shape == (lc, self.B, T, self.Hkv, self.d) and v.shape == k.shape and k.dtype == self.dtype
        if out is not None:
            assert q is not None and q.shape == (lc, self.B, T, self.H, self.d) and out.shape == q.shape
        _check(self.lib.glide_prefill(self._h, layer_begin, lc, T, _ptr(q), _ptr(k), _ptr(v), _ptr(out),
                                      _stream(stream)), "glide_prefill")

    def glide_decode_step(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                          stream=None) -> None:
        rc = self.lib.glide_decode_step(self._h, *self._step_args(q, k, v, out, self.L), _stream(stream))
        if rc:
            _check(rc, "glide_decode_step")

    def glide_prefill_gated(self, q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor,
                            gate: Optional[torch.Tensor], out: Optional[torch.Tensor] = None, layer_begin: int = 0,
                            layer_count: Optional[int] = None, stream=None) -> None:
        """glide_prefill of a gated context: gate fp32 [layer_count][B][T][H_kv] in (0, 1], or None for gates of 1."""
        lc = self.L - layer_begin if layer_count is None else layer_count
        T = k.shape[2]
        assert k.shape == (lc, self.B, T, self.Hkv, self.d) and v.shape == k.shape and k.dtype == self.dtype
        assert gate is None or (gate.shape == (lc, self.B, T, self.Hkv) and gate.dtype == torch.float32)
        if out is not None:
            assert q is not None and q.shape == (lc, self.B, T, self.H, self.d) and out.shape == q.shape
        _check(self.lib.glide_prefill_gated(self._h, layer_begin, lc, T, _ptr(q), _ptr(k), _ptr(v), _ptr(gate), _ptr(out),
                                            _stream(stream)), "glide_prefill_gated")

    def glide_decode_step_gated(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, gate: Optional[torch.Tensor],
                                out: torch.Tensor, stream=None) -> None:
        """glide_decode_step of a gated context: gate fp32 [L][B][H_kv] in (0, 1], or None for gates of 1."""
        args = self._step_args(q, k, v, out, self.L)
        assert gate is None or (gate.shape == (self.L, self.B, self.Hkv) and gate.dtype == torch.float32)
        _check(self.lib.glide_decode_step_gated(self._h, *args[:3], _ptr(gate), args[3], _stream(stream)),
               "glide_decode_step_gated")

    def glide_decode_step_layers(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                                 layer_begin: int, layer_count: int, stream=None) -> None:
        """glide_decode_step for the layers [layer_begin, layer_begin + layer_count); tensors are the range's."""
        rc = self.lib.glide_decode_step_layers(self._h, int(layer_begin), int(layer_count), *self._step_args(q, k, v, out, layer_count),
                                               _stream(stream))
        if rc:
            _check(rc, "glide_decode_step_layers")

    def glide_decode_step_noalloc(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                                  stream=None) -> None:
        """glide_decode_step for callers that must not allocate: the step's split-K scratch lives in a static
        buffer inside the library instead of the workspace (see include/glide.h for the limits)."""
        assert q.shape == (self.L, self.B, self.H, self.d) and out.shape == q.shape
        assert k.shape == (self.L, self.B, self.Hkv, self.d) and v.shape == k.shape
        assert q.dtype == k.dtype == v.dtype == out.dtype == self.dtype
        _check(self.lib.glide_decode_step_noalloc(self._h, _ptr(q), _ptr(k), _ptr(v), _ptr(out), _stream(stream)),
               "glide_decode_step_noalloc")

    # -- sequences of different lengths: every slot of the batch has its own position ---------------
    def glide_reset_seq(self, b: int, stream=None) -> None:
        """Slot b starts an empty sequence; the other slots are untouched."""
        _check(self.lib.glide_reset_seq(self._h, int(b), _stream(stream)), "glide_reset_seq")

    def glide_park_seq(self, b: int, stream=None) -> None:
        """Slot b holds no sequence: decode steps skip it until glide_reset_seq starts a new one there."""
        _check(self.lib.glide_park_seq(self._h, int(b), _stream(stream)), "glide_park_seq")

    def glide_prefill_seq(self, b: int, q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor,
                          out: Optional[torch.Tensor] = None, stream=None) -> None:
        """glide_prefill for slot b alone, all layers: q, out [L][T][H][d]; k, v [L][T][H_kv][d]."""
        T = k.shape[1]
        assert k.shape == (self.L, T, self.Hkv, self.d) and v.shape == k.shape and k.dtype == self.dtype
        if out is not None:
            assert q is not None and q.shape == (self.L, T, self.H, self.d) and out.shape == q.shape
        _check(self.lib.glide_prefill_seq(self._h, int(b), T, _ptr(q), _ptr(k), _ptr(v), _ptr(out), _stream(stream)),
               "glide_prefill_seq")

    def glide_seq_tokens(self, b: int) -> int:
        n = ctypes.c_int64(0)
        _check(self.lib.glide_seq_tokens(self._h, int(b), ctypes.byref(n)), "glide_seq_tokens")
        return int(n.value)

    def glide_seq_layer_info(self, layer: int, b: int) -> dict:
        info = glide_layer_info_t()
        _check(self.lib.glide_seq_layer_info(self._h, layer, int(b), _stream(None), ctypes.byref(info)),
               "glide_seq_layer_info")
        return {n: int(getattr(info, n)) for n, _ in glide_layer_info_t._fields_}

    def glide_destroy(self) -> None:
        if getattr(self, "_h", None):
            self.lib.glide_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.glide_destroy()
        except Exception:
            pass

    # -- support ----------------------------------------------------------------------------------
    def glide_layer_info(self, layer: int) -> dict:
        info = glide_layer_info_t()
        _check(self.lib.glide_layer_info(self._h, layer, _stream(None), ctypes.byref(info)), "glide_layer_info")
        return {n: int(getattr(info, n)) for n, _ in glide_layer_info_t._fields_}

    def capacity(self, layer: int) -> int:
        return min(self.windows[layer], self.max_tokens)

    def glide_export_state(self, layer: int):
        cap = self.capacity(layer)
        rk = torch.empty((self.B, self.Hkv, cap, self.d), dtype=self.dtype, device=self.device)
        rv = torch.empty_like(rk)
        S = torch.empty((self.B, self.Hkv, self.dp, self.d), dtype=torch.float32, device=self.device)
        z = torch.empty((self.B, self.Hkv, self.dp), dtype=torch.float32, device=self.device)
        _check(self.lib.glide_export_state(self._h, layer, _ptr(rk) if cap else None, _ptr(rv) if cap else None,
                                           _ptr(S), _ptr(z), _stream(None)), "glide_export_state")
        return rk, rv, S, z

    def glide_import_state(self, layer: int, n: int, ringK=None, ringV=None, S=None, z=None) -> None:
        _check(self.lib.glide_import_state(self._h, layer, int(n), _ptr(ringK), _ptr(ringV), _ptr(S), _ptr(z),
                                           _stream(None)), "glide_import_state")

    def glide_export_gates(self, layer: int) -> torch.Tensor:
        """[B][H_kv][capacity] fp32: the gates of the ring's tokens (gated contexts)."""
        gates = torch.empty((self.B, self.Hkv, self.capacity(layer)), dtype=torch.float32, device=self.device)
        _check(self.lib.glide_export_gates(self._h, layer, _ptr(gates), _stream(None)), "glide_export_gates")
        return gates

    def glide_import_gates(self, layer: int, gates: torch.Tensor) -> None:
        assert gates.shape == (self.B, self.Hkv, self.capacity(layer)) and gates.dtype == torch.float32
        _check(self.lib.glide_import_gates(self._h, layer, _ptr(gates), _stream(None)), "glide_import_gates")

    def glide_reset(self) -> None:
        _check(self.lib.glide_reset(self._h, _stream(None)), "glide_reset")

    def glide_device_status(self) -> int:
        out = ctypes.c_int32(0)
        _check(self.lib.glide_device_status(self._h, _stream(None), ctypes.byref(out)), "glide_device_status")
        return int(out.value)

    def glide_decode_launch_info(self) -> dict:
        a, b, c = ctypes.c_int32(0), ctypes.c_int32(0), ctypes.c_int32(0)
        _check(self.lib.glide_decode_launch_info(self._h, ctypes.byref(a), ctypes.byref(b), ctypes.byref(c)),
               "glide_decode_launch_info")
        return dict(launches=a.value, work_items=b.value, grid=c.value)


def paged4_row_bytes(head_dim: int) -> int:
    """Bytes that a slot of a page in 4 bits takes of its KV head's block: the codes, then (behind all slots' codes) the levels."""
    return head_dim // 2 + 4


def make_paged_config(k_pages: torch.Tensor, n_q_heads: int, max_batch: int, max_tokens: int, softmax_scale: float = 0.0,
                      weights: bool = True, head_dim: Optional[int] = None) -> glide_paged_config:
    """The configuration of pages k_pages [L][n_pages][H_kv][page_size][d], which may be a view with other strides; with head_dim, of pages
    in 4 bits: uint8 [L][n_pages][H_kv][page_size * (head_dim / 2 + 4)], a head's block side by side."""
    if head_dim is not None:
        assert k_pages.dim() == 4 and k_pages.dtype is torch.uint8 and k_pages.stride(3) == 1, \
            "pages in 4 bits are uint8 [L][n_pages][H_kv][page_size * (head_dim / 2 + 4)]"
        L, n, hkv, block = k_pages.shape
        row = paged4_row_bytes(head_dim)
        assert block % row == 0, f"pages in 4 bits: {row} bytes for each slot of a block"
        assert hkv == 1 or k_pages.stride(2) >= block, "pages: heads that share memory"
        cfg = glide_paged_config(n_layers=L, n_q_heads=n_q_heads, n_kv_heads=hkv, head_dim=head_dim, io_dtype=GLIDE_BF16_CACHE4, page_size=block // row,
                                 n_pages=n, max_batch=int(max_batch), max_tokens=int(max_tokens), softmax_scale=float(softmax_scale),
                                 weights=int(bool(weights)), row_stride=row)
        cfg.head_stride = int(k_pages.stride(2)) if hkv > 1 else block
        cfg.page_stride = int(k_pages.stride(1)) if n > 1 else hkv * cfg.head_stride
        cfg.layer_stride = int(k_pages.stride(0)) if L > 1 else max(1, n) * cfg.page_stride
        return cfg
    assert k_pages.dim() == 5 and k_pages.stride(4) == 1, "pages are [L][n_pages][H_kv][page_size][d], features side by side"
    L, n, hkv, page, d = k_pages.shape
    assert k_pages.stride(3) >= d, "pages: slots that share memory"   # (strides of 0 would say "side by side" to the library)
    cfg = glide_paged_config(n_layers=L, n_q_heads=n_q_heads, n_kv_heads=hkv, head_dim=d,
                             io_dtype={torch.float32: GLIDE_F32, torch.bfloat16: GLIDE_BF16}[k_pages.dtype], page_size=page, n_pages=n,
                             max_batch=int(max_batch), max_tokens=int(max_tokens), softmax_scale=float(softmax_scale), weights=int(bool(weights)))
    cfg.layer_stride, cfg.page_stride, cfg.head_stride, cfg.row_stride = (int(k_pages.stride(i)) for i in range(4))
    if L == 1:   # (of a single layer any distance will do)
        cfg.layer_stride = max(1, n) * cfg.page_stride
    return cfg


def glide_paged_workspace_bytes(cfg: glide_paged_config) -> int:
    out = ctypes.c_size_t(0)
    _check(load_library().glide_paged_workspace_bytes(ctypes.byref(cfg), ctypes.byref(out)), "glide_paged_workspace_bytes")
    return int(out.value)


class GlideRotation:
    """The rotation of queries and keys by their positions: cos, sin fp32 [n_positions][rot_dim / 2] on the GPU, a row for each position (views of
    equal strides will do).  neighbours: pair i is features 2i and 2i + 1, otherwise i and i + rot_dim / 2."""

    def __init__(self, cos: torch.Tensor, sin: torch.Tensor, neighbours: bool = False):
        assert cos.dtype is torch.float32 and sin.dtype is torch.float32 and cos.dim() == 2 and cos.shape == sin.shape and cos.device == sin.device, \
            "cos and sin: fp32 [n_positions][rot_dim / 2]"
        assert cos.stride() == sin.stride() and cos.stride(1) == 1, "cos and sin: equal strides, a position's entries side by side"
        n, half = cos.shape
        assert n == 1 or cos.stride(0) >= half, "cos and sin: positions that share memory"
        self.device, self._keep = cos.device, (cos, sin)
        self.packed = bytes(glide_rotation(dev_cos=cos.data_ptr(), dev_sin=sin.data_ptr(), n_positions=n, stride=cos.stride(0) if n > 1 else half,
                                           rot_dim=2 * half, neighbours=int(bool(neighbours))))


_I32, _F32 = torch.int32, torch.float32
_MOST_TOKENS = 1 << 30   # of a call
# a call's fields as bytes of its own (one pack instead of a store per field: a step's host time is what counts where the cache is short)
_pack_call = struct.Struct("@iiPiiqPPqqqqqPPPq").pack
assert struct.calcsize("@iiPiiqPPqqqqqPPPq") == ctypes.sizeof(glide_paged_call)


class GlidePaged:
    """Softmax attention over a paged cache (include/glide.h): k_pages, v_pages [L][n_pages][H_kv][page_size][d] are the
    caller's (views of equal strides will do), a torch workspace and the handle are owned here.  Tables are int32 [B][cols], lens,
    seen and new_lens int32 [B], starts int32 [B + 1], weight fp32 and pos int32 [B][H_kv][slots], all on the pages' device.
    With head_dim the pages are held in 4 bits: uint8 [L][n_pages][H_kv][page_size * (head_dim / 2 + 4)], all else bf16 (weights has to be False).
    Calls of one object must follow one another on the GPU, from whichever host threads they come; objects of their own may share
    pages.  The object has to live until its calls on streams other than the one that it was made on have ended."""

    def __init__(self, k_pages: torch.Tensor, v_pages: torch.Tensor, n_q_heads: int, max_batch: int, max_tokens: int,
                 softmax_scale: float = 0.0, weights: bool = True, head_dim: Optional[int] = None):
        self.lib = load_library()
        assert k_pages.is_cuda and v_pages.device == k_pages.device and v_pages.dtype == k_pages.dtype
        assert v_pages.shape == k_pages.shape and v_pages.stride() == k_pages.stride()
        self.device, self.dtype = k_pages.device, torch.bfloat16 if head_dim is not None else k_pages.dtype
        self.cfg = make_paged_config(k_pages, n_q_heads, max_batch, max_tokens, softmax_scale, weights, head_dim)
        self.L, self.n_pages, self.Hkv, self.page_size, self.d = (getattr(self.cfg, n) for n in ("n_layers", "n_pages", "n_kv_heads", "page_size", "head_dim"))
        self.H, self.max_batch, self.max_tokens = int(n_q_heads), int(max_batch), int(max_tokens)
        self.workspace_bytes = glide_paged_workspace_bytes(self.cfg)
        self._keep = (k_pages, v_pages)
        with torch.cuda.device(self.device):
            self.workspace = torch.empty(self.workspace_bytes + 256, dtype=torch.uint8, device=self.device)
            base = (self.workspace.data_ptr() + 255) // 256 * 256
            handle = ctypes.c_void_p()
            _check(self.lib.glide_paged_create(ctypes.byref(self.cfg), k_pages.data_ptr(), v_pages.data_ptr(), base, self.workspace_bytes,
                                               _stream(None), ctypes.byref(handle)), "glide_paged_create")
        self._h = handle
        self._index = self.device.index

    # (A tensor's shape is asked for once, as a whole: .size(i) and .stride(i) take three times as long, and a short step is bound by
    # the host's time for its call.)
    def _ints(self, t: torch.Tensor, n: int, what: str) -> int:
        assert t.dtype is _I32 and t.shape == (n,) and t.is_contiguous() and t.get_device() == self._index, f"{what}: int32 [{n}] on {self.device}"
        return t.data_ptr()

    def _rows(self, t: torch.Tensor, rows: int, heads: int, what: str):
        """Address and token stride (0: side by side) of [rows][heads][d] whose heads lie side by side."""
        assert t.dtype is self.dtype and t.shape == (rows, heads, self.d) and t.get_device() == self._index, \
            f"{what}: {self.dtype} [{rows}][{heads}][{self.d}] on {self.device}"
        if t.is_contiguous():
            return t.data_ptr(), 0
        stride = t.stride()
        assert stride[2] == 1 and (heads == 1 or stride[1] == self.d), f"{what}: a token's heads have to lie side by side"
        if rows == 1:
            return t.data_ptr(), 0
        assert stride[0] >= heads * self.d, f"{what}: tokens that share memory"   # (0 would say "side by side" to the library)
        return t.data_ptr(), stride[0]

    def _track(self, t: torch.Tensor, B: int, dtype, what: str):
        shape = t.shape
        assert t.dtype is dtype and len(shape) == 3 and shape[:2] == (B, self.Hkv) and t.is_contiguous() and t.get_device() == self._index, \
            f"{what}: {dtype} [{B}][{self.Hkv}][slots] on {self.device}"
        return t.data_ptr(), shape[2]

    def _lse(self, lse, rows: int):
        if lse is None:
            return None
        assert lse.dtype is _F32 and lse.shape == (rows, self.H) and lse.is_contiguous() and lse.get_device() == self._index, \
            f"lse: fp32 [{rows}][{self.H}] on {self.device}"
        return lse.data_ptr()

    def _packed_call(self, layer, table, lens, starts, rows, strides, window, n_sink, weight, pos, seen) -> bytes:
        """Checks what the calls share and packs it; rows None: one per sequence."""
        shape = table.shape
        assert table.dtype is _I32 and len(shape) == 2 and table.get_device() == self._index, f"table: int32 [B][cols] on {self.device}"
        B, cols = shape
        stride = cols
        if not table.is_contiguous():
            stride, inner = table.stride()
            assert inner == 1, "table: entries of a sequence side by side"
            stride = stride if B > 1 else cols
        p_weight = p_pos = p_seen = p_starts = track = 0
        if weight is not None:
            p_weight, track = self._track(weight, B, _F32, "weight")
        if pos is not None:
            p_pos, slots = self._track(pos, B, _I32, "pos")
            assert track in (0, slots), "weight and pos: as many slots"
            track = slots
        if seen is not None:
            p_seen = self._ints(seen, B, "seen")
        if starts is not None:
            p_starts = self._ints(starts, B + 1, "starts")
        return _pack_call(layer, B, table.data_ptr(), cols, n_sink, stride, self._ints(lens, B, "lens"), p_starts, B if rows is None else rows,
                          *strides, window, p_weight, p_pos, p_seen, track)

    def _run(self, where: str, stream, fn, call: bytes, *args) -> None:
        if self._index == _current_device():
            rc = fn(self._h, call, *args, _stream(stream))
        else:
            with torch.cuda.device(self.device):
                rc = fn(self._h, call, *args, _stream(stream))
        if rc:
            _check(rc, where)

    def _qkv(self, q, k, v, out, rows: int):
        """Addresses of q, k, v, out as far as there are, and their strides."""
        p_q = p_k = p_v = p_out = None
        q_stride = kv_stride = out_stride = 0
        if q is not None:
            p_q, q_stride = self._rows(q, rows, self.H, "q")
        assert (k is None) == (v is None), "k and v: both or neither"
        if k is not None:
            p_k, kv_stride = self._rows(k, rows, self.Hkv, "k")
            p_v, stride = self._rows(v, rows, self.Hkv, "v")
            assert stride == kv_stride, "k and v: equal strides"
        if out is not None:
            p_out, out_stride = self._rows(out, rows, self.H, "out")
        return (p_q, p_k, p_v, p_out), (q_stride, kv_stride, out_stride)

    def glide_paged_prefill(self, table, lens, starts, q, k, v, out=None, lse=None, window: int = -1, n_sink: int = 0, weight=None,
                            pos=None, seen=None, layer: int = 0, stream=None) -> None:
        """Stores the new tokens (rows starts[b] .. starts[b + 1] - 1 of k, v; None: they are in the cache) and, with out, attends.
        weight, pos: the new slots' account starts at 0 and their positions are written (k, v or not)."""
        rows = (k if k is not None else q).shape[0]
        tensors, strides = self._qkv(q, k, v, out, rows)
        call = self._packed_call(layer, table, lens, starts, rows, strides, window, n_sink, weight, pos, seen)
        self._run("glide_paged_prefill", stream, self.lib.glide_paged_prefill, call, *tensors, self._lse(lse, rows))

    def glide_paged_decode(self, table, lens, q, k, v, out, lse=None, window: int = -1, n_sink: int = 0, weight=None, pos=None,
                           seen=None, layer: int = 0, stream=None) -> None:
        """One new token per sequence: stored at slot lens[b] - 1 (k, v None: it is in the cache), attends; weight: the account, to which
        the step's weights are added (the new slot's starts at 0, with k, v None from what it is); pos: the slot's position is written."""
        rows = table.shape[0]
        tensors, strides = self._qkv(q, k, v, out, rows)
        call = self._packed_call(layer, table, lens, None, rows, strides, window, n_sink, weight, pos, seen)
        self._run("glide_paged_decode", stream, self.lib.glide_paged_decode, call, *tensors, self._lse(lse, rows))

    def glide_paged_weights(self, table, lens, starts, q, lse, weight, window: int = -1, n_sink: int = 0, layer: int = 0, stream=None) -> None:
        """Adds the weights that the tokens q with the row sums lse (of glide_paged_prefill) give every slot to the account."""
        rows = q.shape[0]
        tensors, strides = self._qkv(q, None, None, None, rows)
        call = self._packed_call(layer, table, lens, starts, rows, strides, window, n_sink, weight, None, None)
        self._run("glide_paged_weights", stream, self.lib.glide_paged_weights, call, tensors[0], self._lse(lse, rows))

    def glide_paged_evict(self, table, lens, seen, weight, pos, budget: int, new_lens, recent: int = 0, n_sink: int = 0, weight_out=None,
                          pos_out=None, layer: int = 0, stream=None) -> None:
        """Every (sequence, KV head) keeps min(lens[b], budget) slots; weight_out, pos_out None: the account changes in place.  new_lens may
        be lens unless other layers' calls still have to read those."""
        B = table.shape[0]
        p_weight, slots = self._track(weight if weight_out is None else weight_out, B, _F32, "weight_out")
        p_pos, pos_slots = self._track(pos if pos_out is None else pos_out, B, _I32, "pos_out")
        assert slots == pos_slots == weight.shape[2], "the accounts: as many slots"
        call = self._packed_call(layer, table, lens, None, None, (0, 0, 0), -1, n_sink, weight, pos, seen)
        self._run("glide_paged_evict", stream, self.lib.glide_paged_evict, call, budget, recent, p_weight, p_pos, self._ints(new_lens, B, "new_lens"))

    def glide_paged_append(self, table, lens, starts, q, k, v, q_out=None, rotation: Optional["GlideRotation"] = None, weight=None, pos=None,
                           seen=None, layer: int = 0, stream=None) -> None:
        """Brings in the new tokens (rows starts[b] .. starts[b + 1] - 1; starts None: row b of sequence b): k rotated by the tokens' positions,
        seen - T_b ... seen - 1, and v are stored, q rotated goes to q_out (q itself, or a tensor that does not overlap it; both None: no
        queries).  Prefill or decode with k, v None then attends."""
        assert (q is None) == (q_out is None), "q and q_out: both or neither"
        rows = k.shape[0]
        assert starts is not None or rows == table.shape[0], "without starts: one new token for each sequence"
        (p_q, p_k, p_v, p_out), strides = self._qkv(q, k, v, q_out, rows)
        call = self._packed_call(layer, table, lens, starts, rows, strides, -1, 0, weight, pos, seen)
        turn = None
        if rotation is not None:
            assert rotation.device == self.device, f"rotation: on {self.device}"
            turn = rotation.packed
        self._run("glide_paged_append", stream, self.lib.glide_paged_append, call, turn, p_q, p_k, p_v, p_out)

    def glide_paged_read(self, table, lens, starts, k, v, layer: int = 0, stream=None) -> None:
        """What the slots of the tokens that starts names (None: the newest of each sequence) hold, into the rows of k and v."""
        rows = k.shape[0]
        assert starts is not None or rows == table.shape[0], "without starts: one row for each sequence"
        (_, p_k, p_v, _), strides = self._qkv(None, k, v, None, rows)
        call = self._packed_call(layer, table, lens, starts, rows, strides, -1, 0, None, None, None)
        self._run("glide_paged_read", stream, self.lib.glide_paged_read, call, p_k, p_v)

    def _bounds(self, bounds):
        assert bounds.dtype is self.dtype and bounds.shape == (self.n_pages, self.Hkv, 2, self.d) and bounds.is_contiguous() and \
            bounds.get_device() == self._index, f"bounds: {self.dtype} [{self.n_pages}][{self.Hkv}][2][{self.d}] on {self.device}"
        return bounds.data_ptr()

    def glide_paged_bounds(self, table, lens, starts, bounds, n_tokens: Optional[int] = None, layer: int = 0, stream=None) -> None:
        """bounds [n_pages][H_kv][2][d], of the layer: least and largest key values of the pages that hold the tokens that starts names (None: the
        newest of each sequence).  n_tokens: starts[B] or more (None: as many as the sequences can hold)."""
        most = min(min(self.max_tokens, table.shape[1] * self.page_size) * table.shape[0], _MOST_TOKENS)
        rows = None if starts is None else most if n_tokens is None else int(n_tokens)
        call = self._packed_call(layer, table, lens, starts, rows, (0, 0, 0), -1, 0, None, None, None)
        self._run("glide_paged_bounds", stream, self.lib.glide_paged_bounds, call, self._bounds(bounds))

    def glide_paged_decode_sparse(self, table, lens, q, k, v, out, bounds, picks, scores, lse=None, n_sink: int = 0, pos=None, seen=None,
                                  layer: int = 0, stream=None) -> None:
        """One new token per sequence, over picks.shape[2] of its pages (its own, those of the first n_sink slots, and those of the largest
        score), which go to picks int32 [B][H_kv][n].  bounds [n_pages][H_kv][2][d] takes the new keys in; scores float64 [B][H_kv][cols]
        is work space.  k, v None: the token is in the cache already."""
        B, cols = table.shape
        tensors, strides = self._qkv(q, k, v, out, B)
        assert picks.dtype is _I32 and picks.dim() == 3 and picks.shape[:2] == (B, self.Hkv) and picks.is_contiguous() and picks.get_device() == self._index, \
            f"picks: int32 [{B}][{self.Hkv}][n] on {self.device}"
        assert scores.dtype is torch.float64 and scores.shape == (B, self.Hkv, cols) and scores.is_contiguous() and scores.get_device() == self._index, \
            f"scores: float64 [{B}][{self.Hkv}][{cols}] on {self.device}"
        call = self._packed_call(layer, table, lens, None, B, strides, -1, n_sink, None, pos, seen)
        self._run("glide_paged_decode_sparse", stream, self.lib.glide_paged_decode_sparse, call, *tensors, self._lse(lse, B), self._bounds(bounds),
                  picks.shape[2], picks.data_ptr(), scores.data_ptr())

    def glide_paged_device_status(self, stream=None) -> int:
        """The status word of the device-side checks, read and cleared behind what `stream` has been given (0: nothing was recorded)."""
        out = ctypes.c_int32(0)
        with torch.cuda.device(self.device):
            _check(self.lib.glide_paged_device_status(self._h, _stream(stream), ctypes.byref(out)), "glide_paged_device_status")
        return int(out.value)

    def glide_paged_destroy(self) -> None:
        if getattr(self, "_h", None):
            self.lib.glide_paged_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.glide_paged_destroy()
        except Exception:
            pass
