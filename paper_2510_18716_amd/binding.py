"""ctypes binding of include/ssd.h and include/ssd_hooks.h.  Same names, same argument order; tensors are passed as
`data_ptr()` and the stream as the raw hipStream_t of torch's current stream."""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional

import numpy as np
import torch

SSD_F32, SSD_BF16 = 0, 1
SSD_SPATIAL, SSD_SEMANTIC = 0, 1
SSD_OK = 0
SSD_ERR_INVALID_ARG, SSD_ERR_LAYER_RANGE, SSD_ERR_STAGE_OVERFLOW, SSD_ERR_ORDER, SSD_ERR_HIP = -1, -2, -3, -4, -5

_HERE = os.path.dirname(os.path.abspath(__file__))
lib_path = os.path.join(_HERE, "libssd_hip.so")


def _load():
    if not os.path.exists(lib_path):
        # build only if nothing is built; never fall back to another implementation
        from . import build as _b
        _b.build(force=True, verbose=False)
    return C.CDLL(lib_path)


lib = _load()


class SsdConfig(C.Structure):
    _fields_ = [
        ("n_layers", C.c_int32), ("n_seqs", C.c_int32), ("n_heads", C.c_int32), ("head_dim", C.c_int32),
        ("dtype", C.c_int32), ("window", C.c_int32), ("n_init_sink", C.c_int32), ("budget", C.c_int32),
        ("recent", C.c_int32), ("stage_cap", C.c_int32), ("softmax_scale", C.c_float), ("spatial_row_buffer", C.c_int32),
        ("reserved", C.c_int32 * 4),
    ]


_vp = C.c_void_p
lib.ssd_cache_bytes.argtypes = [C.POINTER(SsdConfig), _vp]
lib.ssd_cache_bytes.restype = C.c_size_t
lib.ssd_cache_init.argtypes = [C.POINTER(SsdConfig), _vp, _vp, C.c_size_t, C.POINTER(_vp)]
lib.ssd_cache_init.restype = C.c_int
lib.ssd_cache_bytes_layered.argtypes = [C.POINTER(SsdConfig), _vp, _vp, _vp]
lib.ssd_cache_bytes_layered.restype = C.c_size_t
lib.ssd_cache_init_layered.argtypes = [C.POINTER(SsdConfig), _vp, _vp, _vp, _vp, C.c_size_t, C.POINTER(_vp)]
lib.ssd_cache_init_layered.restype = C.c_int
lib.ssd_cache_layer_budget.argtypes = [_vp, C.c_int, C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
lib.ssd_cache_layer_budget.restype = C.c_int
lib.ssd_cache_bytes_heads.argtypes = [C.POINTER(SsdConfig), _vp, _vp]
lib.ssd_cache_bytes_heads.restype = C.c_size_t
lib.ssd_cache_init_heads.argtypes = [C.POINTER(SsdConfig), _vp, _vp, _vp, C.c_size_t, C.POINTER(_vp)]
lib.ssd_cache_init_heads.restype = C.c_int
lib.ssd_cache_head_budget.argtypes = [_vp, C.c_int, C.c_int, C.POINTER(C.c_int32)]
lib.ssd_cache_head_budget.restype = C.c_int
lib.ssd_cache_head_runs.argtypes = [_vp, C.c_int, C.c_int, C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
lib.ssd_cache_head_runs.restype = C.c_int
lib.ssd_cache_spatial_slot.argtypes = [_vp, C.c_int, C.c_int, C.c_int, C.POINTER(C.c_int32)]
lib.ssd_cache_spatial_slot.restype = C.c_int
lib.ssd_cache_free.argtypes = [_vp]
lib.ssd_cache_free.restype = None
lib.ssd_cache_reset.argtypes = [_vp]
lib.ssd_cache_reset.restype = C.c_int
lib.ssd_cache_layer_state.argtypes = [_vp, C.c_int, C.POINTER(C.c_int32 * 4)]
lib.ssd_cache_layer_state.restype = C.c_int
lib.ssd_cache_layer_window.argtypes = [_vp, C.c_int, C.POINTER(C.c_int32)]
lib.ssd_cache_layer_window.restype = C.c_int
lib.ssd_cache_set_launch.argtypes = [_vp, C.c_int]
lib.ssd_cache_set_launch.restype = C.c_int
lib.ssd_classify_heads.argtypes = [_vp, _vp, C.c_int, C.c_int, C.c_int, C.c_int, C.c_float, _vp, _vp, _vp]
lib.ssd_classify_heads.restype = C.c_int
lib.ssd_append_token.argtypes = [_vp, C.c_int, C.c_int, _vp, _vp, _vp]
lib.ssd_append_token.restype = C.c_int
lib.ssd_decode_attn.argtypes = [_vp, C.c_int, C.c_int, _vp, _vp, C.c_int, _vp]
lib.ssd_decode_attn.restype = C.c_int
lib.ssd_decode_step.argtypes = [_vp, C.c_int, C.c_int, _vp, _vp, _vp, _vp, C.c_int, C.c_int, _vp]
lib.ssd_decode_step.restype = C.c_int
lib.ssd_decode_step_rope.argtypes = [_vp, C.c_int, C.c_int, _vp, _vp, _vp, _vp, C.c_int, C.c_int, _vp, _vp, C.c_int, _vp]
lib.ssd_decode_step_rope.restype = C.c_int
lib.ssd_bench_stream.argtypes = [_vp, C.c_size_t, C.c_longlong, C.c_int, _vp, _vp]
lib.ssd_bench_stream.restype = C.c_int
lib.ssd_bench_copy.argtypes = [_vp, _vp, C.c_size_t, _vp]
lib.ssd_bench_copy.restype = C.c_int
lib.ssd_compress_kv.argtypes = [_vp, C.c_int, C.c_int, _vp, _vp, _vp, C.c_int, _vp]
lib.ssd_compress_kv.restype = C.c_int
lib.ssd_prefill_scores.argtypes = [_vp, _vp, C.c_int, C.c_int, C.c_int, C.c_int, C.c_float, _vp, _vp]
lib.ssd_prefill_scores.restype = C.c_int
lib.ssd_cfg_mix.argtypes = [_vp, C.c_int, C.c_int, C.c_int, C.c_float, _vp, _vp]
lib.ssd_cfg_mix.restype = C.c_int
lib.ssd_cache_export_slots.argtypes = [_vp]
lib.ssd_cache_export_slots.restype = C.c_int
lib.ssd_cache_export.argtypes = [_vp, C.c_int, _vp, _vp, _vp, _vp]
lib.ssd_cache_export.restype = C.c_int
lib.ssd_dense_workspace_bytes.argtypes = [C.c_int] * 4
lib.ssd_dense_workspace_bytes.restype = C.c_size_t
lib.ssd_dense_decode_attn.argtypes = [_vp, _vp, _vp, _vp, C.c_int, C.c_int, C.c_int, C.c_int, C.c_int, C.c_int,
                                      C.c_float, _vp, _vp, C.c_int, C.c_int, C.c_int, _vp, C.c_size_t, _vp]
lib.ssd_dense_decode_attn.restype = C.c_int
lib.ssd_dense_decode_attn_static.argtypes = [_vp, _vp, _vp, _vp, C.c_int, C.c_int, C.c_int, C.c_int, C.c_int, C.c_int,
                                             C.c_float, _vp, _vp, C.c_int, C.c_int, C.c_int, _vp]
lib.ssd_dense_decode_attn_static.restype = C.c_int
lib.ssd_last_error.argtypes = []
lib.ssd_last_error.restype = C.c_char_p
lib.ssd_version.argtypes = []
lib.ssd_version.restype = C.c_int
lib.ssd_cache_set_launch_shape.argtypes = [_vp, C.c_int, C.c_int, C.c_int]
lib.ssd_cache_set_launch_shape.restype = C.c_int
lib.ssd_cache_last_launch_shape.argtypes = [_vp, C.POINTER(C.c_int32)]
lib.ssd_cache_last_launch_shape.restype = C.c_int
lib.ssd_dense_decode_attn_splits.argtypes = [_vp, _vp, _vp, _vp, C.c_int, C.c_int, C.c_int, C.c_int, C.c_int, C.c_int,
                                             C.c_float, _vp, _vp, C.c_int, C.c_int, C.c_int, C.c_int, _vp, C.c_size_t, _vp]
lib.ssd_dense_decode_attn_splits.restype = C.c_int
lib.ssd_decode_step_split.argtypes = [_vp, C.c_int, C.c_int, _vp, _vp, _vp, _vp, C.c_int, C.c_int, C.POINTER(_vp), C.c_int, C.c_int]
lib.ssd_decode_step_split.restype = C.c_int
lib.ssd_decode_step_split_rope.argtypes = [_vp, C.c_int, C.c_int, _vp, _vp, _vp, _vp, C.c_int, C.c_int, _vp, _vp, C.c_int,
                                           C.POINTER(_vp), C.c_int, C.c_int]
lib.ssd_decode_step_split_rope.restype = C.c_int
lib.ssd_decode_step_split_plan.argtypes = [_vp, C.c_int, C.c_int, C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
lib.ssd_decode_step_split_plan.restype = C.c_int


class SsdError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__("%s failed with %d: %s" % (where, code, ssd_last_error()))


def ssd_last_error() -> str:
    return lib.ssd_last_error().decode()


def ssd_version() -> int:
    return lib.ssd_version()


def _check(rc: int, where: str) -> None:
    if rc != SSD_OK:
        raise SsdError(rc, where)


_Tensor = torch.Tensor


def _ptr(t) -> Optional[int]:
    if type(t) is not _Tensor and (t is None or isinstance(t, int)):
        return t
    assert t.is_contiguous(), "tensors handed to the library must be contiguous"
    return t.data_ptr()


# torch's own accessors of the current stream's raw handle and device; not part of its public interface, so they may be missing
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream=None) -> Optional[int]:
    """Raw handle of `stream`, or of torch's current stream.  The handle itself is asked for where torch lets it be:
    torch.cuda.current_stream() builds a stream object and is_available() counts devices, 2.5 us of a call that takes 5."""
    if stream is not None:
        return stream if isinstance(stream, int) else stream.cuda_stream
    if _raw_stream is not None and _raw_device is not None and torch.cuda.is_initialized():
        return _raw_stream(_raw_device())
    if torch.cuda.is_available():
        return torch.cuda.current_stream().cuda_stream
    return None


_DTYPE_CODES = {torch.bfloat16: SSD_BF16, "bf16": SSD_BF16, torch.float32: SSD_F32, "f32": SSD_F32}


def _dtype_code(dt) -> int:
    if isinstance(dt, int):
        return dt                      # passed through; the library validates it
    code = _DTYPE_CODES.get(dt)
    if code is None:
        raise ValueError("unsupported dtype %r" % (dt,))
    return code


def make_config(L, B, H, d, dtype, W, S, M, R, C_, softmax_scale=0.0, spatial_row_buffer=0) -> SsdConfig:
    cfg = SsdConfig()
    cfg.n_layers, cfg.n_seqs, cfg.n_heads, cfg.head_dim = L, B, H, d
    cfg.dtype = _dtype_code(dtype)
    cfg.window, cfg.n_init_sink, cfg.budget, cfg.recent, cfg.stage_cap = W, S, M, R, C_
    cfg.softmax_scale = softmax_scale
    cfg.spatial_row_buffer = int(spatial_row_buffer)
    return cfg


def _per_layer(x, L):
    """Host int32 [L] array for a per-layer window / budget list, or None."""
    if x is None:
        return None
    a = np.ascontiguousarray(x, dtype=np.int32)
    if a.shape != (L,):
        raise ValueError("per-layer array must have one entry per layer")
    return a


def _per_head(x, L, H):
    """Host int32 [L*H] array of per-head budgets, or None."""
    if x is None:
        return None
    a = np.ascontiguousarray(x, dtype=np.int32)
    if a.size != L * H:
        raise ValueError("per-head array must have one entry per (layer, head)")
    return a.reshape(-1)


def ssd_cache_bytes(cfg: SsdConfig, head_type: np.ndarray, window=None, budget=None, head_budget=None) -> int:
    ht = np.ascontiguousarray(head_type, dtype=np.uint8)
    hb = _per_head(head_budget, cfg.n_layers, cfg.n_heads)
    if hb is not None:
        return lib.ssd_cache_bytes_heads(C.byref(cfg), ht.ctypes.data, hb.ctypes.data)
    w, m = _per_layer(window, cfg.n_layers), _per_layer(budget, cfg.n_layers)
    return lib.ssd_cache_bytes_layered(C.byref(cfg), ht.ctypes.data, None if w is None else w.ctypes.data,
                                       None if m is None else m.ctypes.data)


class Cache:
    """Owner of one ssd_cache descriptor and of the torch tensor that backs it in HBM.

    `device=None` creates a descriptor over a fake, never dereferenced address with launches
    switched off: the host-side logic (validation, counters, error codes) can then be exercised
    on a machine without a GPU.
    """

    def __init__(self, cfg: SsdConfig, head_type: np.ndarray, device="cuda", window=None, budget=None, head_budget=None):
        """window, budget: optional per-layer lists [L] (ssd_cache_init_layered);
        head_budget: optional [L, H] array, W_h of a spatial head / M_h of a semantic head (ssd_cache_init_heads)."""
        self.cfg = cfg
        self.head_type = np.ascontiguousarray(head_type, dtype=np.uint8)
        w, m = _per_layer(window, cfg.n_layers), _per_layer(budget, cfg.n_layers)
        hb = _per_head(head_budget, cfg.n_layers, cfg.n_heads)
        if hb is not None and (w is not None or m is not None):
            raise ValueError("budgets are given per layer or per head, not both")
        wp, mp = (None if w is None else w.ctypes.data), (None if m is None else m.ctypes.data)
        if hb is not None:
            nbytes = lib.ssd_cache_bytes_heads(C.byref(cfg), self.head_type.ctypes.data, hb.ctypes.data)
        else:
            nbytes = lib.ssd_cache_bytes_layered(C.byref(cfg), self.head_type.ctypes.data, wp, mp)
        if nbytes == 0:
            raise SsdError(SSD_ERR_INVALID_ARG, "ssd_cache_bytes")
        self.head_type = self.head_type.reshape(cfg.n_layers, cfg.n_heads)
        self.nbytes = nbytes
        self._h = _vp()
        if device is None:
            self.mem = None
            base = 1 << 20
        else:
            self.mem = torch.empty(nbytes + 256, dtype=torch.uint8, device=device)
            base = (self.mem.data_ptr() + 255) // 256 * 256
        if hb is not None:
            _check(lib.ssd_cache_init_heads(C.byref(cfg), self.head_type.ctypes.data, hb.ctypes.data, base, nbytes, C.byref(self._h)),
                   "ssd_cache_init_heads")
        else:
            _check(lib.ssd_cache_init_layered(C.byref(cfg), self.head_type.ctypes.data, wp, mp, base, nbytes, C.byref(self._h)),
                   "ssd_cache_init")
        if device is None:
            _check(lib.ssd_cache_set_launch(self._h, 0), "ssd_cache_set_launch")
        self.torch_dtype = torch.bfloat16 if cfg.dtype == SSD_BF16 else torch.float32

    def __del__(self):
        h = getattr(self, "_h", None)
        if h is not None and h.value:
            lib.ssd_cache_free(h)
            self._h = None

    @property
    def handle(self):
        return self._h

    def reset(self):
        _check(lib.ssd_cache_reset(self._h), "ssd_cache_reset")

    def set_launch_shape(self, ch: int = 0, wpb: int = 0, new_rows: int = 0):
        """Test / sweep hook: override the attention launch shape of this cache ((0, 0, 0) = the library's choice)."""
        _check(lib.ssd_cache_set_launch_shape(self._h, ch, wpb, new_rows), "ssd_cache_set_launch_shape")

    def last_launch_shape(self):
        """Test hook: (ch, wpb, new_rows) of the newest attention / step launch, in set_launch_shape's codes."""
        out = (C.c_int32 * 3)()
        _check(lib.ssd_cache_last_launch_shape(self._h, out), "ssd_cache_last_launch_shape")
        return tuple(out)

    def split_plan(self, layers_per_call: int, n_streams: int):
        """(sequences per part, number of parts) of ssd_decode_step_split for a call over that many layers."""
        p, n = C.c_int32(0), C.c_int32(0)
        _check(lib.ssd_decode_step_split_plan(self._h, layers_per_call, n_streams, C.byref(p), C.byref(n)), "ssd_decode_step_split_plan")
        return p.value, n.value

    def layer_state(self, layer: int):
        out = (C.c_int32 * 4)()
        _check(lib.ssd_cache_layer_state(self._h, layer, C.byref(out)), "ssd_cache_layer_state")
        return tuple(out)

    def layer_budget(self, layer: int):
        """(W, M) of one layer."""
        w, m = C.c_int32(0), C.c_int32(0)
        _check(lib.ssd_cache_layer_budget(self._h, layer, C.byref(w), C.byref(m)), "ssd_cache_layer_budget")
        return w.value, m.value

    def head_budget(self, layer: int, head: int) -> int:
        """W_h of a spatial head, M_h of a semantic head."""
        v = C.c_int32(0)
        _check(lib.ssd_cache_head_budget(self._h, layer, head, C.byref(v)), "ssd_cache_head_budget")
        return v.value

    def head_runs(self, layer: int, head: int):
        """[(start, len), ...] of the valid-slot runs of one head's unit (host arithmetic only)."""
        st, ln = (C.c_int32 * 3)(), (C.c_int32 * 3)()
        _check(lib.ssd_cache_head_runs(self._h, layer, head, st, ln), "ssd_cache_head_runs")
        return [(st[k], ln[k]) for k in range(3) if ln[k] > 0]

    def spatial_slot(self, layer: int, head: int, position: int) -> int:
        v = C.c_int32(0)
        _check(lib.ssd_cache_spatial_slot(self._h, layer, head, position, C.byref(v)), "ssd_cache_spatial_slot")
        return v.value

    def layer_window(self, layer: int) -> int:
        out = C.c_int32(0)
        _check(lib.ssd_cache_layer_window(self._h, layer, C.byref(out)), "ssd_cache_layer_window")
        return out.value

    @property
    def export_slots(self) -> int:
        return lib.ssd_cache_export_slots(self._h)

    def export(self, layer: int, stream=None):
        """(pos int32 [B,H,slots], count int32 [B,H], score float32 [B,H,slots]) on the cache's device."""
        B, H, slots = self.cfg.n_seqs, self.cfg.n_heads, self.export_slots
        dev = self.mem.device
        pos = torch.empty((B, H, slots), dtype=torch.int32, device=dev)
        cnt = torch.empty((B, H), dtype=torch.int32, device=dev)
        sc = torch.empty((B, H, slots), dtype=torch.float32, device=dev)
        _check(lib.ssd_cache_export(self._h, layer, _ptr(pos), _ptr(cnt), _ptr(sc), _stream(stream)), "ssd_cache_export")
        return pos, cnt, sc


def ssd_append_token(cache: Cache, layer_begin: int, layer_end: int, k_new, v_new, stream=None) -> None:
    _check(lib.ssd_append_token(cache.handle, layer_begin, layer_end, _ptr(k_new), _ptr(v_new), _stream(stream)),
           "ssd_append_token")


def ssd_decode_attn(cache: Cache, layer_begin: int, layer_end: int, q, out, accumulate_scores: bool = True,
                    stream=None) -> None:
    _check(lib.ssd_decode_attn(cache.handle, layer_begin, layer_end, _ptr(q), _ptr(out), int(bool(accumulate_scores)),
                               _stream(stream)), "ssd_decode_attn")


def ssd_decode_step(cache: Cache, layer_begin: int, layer_end: int, q, k_new, v_new, out, accumulate_scores: bool = True,
                    compress: bool = True, stream=None) -> None:
    _check(lib.ssd_decode_step(cache.handle, layer_begin, layer_end, _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(out),
                               int(bool(accumulate_scores)), int(bool(compress)), _stream(stream)), "ssd_decode_step")


SSD_MAX_SPLIT = 4
SSD_SPLIT_FORK, SSD_SPLIT_JOIN = 1, 2


def stream_array(streams):
    """ctypes array of raw hipStream_t for ssd_decode_step_split (torch streams or raw handles)."""
    raw = [(s if isinstance(s, int) else s.cuda_stream) for s in streams]
    return (_vp * len(raw))(*raw)


def ssd_decode_step_split(cache: Cache, layer_begin: int, layer_end: int, q, k_new, v_new, out, streams, sync: int = 0,
                          accumulate_scores: bool = True, compress: bool = True) -> None:
    arr = streams if isinstance(streams, C.Array) else stream_array(streams)
    _check(lib.ssd_decode_step_split(cache.handle, layer_begin, layer_end, _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(out),
                                     int(bool(accumulate_scores)), int(bool(compress)), arr, len(arr), int(sync)),
           "ssd_decode_step_split")


SSD_ROPE_HALF, SSD_ROPE_INTERLEAVED = 1, 2


def ssd_decode_step_split_rope(cache: Cache, layer_begin: int, layer_end: int, q, k_new, v_new, out, cos, sin, rope_layout: int,
                               streams, sync: int = 0, accumulate_scores: bool = True, compress: bool = True) -> None:
    arr = streams if isinstance(streams, C.Array) else stream_array(streams)
    _check(lib.ssd_decode_step_split_rope(cache.handle, layer_begin, layer_end, _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(out),
                                          int(bool(accumulate_scores)), int(bool(compress)), _ptr(cos), _ptr(sin), int(rope_layout),
                                          arr, len(arr), int(sync)), "ssd_decode_step_split_rope")


def ssd_decode_step_rope(cache: Cache, layer_begin: int, layer_end: int, q, k_new, v_new, out, cos, sin, rope_layout: int,
                         accumulate_scores: bool = True, compress: bool = True, stream=None) -> None:
    _check(lib.ssd_decode_step_rope(cache.handle, layer_begin, layer_end, _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(out),
                                    int(bool(accumulate_scores)), int(bool(compress)), _ptr(cos), _ptr(sin), int(rope_layout),
                                    _stream(stream)), "ssd_decode_step_rope")


def ssd_compress_kv(cache: Cache, layer_begin: int, layer_end: int, K_src=None, V_src=None, score_src=None,
                    n_src: int = 0, stream=None) -> None:
    _check(lib.ssd_compress_kv(cache.handle, layer_begin, layer_end, _ptr(K_src), _ptr(V_src), _ptr(score_src), int(n_src),
                               _stream(stream)), "ssd_compress_kv")


def ssd_prefill_scores(Q, K, n_units: int, n_src: int, d: int, dtype, score_out, softmax_scale: float = 0.0, stream=None) -> None:
    _check(lib.ssd_prefill_scores(_ptr(Q), _ptr(K), int(n_units), int(n_src), int(d), _dtype_code(dtype), float(softmax_scale),
                                  _ptr(score_out), _stream(stream)), "ssd_prefill_scores")


def ssd_cfg_mix(p, n_seqs: int, V: int, dtype, gamma: float, out, stream=None) -> None:
    _check(lib.ssd_cfg_mix(_ptr(p), int(n_seqs), int(V), _dtype_code(dtype), float(gamma), _ptr(out), _stream(stream)), "ssd_cfg_mix")


def ssd_classify_heads(far, tot, L: int, P: int, H: int, T: int, tau: float, s_out, type_out, stream=None) -> None:
    _check(lib.ssd_classify_heads(_ptr(far), _ptr(tot), L, P, H, T, float(tau), _ptr(s_out), _ptr(type_out),
                                  _stream(stream)), "ssd_classify_heads")


def ssd_dense_workspace_bytes(B: int, H: int, d: int, n: int) -> int:
    return lib.ssd_dense_workspace_bytes(B, H, d, n)


def ssd_dense_decode_attn(q, K, V, out, B: int, H: int, d: int, dtype, n_cap: int, n: int, softmax_scale: float = 0.0,
                          far=None, tot=None, mass_stride: int = 1, vis_start: int = 0, w: int = 32, workspace=None,
                          stream=None, splits: Optional[int] = None) -> None:
    """splits=None: ssd_dense_decode_attn; an integer: the test hook ssd_dense_decode_attn_splits with that many row splits."""
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    if splits is None:
        _check(lib.ssd_dense_decode_attn(_ptr(q), _ptr(K), _ptr(V), _ptr(out), B, H, d, _dtype_code(dtype), n_cap, n,
                                         float(softmax_scale), _ptr(far), _ptr(tot), mass_stride, vis_start, w,
                                         _ptr(workspace), ws_bytes, _stream(stream)), "ssd_dense_decode_attn")
    else:
        _check(lib.ssd_dense_decode_attn_splits(_ptr(q), _ptr(K), _ptr(V), _ptr(out), B, H, d, _dtype_code(dtype), n_cap, n,
                                                float(softmax_scale), _ptr(far), _ptr(tot), mass_stride, vis_start, w,
                                                int(splits), _ptr(workspace), ws_bytes, _stream(stream)),
               "ssd_dense_decode_attn_splits")


SSD_DENSE_STATIC_SCRATCH_BYTES = 8 << 20


def ssd_dense_decode_attn_static(q, K, V, out, B: int, H: int, d: int, dtype, n_cap: int, n: int, softmax_scale: float = 0.0,
                                 far=None, tot=None, mass_stride: int = 1, vis_start: int = 0, w: int = 32, stream=None) -> None:
    _check(lib.ssd_dense_decode_attn_static(_ptr(q), _ptr(K), _ptr(V), _ptr(out), B, H, d, _dtype_code(dtype), n_cap, n,
                                            float(softmax_scale), _ptr(far), _ptr(tot), mass_stride, vis_start, w,
                                            _stream(stream)), "ssd_dense_decode_attn_static")


# ---- serving batches of unequal lengths: the cache in pages, the step's logits ----

SSD_MXFP4, SSD_MXFP8 = 4, 8
_FORMATS = {"mxfp4": SSD_MXFP4, "mxfp8": SSD_MXFP8, SSD_MXFP4: SSD_MXFP4, SSD_MXFP8: SSD_MXFP8}
_INT, _F32 = torch.int32, torch.float32


def _format_code(format) -> int:
    if format not in _FORMATS:
        raise ValueError("format %r: \"mxfp4\" or \"mxfp8\" is expected" % (format,))
    return _FORMATS[format]


class SsdPagedConfig(C.Structure):
    _fields_ = [
        ("n_seqs", C.c_int32), ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32),
        ("page_size", C.c_int32), ("n_pages", C.c_int32), ("max_blocks", C.c_int32), ("softmax_scale", C.c_float),
        ("reserved", C.c_int32 * 3), ("page_stride", C.c_int64), ("head_stride", C.c_int64), ("row_stride", C.c_int64),
        ("q_stride", C.c_int64), ("new_stride", C.c_int64),
    ]

    def __setattr__(self, name, value):
        super().__setattr__(name, value)
        self.__dict__.pop("strides", None)
        self.__dict__.pop("mx_strides", None)

    def __getattr__(self, name):
        """strides: what the config says of the pool, q and new rows as torch says it of tensors [n_pages, n_kv_heads, page_size, d],
        [n_seqs, n_heads, d] and [n_new, n_kv_heads, d]; mx_strides: by a format's name or bits, what the calls on quantised pages expect of their tensors (_mx_call).
        Found when they are first asked for after a field was set."""
        if name == "mx_strides":
            got = self.__dict__[name] = {key: _mx_call(self, bits) for key, bits in _FORMATS.items()}
            return got
        if name != "strides":
            raise AttributeError(name)
        d, row = self.head_dim, self.row_stride or self.head_dim
        head = self.head_stride or row * self.page_size
        got = self.__dict__["strides"] = ((self.page_stride or head * self.n_kv_heads, head, row, 1), (self.q_stride or self.n_heads * d, d, 1),
                                          (self.new_stride or self.n_kv_heads * d, d, 1))
        return got


class SsdLogitsParams(C.Structure):
    _fields_ = [
        ("tokens", _vp), ("n_tokens", _vp), ("n_prompt", _vp), ("repetition", _vp), ("presence", _vp), ("frequency", _vp),
        ("temperature", _vp), ("bias", _vp), ("mask", _vp), ("token_stride", C.c_int64), ("bias_stride", C.c_int64),
        ("mask_stride", C.c_int64),
    ]


_pcfg = C.POINTER(SsdPagedConfig)
lib.ssd_paged_append.argtypes = [_pcfg] + [_vp] * 10 + [C.c_int, _vp, _vp]
lib.ssd_paged_append.restype = C.c_int
lib.ssd_paged_workspace_bytes.argtypes = [_pcfg, C.c_int, C.c_int]
lib.ssd_paged_workspace_bytes.restype = C.c_size_t
lib.ssd_paged_decode_attn.argtypes = [_pcfg] + [_vp] * 9 + [C.c_int, _vp, C.c_size_t, _vp]
lib.ssd_paged_decode_attn.restype = C.c_int
lib.ssd_paged_decode_step.argtypes = [_pcfg] + [_vp] * 13 + [C.c_int, _vp, C.c_size_t, _vp]
lib.ssd_paged_decode_step.restype = C.c_int
lib.ssd_paged_evict_workspace_bytes.argtypes = [_pcfg, C.c_int]
lib.ssd_paged_evict_workspace_bytes.restype = C.c_size_t
lib.ssd_paged_evict.argtypes = [_pcfg] + [_vp] * 6 + [C.c_int, C.c_int] + [_vp] * 5 + [C.c_int, _vp, C.c_size_t, _vp]
lib.ssd_paged_evict.restype = C.c_int
lib.ssd_paged_mx_append.argtypes = [_pcfg, C.c_int] + [_vp] * 12 + [C.c_int, _vp, _vp]
lib.ssd_paged_mx_append.restype = C.c_int
lib.ssd_paged_mx_read.argtypes = [_pcfg, C.c_int] + [_vp] * 7 + [C.c_int] + [_vp] * 4
lib.ssd_paged_mx_read.restype = C.c_int
lib.ssd_paged_mx_workspace_bytes.argtypes = [_pcfg, C.c_int, C.c_int, C.c_int]
lib.ssd_paged_mx_workspace_bytes.restype = C.c_size_t
lib.ssd_paged_mx_decode_attn.argtypes = [_pcfg, C.c_int] + [_vp] * 11 + [C.c_int, _vp, C.c_size_t, _vp]
lib.ssd_paged_mx_decode_attn.restype = C.c_int
lib.ssd_paged_mx_decode_step.argtypes = [_pcfg, C.c_int] + [_vp] * 15 + [C.c_int, _vp, C.c_size_t, _vp]
lib.ssd_paged_mx_decode_step.restype = C.c_int
lib.ssd_paged_mx_evict_workspace_bytes.argtypes = [_pcfg, C.c_int, C.c_int]
lib.ssd_paged_mx_evict_workspace_bytes.restype = C.c_size_t
lib.ssd_paged_mx_evict.argtypes = [_pcfg, C.c_int] + [_vp] * 8 + [C.c_int, C.c_int] + [_vp] * 5 + [C.c_int, _vp, C.c_size_t, _vp]
lib.ssd_paged_mx_evict.restype = C.c_int
lib.ssd_rope_axes.argtypes = [_vp, _vp, C.c_int, C.c_int, C.c_int, C.c_int, C.c_int64, C.c_int64, _vp, C.c_int, _vp, _vp, C.c_int, C.c_int, C.c_int, _vp]
lib.ssd_rope_axes.restype = C.c_int
lib.ssd_logits_process.argtypes = [_vp, C.c_int, C.c_int, C.c_int, C.c_int64, C.c_int, C.c_float, C.POINTER(SsdLogitsParams), _vp,
                                   C.c_int64, _vp]
lib.ssd_logits_process.restype = C.c_int


def make_paged_config(B, H, H_kv, d, dtype, page_size, n_pages, max_blocks, softmax_scale=0.0, page_stride=0, head_stride=0,
                      row_stride=0, q_stride=0, new_stride=0) -> SsdPagedConfig:
    cfg = SsdPagedConfig()
    cfg.n_seqs, cfg.n_heads, cfg.n_kv_heads, cfg.head_dim = B, H, H_kv, d
    cfg.dtype = _dtype_code(dtype)
    cfg.page_size, cfg.n_pages, cfg.max_blocks, cfg.softmax_scale = page_size, n_pages, max_blocks, softmax_scale
    cfg.page_stride, cfg.head_stride, cfg.row_stride = page_stride, head_stride, row_stride
    cfg.q_stride, cfg.new_stride = q_stride, new_stride
    return cfg


def _runs(t):
    """A tensor's dimensions as (size, stride), those of one element left out and neighbours that are one run of memory joined."""
    runs = []
    for size, stride in zip(t.shape, t.stride()):
        if size == 1:
            continue
        if runs and runs[-1][1] == size * stride:
            runs[-1] = (runs[-1][0] * size, stride)
        else:
            runs.append((size, stride))
    if not runs or runs[-1][1] != 1:
        runs.append((1, 1))
    return runs


def _check_rows(t, what: str, n: int, stride: int, width: int) -> None:
    """n rows of `width` elements, `stride` apart: the tensor's own rows, or memory without gaps that reaches as far."""
    runs = _runs(t)
    fits = runs[-1][1] == 1
    if fits and n > 1 and len(runs) == 1:
        fits = (n - 1) * stride + width <= runs[0][0]
        if fits and t.dim() > 1 and t.shape[0] >= n and t.stride(0) >= width:          # rows of its own
            fits = t.stride(0) == stride
    elif fits and n > 0:
        fits = runs[-1][0] >= width and (n == 1 or any(size >= n and apart == stride for size, apart in runs[:-1]))
    if n > 0 and not fits:
        raise ValueError("%s of shape %s, strides %s: %d rows of %d elements that lie %d apart are expected"
                         % (what, tuple(t.shape), t.stride(), n, width, stride))


def _check_pool(t, what: str, cfg) -> None:
    """[n_pages, n_kv_heads, page_size, d] with the config's strides (or the same with page_size before n_kv_heads, as it lies in memory then), or
    memory without gaps that reaches as far."""
    want, sizes = cfg.strides[0], (cfg.n_pages, cfg.n_kv_heads, cfg.page_size, cfg.head_dim)
    named = False
    if t.dim() == 4:
        for order in ((0, 1, 2, 3), (0, 2, 1, 3)):
            if tuple(t.shape[i] for i in order[1:]) == sizes[1:]:
                named = True
                if all(size == 1 or t.stride(i) == stride for i, size, stride in zip(order, sizes, want)):
                    return
    fits = not named
    if fits and t.is_contiguous():
        fits = sum((size - 1) * stride for size, stride in zip(sizes, want)) < t.numel()
    elif fits:
        runs = [(size, stride) for size, stride in zip(t.shape, t.stride()) if size != 1]
        fits = bool(runs) and runs[-1][1] == 1 and all(stride in want for _, stride in runs[:-1])
    if not fits:
        raise ValueError("%s of shape %s, strides %s: the config says [%d, %d, %d, %d] with strides %s" % ((what, tuple(t.shape), t.stride()) + sizes + (want,)))


def _pool(t, what: str, cfg, want) -> Optional[int]:
    """Address of a pool whose strides the config gives: `want`."""
    if type(t) is _Tensor and t.stride() == want:
        return t.data_ptr()
    if t is None or isinstance(t, int):
        return t
    if t.dim() == 4 or not t.is_contiguous() or t.numel() != cfg.n_pages * want[0] or want[0] < want[1] * cfg.n_kv_heads:
        _check_pool(t, what, cfg)                                  # else the memory of the whole pool, in another shape
    return t.data_ptr()


def _rows(t, what: str, n: int, heads: int, want) -> Optional[int]:
    """Address of n rows of `heads` heads; want: the strides of [n, heads, d]."""
    if type(t) is _Tensor and t.stride() == want:
        return t.data_ptr()
    if t is None or isinstance(t, int):
        return t
    width = heads * want[1]
    if t.is_contiguous() and want[0] == width and t.numel() == n * width:          # of any shape
        return t.data_ptr()
    if t.stride() != (want[0], 1) or t.shape[1] < width:
        _check_rows(t, what, n, want[0], width)
    return t.data_ptr()


def _vocabulary_stride(t, what: str, n: int, V: int, stride: int) -> int:
    """How far n rows of V elements lie apart: as the caller says, or where that is 0 as the tensor does."""
    if t.dim() == 2 and t.shape[0] >= n > 1 and t.shape[1] >= V:
        own, one = t.stride()
        if one == 1 and own >= V and stride in (0, own):
            return own
    if stride == 0:
        runs = _runs(t)
        if len(runs) == 1:                                         # memory without gaps: its own rows, if there are as many of them
            stride = t.shape[-1] if t.dim() > 1 and t.shape[-1] >= V and t.numel() >= n * t.shape[-1] else V
        else:
            stride = next((apart for size, apart in reversed(runs[:-1]) if size >= n), V)
    _check_rows(t, what, n, stride, V)
    return max(stride, V)


def _per_row(t, what: str, n: int, width: int, shared: bool) -> int:
    """The stride of an array (without gaps) with a row of `width` elements for each of n rows, or one for all: 0."""
    if t is not None and not isinstance(t, int):
        rows = 1 if shared else n
        own = width if t.dim() < 2 or t.numel() == rows * width else t.shape[-1]
        if own < width or t.numel() < rows * own:
            raise ValueError("%s of shape %s: %d rows of %d elements are expected" % (what, tuple(t.shape), rows, width))
        width = own
    return 0 if shared else width


def _size(t) -> int:
    return 0 if t is None else t.nbytes


def ssd_paged_append(cfg: SsdPagedConfig, k_pages, v_pages, block_table, seq_len, k_new, v_new, pos=None, weight=None, seq_pos=None,
                     new_start=None, n_new: Optional[int] = None, weight_new=None, stream=None) -> None:
    """n_new: tokens in k_new; None: its first dimension."""
    n = int(k_new.shape[0] if n_new is None else n_new)
    pool, _, new = cfg.strides
    heads = cfg.n_kv_heads
    _check(lib.ssd_paged_append(C.byref(cfg), _pool(k_pages, "k_pages", cfg, pool), _pool(v_pages, "v_pages", cfg, pool), _ptr(pos), _ptr(weight),
                                _ptr(block_table), _ptr(seq_len), _ptr(seq_pos), _rows(k_new, "k_new", n, heads, new), _rows(v_new, "v_new", n, heads, new),
                                _ptr(new_start), n, _ptr(weight_new), _stream(stream)), "ssd_paged_append")


def ssd_paged_workspace_bytes(cfg: SsdPagedConfig, max_len: int = 0, with_weights: bool = False) -> int:
    return lib.ssd_paged_workspace_bytes(C.byref(cfg), int(max_len), int(bool(with_weights)))


def ssd_paged_decode_attn(cfg: SsdPagedConfig, q, k_pages, v_pages, block_table, seq_len, out, lse=None, weight_in=None, weight_out=None,
                          max_len: int = 0, workspace=None, stream=None) -> None:
    pool, queries, _ = cfg.strides
    _check(lib.ssd_paged_decode_attn(C.byref(cfg), _rows(q, "q", cfg.n_seqs, cfg.n_heads, queries), _pool(k_pages, "k_pages", cfg, pool),
                                     _pool(v_pages, "v_pages", cfg, pool), _ptr(weight_in), _ptr(weight_out), _ptr(block_table), _ptr(seq_len),
                                     _ptr(out), _ptr(lse), int(max_len), _ptr(workspace), _size(workspace), _stream(stream)), "ssd_paged_decode_attn")


def ssd_paged_decode_step(cfg: SsdPagedConfig, q, k_new, v_new, k_pages, v_pages, block_table, seq_len, out, pos=None, seq_pos=None, lse=None,
                          weight_in=None, weight_out=None, max_len: int = 0, workspace=None, stream=None) -> None:
    (pool, queries, new), B, heads = cfg.strides, cfg.n_seqs, cfg.n_kv_heads
    _check(lib.ssd_paged_decode_step(C.byref(cfg), _rows(q, "q", B, cfg.n_heads, queries), _rows(k_new, "k_new", B, heads, new),
                                     _rows(v_new, "v_new", B, heads, new), _pool(k_pages, "k_pages", cfg, pool), _pool(v_pages, "v_pages", cfg, pool),
                                     _ptr(pos), _ptr(weight_in), _ptr(weight_out), _ptr(block_table), _ptr(seq_len), _ptr(seq_pos), _ptr(out),
                                     _ptr(lse), int(max_len), _ptr(workspace), _size(workspace), _stream(stream)), "ssd_paged_decode_step")


def ssd_paged_evict_workspace_bytes(cfg: SsdPagedConfig, max_len: int = 0) -> int:
    return lib.ssd_paged_evict_workspace_bytes(C.byref(cfg), int(max_len))


def ssd_paged_evict(cfg: SsdPagedConfig, k_pages, v_pages, block_table, seq_len, budget, pos_in, pos_out, weight_in, weight_out, seq_len_out=None,
                    n_sink: int = 0, recent: int = 0, seq_pos=None, max_len: int = 0, workspace=None, stream=None) -> None:
    pool = cfg.strides[0]
    _check(lib.ssd_paged_evict(C.byref(cfg), _pool(k_pages, "k_pages", cfg, pool), _pool(v_pages, "v_pages", cfg, pool), _ptr(block_table), _ptr(seq_len),
                               _ptr(seq_pos), _ptr(budget), int(n_sink), int(recent), _ptr(pos_in), _ptr(pos_out), _ptr(weight_in), _ptr(weight_out), _ptr(seq_len_out),
                               int(max_len), _ptr(workspace), _size(workspace), _stream(stream)), "ssd_paged_evict")


def _mx_call(cfg, bits: int) -> tuple:
    """What the calls on quantised pages expect of their tensors: (strides of a pool in bytes, its sizes [n_pages, n_kv_heads, page_size, bytes of a row], whether it has no gaps,
    bits, bytes of the scales, and for the calls' own arguments (_rows_of q, _rows_of new rows, type of outputs, elements of an output, an lse, a list of sequences,
    the block table and a table of the pool))."""
    n, kv, page, d, B, H = cfg.n_pages, cfg.n_kv_heads, cfg.page_size, cfg.head_dim, cfg.n_seqs, cfg.n_heads
    pool, q, new = cfg.strides
    row, dtype = d * bits // 8, torch.float32 if cfg.dtype == SSD_F32 else torch.bfloat16            # another type is refused by the library
    strides = tuple(s * bits // 8 for s in pool[:3]) + (1,)
    return (strides, (n, kv, page, row), strides == (kv * page * row, page * row, row, 1), bits, n * kv * page * (d // 32),
            (_rows_of(H, d, q, dtype), _rows_of(kv, d, new, dtype), dtype, B * H * d, B * H, B, B * cfg.max_blocks, n * kv * page))


def _rows_of(heads: int, d: int, strides: tuple, dtype) -> tuple:
    """(heads, d, strides of [n, heads, d], type, bytes of a row where rows have no gaps between them, or 0)."""
    return heads, d, strides, dtype, heads * d * dtype.itemsize if strides[0] == heads * d else 0


def _check_mx_pool(t, what: str, want, sizes) -> None:
    if t.element_size() != 1:
        raise ValueError("%s of type %s: a pool of codes is bytes" % (what, t.dtype))
    if tuple(t.shape) == sizes:
        fits = all(size == 1 or stride == w for size, stride, w in zip(sizes, t.stride(), want))
        if not fits and sizes[1] == sizes[2]:                      # which of the two dimensions is which, the strides say
            fits = t.transpose(1, 2).stride() == want
    elif t.dim() == 4 and tuple(t.transpose(1, 2).shape) == sizes:
        fits = all(size == 1 or stride == w for size, stride, w in zip(sizes, t.transpose(1, 2).stride(), want))
    else:
        fits = t.is_contiguous() and sum((size - 1) * w for size, w in zip(sizes, want)) < t.numel()
    if not fits:
        raise ValueError("%s of shape %s, strides %s: the config says bytes [%d, %d, %d, %d] with strides %s" % ((what, tuple(t.shape), t.stride()) + sizes + (want,)))


def _mx_scales(t, what: str, need: int) -> Optional[int]:
    """Address of the scales: `need` bytes without gaps."""
    if type(t) is not _Tensor and (t is None or isinstance(t, int)):
        return t
    if t.nbytes < need or not t.is_contiguous():
        raise ValueError("%s of shape %s, strides %s, type %s: %d bytes without gaps are expected" % (what, tuple(t.shape), t.stride(), t.dtype, need))
    return t.data_ptr()


def _mx_pool(t, what: str, strides, sizes, dense) -> Optional[int]:
    """Address of a pool of codes: bytes [n_pages, n_kv_heads, page_size, d * bits / 8] with the config's strides (or the same with page_size before
    n_kv_heads, as it lies in memory then), or memory without gaps that reaches as far."""
    if type(t) is _Tensor and t.shape == sizes and (t.is_contiguous() if dense else t.stride() == strides) and t.element_size() == 1:
        return t.data_ptr()
    if t is None or isinstance(t, int):
        return t
    _check_mx_pool(t, what, strides, sizes)
    return t.data_ptr()


def _table(t, what: str, n: int, dtype) -> Optional[int]:
    """Address of at least n elements without gaps, of dtype (or whole numbers of its size where it is one of those)."""
    if t is None:
        return None
    if type(t) is _Tensor and t.dtype is dtype and t.numel() >= n and t.is_contiguous():
        return t.data_ptr()
    if isinstance(t, int):
        return t
    if t.dtype is not dtype and (t.element_size() != dtype.itemsize or not _is_whole(t.dtype) or not _is_whole(dtype)):
        raise ValueError("%s of type %s: %s, elements of %d bytes are expected" % (what, t.dtype, dtype, dtype.itemsize))
    if t.numel() < n or not t.is_contiguous():
        raise ValueError("%s of shape %s, strides %s: %d elements without gaps are expected" % (what, tuple(t.shape), t.stride(), n))
    return t.data_ptr()


def _is_whole(dtype) -> bool:
    return not dtype.is_floating_point and not dtype.is_complex


def _mx_rows(t, what: str, n: int, rows) -> Optional[int]:
    """Address of n rows; rows: _rows_of them."""
    heads, d, strides, dtype, dense = rows
    if type(t) is _Tensor and t.dtype is dtype and (t.nbytes == n * dense and t.is_contiguous() if dense else t.stride() == strides and t.shape == (n, heads, d)):
        return t.data_ptr()
    if t is None or isinstance(t, int):
        return t
    if t.dtype is not dtype:
        raise ValueError("%s of type %s: %s, elements of %d bytes are expected" % (what, t.dtype, dtype, dtype.itemsize))
    if t.dim() != 2 or t.stride() != (strides[0], 1) or t.shape[0] < n or t.shape[1] < heads * d:        # else where a projection has them
        _check_rows(t, what, n, strides[0], heads * d)
    return t.data_ptr()


def _mx_pools(cfg, format, k_pages, v_pages, k_scales, v_scales):
    """The format's code, and the addresses of two pools of codes and their scales."""
    strides, sizes, dense, bits, scales, _ = cfg.mx_strides.get(format) or _format_code(format)
    return (bits, _mx_pool(k_pages, "k_pages", strides, sizes, dense), _mx_pool(v_pages, "v_pages", strides, sizes, dense), _mx_scales(k_scales, "k_scales", scales),
            _mx_scales(v_scales, "v_scales", scales))


def ssd_paged_mx_append(cfg: SsdPagedConfig, format, k_pages, v_pages, k_scales, v_scales, block_table, seq_len, k_new, v_new, pos=None, weight=None,
                        seq_pos=None, new_start=None, n_new: Optional[int] = None, weight_new=None, stream=None) -> None:
    """format: "mxfp4" or "mxfp8" (SSD_MXFP4, SSD_MXFP8).  n_new: tokens in k_new; None: its first dimension."""
    n = int(k_new.shape[0] if n_new is None else n_new)
    bits, k, v, ks, vs = _mx_pools(cfg, format, k_pages, v_pages, k_scales, v_scales)
    _, new, _, _, _, seqs, blocks, places = cfg.mx_strides[bits][5]
    _check(lib.ssd_paged_mx_append(C.byref(cfg), bits, k, v, ks, vs, _table(pos, "pos", places, _INT), _table(weight, "weight", places, _F32),
                                   _table(block_table, "block_table", blocks, _INT), _table(seq_len, "seq_len", seqs, _INT), _table(seq_pos, "seq_pos", seqs, _INT),
                                   _mx_rows(k_new, "k_new", n, new), _mx_rows(v_new, "v_new", n, new), _table(new_start, "new_start", seqs + 1, _INT), n,
                                   _table(weight_new, "weight_new", n * new[0], _F32), _stream(stream)), "ssd_paged_mx_append")


def ssd_paged_mx_read(cfg: SsdPagedConfig, format, k_pages, v_pages, k_scales, v_scales, block_table, seq_len, k_out, v_out, row_start=None,
                      first_slot=None, n_rows: Optional[int] = None, stream=None) -> None:
    """n_rows: rows of k_out; None: its first dimension."""
    n = int(k_out.shape[0] if n_rows is None else n_rows)
    bits, k, v, ks, vs = _mx_pools(cfg, format, k_pages, v_pages, k_scales, v_scales)
    _, new, _, _, _, seqs, blocks, _ = cfg.mx_strides[bits][5]
    _check(lib.ssd_paged_mx_read(C.byref(cfg), bits, k, v, ks, vs, _table(block_table, "block_table", blocks, _INT), _table(seq_len, "seq_len", seqs, _INT),
                                 _table(row_start, "row_start", seqs + 1, _INT), n, _table(first_slot, "first_slot", seqs, _INT), _mx_rows(k_out, "k_out", n, new),
                                 _mx_rows(v_out, "v_out", n, new), _stream(stream)), "ssd_paged_mx_read")


def ssd_paged_mx_workspace_bytes(cfg: SsdPagedConfig, format, max_len: int = 0, with_weights: bool = False) -> int:
    return lib.ssd_paged_mx_workspace_bytes(C.byref(cfg), _format_code(format), int(max_len), int(bool(with_weights)))


def ssd_paged_mx_decode_attn(cfg: SsdPagedConfig, format, q, k_pages, v_pages, k_scales, v_scales, block_table, seq_len, out, lse=None, weight_in=None,
                             weight_out=None, max_len: int = 0, workspace=None, stream=None) -> None:
    bits, k, v, ks, vs = _mx_pools(cfg, format, k_pages, v_pages, k_scales, v_scales)
    queries, _, dtype, size, heads, seqs, blocks, places = cfg.mx_strides[bits][5]
    _check(lib.ssd_paged_mx_decode_attn(C.byref(cfg), bits, _mx_rows(q, "q", seqs, queries), k, v, ks, vs,
                                        _table(weight_in, "weight_in", places, _F32), _table(weight_out, "weight_out", places, _F32),
                                        _table(block_table, "block_table", blocks, _INT), _table(seq_len, "seq_len", seqs, _INT), _table(out, "out", size, dtype),
                                        _table(lse, "lse", heads, _F32), int(max_len), _ptr(workspace), _size(workspace), _stream(stream)), "ssd_paged_mx_decode_attn")


def ssd_paged_mx_decode_step(cfg: SsdPagedConfig, format, q, k_new, v_new, k_pages, v_pages, k_scales, v_scales, block_table, seq_len, out, pos=None,
                             seq_pos=None, lse=None, weight_in=None, weight_out=None, max_len: int = 0, workspace=None, stream=None) -> None:
    bits, k, v, ks, vs = _mx_pools(cfg, format, k_pages, v_pages, k_scales, v_scales)
    queries, new, dtype, size, heads, n, blocks, places = cfg.mx_strides[bits][5]
    _check(lib.ssd_paged_mx_decode_step(C.byref(cfg), bits, _mx_rows(q, "q", n, queries), _mx_rows(k_new, "k_new", n, new),
                                        _mx_rows(v_new, "v_new", n, new), k, v, ks, vs, _table(pos, "pos", places, _INT), _table(weight_in, "weight_in", places, _F32),
                                        _table(weight_out, "weight_out", places, _F32), _table(block_table, "block_table", blocks, _INT),
                                        _table(seq_len, "seq_len", n, _INT), _table(seq_pos, "seq_pos", n, _INT), _table(out, "out", size, dtype),
                                        _table(lse, "lse", heads, _F32), int(max_len), _ptr(workspace), _size(workspace), _stream(stream)), "ssd_paged_mx_decode_step")


def ssd_paged_mx_evict_workspace_bytes(cfg: SsdPagedConfig, format, max_len: int = 0) -> int:
    return lib.ssd_paged_mx_evict_workspace_bytes(C.byref(cfg), _format_code(format), int(max_len))


def ssd_paged_mx_evict(cfg: SsdPagedConfig, format, k_pages, v_pages, k_scales, v_scales, block_table, seq_len, budget, pos_in, pos_out, weight_in,
                       weight_out, seq_len_out=None, n_sink: int = 0, recent: int = 0, seq_pos=None, max_len: int = 0, workspace=None, stream=None) -> None:
    bits, k, v, ks, vs = _mx_pools(cfg, format, k_pages, v_pages, k_scales, v_scales)
    _, _, _, _, _, seqs, blocks, places = cfg.mx_strides[bits][5]
    _check(lib.ssd_paged_mx_evict(C.byref(cfg), bits, k, v, ks, vs, _table(block_table, "block_table", blocks, _INT), _table(seq_len, "seq_len", seqs, _INT),
                                  _table(seq_pos, "seq_pos", seqs, _INT), _table(budget, "budget", seqs, _INT), int(n_sink), int(recent),
                                  _table(pos_in, "pos_in", places, _INT), _table(pos_out, "pos_out", places, _INT), _table(weight_in, "weight_in", places, _F32),
                                  _table(weight_out, "weight_out", places, _F32), _table(seq_len_out, "seq_len_out", seqs, _INT), int(max_len), _ptr(workspace),
                                  _size(workspace), _stream(stream)), "ssd_paged_mx_evict")


def ssd_rope_axes(x, out, n_rows: int, n_heads: int, head_dim: int, dtype, pos, inv_freq, axis=None, n_axes: int = 1, n_pairs: Optional[int] = None,
                  layout: int = SSD_ROPE_HALF, inverse: bool = False, x_stride: int = 0, out_stride: int = 0, stream=None) -> None:
    """n_pairs None: inv_freq's elements.  x_stride, out_stride 0: the tensor's own (query and key heads may be handed over where a projection has them)."""
    rows, code = [], _dtype_code(dtype)
    held = torch.float32 if code == SSD_F32 else torch.bfloat16      # another code is refused by the library
    for t, what, stride in ((x, "x", x_stride), (out, "out", out_stride)):
        if t is not None and not isinstance(t, int):
            if t.dtype is not held:
                raise ValueError("%s of type %s: %s, elements of %d bytes are expected" % (what, t.dtype, held, held.itemsize))
            own = t.stride()
            if len(own) == 3 and own[1] == head_dim and own[2] == 1 and own[0] > 0 and t.shape == (n_rows, n_heads, head_dim) and stride in (0, own[0]):
                stride = own[0] if n_rows > 1 else 0
            else:
                stride = stride or (own[0] if len(own) > 1 and t.shape[0] == n_rows > 1 else 0)
                _check_rows(t, what, n_rows, stride or n_heads * head_dim, n_heads * head_dim)
            t = t.data_ptr()
        rows += [t, stride]
    x, x_stride, out, out_stride = rows
    pairs = int(inv_freq.numel() if n_pairs is None else n_pairs)
    _check(lib.ssd_rope_axes(x, out, int(n_rows), int(n_heads), int(head_dim), code, int(x_stride), int(out_stride),
                             _table(pos, "pos", n_axes * n_rows, _INT), int(n_axes), _table(axis, "axis", pairs, torch.uint8),
                             _table(inv_freq, "inv_freq", pairs, _F32), pairs, int(layout), int(bool(inverse)), _stream(stream)), "ssd_rope_axes")


def ssd_logits_process(logits, n_rows: int, V: int, dtype, out, gamma: Optional[float] = None, tokens=None, n_tokens=None, n_prompt=None,
                       repetition=None, presence=None, frequency=None, temperature=None, bias=None, bias_shared: bool = False, mask=None,
                       mask_shared: bool = False, logits_stride: int = 0, out_stride: int = 0, token_stride: Optional[int] = None,
                       stream=None) -> None:
    """gamma: guidance strength, None: no guidance.  bias [n_rows, V] and mask [n_rows, ceil(V / 32)], or one row of either for all
    (bias_shared, mask_shared).  token_stride: places per row of tokens, None: its last dimension.  logits_stride, out_stride 0: the tensor's own (a view of
    a padded vocabulary may be handed over as it is)."""
    p = SsdLogitsParams()
    p.tokens, p.n_tokens, p.n_prompt = _ptr(tokens), _ptr(n_tokens), _ptr(n_prompt)
    p.repetition, p.presence, p.frequency, p.temperature = _ptr(repetition), _ptr(presence), _ptr(frequency), _ptr(temperature)
    p.bias, p.mask = _ptr(bias), _ptr(mask)
    p.token_stride = int((0 if tokens is None else tokens.shape[-1]) if token_stride is None else token_stride)
    p.bias_stride = _per_row(bias, "bias", n_rows, int(V), bias_shared)
    p.mask_stride = _per_row(mask, "mask", n_rows, -(-int(V) // 32), mask_shared)
    if logits is not None and not isinstance(logits, int):
        n = n_rows if gamma is None else 2 * n_rows
        if logits_stride or logits.numel() != n * V or not logits.is_contiguous():
            logits_stride = _vocabulary_stride(logits, "logits", n, V, logits_stride)
        logits = logits.data_ptr()
    if out is not None and not isinstance(out, int):
        if out_stride or out.numel() != n_rows * V or not out.is_contiguous():
            out_stride = _vocabulary_stride(out, "out", n_rows, V, out_stride)
        out = out.data_ptr()
    _check(lib.ssd_logits_process(logits, int(n_rows), int(V), _dtype_code(dtype), int(logits_stride), int(gamma is not None),
                                  float(gamma or 0.0), C.byref(p), out, int(out_stride), _stream(stream)), "ssd_logits_process")
