"""Thin ctypes binding of libf3dc.so (declared in include/f3dc.h).

Argument marshalling only: every step of the cached denoising step runs in
the library's CUDA kernels.  Device buffers are torch CUDA tensors (passed by
data pointer); host buffers are NumPy arrays.  If the library has not been
built, loading raises -- there is no CPU fallback.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
import re
import threading

import numpy as np

from . import build as _build

F3DC_OK = 0
STATUS_NAMES = {0: "OK", 1: "INVALID_ARG", 2: "CUDA", 3: "OOM", 4: "UNSUPPORTED", 5: "TIMEOUT",
                6: "NONFINITE", 7: "DEVICE"}
REFRESH_PERIOD, REFRESH_LITERAL = 0, 1
EPI_BIAS, EPI_GELU, EPI_RESID = 0, 1, 2
NORM_NONE, NORM_LAYER, NORM_RMS = 0, 1, 2
HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "f3dc.h")


class F3dcError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"f3dc status {STATUS_NAMES.get(status, status)}: {msg}")
        self.status = status


class Config(C.Structure):
    _fields_ = [("grid", C.c_int32), ("channels", C.c_int32), ("width", C.c_int32), ("blocks", C.c_int32),
                ("heads", C.c_int32), ("mlp_ratio", C.c_int32), ("cond_tokens", C.c_int32),
                ("cond_dim", C.c_int32), ("steps", C.c_int32), ("max_batch", C.c_int32),
                ("gamma_up", C.c_int32), ("tau", C.c_int32), ("f_corr", C.c_int32),
                ("refresh_mode", C.c_int32), ("eta", C.c_double), ("rho_a", C.c_double), ("mu", C.c_double),
                ("omega", C.c_double), ("xi", C.c_double), ("rho_cfg_off", C.c_double),
                ("cfg_strength", C.c_double), ("cfg_t_lo", C.c_double), ("ssc_accel", C.c_int32),
                ("decoder", C.c_int32)]


class KernelStats(C.Structure):
    _fields_ = [("name", C.c_char * 24), ("launches", C.c_int64), ("total_ms", C.c_double),
                ("flops", C.c_double), ("bytes", C.c_double)]


class Weights(C.Structure):
    _fields_ = [("layout_version", C.c_int32), ("blob", C.c_void_p), ("blob_elems", C.c_size_t)]


class FaultInjection(C.Structure):
    _fields_ = [("fail_alloc_at", C.c_int32), ("gemm_missing_arrivals", C.c_int32), ("gemm_wait_ns", C.c_int64),
                ("attn_missing_kv", C.c_int32)]


class NormLayer(C.Structure):
    """The constant part of a norm_residual call; keeps its tensors (bf16
    [width], as everywhere also as 16-bit integers, or None) alive."""
    _fields_ = [("width", C.c_int32), ("post", C.c_int32), ("pre", C.c_int32), ("eps", C.c_float),
                ("res_scale", C.c_float), ("post_g", C.c_void_p), ("post_b", C.c_void_p), ("pre_g", C.c_void_p),
                ("pre_b", C.c_void_p)]

    def __init__(self, width, post=NORM_NONE, pre=NORM_LAYER, post_g=None, post_b=None, pre_g=None, pre_b=None,
                 eps=1e-6, res_scale=1.0):
        self._tensors = tuple(t for t in (post_g, post_b, pre_g, pre_b) if t is not None)
        for t in self._tensors:
            if not t.is_cuda or t.dtype not in _fp8_types()["bf16"] or t.numel() < width or not t.is_contiguous():
                raise F3dcError(1, f"gains and biases are bf16 [{width}] on a GPU: got {t.dtype} {tuple(t.shape)} on {t.device}")
        super().__init__(width, post, pre, eps, res_scale, _ptr(post_g), _ptr(post_b), _ptr(pre_g), _ptr(pre_b))
        self._ref = C.pointer(self)


class Rotary(C.Structure):
    """Rotation by positions: `inv_freq` are the dims / 2 pairs' angles per unit of
    position (or base ** (-j / pairs of an axis) for each axis).  Keeps their turns
    on the given (or current) GPU."""
    _fields_ = [("dims", C.c_int32), ("interleaved", C.c_int32), ("axes", C.c_int32), ("turns", C.c_void_p)]

    def __init__(self, dims, inv_freq=None, base=10000.0, interleaved=False, axes=1, device="cuda"):
        import torch
        n = dims // 2
        if inv_freq is None:
            of_axis = max(1, n // max(1, axes))
            inv_freq = [base ** (-(j % of_axis) / of_axis) for j in range(n)]
        if len(inv_freq) != n:
            raise F3dcError(1, f"{dims} rotating elements have {n} frequencies: got {len(inv_freq)}")
        self.host = rotary_turns(inv_freq)
        self._turns = torch.from_numpy(self.host.view(np.int64)).to(device)
        super().__init__(dims, int(interleaved), axes, self._turns.data_ptr())
        self._ref = C.pointer(self)


def _same_device(what, tensors):
    for t in tensors:
        if not t.is_cuda or t.get_device() != tensors[0].get_device():
            raise F3dcError(1, f"{what}: tensors on one GPU are needed, got one on {t.device}")


class KVCache(C.Structure):
    """A pool of pages of 8-bit keys and values, as four tensors (kept alive): k and v
    e4m3 [pages, kv_heads, page_tokens, dh] (bytes; pages may lie apart), their scales
    bytes [pages, kv_heads]."""
    _fields_ = [("pages", C.c_int32), ("page_tokens", C.c_int32), ("kv_heads", C.c_int32), ("dh", C.c_int32),
                ("k", C.c_void_p), ("v", C.c_void_p), ("k_scales", C.c_void_p), ("v_scales", C.c_void_p),
                ("page_stride", C.c_int64), ("scale_stride", C.c_int64)]

    def __init__(self, k, v, k_scales, v_scales):
        self._tensors = (k, v, k_scales, v_scales)
        kinds = _fp8_types()
        for t, n, kind in zip(self._tensors, (4, 4, 2, 2), ("e4m3", "e4m3", "scale", "scale")):
            if t.dtype not in kinds[kind] or t.dim() != n:
                raise F3dcError(1, f"a cache holds {kind} bytes in {n} dimensions: got {t.dtype} {tuple(t.shape)}")
        pages, heads, tokens, dh = k.shape
        if v.shape != k.shape or tuple(k_scales.shape) != (pages, heads) or k_scales.shape != v_scales.shape:
            raise F3dcError(1, "k and v need one shape [pages, kv_heads, page_tokens, dh], their scales [pages, kv_heads]")
        # (the stride of a dimension of one says nothing)
        page_stride, scale_stride = (k.stride(0), k_scales.stride(0)) if pages > 1 else (heads * tokens * dh, heads)
        for t in (k, v):
            want = (page_stride, tokens * dh, dh, 1)
            if any(n > 1 and a != b for n, a, b in zip(t.shape, t.stride(), want)):
                raise F3dcError(1, "a page's bytes must lie together, pages of k and v equally far apart")
        for t in (k_scales, v_scales):
            if any(n > 1 and a != b for n, a, b in zip(t.shape, t.stride(), (scale_stride, 1))):
                raise F3dcError(1, "a page's scales must lie together, pages of k_scales and v_scales equally far apart")
        _same_device("cache", self._tensors)
        super().__init__(pages, tokens, heads, dh, *(t.data_ptr() for t in self._tensors), page_stride, scale_stride)
        self._ref = C.pointer(self)


class KVBatch(C.Structure):
    """The sequences of a call: row_start int32 [batch + 1], lengths int32 [batch] (with the
    call's rows) and page_table int32 [batch, pages] on the GPU, kept alive; `rows` packed rows, and
    bounds on a sequence's rows and length.  A table may be a view of a wider one: a sequence longer than the
    view's columns hold is out of bounds."""
    _fields_ = [("row_start", C.c_void_p), ("lengths", C.c_void_p), ("page_table", C.c_void_p), ("table_stride", C.c_int64),
                ("batch", C.c_int32), ("rows", C.c_int32), ("max_rows", C.c_int32), ("max_length", C.c_int32)]

    def __init__(self, row_start, lengths, page_table, rows, max_rows, max_length):
        self._tensors = (row_start, lengths, page_table)
        for t, n in zip(self._tensors, (1, 1, 2)):
            if t.dtype not in _fp8_types()["int32"] or t.dim() != n or (t.shape[-1] > 1 and t.stride(n - 1) != 1):
                raise F3dcError(1, f"row_start, lengths and page_table are int32 with neighbouring entries: got {t.dtype} {tuple(t.shape)}")
        batch = lengths.shape[0]
        if row_start.shape[0] != batch + 1 or page_table.shape[0] != batch:
            raise F3dcError(1, "row_start needs batch + 1 entries, page_table a row for each sequence")
        if batch > 1 and page_table.stride(0) < page_table.shape[1]:
            raise F3dcError(1, "rows of page_table overlap")
        _same_device("batch", self._tensors)
        # (a single row's stride may be anything, and that of rows without columns)
        columns = page_table.shape[1]
        stride = page_table.stride(0) if batch > 1 and columns else columns
        super().__init__(row_start.data_ptr(), lengths.data_ptr(), page_table.data_ptr(), stride, batch, rows, max_rows, max_length)
        self._ref = C.pointer(self)
        self._columns = columns if columns < stride else None

    def _for(self, cache):
        """The structure for calls with `cache`: to the library a row of the table has as many pages as its stride, so
        the bound on lengths is no larger than what a view's columns hold."""
        if self._columns is None or self.max_length <= self._columns * cache.page_tokens:
            return self._ref
        bounded = KVBatch.from_buffer_copy(self)
        bounded.max_length = self._columns * cache.page_tokens
        return C.pointer(bounded)


_lock = threading.Lock()
_lib = None
_i64 = C.c_int64
_vp, _i32p, _f32p, _f64p, _u32p = C.c_void_p, C.POINTER(C.c_int32), C.POINTER(C.c_float), C.POINTER(
    C.c_double), C.POINTER(C.c_uint32)


def library_path() -> str:
    return _build.LIB


def lib():
    """Loads libf3dc.so (building it first if the sources are newer)."""
    global _lib
    if _lib is not None:  # set once, complete
        return _lib
    with _lock:
        if _lib is None:
            path = _build.build()
            if not os.path.exists(path):
                raise RuntimeError(f"libf3dc.so missing at {path}")
            L = C.CDLL(path)
            cfgp, wp = C.POINTER(Config), C.POINTER(Weights)
            sig = {
                "f3dc_config_default": ([cfgp], C.c_int),
                "f3dc_weights_elems": ([cfgp], C.c_size_t),
                "f3dc_time_schedule": ([cfgp, _f32p], C.c_int),
                "f3dc_pcsc_quota": ([cfgp, C.c_double, C.c_int32, _i32p, _i32p, _i32p], C.c_int),
                "f3dc_create": ([cfgp, wp, _vp, C.POINTER(_vp)], C.c_int),
                "f3dc_destroy": ([_vp], C.c_int),
                "f3dc_last_error": ([_vp], C.c_char_p),
                "f3dc_device_status": ([_vp, _u32p], C.c_int),
                "f3dc_ssc_select": ([_vp, _vp, _vp, C.c_int32, _vp, _vp, _vp, _vp, _vp], C.c_int),
                "f3dc_set_cond": ([_vp, _vp, C.c_int32, _vp], C.c_int),
                "f3dc_step": ([_vp, C.c_int32, C.c_int32, _vp, _vp, _vp, _vp, _vp], C.c_int),
                "f3dc_sample": ([_vp, _vp, _vp, C.c_int32, _f64p, _i32p, _i32p, _f64p, _vp], C.c_int),
                "f3dc_dynamic_voxel_curve": ([_vp, _vp, _vp, C.c_int32, C.POINTER(C.c_int64), _vp], C.c_int),
                "f3dc_fit_mu": ([_f64p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_double, C.c_double,
                                 _f64p, _f64p, _i32p], C.c_int),
                "f3dc_forward": ([_vp, C.c_float, C.c_int32, _vp, _vp, _vp, _vp, _vp], C.c_int),
                "f3dc_profile": ([_vp, C.c_int32], C.c_int),
                "f3dc_profile_read": ([_vp, C.POINTER(KernelStats), C.c_int32, _i32p], C.c_int),
                "f3dc_launch_count": ([_vp, C.POINTER(C.c_int64)], C.c_int),
                "f3dc_set_graphs": ([_vp, C.c_int32], C.c_int),
                "f3dc_gemm": ([_vp, _vp, _vp, _vp, _vp, C.c_int32, C.c_int32, C.c_int32, C.c_int32, _vp], C.c_int),
                "f3dc_gemm_noalloc": ([_vp, _vp, _vp, _vp, _vp, C.c_int32, C.c_int32, C.c_int32, C.c_int32, _vp],
                                      C.c_int),
                "f3dc_gemm_status": ([_u32p], C.c_int),
                "f3dc_set_fault_injection": ([C.POINTER(FaultInjection)], C.c_int),
                "f3dc_attention": ([_vp, C.c_int32, _vp, _vp, C.c_int32, _vp, C.c_int32, C.c_int32, C.c_int32,
                                    C.c_int32, _vp], C.c_int),
                "f3dc_quantize_fp8": ([_vp, C.c_int32, _i64, _vp, _i64, _vp, _i64, C.c_int32, C.c_int32, _vp], C.c_int),
                "f3dc_gemm_fp8": ([_vp, _i64] * 4 + [_vp, _vp] + [_vp, _i64] * 2 + [C.c_int32] * 4 + [_vp], C.c_int),
                "f3dc_norm_residual": ([C.POINTER(NormLayer), _vp, _i64, _vp, _i64, _vp, _i64, _vp, _vp, _vp, _i64, _vp,
                                        C.c_int32, _vp, _i64, _vp, _i64, C.c_int32, _vp], C.c_int),
                "f3dc_rotary_turns": ([_f64p, C.c_int32, C.POINTER(C.c_uint64)], C.c_int),
                "f3dc_kv_append_fp8": ([C.POINTER(KVCache), C.POINTER(KVBatch), C.POINTER(Rotary)] + [_vp, _i64] * 4 +
                                       [C.c_int32, _vp, _vp], C.c_int),
                "f3dc_kv_attention_workspace": ([C.POINTER(KVCache), C.POINTER(KVBatch), C.c_int32], C.c_size_t),
                "f3dc_kv_attention_fp8": ([C.POINTER(KVCache), C.POINTER(KVBatch)] + [_vp, _i64] * 2 +
                                          [_vp, C.c_int32, C.c_float, C.c_int32, _vp, C.c_size_t, _vp], C.c_int),
            }
            for name, (args, res) in sig.items():
                fn = getattr(L, name)
                fn.argtypes = args
                fn.restype = res
            _lib = L
    return _lib


def declared_symbols():
    """Names of the functions include/f3dc.h declares."""
    with open(HEADER) as f:
        text = f.read()
    return sorted(set(re.findall(r"\b(f3dc_\w+)\s*\(", text)))


def _check(status, handle=None):
    if status != F3DC_OK:
        msg = lib().f3dc_last_error(handle)
        raise F3dcError(status, msg.decode() if msg else "")


# Pointer arguments are plain integers (the functions' argtypes convert them):
# a small call is bound by this marshalling, not by its kernel.
def _ptr(t):
    return None if t is None else t.data_ptr()


_current_raw_stream = None


def _stream(stream):
    """The given stream, or the current one of the current device (its handle
    alone: torch.cuda.current_stream() builds a Stream object per call)."""
    global _current_raw_stream
    if stream is not None:
        return stream
    if _current_raw_stream is None:
        import torch
        torch.cuda.init()
        get_stream, get_device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
        # (of the only device there is without asking which one is current)
        _current_raw_stream = functools.partial(get_stream, 0) if torch.cuda.device_count() == 1 else lambda: get_stream(get_device())
    return _current_raw_stream()


def _np_ptr(a, typ):
    return None if a is None else a.ctypes.data_as(typ)


# ---------------------------------------------------------------- host calls

def default_config() -> Config:
    c = Config()
    _check(lib().f3dc_config_default(C.byref(c)))
    return c


def config_for(shape, max_batch: int = 1, **hyper) -> Config:
    """Config for a synth.ModelShape; keyword arguments override fields."""
    c = default_config()
    c.grid, c.channels, c.width, c.blocks = shape.grid, shape.channels, shape.width, shape.blocks
    c.heads, c.mlp_ratio, c.cond_tokens, c.cond_dim = shape.heads, shape.mlp_ratio, shape.cond_tokens, shape.cond_dim
    c.steps, c.gamma_up, c.max_batch = shape.steps, shape.gamma_up, max_batch
    for k, v in hyper.items():
        setattr(c, k, v)
    return c


def weights_elems(cfg: Config) -> int:
    return int(lib().f3dc_weights_elems(C.byref(cfg)))


def time_schedule(cfg: Config) -> np.ndarray:
    out = np.empty(cfg.steps + 1, np.float32)
    _check(lib().f3dc_time_schedule(C.byref(cfg), out.ctypes.data_as(_f32p)))
    return out


def pcsc_quota(cfg: Config, sigma: float, k: int, consec=None):
    """Returns (quota, phase); consec is a one-element int32 array updated in
    place when the tau rule should apply."""
    q, ph = C.c_int32(0), C.c_int32(0)
    cp = consec.ctypes.data_as(_i32p) if consec is not None else None
    _check(lib().f3dc_pcsc_quota(C.byref(cfg), float(sigma), int(k), cp, C.byref(q), C.byref(ph)))
    return q.value, ph.value


# ---------------------------------------------------------------- handle

class Handle:
    """Owns an f3dc_handle.  `blob` is a CUDA tensor of the layout-v2 bf16
    weights (any 16-bit dtype); it may be freed after construction."""

    def __init__(self, cfg: Config, blob, stream=None):
        self.cfg = cfg
        self.h = C.c_void_p()
        w = Weights(2, blob.data_ptr(), blob.numel())
        _check(lib().f3dc_create(C.byref(cfg), C.byref(w), _stream(stream), C.byref(self.h)))

    def close(self):
        if self.h:
            lib().f3dc_destroy(self.h)
            self.h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _ck(self, st):
        _check(st, self.h)

    def device_status(self) -> int:
        v = C.c_uint32(0)
        self._ck(lib().f3dc_device_status(self.h, C.byref(v)))
        return v.value

    def ssc_select(self, v_prev1, v_prev2, B, quota_dev, active_idx_out, n_active_out, cached_mask_out=None,
                   stream=None):
        self._ck(lib().f3dc_ssc_select(self.h, _ptr(v_prev1), _ptr(v_prev2), B, _ptr(quota_dev),
                                       _ptr(active_idx_out), _ptr(n_active_out), _ptr(cached_mask_out),
                                       _stream(stream)))

    def set_cond(self, cond, B, stream=None):
        self._ck(lib().f3dc_set_cond(self.h, _ptr(cond), B, _stream(stream)))

    def step(self, k, B, S, ring, quota_dev, dyn_voxels=None, stream=None):
        self._ck(lib().f3dc_step(self.h, k, B, _ptr(S), _ptr(ring), _ptr(quota_dev), _ptr(dyn_voxels),
                                 _stream(stream)))

    def sample(self, S, cond, B, sigma_override=None, quota_schedule=None, want_log=True, stream=None):
        """Algorithm 1 in place on S; returns (quota_log [T, B], sigma [B]) or
        (None, None) when want_log is False (no host synchronisation)."""
        T = self.cfg.steps
        so = None if sigma_override is None else np.ascontiguousarray(sigma_override, np.float64)
        qs = None if quota_schedule is None else np.ascontiguousarray(quota_schedule, np.int32)
        ql = np.zeros((T, B), np.int32) if want_log else None
        sg = np.zeros(B, np.float64) if want_log else None
        self._ck(lib().f3dc_sample(self.h, _ptr(S), _ptr(cond), B, _np_ptr(so, _f64p), _np_ptr(qs, _i32p),
                                   _np_ptr(ql, _i32p), _np_ptr(sg, _f64p), _stream(stream)))
        return ql, sg

    def dynamic_voxel_curve(self, S, cond, B, stream=None) -> np.ndarray:
        """Eq. 1's dS at every step of an uncached sampler run: int64 [T, B]."""
        out = np.zeros((self.cfg.steps, B), np.int64)
        self._ck(lib().f3dc_dynamic_voxel_curve(self.h, _ptr(S), _ptr(cond), B,
                                                out.ctypes.data_as(C.POINTER(C.c_int64)), _stream(stream)))
        return out

    def profile(self, enable: bool):
        self._ck(lib().f3dc_profile(self.h, 1 if enable else 0))

    def profile_read(self):
        arr = (KernelStats * 32)()
        n = C.c_int32(0)
        self._ck(lib().f3dc_profile_read(self.h, arr, 32, C.byref(n)))
        return [{"name": arr[i].name.decode(), "launches": arr[i].launches, "total_ms": arr[i].total_ms,
                 "flops": arr[i].flops, "bytes": arr[i].bytes} for i in range(min(n.value, 32))]

    def set_graphs(self, enable: bool):
        self._ck(lib().f3dc_set_graphs(self.h, 1 if enable else 0))

    def launch_count(self) -> int:
        n = C.c_int64(0)
        self._ck(lib().f3dc_launch_count(self.h, C.byref(n)))
        return n.value

    def forward(self, t, B, S, active_idx, n_active, v_out, stream=None):
        self._ck(lib().f3dc_forward(self.h, float(t), B, _ptr(S), _ptr(active_idx), _ptr(n_active), _ptr(v_out),
                                    _stream(stream)))


# ---------------------------------------------------------------- kernels

def fit_mu(curves, k_lo=8, k_hi=18, tol=0.1, min_frac=0.6):
    """Data-driven PCSC slope from dS curves [n, T]: (mu, slopes [n], kept [n] bool)."""
    c = np.ascontiguousarray(curves, np.float64)
    n, T = c.shape
    mu = C.c_double(0.0)
    slopes = np.empty(n, np.float64)
    kept = np.empty(n, np.int32)
    _check(lib().f3dc_fit_mu(c.ctypes.data_as(_f64p), n, T, k_lo, k_hi, tol, min_frac, C.byref(mu),
                             slopes.ctypes.data_as(_f64p), kept.ctypes.data_as(_i32p)))
    return mu.value, slopes, kept.astype(bool)


def gemm(A, Bw, bias, gate, out, M, N, K, epilogue, stream=None):
    _check(lib().f3dc_gemm(_ptr(A), _ptr(Bw), _ptr(bias), _ptr(gate), _ptr(out), M, N, K, epilogue,
                           _stream(stream)))


def gemm_noalloc(A, Bw, bias, gate, out, M, N, K, epilogue, stream=None):
    """f3dc_gemm without any allocation (split-K scratch in a static array)."""
    _check(lib().f3dc_gemm_noalloc(_ptr(A), _ptr(Bw), _ptr(bias), _ptr(gate), _ptr(out), M, N, K, epilogue,
                                   _stream(stream)))


def set_fault_injection(fail_alloc_at=-1, gemm_missing_arrivals=0, gemm_wait_ns=0, attn_missing_kv=0):
    """Test-only, host-side fault injection (see f3dc_set_fault_injection);
    called with no arguments it turns everything off."""
    fi = FaultInjection(fail_alloc_at, gemm_missing_arrivals, gemm_wait_ns, attn_missing_kv)
    _check(lib().f3dc_set_fault_injection(C.byref(fi)))


def gemm_status() -> int:
    """Reads and clears the current device's status word of the standalone
    kernel calls: GEMMs and attention (synchronizes the device)."""
    v = C.c_uint32(0)
    _check(lib().f3dc_gemm_status(C.byref(v)))
    return v.value


def attention(q, ldq, k, v, ldkv, out, nq, nk, heads, dh, stream=None):
    _check(lib().f3dc_attention(_ptr(q), ldq, _ptr(k), _ptr(v), ldkv, _ptr(out), nq, nk, heads, dh,
                                _stream(stream)))


# ---------------------------------------------------------------- 8-bit linear layers

_fp8_state = None
_fp8_kinds = None


def _fp8_types():
    """What element types a tensor may have where the library reads or writes one
    kind of element.  Integers of the same size hold an element's bits."""
    global _fp8_kinds
    if _fp8_kinds is None:
        import torch as t
        _fp8_kinds = {"bf16": frozenset((t.bfloat16, t.int16, t.uint16)), "fp32": frozenset((t.float32,)),
                      "int32": frozenset((t.int32,)), "e4m3": frozenset((t.uint8, t.int8, t.float8_e4m3fn)),
                      "scale": frozenset((t.uint8, t.int8, t.float8_e8m0fnu))}
    return _fp8_kinds


class _Args:
    """The tensor arguments of a call and the kind of element of each."""

    def __init__(self, **kinds):
        self.names, self.kinds = tuple(kinds), tuple(kinds.values())
        self.types = tuple(frozenset().union(*(_fp8_types()[k] for k in v.split(" or "))) for v in self.kinds)

    def pointers(self, tensors, current):
        """Pointers of the tensors (None: null), which must be of their types and lie on the current device."""
        if current is None:
            return [None if t is None else t.data_ptr() if t.dtype in types and t.is_cuda else self._refuse(tensors)
                    for t, types in zip(tensors, self.types)]
        here = current()
        return [None if t is None else t.data_ptr() if t.dtype in types and t.get_device() == here and t.is_cuda else
                self._refuse(tensors, here) for t, types in zip(tensors, self.types)]

    def _refuse(self, tensors, here=0):
        for t, types, name, kind in zip(tensors, self.types, self.names, self.kinds):
            if t is not None and t.dtype not in types:
                raise F3dcError(1, f"{name} is {t.dtype}: need {kind}")
            if t is not None and not (t.is_cuda and t.get_device() == here):
                raise F3dcError(1, f"{name} is a tensor on {t.device}, which is not the current device")


def _fp8_args():
    """The arguments of quantize_fp8, of gemm_fp8 by its output (16 bits, fp32, 8 bits) and of
    norm_residual with h in 16 and in 8 bits."""
    ops = dict(A="e4m3", a_scales="scale", Bw="e4m3", b_scales="scale", bias="bf16", gate="fp32")
    rows = dict(x="fp32", x_out="fp32", y="bf16", gate="fp32", scale="fp32", shift="fp32", group_of_row="int32")
    return (_Args(x="bf16 or fp32", q="e4m3", scales="scale"),
            *(_Args(**ops, out=k, out_scales="scale") for k in ("bf16", "fp32", "e4m3")),
            *(_Args(**rows, h=k, h_scales="scale") for k in ("bf16", "e4m3")))


def _fp8():
    """(calls, their arguments, current device's getter or None where there is one
    device only), made on first use: a call is bound by its marshalling."""
    global _fp8_state
    if _fp8_state is None:
        import torch
        torch.cuda.init()
        L = lib()
        _fp8_state = ((L.f3dc_quantize_fp8, L.f3dc_gemm_fp8, L.f3dc_norm_residual), _fp8_args(),
                      torch._C._cuda_getDevice if torch.cuda.device_count() > 1 else None)
    return _fp8_state


def quantize_fp8(x, ldx, q, ldq, scales, lds, rows, cols, stream=None):
    """x [rows, cols] (bf16 or fp32; 16-bit integers are bf16 bits) -> e4m3
    bytes q and one power-of-two scale byte per row and block of 128 columns."""
    calls, args, current = _fp8_state or _fp8()
    px, pq, ps = args[0].pointers((x, q, scales), current)
    x_type = 1 if x is not None and x.dtype in _fp8_kinds["fp32"] else 0
    st = calls[0](px, x_type, ldx, pq, ldq, ps, lds, rows, cols, _stream(stream))
    if st:
        _check(st)


def gemm_fp8(A, lda, a_scales, ldas, Bw, ldb, b_scales, ldbs, bias, gate, out, ldo, out_scales, ldos, M, N, K, epilogue,
             stream=None):
    """Matrix product of two 8-bit matrices with f3dc_gemm's epilogues; with
    out_scales the output is an 8-bit matrix too."""
    calls, args, current = _fp8_state or _fp8()
    pa, psa, pb, psb, pbias, pgate, po, pos = args[3 if out_scales is not None else 2 if epilogue == EPI_RESID else 1].pointers(
        (A, a_scales, Bw, b_scales, bias, gate, out, out_scales), current)
    st = calls[1](pa, lda, psa, ldas, pb, ldb, psb, ldbs, pbias, pgate, po, ldo, pos, ldos, M, N, K, epilogue,
                  _stream(stream))
    if st:
        _check(st)


def norm_residual(layer, x, ldx, x_out, ldxo, y, ldy, gate, scale, shift, ldmod, group_of_row, groups, h, ldh, h_scales,
                  ldhs, rows, stream=None):
    """x_out = alpha x + gate post(y), h = pre(x_out) (1 + scale) + shift in one
    pass (`layer`: a NormLayer); with h_scales h is an 8-bit matrix."""
    calls, args, current = _fp8_state or _fp8()
    px, pxo, py, pg, psc, psh, pgr, ph, phs = args[4 if h_scales is None else 5].pointers(
        (x, x_out, y, gate, scale, shift, group_of_row, h, h_scales), current)
    if current is not None and any(t.get_device() != current() for t in layer._tensors):
        raise F3dcError(1, "a gain or bias is on another device than the current one")
    st = calls[2](layer._ref, px, ldx, pxo, ldxo, py, ldy, pg, psc, psh, ldmod, pgr, groups, ph, ldh, phs, ldhs, rows,
                  _stream(stream))
    if st:
        _check(st)


# ---------------------------------------------------------------- attention over a paged 8-bit cache

_kv_state = None


def rotary_turns(inv_freq) -> np.ndarray:
    """Angles per unit of position (radians) as 64-bit fractions of a turn."""
    f = np.ascontiguousarray(inv_freq, np.float64)
    out = np.empty(f.shape, np.uint64)
    _check(lib().f3dc_rotary_turns(f.ctypes.data_as(_f64p), f.size, out.ctypes.data_as(C.POINTER(C.c_uint64))))
    return out


def _kv_args():
    """The tensor arguments of kv_append_fp8 and of kv_attention_fp8."""
    return (_Args(k="bf16", v="bf16", q="bf16", q_out="bf16", positions="int32"),
            _Args(q="bf16", out="bf16", lse="fp32", workspace="e4m3"))


def _kv():
    """(calls, their arguments, current device's getter or None), made on first use."""
    global _kv_state
    if _kv_state is None:
        current = _fp8()[2]
        L = lib()
        _kv_state = ((L.f3dc_kv_append_fp8, L.f3dc_kv_attention_fp8), _kv_args(), current)
    return _kv_state


def _kv_here(current, *structs):
    for s in structs:
        if s is not None and (s._turns if isinstance(s, Rotary) else s._tensors[0]).get_device() != current():
            raise F3dcError(1, f"a {type(s).__name__} is on another device than the current one")


def kv_append_fp8(cache, batch, k, ldk, v, ldv, q=None, ldq=0, q_out=None, ldqo=0, heads=0, rotary=None, positions=None,
                  stream=None):
    """Keys and values (bf16 rows) of the batch's new tokens into the pages of their
    sequences, rotated by `rotary` (a Rotary) on the way; with q the rows' queries are rotated into q_out too."""
    calls, args, current = _kv_state or _kv()
    pk, pv, pq, pqo, pp = args[0].pointers((k, v, q, q_out, positions), current)
    if current is not None:
        _kv_here(current, cache, batch, rotary)
    if positions is not None and (not positions.is_contiguous() or positions.numel() < batch.rows * (rotary.axes if rotary else 1)):
        raise F3dcError(1, "positions are contiguous int32 [rows, axes]")
    st = calls[0](cache._ref, batch._for(cache), rotary._ref if rotary is not None else None, pk, ldk, pv, ldv, pq, ldq, pqo, ldqo, heads,
                  pp, _stream(stream))
    if st:
        _check(st)


def kv_attention_workspace(cache, batch, heads) -> int:
    """Bytes of workspace for kv_attention_fp8 (0: none is needed)."""
    return int(lib().f3dc_kv_attention_workspace(cache._ref, batch._for(cache), heads))


def kv_attention_fp8(cache, batch, q, ldq, out, ldo, heads, scale, causal=False, lse=None, workspace=None, stream=None):
    """Attention of packed bf16 query rows over their sequences' cached tokens; lse
    fp32 [rows, heads]; `workspace` a byte tensor of kv_attention_workspace() bytes."""
    calls, args, current = _kv_state or _kv()
    pq, po, pl, pw = args[1].pointers((q, out, lse, workspace), current)
    if current is not None:
        _kv_here(current, cache, batch)
    if lse is not None and (not lse.is_contiguous() or lse.numel() < batch.rows * heads):
        raise F3dcError(1, "lse is contiguous fp32 [rows, heads]")
    st = calls[1](cache._ref, batch._for(cache), pq, ldq, po, ldo, pl, heads, scale, 1 if causal else 0, pw,
                  workspace.numel() if workspace is not None else 0, _stream(stream))
    if st:
        _check(st)
