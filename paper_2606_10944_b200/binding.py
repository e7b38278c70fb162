"""ctypes binding of the C-ABI CUDA library (argument marshalling only).

Each function mirrors one entry point declared in ``include/elm.h``.  PyTorch is used for
device memory and the current stream; every arithmetic step runs inside the library's
kernels.  There is no CPU fallback: if ``csrc/libelm.so`` has not been built, or no CUDA
device is present when a compute call is made, an :class:`ElmError` is raised.
"""
from __future__ import annotations

import ctypes
from pathlib import Path

import torch

ELM_F32, ELM_BF16, ELM_E4M3 = 0, 1, 2
PREC_FP64_DET, PREC_FP32 = 0, 1
_PRECISIONS = {"fp64": PREC_FP64_DET, "fp64_det": PREC_FP64_DET, "fp32": PREC_FP32,
               PREC_FP64_DET: PREC_FP64_DET, PREC_FP32: PREC_FP32}
STAGE_NAMES = ["prepass", "level_prep", "gram", "walk", "emit", "gather", "attend"]

EXPORTED_SYMBOLS = [
    "elm_workspace_bytes", "elm_default_delta_levels", "elm_compress", "elm_attend",
    "elm_attend_workspace_bytes", "elm_attend_static", "elm_attend_static_status", "elm_compress_ragged_count", "elm_compress_ragged", "elm_express_workspace_bytes", "elm_express_compress",
    "elm_express_prefill_workspace_bytes", "elm_express_prefill",
    "elm_stream_workspace_bytes", "elm_stream_init", "elm_stream_step", "elm_stream_steps", "elm_stream_cache",
    "elm_rope", "elm_rope_frequencies", "elm_page_plan", "elm_page_release", "elm_cache4_row_bytes", "elm_cache4_append", "elm_cache4_read",
    "elm_cache4_attend_workspace_bytes", "elm_cache4_attend", "elm_cache4_attend_status",
    "elm_host_call_scratch_bytes", "elm_compress_attend_host",
    "elm_compress_status", "elm_attend_status", "elm_debug_set", "elm_debug_round_check", "elm_debug_decode_grid", "elm_debug_stream_form", "elm_profile_enable", "elm_profile_read", "elm_launch_count", "elm_strerror", "elm_version",
]


class ElmError(RuntimeError):
    pass


class ElmParams(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("q_heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
        ("n_kv", ctypes.c_int32), ("n_q", ctypes.c_int32), ("d", ctypes.c_int32),
        ("log2_nout", ctypes.c_int32), ("m", ctypes.c_int32),
        ("dtype", ctypes.c_int32), ("precision", ctypes.c_int32),
        ("delta", ctypes.c_double), ("delta_level", ctypes.POINTER(ctypes.c_double)),
    ]


class ElmStream(ctypes.Structure):
    _fields_ = [
        ("n", ctypes.c_int64), ("ell", ctypes.c_int64), ("n_E", ctypes.c_int64),
        ("m", ctypes.c_int32), ("b", ctypes.c_int32), ("q", ctypes.c_int32), ("mbar", ctypes.c_int32),
        ("n_S", ctypes.c_int64 * 16), ("calls", ctypes.c_int64 * 16),
        ("n_known", ctypes.c_int64), ("seed", ctypes.c_uint64),
    ]


class RopeParams(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("heads", ctypes.c_int32), ("n_tokens", ctypes.c_int32), ("d", ctypes.c_int32),
        ("dtype", ctypes.c_int32), ("rotary_dim", ctypes.c_int32), ("layout", ctypes.c_int32), ("inverse", ctypes.c_int32),
        ("scale", ctypes.c_double), ("inv_freq", ctypes.POINTER(ctypes.c_double)),
        ("x_stride", ctypes.c_int64 * 3), ("out_stride", ctypes.c_int64 * 3),
    ]


class PageParams(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("page_rows", ctypes.c_int32),
                ("max_tokens", ctypes.c_int32), ("n_free", ctypes.c_int32)]


class AppendParams(ctypes.Structure):
    _fields_ = [
        ("n_tokens", ctypes.c_int32), ("q_heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("d", ctypes.c_int32),
        ("dtype", ctypes.c_int32), ("page_rows", ctypes.c_int32), ("n_pages", ctypes.c_int32),
        ("rotary_dim", ctypes.c_int32), ("layout", ctypes.c_int32),
        ("scale", ctypes.c_double), ("inv_freq", ctypes.POINTER(ctypes.c_double)),
        ("q_stride", ctypes.c_int64 * 2), ("k_stride", ctypes.c_int64 * 2), ("v_stride", ctypes.c_int64 * 2),
        ("q_out_stride", ctypes.c_int64 * 2),
    ]


class Cache4Params(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("q_heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("d", ctypes.c_int32),
        ("dtype", ctypes.c_int32), ("page_rows", ctypes.c_int32), ("n_pages", ctypes.c_int32), ("max_pages", ctypes.c_int32),
        ("n_kv", ctypes.c_int32), ("n_q", ctypes.c_int32), ("n_tokens", ctypes.c_int32), ("causal", ctypes.c_int32),
        ("q_stride", ctypes.c_int64 * 3), ("o_stride", ctypes.c_int64 * 3),
    ]


_lib = None


def library_path() -> Path:
    return Path(__file__).resolve().parent / "csrc" / "libelm.so"


def load_library():
    global _lib
    if _lib is not None:
        return _lib
    path = library_path()
    if not path.exists():
        raise ElmError(f"{path} is missing: build it with `python -m paper_2606_10944_b200.build` "
                       "(there is no CPU fallback)")
    lib = ctypes.CDLL(str(path))
    vp, sz = ctypes.c_void_p, ctypes.c_size_t
    pp = ctypes.POINTER(ElmParams)
    szp = ctypes.POINTER(sz)
    lib.elm_workspace_bytes.argtypes = [pp, szp, szp]
    lib.elm_default_delta_levels.argtypes = [ctypes.c_int32, ctypes.c_double, ctypes.POINTER(ctypes.c_double)]
    lib.elm_compress.argtypes = [vp, vp, pp, ctypes.c_uint64, vp, vp, vp, sz, vp]
    lib.elm_attend.argtypes = [vp, vp, vp, vp, vp, ctypes.c_int32, pp, vp, vp, sz, vp]
    lib.elm_attend_workspace_bytes.argtypes = [pp, ctypes.c_int32, szp]
    lib.elm_attend_static.argtypes = [vp, vp, vp, vp, vp, ctypes.c_int32, pp, vp, vp]
    lib.elm_attend_static_status.argtypes = [pp, ctypes.c_int32, ctypes.POINTER(ctypes.c_int32), vp]
    lib.elm_compress_ragged_count.argtypes = [pp, ctypes.c_int32, ctypes.c_int32, ctypes.POINTER(ctypes.c_int32), szp]
    lib.elm_compress_ragged.argtypes = [vp, vp, pp, ctypes.c_int32, ctypes.c_int32, ctypes.c_uint64, vp, vp, vp, sz, vp]
    lib.elm_express_workspace_bytes.argtypes = [pp, ctypes.c_int32, szp]
    lib.elm_express_compress.argtypes = [vp, vp, pp, ctypes.c_int32, ctypes.c_uint64, vp, vp, vp, sz, vp]
    lib.elm_express_prefill_workspace_bytes.argtypes = [pp, ctypes.c_int32, szp]
    lib.elm_express_prefill.argtypes = [vp, vp, vp, pp, ctypes.c_int32, ctypes.c_uint64, vp, vp, vp, vp, sz, vp]
    sp = ctypes.POINTER(ElmStream)
    lib.elm_stream_workspace_bytes.argtypes = [pp, ctypes.c_int32, szp]
    lib.elm_stream_init.argtypes = [sp, vp, vp, ctypes.c_int64, pp, ctypes.c_int32, ctypes.c_uint64, vp, sz, vp]
    lib.elm_stream_step.argtypes = [sp, vp, vp, vp, pp, vp, vp, sz, vp]
    lib.elm_stream_steps.argtypes = [sp, ctypes.c_int32, vp, vp, vp, pp, vp, vp, sz, vp]
    lib.elm_stream_cache.argtypes = [sp, pp, vp, vp, ctypes.POINTER(ctypes.c_int32), vp, sz, vp]
    i32, i32p, f64, f64p = ctypes.c_int32, ctypes.POINTER(ctypes.c_int32), ctypes.c_double, ctypes.POINTER(ctypes.c_double)
    gp, cp = ctypes.POINTER(PageParams), ctypes.POINTER(Cache4Params)
    lib.elm_rope.argtypes = [vp, vp, ctypes.c_int64, ctypes.POINTER(RopeParams), vp, vp]
    lib.elm_rope_frequencies.argtypes = [i32, f64, i32, f64, f64, f64, f64, f64p, f64p]
    lib.elm_page_plan.argtypes = [vp, vp, vp, vp, vp, gp, vp, vp, vp, vp, vp, vp, vp]
    lib.elm_page_release.argtypes = [vp, vp, vp, vp, vp, gp, vp]
    lib.elm_cache4_row_bytes.argtypes = [i32, szp]
    lib.elm_cache4_append.argtypes = [vp, vp, vp, vp, vp, ctypes.POINTER(AppendParams), vp, vp, vp]
    lib.elm_cache4_read.argtypes = [vp, vp, vp, vp, cp, vp, vp, vp]
    lib.elm_cache4_attend_workspace_bytes.argtypes = [cp, i32, szp]
    lib.elm_cache4_attend.argtypes = [vp, vp, vp, vp, vp, vp, vp, cp, vp, vp, sz, vp]
    lib.elm_cache4_attend_status.argtypes = [vp, cp, i32, i32p, vp]
    lib.elm_host_call_scratch_bytes.argtypes = [pp, szp]
    lib.elm_compress_attend_host.argtypes = [vp, vp, vp, vp, vp, vp, pp, ctypes.c_uint64, vp, sz, vp]
    lib.elm_compress_status.argtypes = [vp, pp, ctypes.POINTER(ctypes.c_int32), vp]
    lib.elm_attend_status.argtypes = [vp, pp, ctypes.c_int32, ctypes.POINTER(ctypes.c_int32), vp]
    lib.elm_debug_set.argtypes = [ctypes.c_int32, ctypes.c_int64]
    lib.elm_debug_decode_grid.argtypes = [pp, ctypes.c_int32, ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int32)]
    lib.elm_debug_stream_form.argtypes = [pp, ctypes.c_int32, ctypes.c_int32, ctypes.POINTER(ctypes.c_int32)]
    lib.elm_debug_round_check.argtypes = [ctypes.POINTER(ElmParams), ctypes.c_int32, ctypes.c_int32, ctypes.c_uint64,
                                          ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_int64),
                                          ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_int64)]
    lib.elm_profile_enable.argtypes = [ctypes.c_int]
    lib.elm_profile_read.argtypes = [ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_int64), ctypes.c_int32]
    lib.elm_launch_count.argtypes = []
    lib.elm_launch_count.restype = ctypes.c_int64
    lib.elm_strerror.argtypes = [ctypes.c_int]
    lib.elm_strerror.restype = ctypes.c_char_p
    lib.elm_version.argtypes = []
    for name in EXPORTED_SYMBOLS:
        if name not in ("elm_launch_count", "elm_strerror"):
            getattr(lib, name).restype = ctypes.c_int
    _lib = lib
    return lib


def _check(rc: int, what: str):
    if rc != 0:
        raise ElmError(f"{what} failed: {load_library().elm_strerror(rc).decode()} ({rc})")


def _require_cuda(*tensors):
    for t in tensors:
        if not t.is_cuda or not t.is_contiguous():
            # (asked only now: a CUDA tensor answers it, and the question costs more than a kernel launch)
            if not torch.cuda.is_available():
                raise ElmError("no CUDA device: the library has no CPU fallback")
            raise ElmError("tensors must be contiguous CUDA tensors")


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return ELM_F32
    if t.dtype == torch.bfloat16:
        return ELM_BF16
    if t.dtype == torch.float8_e4m3fn:
        return ELM_E4M3
    raise ElmError(f"unsupported dtype {t.dtype}")


def _stream() -> int:
    # the current device's current stream; torch's own accessor saves the torch.cuda.Stream object made for every call,
    # but is not public, so a build of torch may lack it
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(torch.cuda.current_device()) if raw is not None else torch.cuda.current_stream().cuda_stream


def make_params(batch, q_heads, kv_heads, n_kv, n_q, d, log2_nout, m, dtype_code, precision="fp32",
                delta=0.5, delta_level=None):
    """Fill an ``elm_params``; returns (params, keepalive) where keepalive owns delta_level."""
    p = ElmParams()
    p.batch, p.q_heads, p.kv_heads = batch, q_heads, kv_heads
    p.n_kv, p.n_q, p.d = n_kv, n_q, d
    p.log2_nout, p.m = log2_nout, m
    p.dtype, p.precision = dtype_code, _PRECISIONS[precision]
    p.delta = float(delta)
    keep = None
    if delta_level is not None:
        keep = (ctypes.c_double * len(delta_level))(*[float(x) for x in delta_level])
        p.delta_level = ctypes.cast(keep, ctypes.POINTER(ctypes.c_double))
    return p, keep


def version() -> int:
    return int(load_library().elm_version())


def default_delta_levels(m: int, delta: float = 0.5):
    out = (ctypes.c_double * max(m, 1))()
    _check(load_library().elm_default_delta_levels(m, delta, out), "elm_default_delta_levels")
    return [out[i] for i in range(m)]


def workspace_bytes(params: ElmParams):
    c, a = ctypes.c_size_t(0), ctypes.c_size_t(0)
    _check(load_library().elm_workspace_bytes(ctypes.byref(params), ctypes.byref(c), ctypes.byref(a)),
           "elm_workspace_bytes")
    return int(c.value), int(a.value)


def _workspace(nbytes: int, device):
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)


def compress(K, V, log2_nout: int, m: int, seed: int = 1, precision="fp32", delta: float = 0.5,
             delta_level=None, workspace=None):
    """elm_compress: K, V [B, Hkv, n, d] -> (idx int32 [B, Hkv, n_out], w float32 [B, Hkv, n_out])."""
    lib = load_library()
    _require_cuda(K, V)
    B, H, n, d = K.shape
    p, keep = make_params(B, H, H, n, 1, d, log2_nout, m, _dtype_code(K), precision, delta, delta_level)
    need, _ = workspace_bytes(p)
    ws = workspace if workspace is not None else _workspace(need, K.device)
    n_out = 1 << log2_nout
    idx = torch.empty((B, H, n_out), dtype=torch.int32, device=K.device)
    w = torch.empty((B, H, n_out), dtype=torch.float32, device=K.device)
    _check(lib.elm_compress(K.data_ptr(), V.data_ptr(), ctypes.byref(p), seed, idx.data_ptr(),
                            w.data_ptr(), ws.data_ptr(), ws.numel(), _stream()), "elm_compress")
    return idx, w


def compress_ragged_count(params: ElmParams, n_sink: int = 0, n_window: int = 0):
    """elm_compress_ragged_count -> (entries per attention problem, workspace bytes)."""
    c, b = ctypes.c_int32(0), ctypes.c_size_t(0)
    _check(load_library().elm_compress_ragged_count(ctypes.byref(params), n_sink, n_window, ctypes.byref(c),
                                                    ctypes.byref(b)), "elm_compress_ragged_count")
    return int(c.value), int(b.value)


def compress_ragged(K, V, log2_nout: int, m: int, n_sink: int = 0, n_window: int = 0, seed: int = 1, precision="fp32",
                    delta: float = 0.5, delta_level=None, workspace=None):
    """elm_compress_ragged: K, V [B, Hkv, n, d] with any n -> (idx, w) [B, Hkv, count]: the sink rows,
    Compress2's weighted cache after the middle rows, the window rows."""
    lib = load_library()
    _require_cuda(K, V)
    B, H, n, d = K.shape
    p, keep = make_params(B, H, H, n, 1, d, log2_nout, m, _dtype_code(K), precision, delta, delta_level)
    count, need = compress_ragged_count(p, n_sink, n_window)
    ws = workspace if workspace is not None else _workspace(need, K.device)
    idx = torch.empty((B, H, max(count, 1)), dtype=torch.int32, device=K.device)[:, :, :count]
    w = torch.empty((B, H, max(count, 1)), dtype=torch.float32, device=K.device)[:, :, :count]
    _check(lib.elm_compress_ragged(K.data_ptr(), V.data_ptr(), ctypes.byref(p), n_sink, n_window, seed, idx.data_ptr(),
                                   w.data_ptr(), ws.data_ptr(), ws.numel(), _stream()), "elm_compress_ragged")
    return idx, w


def express_compress(K, V, log2_nout: int, mbar: int, seed: int = 1, precision="fp32", delta: float = 0.5,
                     workspace=None):
    """elm_express_compress: K, V [B, Hkv, n, d] with n = n_out 4^R -> (idx, w) of the Express cache
    after the whole sequence (Offline-Express with KH-Express failure parameters)."""
    lib = load_library()
    _require_cuda(K, V)
    B, H, n, d = K.shape
    p, _ = make_params(B, H, H, n, 1, d, log2_nout, 0, _dtype_code(K), precision, delta)
    need = ctypes.c_size_t(0)
    _check(lib.elm_express_workspace_bytes(ctypes.byref(p), mbar, ctypes.byref(need)), "elm_express_workspace_bytes")
    ws = workspace if workspace is not None else _workspace(int(need.value), K.device)
    n_out = 1 << log2_nout
    idx = torch.empty((B, H, n_out), dtype=torch.int32, device=K.device)
    w = torch.empty((B, H, n_out), dtype=torch.float32, device=K.device)
    _check(lib.elm_express_compress(K.data_ptr(), V.data_ptr(), ctypes.byref(p), mbar, seed, idx.data_ptr(),
                                    w.data_ptr(), ws.data_ptr(), ws.numel(), _stream()), "elm_express_compress")
    return idx, w


def express_prefill(Q, K, V, log2_nout: int, mbar: int, seed: int = 1, precision="fp32", delta: float = 0.5,
                    workspace=None, out=None):
    """elm_express_prefill: Q [B, Hq, n, d], K, V [B, Hkv, n, d] -> (O like Q, idx, w): every token attends
    over the Express cache as of its own position plus itself (Thinformer Express in prefill)."""
    lib = load_library()
    _require_cuda(Q, K, V)
    B, Hq, nq, d = Q.shape
    H, n = K.shape[1], K.shape[2]
    p, _ = make_params(B, Hq, H, n, nq, d, log2_nout, 0, _dtype_code(K), precision, delta)
    need = ctypes.c_size_t(0)
    _check(lib.elm_express_prefill_workspace_bytes(ctypes.byref(p), mbar, ctypes.byref(need)),
           "elm_express_prefill_workspace_bytes")
    ws = workspace if workspace is not None else _workspace(int(need.value), K.device)
    n_out = 1 << log2_nout
    O = out if out is not None else torch.empty_like(Q)
    idx = torch.empty((B, H, n_out), dtype=torch.int32, device=K.device)
    w = torch.empty((B, H, n_out), dtype=torch.float32, device=K.device)
    _check(lib.elm_express_prefill(Q.data_ptr(), K.data_ptr(), V.data_ptr(), ctypes.byref(p), mbar, seed, O.data_ptr(),
                                   idx.data_ptr(), w.data_ptr(), ws.data_ptr(), ws.numel(), _stream()),
           "elm_express_prefill")
    return O, idx, w


class Stream:
    """elm_stream_*: streaming Thinformer Express over K, V [B, Hkv, capacity, d] (one token per step)."""

    def __init__(self, K, V, q_heads: int, log2_nout: int, mbar: int, seed: int = 1, precision="fp32",
                 delta: float = 0.5, n_known=None):
        lib = load_library()
        _require_cuda(K, V)
        B, H, n, d = K.shape
        self.K, self.V = K, V
        self.params, _ = make_params(B, q_heads, H, n, 1, d, log2_nout, 0, _dtype_code(K), precision, delta)
        need = ctypes.c_size_t(0)
        _check(lib.elm_stream_workspace_bytes(ctypes.byref(self.params), mbar, ctypes.byref(need)),
               "elm_stream_workspace_bytes")
        self.ws = _workspace(int(need.value), K.device)
        self.state = ElmStream()
        _check(lib.elm_stream_init(ctypes.byref(self.state), K.data_ptr(), V.data_ptr(), n if n_known is None else n_known,
                                   ctypes.byref(self.params), mbar, seed, self.ws.data_ptr(), self.ws.numel(), _stream()),
               "elm_stream_init")

    def step(self, q_t, out=None):
        """q_t [B, Hq, 1, d] -> O_t; the token is row state.n of K and V."""
        O = out if out is not None else torch.empty_like(q_t)
        _check(load_library().elm_stream_step(ctypes.byref(self.state), q_t.data_ptr(), self.K.data_ptr(), self.V.data_ptr(),
                                              ctypes.byref(self.params), O.data_ptr(), self.ws.data_ptr(), self.ws.numel(),
                                              _stream()), "elm_stream_step")
        return O

    def steps(self, q_T, out=None):
        """q_T [T, B, Hq, 1, d] -> O_T of the same shape: T tokens by one library call (elm_stream_steps)."""
        O = out if out is not None else torch.empty_like(q_T)
        _check(load_library().elm_stream_steps(ctypes.byref(self.state), q_T.shape[0], q_T.data_ptr(), self.K.data_ptr(),
                                               self.V.data_ptr(), ctypes.byref(self.params), O.data_ptr(), self.ws.data_ptr(),
                                               self.ws.numel(), _stream()), "elm_stream_steps")
        return O

    def cache(self):
        """(idx int32 [B, Hkv, count], w float32 [B, Hkv, count]) of wtd_cache()."""
        p = self.params
        cap = 6 * (1 << p.log2_nout) + 1
        idx = torch.empty((p.batch, p.kv_heads, cap), dtype=torch.int32, device=self.K.device)
        w = torch.empty((p.batch, p.kv_heads, cap), dtype=torch.float32, device=self.K.device)
        count = ctypes.c_int32(0)
        # the library writes dense [problem][count] arrays at the front of the buffers
        _check(load_library().elm_stream_cache(ctypes.byref(self.state), ctypes.byref(p), idx.data_ptr(), w.data_ptr(),
                                               ctypes.byref(count), self.ws.data_ptr(), self.ws.numel(), _stream()),
               "elm_stream_cache")
        c = int(count.value)
        flat_i = idx.reshape(-1)[: p.batch * p.kv_heads * c].reshape(p.batch, p.kv_heads, c)
        flat_w = w.reshape(-1)[: p.batch * p.kv_heads * c].reshape(p.batch, p.kv_heads, c)
        return flat_i, flat_w


def attend_workspace_bytes(params: ElmParams, n_core: int) -> int:
    need = ctypes.c_size_t(0)
    _check(load_library().elm_attend_workspace_bytes(ctypes.byref(params), n_core, ctypes.byref(need)),
           "elm_attend_workspace_bytes")
    return int(need.value)


def attend(Q, K, V, idx, w, precision="fp32", workspace=None, out=None):
    """elm_attend: Q [B, Hq, nq, d]; K, V [B, Hkv, n, d]; idx, w [B, Hkv, n_core] -> O like Q."""
    lib = load_library()
    _require_cuda(Q, K, V, idx, w)
    B, Hq, nq, d = Q.shape
    Hkv, n = K.shape[1], K.shape[2]
    n_core = idx.shape[-1]
    if idx.dtype != torch.int32 or w.dtype != torch.float32:
        raise ElmError("idx must be int32 and w float32")
    # log2_nout / m only describe compression; any consistent pair passes validation
    p, _ = make_params(B, Hq, Hkv, n, nq, d, n.bit_length() - 1, 0, _dtype_code(Q), precision)
    need = ctypes.c_size_t(0)
    _check(lib.elm_attend_workspace_bytes(ctypes.byref(p), n_core, ctypes.byref(need)),
           "elm_attend_workspace_bytes")
    ws = workspace if workspace is not None else _workspace(int(need.value), Q.device)
    # 8-bit inputs: the output is bf16
    O = out if out is not None else torch.empty(Q.shape, dtype=torch.bfloat16 if Q.dtype == torch.float8_e4m3fn else Q.dtype,
                                                device=Q.device)
    _check(lib.elm_attend(Q.data_ptr(), K.data_ptr(), V.data_ptr(), idx.data_ptr(), w.data_ptr(),
                          n_core, ctypes.byref(p), O.data_ptr(), ws.data_ptr(), ws.numel(), _stream()),
           "elm_attend")
    return O


ATTEND_STATIC_SCRATCH_BYTES = 16 << 20


def attend_static(Q, K, V, idx, w, precision="fp32", out=None):
    """elm_attend_static: elm_attend without a workspace argument.

    For callers that may not allocate device memory: the coreset operands are staged in a
    fixed array inside the library (ATTEND_STATIC_SCRATCH_BYTES), so this wrapper allocates
    nothing when ``out`` is supplied.  Calls on one device share that array; do not let two of
    them overlap on the GPU.
    """
    lib = load_library()
    _require_cuda(Q, K, V, idx, w)
    B, Hq, nq, d = Q.shape
    Hkv, n = K.shape[1], K.shape[2]
    if idx.dtype != torch.int32 or w.dtype != torch.float32:
        raise ElmError("idx must be int32 and w float32")
    p, _ = make_params(B, Hq, Hkv, n, nq, d, n.bit_length() - 1, 0, _dtype_code(Q), precision)
    O = out if out is not None else torch.empty_like(Q)
    _check(lib.elm_attend_static(Q.data_ptr(), K.data_ptr(), V.data_ptr(), idx.data_ptr(), w.data_ptr(),
                                 idx.shape[-1], ctypes.byref(p), O.data_ptr(), _stream()),
           "elm_attend_static")
    return O


def attend_static_status(Q, K, n_core: int, precision="fp32") -> int:
    """elm_attend_static_status after an attend_static call with these tensors' shapes: 0 unless a bounded
    device wait expired during it."""
    B, Hq, nq, d = Q.shape
    Hkv, n = K.shape[1], K.shape[2]
    p, _ = make_params(B, Hq, Hkv, n, nq, d, n.bit_length() - 1, 0, _dtype_code(Q), precision)
    out = ctypes.c_int32(-1)
    _check(load_library().elm_attend_static_status(ctypes.byref(p), n_core, ctypes.byref(out), _stream()),
           "elm_attend_static_status")
    return int(out.value)


# ------------------------------------------------------------------------------------------------
# rotary positions, pages, rows held in 4 bits
# ------------------------------------------------------------------------------------------------
# The calls below run on their tensors' device, on its current stream, whatever the current device is: one that finds another current
# device calls itself again under that of its tensors.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_of(device: int) -> int:
    return _raw_stream(device) if _raw_stream is not None else torch.cuda.current_stream(device).cuda_stream


def _device(first, *tensors):
    """Ordinal of the one device that the tensors (or None) are on."""
    index = first.get_device()
    if index < 0:
        _require_cuda(first)
    for t in tensors:
        if t is not None and t.get_device() != index:
            raise ElmError("tensors must be CUDA tensors of one device")
    return index


class _Kept(dict):
    """What a call has found out about sizes, strides and types (nothing of the tensors themselves), for the next one with the same.
    A call of sizes that are not here looks at everything (up to 9 us more), and all are forgotten at the 256th, so steps whose number of tokens changes
    are best padded to a few sizes, as page_plan() allows."""

    def keep(self, key, value):
        if len(self) >= 256:
            self.clear()
        self[key] = value
        return value


def _rows(x, dims, what):
    """x with its last numbers side by side, and its other strides; a broadcast of one row is copied (strides of 0 mean dense)."""
    if x.dim() != dims:
        raise ElmError(f"{what} must have {dims} dimensions")
    if x.numel() == 0:
        raise ElmError(f"{what} is empty")
    st = x.stride()
    if st[-1] != 1 and x.shape[-1] > 1:
        raise ElmError(f"{what}: the numbers of a head must lie side by side")
    if not any(st[:-1]) and x.numel() > x.shape[-1]:
        x = x.contiguous()
        st = x.stride()
    return x, st


def _int32(t, what, shape=None):
    if t.dtype != torch.int32 or not t.is_contiguous() or (shape is not None and tuple(t.shape) != tuple(shape)):
        raise ElmError(f"{what} must be a contiguous int32 tensor" + (f" of shape {tuple(shape)}" if shape is not None else ""))
    return t


def _storage_code(t):
    code = _dtype_code(t)
    if code == ELM_E4M3:
        raise ElmError(f"unsupported dtype {t.dtype}")
    return code


def _ptr(t):
    return None if t is None else t.data_ptr()


_ROPE_LAYOUTS = {"halves": 0, "pairs": 1}
_ROPE_SCALINGS = {"plain": 0, "linear": 1, "base": 2, "ramp": 3, "smooth": 4}


class Rope:
    """Frequencies of a rotation (elm_rope_frequencies): the first ``rotary_dim`` numbers of a head turn in pairs, (i, i +
    rotary_dim / 2) with layout "halves", (2i, 2i + 1) with "pairs".  ``scaling``: "plain", "linear", "base", "ramp" or "smooth",
    with its ``factor``, the trained length ``original`` and the turns ``low`` and ``high`` of the blends (see include/elm.h)."""

    def __init__(self, rotary_dim, base=10000.0, layout="halves", scaling="plain", factor=1.0, original=0.0, low=1.0, high=32.0):
        if layout not in _ROPE_LAYOUTS or scaling not in _ROPE_SCALINGS:
            raise ElmError(f"unknown layout {layout!r} or scaling {scaling!r}")
        self.rotary_dim, self.layout = int(rotary_dim), _ROPE_LAYOUTS[layout]
        self._freq = (ctypes.c_double * max(1, self.rotary_dim // 2))()
        scale = ctypes.c_double(1.0)
        _check(load_library().elm_rope_frequencies(self.rotary_dim, base, _ROPE_SCALINGS[scaling], factor, original, low, high, self._freq,
                                                   ctypes.byref(scale)), "elm_rope_frequencies")
        self.scale = scale.value
        self._freq_ptr = ctypes.cast(self._freq, ctypes.POINTER(ctypes.c_double))
        self._kept = _Kept()

    @property
    def inv_freq(self):
        return list(self._freq)


def rope(X, positions, rope: Rope, inverse=False, out=None):
    """elm_rope: X [B, H, n, d] (any strides, a head's numbers side by side) rotated by positions, an int32 tensor [B, n] or the first
    position of every sequence; ``inverse``: rotated back (the gradient).  ``out``: X itself, or another tensor of its shape.  Where X requires
    a gradient, the result has one (without ``out``)."""
    tensor = isinstance(positions, torch.Tensor)
    device = _device(X, out, positions if tensor else None)
    if X.requires_grad and torch.is_grad_enabled():
        if out is not None:
            raise ElmError("out: X requires a gradient, which a given place for the result does not have")
        return _Rotation.apply(X, positions, rope, inverse)
    if device != torch.cuda.current_device():
        with torch.cuda.device(device):
            return _rope_again(X, positions, rope, inverse, out)
    key = (X.shape, X.stride(), X.dtype, inverse, positions.shape if tensor else None)
    if out is not None:
        key += (out.shape, out.stride(), out.dtype)
    p = rope._kept.get(key)
    if p is None:
        Y, xs = _rows(X, 4, "X")
        if Y is not X:                                      # (a broadcast of one row)
            if out is X:
                raise ElmError("out: rows must lie apart")
            return _rope_again(Y, positions, rope, inverse, out)
        B, H, n, d = X.shape
        if out is not None:
            if out.shape != X.shape or out.dtype != X.dtype:
                raise ElmError("out must have X's shape and dtype")
            os_ = out.stride()
            if (os_[-1] != 1 and d > 1) or not any(os_[:-1]) and out.numel() > d:
                raise ElmError("out: the numbers of a head must lie side by side, rows apart")
        if tensor:
            _int32(positions, "positions", (B, n))
        p = RopeParams(B, H, n, d, _storage_code(X), rope.rotary_dim, rope.layout, int(bool(inverse)), rope.scale, rope._freq_ptr)
        p.x_stride[:] = xs[:3]
        p.out_stride[:] = os_[:3] if out is not None else (0, 0, 0)
        rope._kept.keep(key, p)
    if tensor:
        if positions.dtype is not torch.int32 or not positions.is_contiguous():
            raise ElmError("positions must be a contiguous int32 tensor")
        pos, first = positions.data_ptr(), 0
    else:
        pos, first = None, int(positions)
    O = out if out is not None else torch.empty_like(X, memory_format=torch.contiguous_format)
    rc = load_library().elm_rope(X.data_ptr(), pos, first, p, O.data_ptr(), _stream_of(device))
    if rc:
        _check(rc, "elm_rope")
    return O


def _rope_again(X, positions, turn, inverse, out):              # (where ``rope`` is the name of an argument)
    return rope(X, positions, turn, inverse, out)


class _Rotation(torch.autograd.Function):
    """The rotation is linear: its gradient is the transposed one, elm_rope's inverse, and that one's is the rotation again."""

    @staticmethod
    def forward(ctx, X, positions, turn, inverse):
        ctx.turn, ctx.inverse, ctx.first = turn, inverse, None
        if isinstance(positions, torch.Tensor):
            ctx.save_for_backward(positions)                    # (a later change of theirs is noticed)
        else:
            ctx.first = positions
        return rope(X.detach(), positions, turn, inverse)

    @staticmethod
    def backward(ctx, dY):
        if dY.stride(-1) != 1:
            dY = dY.contiguous()
        return rope(dY, ctx.saved_tensors[0] if ctx.first is None else ctx.first, ctx.turn, not ctx.inverse), None, None, None


class PagePlan:
    """What page_plan() returns: start, length [B], free_count [1], cu [B + 1], positions, slots [max_tokens]."""

    __slots__ = ("start", "length", "free_count", "cu", "positions", "slots")


_plan_kept = _Kept()


def page_plan(table, length, n_new, free, free_count, page_rows: int, max_tokens: int, length_out=None, free_count_out=None) -> PagePlan:
    """elm_page_plan: pages, positions and slots of the n_new [B] tokens that come to requests of length [B].  ``table`` [B, max_pages]
    gets the new pages' numbers; length_out and free_count_out may be length and free_count."""
    device = _device(table, length, n_new, free, free_count, length_out, free_count_out)
    if device != torch.cuda.current_device():
        with torch.cuda.device(device):
            return page_plan(table, length, n_new, free, free_count, page_rows, max_tokens, length_out, free_count_out)
    key = (table.shape, length.shape, n_new.shape, free.shape, free_count.shape, page_rows, max_tokens)
    kept = _plan_kept.get(key)
    if kept is None:
        if table.dim() != 2:
            raise ElmError("table must be [B, max_pages]")
        B, max_pages = table.shape
        _int32(length, "length", (B,)), _int32(n_new, "n_new", (B,)), _int32(free, "free"), _int32(free_count, "free_count", (1,))
        # (one allocation for all that comes out)
        sizes = [max(0, max_tokens), max(0, max_tokens), B, B, B + 1, 1]
        kept = _plan_kept.keep(key, (PageParams(B, max_pages, page_rows, max_tokens, free.numel()), sum(sizes), sizes))
    p, total, cuts = kept
    for t in (table, length, n_new, free, free_count):
        if t.dtype is not torch.int32 or not t.is_contiguous():
            raise ElmError("table, length, n_new, free and free_count must be contiguous int32 tensors")
    buf = torch.empty(total, dtype=torch.int32, device=table.device)
    r = PagePlan()
    r.positions, r.slots, r.start, r.length, r.cu, r.free_count = buf.split_with_sizes(cuts)
    if length_out is not None:
        r.length = _int32(length_out, "length_out", length.shape)
    if free_count_out is not None:
        r.free_count = _int32(free_count_out, "free_count_out", (1,))
    rc = load_library().elm_page_plan(table.data_ptr(), length.data_ptr(), n_new.data_ptr(), free.data_ptr(), free_count.data_ptr(), p,
                                      r.start.data_ptr(), r.length.data_ptr(), r.free_count.data_ptr(), r.cu.data_ptr(),
                                      r.positions.data_ptr(), r.slots.data_ptr(), _stream_of(device))
    if rc:
        _check(rc, "elm_page_plan")
    return r


def page_release(table, length, done, free, free_count, page_rows: int):
    """elm_page_release: the pages of the requests with done [B] != 0 go back to the end of free; everything in place."""
    lib = load_library()
    device = _device(table, length, done, free, free_count)
    with torch.cuda.device(device):
        B, max_pages = _int32(table, "table").shape
        _int32(length, "length", (B,)), _int32(done, "done", (B,)), _int32(free, "free"), _int32(free_count, "free_count", (1,))
        p = PageParams(B, max_pages, page_rows, 0, free.numel())
        _check(lib.elm_page_release(table.data_ptr(), length.data_ptr(), done.data_ptr(), free.data_ptr(), free_count.data_ptr(),
                                    ctypes.byref(p), _stream_of(device)), "elm_page_release")


def cache4_row_bytes(d: int) -> int:
    b = ctypes.c_size_t(0)
    _check(load_library().elm_cache4_row_bytes(d, ctypes.byref(b)), "elm_cache4_row_bytes")
    return int(b.value)


def cache4_pool(n_pages: int, kv_heads: int, page_rows: int, d: int, device="cuda"):
    """An empty pool of rows held in 4 bits: uint8 [n_pages, kv_heads, page_rows, row bytes]."""
    return torch.empty(n_pages, kv_heads, page_rows, cache4_row_bytes(d), dtype=torch.uint8, device=device)


def _pool_d(rows):
    if rows.dtype != torch.uint8 or rows.dim() != 4 or not rows.is_contiguous():
        raise ElmError("rows must be a contiguous uint8 tensor [n_pages, kv_heads, page_rows, row bytes]")
    d = {80: 64, 144: 128}.get(rows.shape[3])
    if d is None:
        raise ElmError(f"rows of {rows.shape[3]} bytes are of no head dimension")
    return d


_append_kept = _Kept()


def cache4_append(rows, K, V, slots, rope: Rope = None, positions=None, Q=None, q_out=None):
    """elm_cache4_append: K, V [T, Hkv, d] into the pool's rows slots [T] (a slot outside the pool: passed over), keys rotated by
    ``rope`` at positions [T].  Q [T, Hq, d] comes back rotated (in q_out, which may be Q; of tokens passed over, as q_out was: without q_out
    those rows are uninitialised memory, NaN possibly)."""
    device = _device(rows, K, V, slots, positions, Q, q_out)
    if device != torch.cuda.current_device():
        with torch.cuda.device(device):
            return cache4_append(rows, K, V, slots, rope, positions, Q, q_out)
    kept = _append_kept if rope is None else rope._kept
    key = (rows.shape, K.shape, K.stride(), K.dtype, V.shape, V.stride(), V.dtype, slots.shape)
    if positions is not None:
        key += (positions.shape,)
    if Q is not None:
        key += (Q.shape, Q.stride(), Q.dtype)
        if q_out is not None:
            key += (q_out.shape, q_out.stride(), q_out.dtype)
    p = kept.get(key)
    if p is None:
        d = _pool_d(rows)
        K2, ks = _rows(K, 3, "K")
        V2, vs = _rows(V, 3, "V")
        Q2, qs = (None, None) if Q is None else _rows(Q, 3, "Q")
        if K2 is not K or V2 is not V or Q2 is not Q:       # (a broadcast of one row)
            if Q2 is not Q and q_out is Q:
                raise ElmError("q_out: rows must lie apart")
            return cache4_append(rows, K2, V2, slots, rope, positions, Q2, q_out)
        T, H = K.shape[:2]
        if K.shape != V.shape or K.dtype != V.dtype or K.shape[2] != d or H != rows.shape[1]:
            raise ElmError("K and V must be [tokens, kv_heads, d] of the pool's heads, of one dtype")
        _int32(slots, "slots", (T,))
        if rope is not None:
            if positions is None:
                raise ElmError("a rotation needs positions")
            _int32(positions, "positions", (T,))
        p = AppendParams(T, 0, H, d, _storage_code(K), rows.shape[2], rows.shape[0])
        if rope is not None:
            p.rotary_dim, p.layout, p.scale, p.inv_freq = rope.rotary_dim, rope.layout, rope.scale, rope._freq_ptr
        p.k_stride[:] = ks[:2]
        p.v_stride[:] = vs[:2]
        if Q is not None:
            if Q.shape[0] != T or Q.shape[2] != d or Q.dtype != K.dtype:
                raise ElmError("Q must be [tokens, q_heads, d] of K's dtype")
            p.q_heads = Q.shape[1]
            p.q_stride[:] = qs[:2]
            if q_out is not None:
                if q_out.shape != Q.shape or q_out.dtype != Q.dtype or q_out.stride(2) != 1:
                    raise ElmError("q_out must have Q's shape and dtype, the numbers of a head side by side")
                if not any(q_out.stride()[:2]) and q_out.numel() > d:
                    raise ElmError("q_out: rows must lie apart")
                p.q_out_stride[:] = q_out.stride()[:2]
        kept.keep(key, p)
    if rows.dtype is not torch.uint8 or not rows.is_contiguous() or slots.dtype is not torch.int32 or not slots.is_contiguous():
        raise ElmError("rows must be contiguous uint8 and slots contiguous int32")
    pos = None
    if rope is not None:
        if positions.dtype is not torch.int32 or not positions.is_contiguous():
            raise ElmError("positions must be contiguous int32")
        pos = positions.data_ptr()
    O = None if Q is None else q_out if q_out is not None else torch.empty_like(Q, memory_format=torch.contiguous_format)
    rc = load_library().elm_cache4_append(_ptr(Q), K.data_ptr(), V.data_ptr(), pos, slots.data_ptr(), p, _ptr(O), rows.data_ptr(), _stream_of(device))
    if rc:
        _check(rc, "elm_cache4_append")
    return O


def _cache4_params(rows, table, q_heads, dtype_code, n_kv, n_q=1, n_tokens=0, causal=True):
    d = _pool_d(rows)
    B, max_pages = _int32(table, "table").shape
    return Cache4Params(B, q_heads, rows.shape[1], d, dtype_code, rows.shape[2], rows.shape[0], max_pages, n_kv, n_q, n_tokens, int(bool(causal)))


_cache4_kept = _Kept()


def cache4_read(rows, table, n: int, idx=None, length=None, dtype=torch.bfloat16, out=None):
    """elm_cache4_read -> K, V [B, Hkv, n, d]: rows 0 .. n - 1 of every request, or rows idx [B, Hkv, n]; a row that is not there (past
    length [B], on no page) is zeros.  ``out``: a pair of tensors for them."""
    device = _device(rows, table, idx, length, *(out or ()))
    if device != torch.cuda.current_device():
        with torch.cuda.device(device):
            return cache4_read(rows, table, n, idx, length, dtype, out)
    key = (rows.shape, table.shape, n, idx if idx is None else idx.shape, length if length is None else length.shape, dtype)
    kept = _cache4_kept.get(key)
    if kept is None:
        code = {torch.float32: ELM_F32, torch.bfloat16: ELM_BF16}.get(dtype)
        if code is None:
            raise ElmError(f"unsupported dtype {dtype}")
        p = _cache4_params(rows, table, rows.shape[1], code, n)
        shape = (p.batch, p.kv_heads, n, p.d)
        if idx is not None:
            _int32(idx, "idx", shape[:3])
        if length is not None:
            _int32(length, "length", shape[:1])
        kept = _cache4_kept.keep(key, (p, shape))
    p, shape = kept
    _int32_all(rows, table, idx, length)
    if out is not None:
        K, V = out
        if any(tuple(t.shape) != shape or t.dtype != dtype or not t.is_contiguous() for t in out):
            raise ElmError(f"out must be two contiguous tensors of shape {shape} and dtype {dtype}")
    else:
        K = torch.empty_strided(shape, (shape[1] * n * shape[3], n * shape[3], shape[3], 1), dtype=dtype, device=rows.device)
        V = torch.empty_like(K)
    rc = load_library().elm_cache4_read(rows.data_ptr(), table.data_ptr(), _ptr(length), _ptr(idx), p, K.data_ptr(), V.data_ptr(), _stream_of(device))
    if rc:
        _check(rc, "elm_cache4_read")
    return K, V


def _int32_all(rows, *tensors):
    if rows.dtype is not torch.uint8 or not rows.is_contiguous():
        raise ElmError("rows must be a contiguous uint8 tensor")
    for t in tensors:
        if t is not None and (t.dtype is not torch.int32 or not t.is_contiguous()):
            raise ElmError("table, length, cu and idx must be contiguous int32 tensors")


def _attend4_params(Q, rows, table, cu, idx, w, length, n_kv, max_q, causal, out):
    if (idx is None) == (length is None):
        raise ElmError("give either length (a request's rows) or idx and w (a list of them)")
    Q2, qs = _rows(Q, 3 if cu is not None else 4, "Q")
    if Q2 is not Q:
        return None                                             # (a broadcast of one row)
    if cu is not None:
        if max_q is None:
            raise ElmError("cu needs max_q, the most tokens of any request")
        T, Hq, d = Q.shape
        p = _cache4_params(rows, table, Hq, _storage_code(Q), 0, max_q, T, causal)
        _int32(cu, "cu", (p.batch + 1,))
        qs = (0, qs[1], qs[0])
    else:
        B, Hq, n_q, d = Q.shape
        p = _cache4_params(rows, table, Hq, _storage_code(Q), 0, n_q, 0, causal)
        if B != p.batch:
            raise ElmError("Q and table must have one batch")
        qs = qs[:3]
    if d != p.d:
        raise ElmError("Q must have the pool's head dimension")
    if idx is not None:
        if cu is not None or w is None or w.dtype != torch.float32 or not w.is_contiguous() or idx.shape != w.shape:
            raise ElmError("idx goes with w, a contiguous float32 tensor of its shape, and with Q [B, Hq, n, d]")
        p.n_kv = _int32(idx, "idx").shape[-1]
        if tuple(idx.shape) != (p.batch, p.kv_heads, p.n_kv):
            raise ElmError("idx must be [B, Hkv, n]")
    else:
        _int32(length, "length", (p.batch,))
        p.n_kv = int(n_kv) if n_kv is not None else 0
    # dense tensors are told to the library as such: its tensor-core form takes no others
    if not Q.is_contiguous() or cu is not None:
        p.q_stride[:] = qs
    if out is not None:
        os_ = out.stride()
        if out.shape != Q.shape or out.dtype != Q.dtype or os_[-1] != 1 or (not any(os_[:-1]) and out.numel() > d):
            raise ElmError("out must have Q's shape and dtype, the numbers of a head side by side")
        if cu is not None:
            p.o_stride[:] = (0, os_[1], os_[0])
        elif not out.is_contiguous():
            p.o_stride[:] = os_[:3]
    return p


def cache4_attend_workspace_bytes(params: Cache4Params, with_list: bool) -> int:
    need = ctypes.c_size_t(0)
    _check(load_library().elm_cache4_attend_workspace_bytes(ctypes.byref(params), int(with_list), ctypes.byref(need)),
           "elm_cache4_attend_workspace_bytes")
    return int(need.value)


def cache4_attend(Q, rows, table, length=None, idx=None, w=None, cu=None, max_q=None, n_kv=None, causal=True, workspace=None, out=None):
    """elm_cache4_attend: Q [B, Hq, n, d] over the rows of the requests of table [B, max_pages]: the first length [B] of them (n_kv: a bound
    of the lengths that the host knows; causal: a request's queries are its last tokens), or the list idx with weights w
    [B, Hkv, n_core].  With cu [B + 1]: Q [T, Hq, d], request b has the tokens cu[b] .. cu[b + 1] - 1, max_q at most.  O like Q: tokens
    outside cu, and those of a request that has more than max_q, are as ``out`` was (without it uninitialised memory, NaN possibly)."""
    device = _device(rows, Q, table, length, idx, w, cu, workspace, out)
    if device != torch.cuda.current_device():
        with torch.cuda.device(device):
            return cache4_attend(Q, rows, table, length, idx, w, cu, max_q, n_kv, causal, workspace, out)
    key = (device, Q.shape, Q.stride(), Q.dtype, rows.shape, table.shape, max_q, n_kv, causal,
           length if length is None else length.shape, cu if cu is None else cu.shape,
           idx if idx is None else (idx.shape, w if w is None else (w.shape, w.dtype, w.is_contiguous())),
           out if out is None else (out.shape, out.stride(), out.dtype))
    kept = _cache4_kept.get(key)
    if kept is None:
        p = _attend4_params(Q, rows, table, cu, idx, w, length, n_kv, max_q, causal, out)
        if p is None:
            if out is Q:
                raise ElmError("out: rows must lie apart")
            return cache4_attend(Q.contiguous(), rows, table, length, idx, w, cu, max_q, n_kv, causal, workspace, out)
        kept = _cache4_kept.keep(key, (p, cache4_attend_workspace_bytes(p, idx is not None)))
    p, need = kept
    _int32_all(rows, table, length, idx, cu)
    ws = workspace if workspace is not None else torch.empty(need, dtype=torch.uint8, device=Q.device)
    O = out if out is not None else torch.empty_like(Q, memory_format=torch.contiguous_format)
    rc = load_library().elm_cache4_attend(Q.data_ptr(), rows.data_ptr(), table.data_ptr(), _ptr(length), _ptr(cu), _ptr(idx), _ptr(w), p,
                                          O.data_ptr(), ws.data_ptr(), ws.numel(), _stream_of(device))
    if rc:
        _check(rc, "elm_cache4_attend")
    return O


def cache4_attend_status(workspace, params: Cache4Params, with_list: bool) -> int:
    """elm_cache4_attend_status: 0 unless a bounded device wait expired during the last cache4_attend call with this workspace."""
    out = ctypes.c_int32(-1)
    device = _device(workspace)
    with torch.cuda.device(device):
        _check(load_library().elm_cache4_attend_status(workspace.data_ptr(), ctypes.byref(params), int(with_list), ctypes.byref(out),
                                                       _stream_of(device)), "elm_cache4_attend_status")
    return int(out.value)


def compress_attend_host(Q, K, V, log2_nout: int, m: int, seed: int = 1, precision="fp32",
                         delta: float = 0.5, scratch=None, out=None, want_coreset=False):
    """elm_compress_attend_host: CPU tensors in, CPU tensor out; copies happen inside the call."""
    lib = load_library()
    if not torch.cuda.is_available():
        raise ElmError("no CUDA device: the library has no CPU fallback")
    for t in (Q, K, V):
        if t.is_cuda or not t.is_contiguous():
            raise ElmError("host call takes contiguous CPU tensors")
    B, Hq, nq, d = Q.shape
    Hkv, n = K.shape[1], K.shape[2]
    p, _ = make_params(B, Hq, Hkv, n, nq, d, log2_nout, m, _dtype_code(Q), precision, delta)
    need = ctypes.c_size_t(0)
    _check(lib.elm_host_call_scratch_bytes(ctypes.byref(p), ctypes.byref(need)), "elm_host_call_scratch_bytes")
    dev = torch.device("cuda", torch.cuda.current_device())
    sc = scratch if scratch is not None else _workspace(int(need.value), dev)
    O = out if out is not None else torch.empty_like(Q)
    n_out = 1 << log2_nout
    idx = torch.empty((B, Hkv, n_out), dtype=torch.int32) if want_coreset else None
    w = torch.empty((B, Hkv, n_out), dtype=torch.float32) if want_coreset else None
    _check(lib.elm_compress_attend_host(Q.data_ptr(), K.data_ptr(), V.data_ptr(), O.data_ptr(),
                                        idx.data_ptr() if want_coreset else None,
                                        w.data_ptr() if want_coreset else None,
                                        ctypes.byref(p), seed, sc.data_ptr(), sc.numel(), _stream()),
           "elm_compress_attend_host")
    return (O, idx, w) if want_coreset else O


def host_call_scratch_bytes(B, Hq, Hkv, n, nq, d, log2_nout, m, dtype, precision="fp32") -> int:
    code = ELM_BF16 if dtype == torch.bfloat16 else ELM_F32
    p, _ = make_params(B, Hq, Hkv, n, nq, d, log2_nout, m, code, precision)
    need = ctypes.c_size_t(0)
    _check(load_library().elm_host_call_scratch_bytes(ctypes.byref(p), ctypes.byref(need)),
           "elm_host_call_scratch_bytes")
    return int(need.value)


def compress_status(workspace, params: ElmParams) -> int:
    """elm_compress_status: 0 unless a bounded device wait expired during the last compress call."""
    out = ctypes.c_int32(-1)
    _check(load_library().elm_compress_status(workspace.data_ptr(), ctypes.byref(params), ctypes.byref(out), _stream()),
           "elm_compress_status")
    return int(out.value)


def attend_status(workspace, params: ElmParams, n_core: int) -> int:
    """elm_attend_status: 0 unless a bounded device wait expired during the last attend call."""
    out = ctypes.c_int32(-1)
    _check(load_library().elm_attend_status(workspace.data_ptr(), ctypes.byref(params), n_core, ctypes.byref(out),
                                            _stream()), "elm_attend_status")
    return int(out.value)


def debug_round_check(B, Hq, Hkv, n, d, log2_nout, mbar, r, seed=1, dtype_code=None, precision="fp32"):
    """elm_debug_round_check (host only): (missing, listed_blocks, needed_blocks, partly_blocks) for Express round r of a prefill, or
    None when that round does not take the one-launch form."""
    lib = load_library()
    p, _ = make_params(B, Hq, Hkv, n, n, d, log2_nout, 0, ELM_BF16 if dtype_code is None else dtype_code, precision)
    out = [ctypes.c_int64(0) for _ in range(4)]
    rc = lib.elm_debug_round_check(ctypes.byref(p), mbar, r, seed, *[ctypes.byref(o) for o in out])
    if rc == -2:                     # ELM_ERR_SHAPE: the round is taken in windows
        return None
    _check(rc, "elm_debug_round_check")
    return tuple(int(o.value) for o in out)


def debug_decode_grid(B, Hq, Hkv, n, d, n_core, n_q=1, dtype_code=None):
    """elm_debug_decode_grid: (CTAs a decode call launches, CTAs the device holds at once)."""
    lib = load_library()
    p, _ = make_params(B, Hq, Hkv, n, n_q, d, n.bit_length() - 1, 0, ELM_BF16 if dtype_code is None else dtype_code)
    ctas, resident = ctypes.c_int32(0), ctypes.c_int32(0)
    _check(lib.elm_debug_decode_grid(ctypes.byref(p), n_core, ctypes.byref(ctas), ctypes.byref(resident)), "elm_debug_decode_grid")
    return int(ctas.value), int(resident.value)


def debug_stream_form(B, Hq, Hkv, n, d, seen, tokens) -> int:
    """elm_debug_stream_form: how a stream's call over bf16 rows attends these tokens (0 one by one, 1 clusters, 2 CTAs that walk)."""
    p, _ = make_params(B, Hq, Hkv, n, 1, d, n.bit_length() - 1, 0, ELM_BF16)
    form = ctypes.c_int32(-1)
    _check(load_library().elm_debug_stream_form(ctypes.byref(p), seen, tokens, ctypes.byref(form)), "elm_debug_stream_form")
    return int(form.value)


def profile_enable(on=True):
    """0 / False: off; 1 / True: every stage; 2: the attention stage only (see include/elm.h)."""
    _check(load_library().elm_profile_enable(int(on)), "elm_profile_enable")


def profile_read():
    """Per-stage (milliseconds, launches) since the last read, as a dict keyed by stage name."""
    n = len(STAGE_NAMES)
    ms = (ctypes.c_float * n)()
    ln = (ctypes.c_int64 * n)()
    _check(load_library().elm_profile_read(ms, ln, n), "elm_profile_read")
    return {STAGE_NAMES[i]: (float(ms[i]), int(ln[i])) for i in range(n)}


def launch_count() -> int:
    return int(load_library().elm_launch_count())
