"""ctypes binding of libexfold.so: argument marshalling only.

Every function has the name and the arguments of its C counterpart in include/exfold.h;
tensors are torch tensors whose data pointers are passed through. All computation happens
in the CUDA library; there is no fallback: if the library is missing, importing fails.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libexfold.so")

EXFOLD_F32, EXFOLD_BF16 = 0, 1
EXFOLD_OK = 0
EXFOLD_ERR_INVALID_ARG = -1
EXFOLD_ERR_UNSUPPORTED = -2
EXFOLD_ERR_WORKSPACE_TOO_SMALL = -3
EXFOLD_ERR_CUDA = -4
EXFOLD_ERR_DEVICE_TIMEOUT = -5
EXFOLD_ERR_EXCEEDS_STATIC_SCRATCH = -6
EXFOLD_STATIC_SCRATCH_BYTES = 8 << 20
EXFOLD_WARN_UNOBSERVED_EXPERT = 1
SCORES = {"softmax": 0, "sigmoid": 1}
GROUP_SCORES = {"max": 0, "top2": 1}
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}

EXPORTS = ["exfold_workspace_bytes", "exfold_host_staging_bytes", "exfold_calibrate", "exfold_moe_prefill",
           "exfold_moe_decode", "exfold_moe_prefill_host", "exfold_moe_decode_host", "exfold_device_status",
           "exfold_status_string", "exfold_launch_count", "exfold_profile_enable", "exfold_profile_read",
           "exfold_moe_decode_noalloc", "exfold_static_pool_build", "exfold_moe_decode_static",
           "exfold_moe_prefill_ex", "exfold_router_logits", "exfold_calibrate_layers", "exfold_device_status_noalloc",
           "exfold_static_scratch_address", "exfold_thread_release", "exfold_moe_prefill_layer", "exfold_moe_decode_layer",
           "exfold_route", "exfold_route_backward", "exfold_moe_prefill_routed", "exfold_moe_decode_routed",
           "exfold_linear_workspace_bytes", "exfold_linear"]
PROFILE_SLOTS = ["prefill_route", "prefill_scan", "prefill_scatter", "gemm1_gateup_swiglu", "gemm2_down_combine",
                 "convert_bf16", "decode_route", "decode_gather", "decode_gateup", "decode_down", "ffn_f32",
                 "combine_f32", "gemm1_pair_pass", "gemm2_pair_pass", "decode_ffn"]


class exfold_layer(C.Structure):
    _fields_ = [("n_experts", C.c_int32), ("n_shared", C.c_int32), ("hidden", C.c_int32), ("inter", C.c_int32),
                ("top_k", C.c_int32), ("dtype", C.c_int32)]


class exfold_tables(C.Structure):
    _fields_ = [("S", C.c_void_p), ("L", C.c_void_p), ("h", C.c_void_p), ("lnh", C.c_void_p), ("n_obs", C.c_void_p)]


class exfold_calib_opts(C.Structure):
    _fields_ = [("lambda_", C.c_float), ("clip_lo", C.c_float), ("clip_hi", C.c_float), ("eps", C.c_float),
                ("mode", C.c_int32)]


class exfold_calib_job(C.Structure):
    _fields_ = [("x_cal", C.c_void_p), ("logits_cal", C.c_void_p), ("m", C.c_int64), ("w_gate", C.c_void_p),
                ("w_up", C.c_void_p), ("w_down", C.c_void_p), ("out", C.POINTER(exfold_tables))]


class exfold_prefill_meta(C.Structure):
    _fields_ = [("ids", C.c_void_p), ("w", C.c_void_p), ("omit_src", C.c_void_p), ("omit_tgt", C.c_void_p),
                ("perm", C.c_void_p), ("offsets", C.c_void_p)]


class exfold_decode_meta(C.Structure):
    _fields_ = [("pool_ids", C.c_void_p), ("pool_size", C.c_void_p), ("pool_mask", C.c_void_p), ("ids", C.c_void_p),
                ("w", C.c_void_p), ("target", C.c_void_p), ("scale", C.c_void_p)]


class exfold_fold_opts(C.Structure):
    _fields_ = [("loss_threshold", C.c_float), ("rescale", C.c_int32), ("confidence_split", C.c_int32),
                ("gemm_path", C.c_int32)]


class exfold_static_pool(C.Structure):
    _fields_ = [("pool_ids", C.c_void_p), ("target", C.c_void_p), ("scale", C.c_void_p), ("pool_m", C.c_int32)]


class exfold_router(C.Structure):
    bias_tensor = None  # make_router: what `bias` points to
    _fields_ = [("score", C.c_int32), ("n_groups", C.c_int32), ("top_groups", C.c_int32), ("group_score", C.c_int32),
                ("renormalise", C.c_int32), ("scale", C.c_float), ("bias", C.c_void_p)]


class exfold_linear_desc(C.Structure):
    _fields_ = [("in_features", C.c_int64), ("out_features", C.c_int64), ("dtype", C.c_int32), ("out_dtype", C.c_int32),
                ("activation", C.c_int32), ("ldx", C.c_int64), ("ldw", C.c_int64), ("ldy", C.c_int64), ("ldr", C.c_int64)]


def _load() -> C.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: run `python -m paper_2608_24938_b200.build` "
                          "(there is no CPU or PyTorch fallback)")
    lib = C.CDLL(LIB_PATH)
    vp, i64, i32, sz = C.c_void_p, C.c_int64, C.c_int32, C.c_size_t
    lib.exfold_workspace_bytes.restype = sz
    lib.exfold_workspace_bytes.argtypes = [C.POINTER(exfold_layer), i64, i32]
    lib.exfold_host_staging_bytes.restype = sz
    lib.exfold_host_staging_bytes.argtypes = [C.POINTER(exfold_layer), i64]
    lib.exfold_calibrate.restype = C.c_int
    lib.exfold_calibrate.argtypes = [C.POINTER(exfold_layer), vp, vp, i64, vp, vp, vp, C.POINTER(exfold_calib_opts),
                                     C.POINTER(exfold_tables), vp, sz, vp]
    lib.exfold_calibrate_layers.restype = C.c_int
    lib.exfold_calibrate_layers.argtypes = [C.POINTER(exfold_layer), C.POINTER(exfold_calib_job), i32,
                                            C.POINTER(exfold_calib_opts), C.POINTER(C.c_int32), vp, sz, vp]
    for fn in (lib.exfold_moe_prefill, lib.exfold_moe_prefill_host):
        fn.restype = C.c_int
        fn.argtypes = [C.POINTER(exfold_layer), vp, vp, i64, vp, vp, vp, C.POINTER(exfold_tables), i32, vp,
                       C.POINTER(exfold_prefill_meta), vp, sz, vp]
    for fn in (lib.exfold_moe_decode, lib.exfold_moe_decode_host):
        fn.restype = C.c_int
        fn.argtypes = [C.POINTER(exfold_layer), vp, vp, i64, vp, vp, vp, C.POINTER(exfold_tables), i32, vp,
                       C.POINTER(exfold_decode_meta), vp, sz, vp]
    lib.exfold_moe_prefill_layer.restype = C.c_int
    lib.exfold_moe_prefill_layer.argtypes = [C.POINTER(exfold_layer), vp, vp, i64, vp, vp, vp, C.POINTER(exfold_tables),
                                             i32, vp, vp, C.POINTER(exfold_prefill_meta), vp, sz, vp]
    lib.exfold_moe_decode_layer.restype = C.c_int
    lib.exfold_moe_decode_layer.argtypes = [C.POINTER(exfold_layer), vp, vp, i64, vp, vp, vp, C.POINTER(exfold_tables),
                                            i32, vp, vp, C.POINTER(exfold_decode_meta), vp, sz, vp]
    lib.exfold_moe_decode_noalloc.restype = C.c_int
    lib.exfold_moe_decode_noalloc.argtypes = [C.POINTER(exfold_layer), vp, vp, i64, vp, vp, vp, C.POINTER(exfold_tables),
                                              i32, vp, C.POINTER(exfold_decode_meta), vp]
    lib.exfold_moe_prefill_ex.restype = C.c_int
    lib.exfold_moe_prefill_ex.argtypes = [C.POINTER(exfold_layer), vp, vp, i64, vp, vp, vp, C.POINTER(exfold_tables), i32,
                                          C.POINTER(exfold_fold_opts), vp, C.POINTER(exfold_prefill_meta), vp, sz, vp]
    lib.exfold_router_logits.restype = C.c_int
    lib.exfold_router_logits.argtypes = [C.POINTER(exfold_layer), vp, vp, i64, vp, vp, sz, vp]
    lib.exfold_static_pool_build.restype = C.c_int
    lib.exfold_static_pool_build.argtypes = [C.POINTER(exfold_layer), C.POINTER(exfold_tables), i32,
                                             C.POINTER(exfold_static_pool), vp]
    lib.exfold_moe_decode_static.restype = C.c_int
    lib.exfold_moe_decode_static.argtypes = [C.POINTER(exfold_layer), vp, vp, i64, vp, vp, vp,
                                             C.POINTER(exfold_static_pool), vp, C.POINTER(exfold_decode_meta), vp, sz, vp]
    lib.exfold_route.restype = C.c_int
    lib.exfold_route.argtypes = [C.POINTER(exfold_layer), vp, i64, C.POINTER(exfold_router), vp, vp, vp, vp]
    lib.exfold_route_backward.restype = C.c_int
    lib.exfold_route_backward.argtypes = [C.POINTER(exfold_layer), vp, vp, vp, i64, C.POINTER(exfold_router), vp, vp]
    lib.exfold_moe_prefill_routed.restype = C.c_int
    lib.exfold_moe_prefill_routed.argtypes = [C.POINTER(exfold_layer), vp, vp, vp, i64, vp, vp, vp, C.POINTER(exfold_tables), i32,
                                              C.POINTER(exfold_fold_opts), vp, C.POINTER(exfold_prefill_meta), vp, sz, vp]
    lib.exfold_moe_decode_routed.restype = C.c_int
    lib.exfold_moe_decode_routed.argtypes = [C.POINTER(exfold_layer), vp, vp, vp, i64, vp, vp, vp, C.POINTER(exfold_tables), i32,
                                             vp, C.POINTER(exfold_decode_meta), vp, sz, vp]
    lib.exfold_linear_workspace_bytes.restype = sz
    lib.exfold_linear_workspace_bytes.argtypes = [C.POINTER(exfold_linear_desc), i64]
    lib.exfold_linear.restype = C.c_int
    lib.exfold_linear.argtypes = [C.POINTER(exfold_linear_desc), vp, vp, vp, vp, i64, vp, vp, sz, vp]
    lib.exfold_device_status.restype = C.c_int
    lib.exfold_device_status.argtypes = [vp, vp]
    lib.exfold_device_status_noalloc.restype = C.c_int
    lib.exfold_device_status_noalloc.argtypes = [vp]
    lib.exfold_static_scratch_address.restype = C.c_int
    lib.exfold_static_scratch_address.argtypes = [C.POINTER(vp)]
    lib.exfold_thread_release.restype = C.c_int
    lib.exfold_thread_release.argtypes = []
    lib.exfold_status_string.restype = C.c_char_p
    lib.exfold_status_string.argtypes = [C.c_int]
    lib.exfold_launch_count.restype = i64
    lib.exfold_launch_count.argtypes = []
    lib.exfold_profile_enable.restype = C.c_int
    lib.exfold_profile_enable.argtypes = [C.c_int]
    lib.exfold_profile_read.restype = C.c_int
    lib.exfold_profile_read.argtypes = [C.POINTER(C.c_float), i32]
    return lib


lib = _load()


class ExfoldError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: {exfold_status_string(code)} ({code})")
        self.code = code


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    assert t.is_contiguous(), "tensors passed to the library must be contiguous"
    return t.data_ptr()


def _stream(stream: Optional[torch.cuda.Stream]) -> int:
    # the raw handle of the current stream: torch.cuda.current_stream() builds a Stream object first, 3.3 us per call
    return stream.cuda_stream if stream is not None else torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def make_layer(n_experts: int, n_shared: int, hidden: int, inter: int, top_k: int, dtype) -> exfold_layer:
    if isinstance(dtype, torch.dtype):
        dtype = {torch.float32: EXFOLD_F32, torch.bfloat16: EXFOLD_BF16}[dtype]
    elif isinstance(dtype, str):
        dtype = {"f32": EXFOLD_F32, "bf16": EXFOLD_BF16}[dtype]
    return exfold_layer(n_experts, n_shared, hidden, inter, top_k, dtype)


def make_tables(S, L, h, lnh, n_obs=None) -> exfold_tables:
    for t in (S, L, h, lnh):
        assert t.dtype == torch.float32
    return exfold_tables(_ptr(S), _ptr(L), _ptr(h), _ptr(lnh), _ptr(n_obs))


def exfold_status_string(code: int) -> str:
    return lib.exfold_status_string(code).decode()


def exfold_launch_count() -> int:
    return int(lib.exfold_launch_count())


def exfold_profile_enable(enable: bool) -> int:
    return int(lib.exfold_profile_enable(1 if enable else 0))


def exfold_profile_read() -> dict:
    """Milliseconds of each kernel of the last call (kernels that did not run are left out)."""
    n = len(PROFILE_SLOTS)
    buf = (C.c_float * n)()
    rc = lib.exfold_profile_read(buf, n)
    if rc != 0:
        raise ExfoldError(rc, "exfold_profile_read")
    return {PROFILE_SLOTS[i]: float(buf[i]) for i in range(n) if buf[i] >= 0}


def exfold_workspace_bytes(layer: exfold_layer, max_tokens: int, routes_per_token: int) -> int:
    return int(lib.exfold_workspace_bytes(C.byref(layer), max_tokens, routes_per_token))


def exfold_host_staging_bytes(layer: exfold_layer, max_tokens: int) -> int:
    return int(lib.exfold_host_staging_bytes(C.byref(layer), max_tokens))


def alloc_workspace(layer: exfold_layer, max_tokens: int, routes_per_token: int, device="cuda",
                    host_staging: bool = False) -> torch.Tensor:
    n = exfold_workspace_bytes(layer, max_tokens, routes_per_token)
    if n == 0:
        raise ExfoldError(EXFOLD_ERR_INVALID_ARG, "exfold_workspace_bytes")
    if host_staging:
        n += exfold_host_staging_bytes(layer, max_tokens)
    return torch.empty(n, dtype=torch.uint8, device=device)


def exfold_router_logits(layer, x, w_router, logits, ws, stream=None) -> int:
    return int(lib.exfold_router_logits(C.byref(layer), _ptr(x), _ptr(w_router), x.shape[0], _ptr(logits), _ptr(ws),
                                        ws.numel(), _stream(stream)))


def exfold_device_status(ws: torch.Tensor, stream=None) -> int:
    return int(lib.exfold_device_status(_ptr(ws), _stream(stream)))


def exfold_device_status_noalloc(stream=None) -> int:
    return int(lib.exfold_device_status_noalloc(_stream(stream)))


def exfold_static_scratch_address() -> int:
    out = C.c_void_p()
    rc = lib.exfold_static_scratch_address(C.byref(out))
    if rc != 0:
        raise ExfoldError(rc, "exfold_static_scratch_address")
    return int(out.value)


def exfold_thread_release() -> int:
    return int(lib.exfold_thread_release())


def exfold_calibrate(layer, x_cal, logits_cal, w_gate, w_up, w_down, out: exfold_tables, ws, lam=1e-3,
                     clip_lo=-4.0, clip_hi=4.0, eps=1e-12, mode=0, stream=None) -> int:
    opts = exfold_calib_opts(lam, clip_lo, clip_hi, eps, mode)
    rc = lib.exfold_calibrate(C.byref(layer), _ptr(x_cal), _ptr(logits_cal), x_cal.shape[0], _ptr(w_gate),
                              _ptr(w_up), _ptr(w_down), C.byref(opts), C.byref(out), _ptr(ws), ws.numel(),
                              _stream(stream))
    if rc < 0:
        raise ExfoldError(rc, "exfold_calibrate")
    return rc


def exfold_calibrate_layers(layer, jobs, ws, lam=1e-3, clip_lo=-4.0, clip_hi=4.0, eps=1e-12, mode=0, stream=None):
    """jobs: sequence of (x_cal, logits_cal, w_gate, w_up, w_down, out_tables). Returns (status, unobserved per job)."""
    opts = exfold_calib_opts(lam, clip_lo, clip_hi, eps, mode)
    arr = (exfold_calib_job * len(jobs))()
    for j, (x_cal, logits_cal, w_gate, w_up, w_down, out) in enumerate(jobs):
        arr[j] = exfold_calib_job(_ptr(x_cal), _ptr(logits_cal), x_cal.shape[0], _ptr(w_gate), _ptr(w_up),
                                  _ptr(w_down), C.pointer(out))
    un = (C.c_int32 * len(jobs))()
    rc = lib.exfold_calibrate_layers(C.byref(layer), arr, len(jobs), C.byref(opts), un, _ptr(ws), ws.numel(),
                                     _stream(stream))
    if rc < 0:
        raise ExfoldError(rc, "exfold_calibrate_layers")
    return rc, list(un)


def _prefill_meta(meta: Optional[dict]):
    if not meta:
        return None
    return C.byref(exfold_prefill_meta(*[_ptr(meta.get(k)) for k in
                                         ("ids", "w", "omit_src", "omit_tgt", "perm", "offsets")]))


def _decode_meta(meta: Optional[dict]):
    if not meta:
        return None
    return C.byref(exfold_decode_meta(*[_ptr(meta.get(k)) for k in
                                        ("pool_ids", "pool_size", "pool_mask", "ids", "w", "target", "scale")]))


def exfold_moe_prefill(layer, x, logits, w_gate, w_up, w_down, tables: exfold_tables, k_pre: int, y, ws,
                       meta: Optional[dict] = None, stream=None, check: bool = True) -> int:
    rc = lib.exfold_moe_prefill(C.byref(layer), _ptr(x), _ptr(logits), x.shape[0], _ptr(w_gate), _ptr(w_up),
                                _ptr(w_down), C.byref(tables), k_pre, _ptr(y), _prefill_meta(meta), _ptr(ws),
                                ws.numel(), _stream(stream))
    if check and rc != 0:
        raise ExfoldError(rc, "exfold_moe_prefill")
    return rc


def exfold_moe_decode(layer, x, logits, w_gate, w_up, w_down, tables: exfold_tables, pool_m: int, y, ws,
                      meta: Optional[dict] = None, stream=None, check: bool = True) -> int:
    rc = lib.exfold_moe_decode(C.byref(layer), _ptr(x), _ptr(logits), x.shape[0], _ptr(w_gate), _ptr(w_up),
                               _ptr(w_down), C.byref(tables), pool_m, _ptr(y), _decode_meta(meta), _ptr(ws),
                               ws.numel(), _stream(stream))
    if check and rc != 0:
        raise ExfoldError(rc, "exfold_moe_decode")
    return rc


def exfold_moe_prefill_layer(layer, x, w_router, w_gate, w_up, w_down, tables: exfold_tables, k_pre: int, y, ws,
                             logits_out, meta: Optional[dict] = None, stream=None, check: bool = True) -> int:
    rc = lib.exfold_moe_prefill_layer(C.byref(layer), _ptr(x), _ptr(w_router), x.shape[0], _ptr(w_gate), _ptr(w_up),
                                      _ptr(w_down), C.byref(tables), k_pre, _ptr(logits_out), _ptr(y),
                                      _prefill_meta(meta), _ptr(ws), ws.numel(), _stream(stream))
    if check and rc != 0:
        raise ExfoldError(rc, "exfold_moe_prefill_layer")
    return rc


def exfold_moe_decode_layer(layer, x, w_router, w_gate, w_up, w_down, tables: exfold_tables, pool_m: int, y, ws,
                            logits_out, meta: Optional[dict] = None, stream=None, check: bool = True) -> int:
    rc = lib.exfold_moe_decode_layer(C.byref(layer), _ptr(x), _ptr(w_router), x.shape[0], _ptr(w_gate), _ptr(w_up),
                                     _ptr(w_down), C.byref(tables), pool_m, _ptr(logits_out), _ptr(y),
                                     _decode_meta(meta), _ptr(ws), ws.numel(), _stream(stream))
    if check and rc != 0:
        raise ExfoldError(rc, "exfold_moe_decode_layer")
    return rc


def exfold_moe_prefill_host(layer, x_host, logits_host, w_gate, w_up, w_down, tables, k_pre, y_host, ws,
                            meta=None, stream=None, check: bool = True) -> int:
    rc = lib.exfold_moe_prefill_host(C.byref(layer), _ptr(x_host), _ptr(logits_host), x_host.shape[0], _ptr(w_gate),
                                     _ptr(w_up), _ptr(w_down), C.byref(tables), k_pre, _ptr(y_host),
                                     _prefill_meta(meta), _ptr(ws), ws.numel(), _stream(stream))
    if check and rc != 0:
        raise ExfoldError(rc, "exfold_moe_prefill_host")
    return rc


def exfold_moe_decode_host(layer, x_host, logits_host, w_gate, w_up, w_down, tables, pool_m, y_host, ws,
                           meta=None, stream=None, check: bool = True) -> int:
    rc = lib.exfold_moe_decode_host(C.byref(layer), _ptr(x_host), _ptr(logits_host), x_host.shape[0], _ptr(w_gate),
                                    _ptr(w_up), _ptr(w_down), C.byref(tables), pool_m, _ptr(y_host),
                                    _decode_meta(meta), _ptr(ws), ws.numel(), _stream(stream))
    if check and rc != 0:
        raise ExfoldError(rc, "exfold_moe_decode_host")
    return rc


def exfold_moe_decode_noalloc(layer, x, logits, w_gate, w_up, w_down, tables: exfold_tables, pool_m: int, y,
                              meta: Optional[dict] = None, stream=None, check: bool = True) -> int:
    """Decode without a caller workspace, for hosts that may not allocate device memory: the scratch is
    the library's own fixed array (EXFOLD_STATIC_SCRATCH_BYTES per GPU). Same results as
    exfold_moe_decode. Calls on one device share that array, so keep them ordered on one stream; make
    the first call on a device outside any stream capture."""
    rc = lib.exfold_moe_decode_noalloc(C.byref(layer), _ptr(x), _ptr(logits), x.shape[0], _ptr(w_gate), _ptr(w_up),
                                       _ptr(w_down), C.byref(tables), pool_m, _ptr(y), _decode_meta(meta),
                                       _stream(stream))
    if check and rc != 0:
        raise ExfoldError(rc, "exfold_moe_decode_noalloc")
    return rc


def exfold_static_pool_build(layer, tables: exfold_tables, pool_m: int, pool_ids, target, scale,
                             stream=None) -> exfold_static_pool:
    """Fills the caller's device arrays pool_ids [M], target [N], scale [N] and returns the struct to pass to
    exfold_moe_decode_static (the tensors must stay alive as long as the struct is used)."""
    sp = exfold_static_pool(_ptr(pool_ids), _ptr(target), _ptr(scale), pool_m)
    rc = lib.exfold_static_pool_build(C.byref(layer), C.byref(tables), pool_m, C.byref(sp), _stream(stream))
    if rc != 0:
        raise ExfoldError(rc, "exfold_static_pool_build")
    return sp


def exfold_moe_decode_static(layer, x, logits, w_gate, w_up, w_down, pool: exfold_static_pool, y, ws,
                             meta: Optional[dict] = None, stream=None, check: bool = True) -> int:
    rc = lib.exfold_moe_decode_static(C.byref(layer), _ptr(x), _ptr(logits), x.shape[0], _ptr(w_gate), _ptr(w_up),
                                      _ptr(w_down), C.byref(pool), _ptr(y), _decode_meta(meta), _ptr(ws), ws.numel(),
                                      _stream(stream))
    if check and rc != 0:
        raise ExfoldError(rc, "exfold_moe_decode_static")
    return rc


def exfold_moe_prefill_ex(layer, x, logits, w_gate, w_up, w_down, tables: exfold_tables, k_pre: int, y, ws,
                          loss_threshold: float = float("inf"), rescale: bool = False, confidence_split: bool = False,
                          gemm_path: int = 0, meta: Optional[dict] = None, stream=None, check: bool = True) -> int:
    opts = exfold_fold_opts(loss_threshold, int(rescale), int(confidence_split), int(gemm_path))
    rc = lib.exfold_moe_prefill_ex(C.byref(layer), _ptr(x), _ptr(logits), x.shape[0], _ptr(w_gate), _ptr(w_up),
                                   _ptr(w_down), C.byref(tables), k_pre, C.byref(opts), _ptr(y), _prefill_meta(meta),
                                   _ptr(ws), ws.numel(), _stream(stream))
    if check and rc != 0:
        raise ExfoldError(rc, "exfold_moe_prefill_ex")
    return rc


def make_router(score: str = "softmax", bias: Optional[torch.Tensor] = None, n_groups: int = 1, top_groups: int = 1,
                group_score: str = "max", renormalise: bool = True, scale: float = 1.0) -> exfold_router:
    """A model's own router (exfold_route). `bias`: fp32 [N] on the device, kept alive by the returned struct."""
    assert bias is None or bias.dtype == torch.float32
    r = exfold_router(SCORES[score], n_groups, top_groups, GROUP_SCORES[group_score], int(renormalise), scale, _ptr(bias))
    r.bias_tensor = bias
    return r


def _here(*tensors) -> None:
    """The calls run on the current device: its tensors only (not the host's, nor another GPU's)."""
    dev = torch._C._cuda_getDevice()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise AssertionError(f"tensor on {t.device}, the current device is cuda:{dev}")


def _typed(t: Optional[torch.Tensor], dtype, shape) -> Optional[int]:
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        raise AssertionError(f"expected contiguous {dtype} {tuple(shape)}, got {t.dtype} {tuple(t.shape)} {t.stride()}")
    return t.data_ptr()


def exfold_route(layer, logits, router: exfold_router, ids, w, load=None, stream=None, check: bool = True) -> int:
    """logits [T][N] fp32 -> ids [T][K] int32, w [T][K] fp32, load [N] int32 (tokens per expert)."""
    (T, N), K, bias = logits.shape, layer.top_k, router.bias_tensor
    if not (logits.dtype is torch.float32 and N == layer.n_experts and ids.dtype is torch.int32 and w.dtype is torch.float32 and
            ids.shape == w.shape == (T, K) and logits.is_contiguous() and ids.is_contiguous() and w.is_contiguous()):
        _typed(logits, torch.float32, (T, layer.n_experts)), _typed(ids, torch.int32, (T, K)), _typed(w, torch.float32, (T, K))
    if bias is not None and bias.shape != (N,):
        raise AssertionError(f"expected a bias of {N} experts, got {tuple(bias.shape)}")
    load_ptr = _typed(load, torch.int32, (N,)) if load is not None else None
    dev = torch._C._cuda_getDevice()
    if not (logits.get_device() == ids.get_device() == w.get_device() == dev and (bias is None or bias.get_device() == dev) and
            (load is None or load.get_device() == dev)):
        _here(logits, bias, ids, w, load)
    rc = lib.exfold_route(layer, logits.data_ptr(), T, router, ids.data_ptr(), w.data_ptr(), load_ptr,
                          stream.cuda_stream if stream is not None else torch._C._cuda_getCurrentRawStream(dev))
    if check and rc != 0:
        raise ExfoldError(rc, "exfold_route")
    return rc


def exfold_route_backward(layer, logits, ids, dw, router: exfold_router, dlogits, stream=None, check: bool = True) -> int:
    """dw [T][K], the gradient of exfold_route's weights -> dlogits [T][N]."""
    (T, N), K = logits.shape, layer.top_k
    if not (logits.dtype is dw.dtype is dlogits.dtype is torch.float32 and ids.dtype is torch.int32 and N == layer.n_experts and
            ids.shape == dw.shape == (T, K) and dlogits.shape == logits.shape and logits.is_contiguous() and ids.is_contiguous() and
            dw.is_contiguous() and dlogits.is_contiguous()):
        _typed(logits, torch.float32, (T, layer.n_experts)), _typed(ids, torch.int32, (T, K)), _typed(dw, torch.float32, (T, K))
        _typed(dlogits, torch.float32, (T, N))
    dev = torch._C._cuda_getDevice()
    if not logits.get_device() == ids.get_device() == dw.get_device() == dlogits.get_device() == dev:
        _here(logits, ids, dw, dlogits)
    rc = lib.exfold_route_backward(layer, logits.data_ptr(), ids.data_ptr(), dw.data_ptr(), T, router, dlogits.data_ptr(),
                                   stream.cuda_stream if stream is not None else torch._C._cuda_getCurrentRawStream(dev))
    if check and rc != 0:
        raise ExfoldError(rc, "exfold_route_backward")
    return rc


def exfold_moe_prefill_routed(layer, x, ids, w, w_gate, w_up, w_down, tables: Optional[exfold_tables], k_pre: int, y, ws,
                              loss_threshold: float = float("inf"), rescale: bool = False, confidence_split: bool = False,
                              gemm_path: int = 0, meta: Optional[dict] = None, stream=None, check: bool = True) -> int:
    """exfold_moe_prefill_ex on given routes ids, w [T][K]. tables may be None where k_pre = K."""
    T, K = x.shape[0], layer.top_k
    opts = exfold_fold_opts(loss_threshold, int(rescale), int(confidence_split), int(gemm_path))
    _here(x, ids, w, w_gate, w_up, w_down, y, ws)
    rc = lib.exfold_moe_prefill_routed(C.byref(layer), _ptr(x), _typed(ids, torch.int32, (T, K)),
                                       _typed(w, torch.float32, (T, K)), T, _ptr(w_gate), _ptr(w_up), _ptr(w_down),
                                       C.byref(tables) if tables is not None else None, k_pre, C.byref(opts), _ptr(y),
                                       _prefill_meta(meta), _ptr(ws), ws.numel(), _stream(stream))
    if check and rc != 0:
        raise ExfoldError(rc, "exfold_moe_prefill_routed")
    return rc


def exfold_moe_decode_routed(layer, x, ids, w, w_gate, w_up, w_down, tables: exfold_tables, pool_m: int, y, ws,
                             meta: Optional[dict] = None, stream=None, check: bool = True) -> int:
    """exfold_moe_decode on given routes ids, w [B][K]."""
    B, K = x.shape[0], layer.top_k
    _here(x, ids, w, w_gate, w_up, w_down, y, ws)
    rc = lib.exfold_moe_decode_routed(C.byref(layer), _ptr(x), _typed(ids, torch.int32, (B, K)),
                                      _typed(w, torch.float32, (B, K)), B, _ptr(w_gate), _ptr(w_up), _ptr(w_down),
                                      C.byref(tables), pool_m, _ptr(y), _decode_meta(meta), _ptr(ws), ws.numel(),
                                      _stream(stream))
    if check and rc != 0:
        raise ExfoldError(rc, "exfold_moe_decode_routed")
    return rc


_LINEAR_DTYPES = {torch.float32: EXFOLD_F32, torch.bfloat16: EXFOLD_BF16}


def _rows(t: torch.Tensor, dtype, rows: int, cols: int) -> int:
    """Row distance of a matrix whose rows are contiguous (0: dense)."""
    assert t.dtype == dtype and t.shape == (rows, cols), f"expected {dtype} {(rows, cols)}, got {t.dtype} {tuple(t.shape)}"
    ld, step = t.stride()
    assert step == 1 or cols == 1, "rows must be contiguous"
    if rows <= 1 and not cols <= ld < 1 << 31:
        return 0
    assert ld >= cols, "rows must not overlap"
    return ld


@functools.lru_cache(maxsize=1024)
def _linear_desc(*fields):
    return C.byref(exfold_linear_desc(*fields))  # by value of its fields; making one costs 2 us of a call


def exfold_linear_workspace_bytes(desc: exfold_linear_desc, max_tokens: int) -> int:
    return int(lib.exfold_linear_workspace_bytes(C.byref(desc), max_tokens))


def alloc_linear_workspace(in_features: int, out_features: int, max_tokens: int, dtype, out_dtype=None, device="cuda",
                           ldx: int = 0, ldw: int = 0) -> torch.Tensor:
    """Workspace of exfold_linear for products of this shape with up to max_tokens rows, ldx and ldw elements apart (0: dense)."""
    desc = exfold_linear_desc(in_features, out_features, _LINEAR_DTYPES[dtype], _LINEAR_DTYPES[out_dtype or dtype], 0, ldx, ldw, 0, 0)
    n = exfold_linear_workspace_bytes(desc, max_tokens)
    if n == 0:
        raise ExfoldError(EXFOLD_ERR_INVALID_ARG, "exfold_linear_workspace_bytes")
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    ws[:256].zero_()  # the status record: a call without tokens leaves it as it is
    return ws


def exfold_linear(x, w, y, ws, bias=None, residual=None, activation: str = "none", stream=None, check: bool = True) -> int:
    """y = act(x w^T + bias) + residual. x [T][in], w [out][in], bias [out] of one type; y, residual [T][out]. The matrices may
    have any distance between their rows."""
    T, i = x.shape
    o, dt, out, ldr, rp, bp = w.shape[0], x.dtype, y.dtype, 0, None, None
    (ldx, sx), (ldw, sw), (ldy, sy) = x.stride(), w.stride(), y.stride()
    if not (sx == sw == sy == 1 and ldx >= i and ldw >= i and ldy >= o and w.shape[1] == i and w.dtype is dt and y.shape == (T, o)):
        ldx, ldw, ldy = _rows(x, dt, T, i), _rows(w, dt, o, i), _rows(y, out, T, o)  # matrices of one row or column, or not usable
    if residual is not None:
        ldr, sr = residual.stride()
        if not (sr == 1 and ldr >= o and residual.dtype is out and residual.shape == y.shape):
            ldr = _rows(residual, out, T, o)
        rp = residual.data_ptr()
    if bias is not None:
        if bias.dtype is not dt or bias.shape != (o,) or not bias.is_contiguous():
            raise AssertionError(f"expected bias {dt} {(o,)}, got {bias.dtype} {tuple(bias.shape)}")
        bp = bias.data_ptr()
    dev = torch._C._cuda_getDevice()
    if not (x.get_device() == w.get_device() == y.get_device() == ws.get_device() == dev and (bp is None or bias.get_device() == dev) and
            (rp is None or residual.get_device() == dev)):
        _here(x, w, bias, residual, y, ws)
    rc = lib.exfold_linear(_linear_desc(i, o, _LINEAR_DTYPES[dt], _LINEAR_DTYPES[out], ACTIVATIONS[activation], ldx, ldw, ldy, ldr),
                           x.data_ptr(), w.data_ptr(), bp, rp, T, y.data_ptr(), ws.data_ptr(), ws.numel(),
                           stream.cuda_stream if stream is not None else torch._C._cuda_getCurrentRawStream(dev))
    if check and rc != 0:
        raise ExfoldError(rc, "exfold_linear")
    return rc
