"""Python binding of libdn (include/dn.h): argument marshalling only.

Every function here has the name of the C entry point it calls, takes torch
tensors that live on the GPU, passes their device pointers and sizes through
ctypes, and launches on the current torch stream (or the one given: what the
call makes itself then belongs to that stream, as inside torch.cuda.stream).  All
arithmetic happens in the HIP kernels; nothing here computes on the host, and
there is no fallback: if ``libdn.so`` is missing the import fails.
"""
from __future__ import annotations

import ctypes
import dataclasses
import math
import os
from typing import Optional

import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libdn.so")

DN_F32, DN_BF16, DN_E4M3 = 0, 1, 2
DN_LN_LAYOUT_VERSION = 2
DN_SWIGLU_LAYOUT_VERSION = 0x102
STATUS = {0: "DN_OK", 1: "DN_ERR_INVALID_ARG", 2: "DN_ERR_UNSUPPORTED", 3: "DN_ERR_MISALIGNED", 4: "DN_ERR_HIP"}
SYMBOLS = ("dn_status_string", "dn_version", "ln_linear_packed_bytes", "ln_linear_prepare",
           "ln_linear_deferred", "rms_linear_deferred", "ln_linear_prepare_centered", "ln_linear_serial",
           "ln_linear_norm_on_load", "ln_linear_deferred_post", "rms_linear_deferred_post",
           "swiglu_packed_bytes", "swiglu_prepare", "rms_swiglu_deferred", "softmax_pv_deferred",
           "attention_deferred", "attention_gqa_deferred", "attention_decode_workspace_bytes",
           "attention_decode_deferred", "attention_decode_deferred_noalloc", "layernorm",
           "rmsnorm", "silu_mul", "softmax", "gemm", "rotary_table", "rotary_apply", "kv_cache_bytes",
           "kv_cache_describe", "kv_cache_append", "kv_cache_read", "attention_cache_workspace_bytes",
           "attention_cache_deferred", "attention_shared_prefix_deferred", "residual_rmsnorm", "residual_rmsnorm_fp8",
           "rows_fp8", "linear_fp8_packed_bytes", "linear_fp8_prepare", "linear_fp8_workspace_bytes", "linear_fp8",
           "token_logprobs_workspace_bytes", "token_logprobs")
DN_KV_PAGE = 64
DN_KV_LAYOUT_VERSION = 1
KV_FORMATS = {"bf16": 1, "fp8": 2}  # DN_KV_BF16, DN_KV_FP8
DN_FP8_LAYOUT_VERSION = 1
ACTIVATIONS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3, "gelu_tanh": 4}  # dn_activation


class DNError(RuntimeError):
    def __init__(self, fn: str, status: int):
        super().__init__(f"{fn} failed: {STATUS.get(status, status)}")
        self.status = status


class LnLinearWeights(ctypes.Structure):
    """Mirror of ``ln_linear_weights`` in dn.h."""
    _fields_ = [("K", ctypes.c_int64), ("N", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("layout_version", ctypes.c_int32), ("packed", ctypes.c_void_p)]


class KVCacheDesc(ctypes.Structure):
    """Mirror of ``kv_cache`` in dn.h."""
    _fields_ = [("pages", ctypes.c_int64), ("heads", ctypes.c_int64), ("d", ctypes.c_int64),
                ("format", ctypes.c_int32), ("layout_version", ctypes.c_int32), ("data", ctypes.c_void_p)]


class LinearFp8Weights(ctypes.Structure):
    """Mirror of ``linear_fp8_weights`` in dn.h."""
    _fields_ = [("K", ctypes.c_int64), ("N", ctypes.c_int64), ("gated", ctypes.c_int32),
                ("layout_version", ctypes.c_int32), ("packed", ctypes.c_void_p)]


def load_library(path: str = _LIB_PATH) -> ctypes.CDLL:
    if not os.path.exists(path):
        raise ImportError(f"libdn.so not found at {path}; build it with "
                          f"`python -m paper_2502_17728_amd.build` (needs hipcc for gfx950)")
    lib = ctypes.CDLL(path)
    vp, i64, i32, f32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_float
    lib.dn_status_string.argtypes, lib.dn_status_string.restype = [i32], ctypes.c_char_p
    lib.dn_version.argtypes, lib.dn_version.restype = [], i32
    lib.ln_linear_packed_bytes.argtypes, lib.ln_linear_packed_bytes.restype = [i64, i64, i32], ctypes.c_size_t
    lib.ln_linear_prepare.argtypes = [vp, vp, vp, vp, i64, i64, i32, vp, ctypes.c_size_t,
                                      ctypes.POINTER(LnLinearWeights), vp]
    lib.ln_linear_deferred.argtypes = [vp, ctypes.POINTER(LnLinearWeights), i64, f32, vp, vp]
    lib.ln_linear_prepare_centered.argtypes = lib.ln_linear_prepare.argtypes
    lib.ln_linear_serial.argtypes = [vp, ctypes.POINTER(LnLinearWeights), i64, f32, vp, vp, vp]
    lib.ln_linear_norm_on_load.argtypes = [vp, ctypes.POINTER(LnLinearWeights), i64, f32, vp, vp, vp]
    lib.ln_linear_deferred_post.argtypes = [vp, ctypes.POINTER(LnLinearWeights), i64, f32, vp, vp, vp, vp, vp, vp]
    lib.rms_linear_deferred_post.argtypes = [vp, ctypes.POINTER(LnLinearWeights), i64, f32, vp, vp, vp, vp, vp]
    lib.rms_linear_deferred.argtypes = [vp, ctypes.POINTER(LnLinearWeights), i64, f32, vp, vp]
    lib.swiglu_packed_bytes.argtypes, lib.swiglu_packed_bytes.restype = [i64, i64, i32], ctypes.c_size_t
    lib.swiglu_prepare.argtypes = [vp, vp, vp, i64, i64, i32, vp, ctypes.c_size_t, ctypes.POINTER(LnLinearWeights),
                                   vp]
    lib.rms_swiglu_deferred.argtypes = [vp, ctypes.POINTER(LnLinearWeights), i64, f32, vp, vp]
    lib.silu_mul.argtypes = [vp, vp, i64, i32, vp, vp]
    lib.softmax_pv_deferred.argtypes = [vp, vp, i64, i64, i64, i64, i32, i32, vp, vp]
    lib.attention_deferred.argtypes = [vp, vp, vp, i64, i64, i64, i64, i32, f32, i32, vp, vp]
    lib.attention_gqa_deferred.argtypes = [vp, vp, vp, i64, i64, i64, i64, i64, i32, f32, i32, vp, vp]
    lib.attention_decode_workspace_bytes.argtypes = [i64, i64, i64, i64]
    lib.attention_decode_workspace_bytes.restype = ctypes.c_size_t
    lib.attention_decode_deferred.argtypes = [vp, vp, vp, i64, i64, i64, i64, f32, i32, vp, ctypes.c_size_t, vp, vp]
    lib.attention_decode_deferred_noalloc.argtypes = [vp, vp, vp, i64, i64, i64, i64, f32, i32, vp, vp]
    lib.layernorm.argtypes = [vp, vp, vp, i64, i64, f32, i32, vp, vp]
    lib.rmsnorm.argtypes = [vp, vp, i64, i64, f32, i32, vp, vp]
    lib.softmax.argtypes = [vp, i64, i64, i64, i32, i32, vp, vp]
    lib.gemm.argtypes = [vp, vp, vp, i64, i64, i64, i64, i32, i32, i32, vp, vp]
    kv, sz = ctypes.POINTER(KVCacheDesc), ctypes.c_size_t
    lib.rotary_table.argtypes = [vp, i64, i64, ctypes.c_double, vp, vp]
    lib.rotary_apply.argtypes = [vp, i64, vp, vp, i64, i64, i64, i64, i64, i32, i32, i32, vp, i64, vp]
    lib.kv_cache_bytes.argtypes, lib.kv_cache_bytes.restype = [i64, i64, i64, i32], sz
    lib.kv_cache_describe.argtypes = [vp, sz, i64, i64, i64, i32, kv]
    lib.kv_cache_append.argtypes = [kv, vp, i64, vp, vp, vp, i64, i64, i32, i64, i64, i32, vp, vp]
    lib.kv_cache_read.argtypes = [kv, vp, i64, i32, vp, vp, vp]
    lib.attention_cache_workspace_bytes.argtypes, lib.attention_cache_workspace_bytes.restype = [i64] * 7, sz
    lib.attention_cache_deferred.argtypes = [vp, i64, i64, i64, kv, vp, i64, vp, vp, i64, f32, i32, vp, sz, vp, vp]
    lib.attention_shared_prefix_deferred.argtypes = [vp, i64, i64, i64, kv, vp, i64, vp, i64, vp, vp, i64, f32, i32, vp,
                                                     sz, vp, vp]
    fw = ctypes.POINTER(LinearFp8Weights)
    lib.residual_rmsnorm.argtypes = [vp, vp, vp, i64, i64, f32, i32, vp, vp, vp]
    lib.residual_rmsnorm_fp8.argtypes = [vp, vp, vp, i64, i64, f32, i32, vp, vp, vp, vp]
    lib.rows_fp8.argtypes = [vp, i64, i64, i32, vp, vp, vp]
    lib.linear_fp8_packed_bytes.argtypes, lib.linear_fp8_packed_bytes.restype = [i64, i64, i32], sz
    lib.linear_fp8_prepare.argtypes = [vp] * 7 + [i64, i64, i32, vp, sz, fw, vp]
    lib.linear_fp8_workspace_bytes.argtypes, lib.linear_fp8_workspace_bytes.restype = [i64, fw], sz
    lib.linear_fp8.argtypes = [vp, vp, fw, i64, i32, vp, i32, vp, sz, vp, vp]
    lib.token_logprobs_workspace_bytes.argtypes, lib.token_logprobs_workspace_bytes.restype = [i64] * 3, sz
    lib.token_logprobs.argtypes = [vp, i64, i64, i64, i32, f32, vp, i64, i64, vp, vp, vp, vp, vp, sz, vp]
    for f in ("ln_linear_prepare", "ln_linear_deferred", "rms_linear_deferred", "ln_linear_prepare_centered",
              "ln_linear_serial", "ln_linear_norm_on_load", "ln_linear_deferred_post",
              "rms_linear_deferred_post", "swiglu_prepare", "rms_swiglu_deferred", "softmax_pv_deferred",
              "attention_deferred", "attention_gqa_deferred", "attention_decode_deferred",
              "attention_decode_deferred_noalloc", "layernorm", "rmsnorm",
              "silu_mul", "softmax",
              "gemm", "rotary_table", "rotary_apply", "kv_cache_describe", "kv_cache_append", "kv_cache_read",
              "attention_cache_deferred", "attention_shared_prefix_deferred", "residual_rmsnorm", "residual_rmsnorm_fp8",
              "rows_fp8", "linear_fp8_prepare", "linear_fp8", "token_logprobs"):
        getattr(lib, f).restype = i32
    return lib


_lib = load_library()


def library_path() -> str:
    return _LIB_PATH


def _dt(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return DN_F32
    if t.dtype == torch.bfloat16:
        return DN_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _dev(t: Optional[torch.Tensor], name: str):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _expect(t: Optional[torch.Tensor], name: str, shape=None, dtype=None, device=None, numel=None):
    """Check a tensor before its pointer reaches the C ABI, which sees only raw pointers and
    sizes: a wrong shape there becomes an out-of-bounds access on the GPU.  Raises ValueError
    on any mismatch; shape entries of None match any size."""
    if t is None:
        return
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if shape is not None and t.shape != shape:
        ok = t.dim() == len(shape) and all(s is None or int(a) == int(s) for a, s in zip(t.shape, shape))
        if not ok:
            want = "[" + ", ".join("*" if s is None else str(int(s)) for s in shape) + "]"
            raise ValueError(f"{name} has shape {list(t.shape)}, expected {want}")
    if numel is not None and t.numel() != numel:
        raise ValueError(f"{name} has {t.numel()} elements, expected {numel}")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device} (all tensors of a call share one device)")


_TORCH_DT = {DN_F32: torch.float32, DN_BF16: torch.bfloat16}


# the current stream's handle without building a Stream object (a private name of torch's)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int:
    if stream is None:
        if _raw_stream is None:
            return torch.cuda.current_stream().cuda_stream
        return _raw_stream(torch.cuda.current_device())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _on(stream, x: torch.Tensor):
    """The stream given, as torch's current one on x's device.  What a call makes for itself on another
    stream than the current one (outputs, scratch, copies) is made in this: torch's allocator orders a
    block's uses by the stream that it was made on, so a block made on the current stream could still
    be in use there when the call's kernels write it, or be given to someone else before they end."""
    if not isinstance(stream, torch.cuda.Stream):
        handle = _stream(stream)
        stream = torch.cuda.ExternalStream(handle, device=x.device) if handle else torch.cuda.default_stream(x.device)
    return torch.cuda.stream(stream)


def _empty(x: torch.Tensor, shape, stream, dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """A tensor made for a call on `stream`, of x's dtype (or the one given) on x's device."""
    if stream is not None and _stream(stream) != _stream_of(None, x):
        with _on(stream, x):
            return _empty(x, shape, None, dtype)
    return x.new_empty(shape) if dtype is None else torch.empty(shape, dtype=dtype, device=x.device)


# The wrappers below run on every token of a decode loop, where the kernels take 5-20 us: a
# call's checks are one comparison each in the usual case, and _expect, which words the error,
# runs only where one fails.
def _like(t: Optional[torch.Tensor], shape, x: torch.Tensor) -> bool:
    """t is None, or has this shape and x's dtype and device."""
    return t is None or (isinstance(t, torch.Tensor) and t.shape == shape and t.dtype == x.dtype
                         and t.get_device() == x.get_device())


def _check(fn: str, status: int):
    if status != 0:
        raise DNError(fn, status)


def _check_rows(x: torch.Tensor, w, out: Optional[torch.Tensor], stats: Optional[torch.Tensor] = None) -> int:
    """x[M, w.K] in the weights' dtype; out (if given) [M, w.N] like x; stats (if given) 2 M fp32."""
    if not isinstance(w, PreparedLinear):
        raise TypeError("w must come from ln_linear_prepare / swiglu_prepare")
    if x.dim() != 2:
        raise ValueError(f"x has shape {list(x.shape)}, expected [M, {w.K}]")
    M, K = x.shape
    desc = w.desc
    if (K == desc.K and x.dtype == _TORCH_DT.get(desc.dtype) and x.is_cuda and x.get_device() == w.packed.get_device()
            and stats is None and _like(out, (M, desc.N), x)):
        return M
    _expect(x, "x", (M, w.K), _TORCH_DT.get(w.desc.dtype), w.packed.device)
    _expect(out, "out", (M, w.N), x.dtype, x.device)
    _expect(stats, "stats", None, torch.float32, x.device, numel=2 * M)
    return M


@dataclasses.dataclass
class PreparedLinear:
    """Prepared static weights: the packed device buffer and its descriptor."""
    packed: torch.Tensor
    desc: LnLinearWeights

    @property
    def K(self):
        return self.desc.K

    @property
    def N(self):
        return self.desc.N


def ln_linear_packed_bytes(K: int, N: int, dtype: int) -> int:
    return int(_lib.ln_linear_packed_bytes(K, N, dtype))


def ln_linear_prepare(W: torch.Tensor, gamma: torch.Tensor, beta: Optional[torch.Tensor] = None,
                      bias: Optional[torch.Tensor] = None, stream=None, centered: bool = False) -> PreparedLinear:
    """centered=True calls ln_linear_prepare_centered (the literal Eq. (5) weight)."""
    if W.dim() != 2:
        raise ValueError(f"W has shape {list(W.shape)}, expected [K, N]")
    K, N = W.shape
    dt = _dt(W)
    _expect(gamma, "gamma", (K,), W.dtype, W.device)
    _expect(beta, "beta", (K,), W.dtype, W.device)
    _expect(bias, "bias", (N,), W.dtype, W.device)
    nbytes = ln_linear_packed_bytes(K, N, dt)
    if nbytes == 0:
        raise DNError("ln_linear_packed_bytes", 1)
    packed = _empty(W, nbytes, stream, torch.uint8)
    desc = LnLinearWeights()
    fn = "ln_linear_prepare_centered" if centered else "ln_linear_prepare"
    _check(fn, getattr(_lib, fn)(
        _dev(W, "W"), _dev(gamma, "gamma"), _dev(beta, "beta"), _dev(bias, "bias"), K, N, dt,
        _dev(packed, "packed"), nbytes, ctypes.byref(desc), _stream(stream)))
    return PreparedLinear(packed, desc)


def ln_linear_deferred(x: torch.Tensor, w: PreparedLinear, eps: float = 1e-5,
                       out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    M = _check_rows(x, w, out)
    if out is None:
        out = x.new_empty((M, w.desc.N)) if stream is None else _empty(x, (M, w.desc.N), stream)
    _check("ln_linear_deferred", _lib.ln_linear_deferred(
        _dev(x, "x"), ctypes.byref(w.desc), M, eps, _dev(out, "out"), _stream(stream)))
    return out


def ln_linear_serial(x: torch.Tensor, w: PreparedLinear, eps: float = 1e-5, stats: Optional[torch.Tensor] = None,
                     out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    M = _check_rows(x, w, out, stats)
    if out is None:
        out = _empty(x, (M, w.N), stream)
    if stats is None:
        stats = _empty(x, 2 * M, stream, torch.float32)
    _check("ln_linear_serial", _lib.ln_linear_serial(
        _dev(x, "x"), ctypes.byref(w.desc), M, eps, _dev(stats, "stats"), _dev(out, "out"), _stream(stream)))
    return out


def ln_linear_norm_on_load(x: torch.Tensor, w: PreparedLinear, eps: float = 1e-5,
                           stats: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                           stream=None) -> torch.Tensor:
    """Ablation: statistics pre-pass, then x normalized on load into the product (no deferral)."""
    M = _check_rows(x, w, out, stats)
    if out is None:
        out = _empty(x, (M, w.N), stream)
    if stats is None:
        stats = _empty(x, 2 * M, stream, torch.float32)
    _check("ln_linear_norm_on_load", _lib.ln_linear_norm_on_load(
        _dev(x, "x"), ctypes.byref(w.desc), M, eps, _dev(stats, "stats"), _dev(out, "out"), _stream(stream)))
    return out


def linear_deferred_post(x: torch.Tensor, w: PreparedLinear, gamma: torch.Tensor, beta: Optional[torch.Tensor] = None,
                         eps: float = 1e-5, rms: bool = False, stats: Optional[torch.Tensor] = None,
                         y: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                         stream=None):
    """Post-LN placement: (out, y, stats) -- the deferred product and the normalized rows."""
    M = _check_rows(x, w, out, stats)
    K = w.K
    _expect(gamma, "gamma", (K,), x.dtype, x.device)
    _expect(beta, "beta", (K,), x.dtype, x.device)
    _expect(y, "y", (M, K), x.dtype, x.device)
    if out is None:
        out = _empty(x, (M, w.N), stream)
    if y is None:
        y = _empty(x, (M, K), stream)
    if stats is None:
        stats = _empty(x, 2 * M, stream, torch.float32)
    if rms:
        if beta is not None:
            raise ValueError("RMSNorm has no shift")
        st = _lib.rms_linear_deferred_post(_dev(x, "x"), ctypes.byref(w.desc), M, eps, _dev(gamma, "gamma"),
                                           _dev(stats, "stats"), _dev(y, "y"), _dev(out, "out"), _stream(stream))
        _check("rms_linear_deferred_post", st)
    else:
        st = _lib.ln_linear_deferred_post(_dev(x, "x"), ctypes.byref(w.desc), M, eps, _dev(gamma, "gamma"),
                                          _dev(beta, "beta"), _dev(stats, "stats"), _dev(y, "y"), _dev(out, "out"),
                                          _stream(stream))
        _check("ln_linear_deferred_post", st)
    return out, y, stats


def rms_linear_deferred(x: torch.Tensor, w: PreparedLinear, eps: float = 1e-5,
                        out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    M = _check_rows(x, w, out)
    if out is None:
        out = x.new_empty((M, w.desc.N)) if stream is None else _empty(x, (M, w.desc.N), stream)
    _check("rms_linear_deferred", _lib.rms_linear_deferred(
        _dev(x, "x"), ctypes.byref(w.desc), M, eps, _dev(out, "out"), _stream(stream)))
    return out


def swiglu_packed_bytes(K: int, N: int, dtype: int) -> int:
    return int(_lib.swiglu_packed_bytes(K, N, dtype))


def swiglu_prepare(W_gate: torch.Tensor, W_up: torch.Tensor, gamma: torch.Tensor, stream=None) -> PreparedLinear:
    if W_gate.dim() != 2:
        raise ValueError(f"W_gate has shape {list(W_gate.shape)}, expected [K, N]")
    K, N = W_gate.shape
    _expect(W_up, "W_up", (K, N), W_gate.dtype, W_gate.device)
    _expect(gamma, "gamma", (K,), W_gate.dtype, W_gate.device)
    dt = _dt(W_gate)
    nbytes = swiglu_packed_bytes(K, N, dt)
    if nbytes == 0:
        raise DNError("swiglu_packed_bytes", 1)
    packed = _empty(W_gate, nbytes, stream, torch.uint8)
    desc = LnLinearWeights()
    _check("swiglu_prepare", _lib.swiglu_prepare(
        _dev(W_gate, "W_gate"), _dev(W_up, "W_up"), _dev(gamma, "gamma"), K, N, dt, _dev(packed, "packed"),
        nbytes, ctypes.byref(desc), _stream(stream)))
    return PreparedLinear(packed, desc)


def rms_swiglu_deferred(x: torch.Tensor, w: PreparedLinear, eps: float = 1e-5,
                        out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    M = _check_rows(x, w, out)
    if out is None:
        out = x.new_empty((M, w.desc.N)) if stream is None else _empty(x, (M, w.desc.N), stream)
    _check("rms_swiglu_deferred", _lib.rms_swiglu_deferred(
        _dev(x, "x"), ctypes.byref(w.desc), M, eps, _dev(out, "out"), _stream(stream)))
    return out


def softmax_pv_deferred(S: torch.Tensor, V: torch.Tensor, causal: bool = False,
                        out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    if S.dim() != 3 or V.dim() != 3:
        raise ValueError(f"S must be [BH, Lq, Lk] and V [BH, Lk, d]; got {list(S.shape)} and {list(V.shape)}")
    BH, Lq, Lk = S.shape
    d = V.shape[-1]
    if not (_like(V, (BH, Lk, d), S) and _like(out, (BH, Lq, d), S)):
        _expect(V, "V", (BH, Lk, d), S.dtype, S.device)
        _expect(out, "out", (BH, Lq, d), S.dtype, S.device)
    if out is None:
        out = S.new_empty((BH, Lq, d)) if stream is None else _empty(S, (BH, Lq, d), stream)
    _check("softmax_pv_deferred", _lib.softmax_pv_deferred(
        _dev(S, "S"), _dev(V, "V"), BH, Lq, Lk, d, int(causal), _dt(S), _dev(out, "out"), _stream(stream)))
    return out


def _check_qkv(Q, K, V, out):
    """Q[BHq, Lq, d], K and V [BH, Lk, d] with BHq a multiple of BH, one dtype and device; out like Q."""
    if Q.dim() != 3 or K.dim() != 3:
        raise ValueError(f"Q must be [BHq, Lq, d] and K, V [BH, Lk, d]; got {list(Q.shape)} and {list(K.shape)}")
    BHq, Lq, d = Q.shape
    BH, Lk = K.shape[0], K.shape[1]
    if not (_like(K, (BH, Lk, d), Q) and _like(V, (BH, Lk, d), Q)):
        _expect(K, "K", (BH, Lk, d), Q.dtype, Q.device)
        _expect(V, "V", (BH, Lk, d), Q.dtype, Q.device)
    if BH < 1 or BHq % BH:
        raise ValueError(f"the query heads ({BHq}) must be a multiple of the key/value heads ({BH})")
    if not _like(out, Q.shape, Q):
        _expect(out, "out", tuple(Q.shape), Q.dtype, Q.device)
    return BHq, Lq, d, BH, Lk


def attention_deferred(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, causal: bool = False,
                       scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                       stream=None) -> torch.Tensor:
    """softmax(scale * Q K^T) V per query head; scale defaults to 1/sqrt(d).

    Q[BH * g, Lq, d], K/V[BH, Lk, d]: g = 1 is one key/value head per query head; g > 1 is
    grouped-query attention, query head h reading key/value head h // g.
    """
    BHq, Lq, d, BH, Lk = _check_qkv(Q, K, V, out)
    g = BHq // BH
    if scale is None:
        scale = 1.0 / float(d) ** 0.5
    if out is None:
        out = _empty(Q, Q.shape, stream)
    if g == 1:
        st = _lib.attention_deferred(_dev(Q, "Q"), _dev(K, "K"), _dev(V, "V"), BH, Lq, Lk, d, int(causal),
                                     float(scale), _dt(Q), _dev(out, "out"), _stream(stream))
        _check("attention_deferred", st)
    else:
        st = _lib.attention_gqa_deferred(_dev(Q, "Q"), _dev(K, "K"), _dev(V, "V"), BH, g, Lq, Lk, d, int(causal),
                                         float(scale), _dt(Q), _dev(out, "out"), _stream(stream))
        _check("attention_gqa_deferred", st)
    return out


def attention_decode_workspace_bytes(BH: int, Lq: int, Lk: int, d: int) -> int:
    return int(_lib.attention_decode_workspace_bytes(BH, Lq, Lk, d))


def attention_decode_deferred(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, scale: Optional[float] = None,
                              workspace: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                              stream=None) -> torch.Tensor:
    """Decode attention (every key visible) split over key ranges, then merged.

    Q[BH * g, Lq, d] against K, V[BH, Lk, d]: with g > 1 (grouped-query attention) query
    heads h * g .. h * g + g - 1 share key/value head h, and the g heads' rows go through
    the kernel together as g * Lq (<= 16) queries of that head.
    """
    BHq, Lq, d, BH, Lk = _check_qkv(Q, K, V, out)
    _expect(workspace, "workspace", None, torch.uint8, Q.device)
    g = BHq // BH
    if out is None:
        out = _empty(Q, Q.shape, stream)
    out_k = out
    if not (Q.is_contiguous() and out.is_contiguous()):  # contiguous ones are [BH, g * Lq, d] as they lie
        if stream is None:
            Q = Q.reshape(BH, g * Lq, d)
        else:
            with _on(stream, Q):
                Q = Q.reshape(BH, g * Lq, d)
        out_k = out.view(BH, g * Lq, d)
    Lq = g * Lq
    if scale is None:
        scale = 1.0 / float(d) ** 0.5
    if workspace is None:
        nbytes = attention_decode_workspace_bytes(BH, Lq, Lk, d)
        workspace = _empty(Q, max(nbytes, 16), stream, torch.uint8)
    _check("attention_decode_deferred", _lib.attention_decode_deferred(
        _dev(Q, "Q"), _dev(K, "K"), _dev(V, "V"), BH, Lq, Lk, d, float(scale), _dt(Q), _dev(workspace, "workspace"),
        workspace.numel(), _dev(out_k, "out"), _stream(stream)))
    return out


def attention_decode_deferred_noalloc(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor,
                                      scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                                      stream=None) -> torch.Tensor:
    """attention_decode_deferred without a workspace: the partials live in the library's own
    device array (the C call allocates nothing; pass `out` to keep this wrapper from allocating
    the output).  Calls overlapping on one GPU share that array."""
    BHq, Lq, d, BH, Lk = _check_qkv(Q, K, V, out)
    g = BHq // BH
    if out is None:
        out = _empty(Q, Q.shape, stream)
    if not (Q.is_contiguous() and out.is_contiguous()):
        raise ValueError("Q and out must be contiguous")
    if scale is None:
        scale = 1.0 / float(d) ** 0.5
    _check("attention_decode_deferred_noalloc", _lib.attention_decode_deferred_noalloc(
        _dev(Q, "Q"), _dev(K, "K"), _dev(V, "V"), BH, g * Lq, Lk, d, float(scale), _dt(Q), _dev(out, "out"),
        _stream(stream)))
    return out


def _check_norm(x, gamma, beta, out):
    if x.dim() != 2:
        raise ValueError(f"x has shape {list(x.shape)}, expected [M, K]")
    M, K = x.shape
    _expect(gamma, "gamma", (K,), x.dtype, x.device)
    _expect(beta, "beta", (K,), x.dtype, x.device)
    _expect(out, "out", (M, K), x.dtype, x.device)
    return M, K


def layernorm(x: torch.Tensor, gamma: torch.Tensor, beta: Optional[torch.Tensor] = None, eps: float = 1e-5,
              out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    M, K = _check_norm(x, gamma, beta, out)
    if out is None:
        out = _empty(x, (M, K), stream)
    _check("layernorm", _lib.layernorm(_dev(x, "x"), _dev(gamma, "gamma"), _dev(beta, "beta"), M, K, eps,
                                       _dt(x), _dev(out, "out"), _stream(stream)))
    return out


def rmsnorm(x: torch.Tensor, gamma: torch.Tensor, eps: float = 1e-5, out: Optional[torch.Tensor] = None,
            stream=None) -> torch.Tensor:
    M, K = _check_norm(x, gamma, None, out)
    if out is None:
        out = _empty(x, (M, K), stream)
    _check("rmsnorm", _lib.rmsnorm(_dev(x, "x"), _dev(gamma, "gamma"), M, K, eps, _dt(x), _dev(out, "out"),
                                   _stream(stream)))
    return out


def silu_mul(g: torch.Tensor, u: torch.Tensor, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    _expect(u, "u", tuple(g.shape), g.dtype, g.device)
    _expect(out, "out", None, g.dtype, g.device, numel=g.numel())
    if out is None:
        out = _empty(g, g.shape, stream)
    _check("silu_mul", _lib.silu_mul(_dev(g, "g"), _dev(u, "u"), g.numel(), _dt(g), _dev(out, "out"),
                                     _stream(stream)))
    return out


def softmax(S: torch.Tensor, causal: int = 0, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    if S.dim() != 3:
        raise ValueError(f"S has shape {list(S.shape)}, expected [BH, Lq, Lk]")
    BH, Lq, Lk = S.shape
    _expect(out, "out", tuple(S.shape), S.dtype, S.device)
    if out is None:
        out = _empty(S, S.shape, stream)
    _check("softmax", _lib.softmax(_dev(S, "S"), BH, Lq, Lk, int(causal), _dt(S), _dev(out, "out"),
                                   _stream(stream)))
    return out


def gemm(A: torch.Tensor, B, bias: Optional[torch.Tensor] = None, b_layout: int = 0,
         a_causal: bool = False, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """C = A . B (+ bias).  B is a tensor ([K, N] for b_layout 0, [N, K] for 1, optionally
    batched) or a PreparedLinear (b_layout 2: the packed weights of ln_linear_prepare)."""
    if A.dim() not in (2, 3):
        raise ValueError(f"A has shape {list(A.shape)}, expected [M, K] or [batch, M, K]")
    squeeze = A.dim() == 2
    A3 = A.unsqueeze(0) if squeeze else A
    batch, M, K = A3.shape
    if isinstance(B, PreparedLinear):
        if B.K != K or _TORCH_DT.get(B.desc.dtype) != A.dtype:
            raise ValueError(f"the prepared weights are [{B.K}, {B.N}] of dtype {_TORCH_DT.get(B.desc.dtype)}; "
                             f"A is [*, {K}] of dtype {A.dtype}")
        if batch != 1:
            raise ValueError("prepared (packed) weights take an unbatched A")
        _expect(B.packed, "B", None, None, A.device)
        b_layout, N = 2, B.N
        bptr = None
    else:
        if b_layout not in (0, 1) or B.dim() not in (2, 3):
            raise ValueError("B must be [K, N] (b_layout 0) or [N, K] (b_layout 1), optionally batched")
        B3 = B.unsqueeze(0) if B.dim() == 2 else B
        N = B3.shape[2] if b_layout == 0 else B3.shape[1]
        _expect(B3, "B", (batch, K, N) if b_layout == 0 else (batch, N, K), A.dtype, A.device)
        bptr = None
    _expect(bias, "bias", (N,), A.dtype, A.device)
    _expect(out, "out", (batch, M, N), A.dtype, A.device)
    bptr = _dev(B.packed, "B") if isinstance(B, PreparedLinear) else _dev(B3, "B")
    if out is None:
        out = _empty(A, (batch, M, N), stream)
    _check("gemm", _lib.gemm(_dev(A3, "A"), bptr, _dev(bias, "bias"), batch, M, K, N, int(b_layout),
                             int(a_causal), _dt(A), _dev(out, "out"), _stream(stream)))
    return out[0] if squeeze else out


# ------------------------------------------------------------------------------- rotary positions
def rotary_frequencies(rot: int, base: float = 10000.0, scaling: Optional[str] = None, factor: float = 1.0,
                       original: int = 8192, low: float = 1.0, high: float = 4.0, device="cuda"):
    """(inv_freq, amplitude) for rotary_table: the rot / 2 frequencies base ** (-2 i / rot), fp64 on
    the device, scaled for contexts ``factor`` times as long as the ``original`` tokens of training:

    - None: as they are.
    - "linear": every frequency divided by factor (positions interpolated).
    - "base": the base raised to base * factor ** (rot / (rot - 2)), which divides the lowest
      frequency by factor and leaves the highest.
    - "parts": a frequency that turns fewer than ``low`` times over the original context is divided
      by factor, one that turns more than ``high`` times is left, those between are blended linearly
      in their number of turns.
    - "parts_log": the same, blended linearly in the dimension (so in the logarithm of the number of
      turns), and with the amplitude 0.1 ln(factor) + 1.  The blend starts and ends where ``high`` and
      ``low`` turns fall, between two dimensions as it may be; for a model whose limits were rounded to
      whole dimensions, or that was trained with other limits than the defaults here (``high`` = 32 is
      common with this scaling), give its limits, or its own frequencies to rotary_table.
    """
    if rot < 2 or rot % 2 or not base > 0 or not factor > 0:
        raise ValueError("rot must be even and positive, base and factor positive")
    freq = float(base) ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    amplitude = 1.0
    if scaling == "linear":
        freq = freq / factor
    elif scaling == "base":
        if rot < 4:
            raise ValueError("scaling the base needs at least two frequencies")
        freq = (float(base) * factor ** (rot / (rot - 2))) ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    elif scaling in ("parts", "parts_log"):
        if not 0 < low < high:
            raise ValueError("0 < low < high is needed")
        turns = original * freq / (2.0 * math.pi)
        if scaling == "parts":
            keep = (turns - low) / (high - low)
        else:
            keep = torch.log(turns / low) / math.log(high / low)
            amplitude = 0.1 * math.log(factor) + 1.0 if factor > 1.0 else 1.0
        keep = keep.clamp(0.0, 1.0)
        freq = keep * freq + (1.0 - keep) * freq / factor
    elif scaling is not None:
        raise ValueError(f"unknown scaling {scaling!r}")
    return freq.to(device), amplitude


def rotary_table(inv_freq: torch.Tensor, positions: int, amplitude: float = 1.0, stream=None) -> torch.Tensor:
    """cos and sin of every position below ``positions``: [positions, rot / 2, 2] fp32."""
    if inv_freq.dim() != 1:
        raise ValueError(f"inv_freq has shape {list(inv_freq.shape)}, expected [rot / 2]")
    _expect(inv_freq, "inv_freq", None, torch.float64)
    half = inv_freq.shape[0]
    table = _empty(inv_freq, (max(int(positions), 0), half, 2), stream, torch.float32)
    _check("rotary_table", _lib.rotary_table(_dev(inv_freq, "inv_freq"), 2 * half, int(positions), float(amplitude),
                                             _dev(table, "table") or None, _stream(stream)))
    return table


def _rows(t: torch.Tensor, name: str):
    """Pointer and token stride of t[T, H, d] (or [T, width]) whose tokens' values lie together."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    T = t.shape[0]
    if t.is_contiguous() and T:
        return t.data_ptr(), t.numel() // T
    st, n = t.stride(), 1
    for k in range(t.dim() - 1, 0, -1):
        if st[k] != n and t.shape[k] != 1:
            raise ValueError(f"{name} must be contiguous within a token")
        n *= t.shape[k]
    return t.data_ptr(), (st[0] if T != 1 else n)  # tokens that lie on one another: refused by the library


def _int32(t: torch.Tensor, name: str, shape, x: torch.Tensor):
    """Pointer of an int32 index tensor of this shape on x's device."""
    if not (isinstance(t, torch.Tensor) and t.dtype is torch.int32 and t.shape == shape and t.is_contiguous()
            and t.get_device() == x.get_device()):
        if t is None:
            raise ValueError(f"{name} is required")
        _expect(t, name, shape, torch.int32, x.device)
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _table_of(table: torch.Tensor, x: torch.Tensor):
    """Pointer, positions and turned dimensions of a rotary table."""
    if isinstance(table, torch.Tensor) and table.dim() == 3:
        rows, half, two = table.shape
        if two == 2 and table.dtype is torch.float32 and table.get_device() == x.get_device() and table.is_contiguous():
            return table.data_ptr(), rows, 2 * half
    if table is None:
        raise ValueError("table is required")
    _expect(table, "table", (None, None, 2), torch.float32, x.device)
    return _dev(table, "table"), table.shape[0], 2 * table.shape[1]


def _stream_of(stream, x: torch.Tensor) -> int:
    """The stream given, or the current one of x's device."""
    if stream is None and _raw_stream is not None:
        return _raw_stream(x.get_device())
    return _stream(stream)


def rotary_apply(x: torch.Tensor, positions: torch.Tensor, table: torch.Tensor, interleaved: bool = False,
                 inverse: bool = False, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """x[T, H, d] turned by each token's position (tokens may be strided, as the query heads of QKV
    rows are; out may be x).  inverse is the transpose: the gradient with respect to x from that with
    respect to the turned x, and the turn back where the table's amplitude is 1."""
    if x.dim() != 3:
        raise ValueError(f"x has shape {list(x.shape)}, expected [T, H, d]")
    T, H, d = x.shape
    xp, xs = _rows(x, "x")
    tp, rows, rot = _table_of(table, x)
    if out is None:
        out = x.new_empty((T, H, d)) if stream is None else _empty(x, (T, H, d), stream)
        op, os_ = out.data_ptr(), H * d
    else:
        if not _like(out, x.shape, x):
            _expect(out, "out", (T, H, d), x.dtype, x.device)
        op, os_ = _rows(out, "out")
    st = _lib.rotary_apply(xp, xs, _int32(positions, "positions", (T,), x), tp, rows, T, H, d, rot, interleaved, inverse,
                           _dt(x), op, os_, _stream_of(stream, x))
    if st:
        raise DNError("rotary_apply", st)
    return out


# ------------------------------------------------------------------------------- paged key/value cache
@dataclasses.dataclass
class KVCache:
    """A paged key/value cache: the device buffer and its descriptor.  Slot s is token s % 64 of
    page s // 64; which pages hold which sequence is the caller's."""
    data: torch.Tensor
    desc: KVCacheDesc

    def __post_init__(self):
        self.ref = ctypes.byref(self.desc)

    @property
    def pages(self):
        return self.desc.pages

    @property
    def heads(self):
        return self.desc.heads

    @property
    def d(self):
        return self.desc.d

    @property
    def format(self):
        return {v: k for k, v in KV_FORMATS.items()}[self.desc.format]


def kv_cache_bytes(pages: int, heads: int, d: int, fmt: str = "bf16") -> int:
    return int(_lib.kv_cache_bytes(pages, heads, d, KV_FORMATS.get(fmt, 0)))


def kv_cache_create(pages: int, heads: int, d: int, fmt: str = "bf16", device="cuda") -> KVCache:
    """A cache of ``pages`` pages of 64 tokens; its memory needs no clearing."""
    n = kv_cache_bytes(pages, heads, d, fmt)
    if n == 0:
        raise DNError("kv_cache_bytes", 1)
    return kv_cache_wrap(torch.empty((pages, heads, n // (pages * heads)), dtype=torch.uint8, device=device), d, fmt)


def kv_cache_wrap(data: torch.Tensor, d: int, fmt: str = "bf16") -> KVCache:
    """The cache held by data[pages, heads, block bytes] (uint8)."""
    if data.dim() != 3:
        raise ValueError(f"data has shape {list(data.shape)}, expected [pages, heads, block bytes]")
    pages, heads = data.shape[:2]
    n = kv_cache_bytes(pages, heads, d, fmt)
    if n == 0:
        raise DNError("kv_cache_bytes", 1)
    _expect(data, "data", (pages, heads, n // (pages * heads)), torch.uint8)
    desc = KVCacheDesc()
    _check("kv_cache_describe", _lib.kv_cache_describe(_dev(data, "data"), data.numel(), pages, heads, d,
                                                       KV_FORMATS[fmt], ctypes.byref(desc)))
    return KVCache(data, desc)


def _check_cache(cache, x: torch.Tensor):
    if not isinstance(cache, KVCache):
        raise TypeError("cache must come from kv_cache_create / kv_cache_wrap")
    if cache.data.get_device() != x.get_device():
        raise ValueError(f"the cache is on {cache.data.device}, expected {x.device} (all tensors of a call share one device)")
    return cache.desc


def kv_cache_append(cache: KVCache, qkv: torch.Tensor, slots: torch.Tensor, positions: Optional[torch.Tensor] = None,
                    table: Optional[torch.Tensor] = None, interleaved: bool = False,
                    q_out: Optional[torch.Tensor] = None, stream=None) -> Optional[torch.Tensor]:
    """Puts the keys and values of qkv[T, (q_heads + 2 heads) d] into the cache at slots[T] (-1: not
    written) and returns the queries [T, q_heads, d] (None where the rows hold none).  With a rotary
    table the queries and keys are turned by positions[T]."""
    desc = _check_cache(cache, qkv)
    if qkv.dim() != 2:
        raise ValueError(f"qkv has shape {list(qkv.shape)}, expected [T, (q_heads + 2 heads) d]")
    T, width = qkv.shape
    heads, d = desc.heads, desc.d
    q_heads = width // d - 2 * heads
    if width % d or q_heads < 0 or q_heads % heads:
        raise ValueError(f"rows of {width} values do not hold a multiple of {heads} query heads and 2 x {heads} key and "
                         f"value heads of {d}")
    qp, qs = _rows(qkv, "qkv")
    op = None
    if q_heads == 0:
        if q_out is not None:
            raise ValueError("the rows hold no queries")
    elif q_out is None:
        q_out = qkv.new_empty((T, q_heads, d)) if stream is None else _empty(qkv, (T, q_heads, d), stream)
        op = q_out.data_ptr()
    else:
        if not _like(q_out, (T, q_heads, d), qkv):
            _expect(q_out, "q_out", (T, q_heads, d), qkv.dtype, qkv.device)
        op = _dev(q_out, "q_out")
    tp, rows, rot, pp = None, 0, 0, None
    if table is not None:
        tp, rows, rot = _table_of(table, qkv)
        pp = _int32(positions, "positions", (T,), qkv)
    st = _lib.kv_cache_append(cache.ref, qp, qs, _int32(slots, "slots", (T,), qkv), pp, tp, rows, rot, interleaved, T,
                              q_heads, _dt(qkv), op, _stream_of(stream, qkv))
    if st:
        raise DNError("kv_cache_append", st)
    return q_out


def kv_cache_read(cache: KVCache, slots: torch.Tensor, K: Optional[torch.Tensor] = None,
                  V: Optional[torch.Tensor] = None, stream=None):
    """(K, V) [T, heads, d] bf16 held at slots[T]; zeros for a slot outside the cache."""
    desc = _check_cache(cache, slots)
    if slots.dim() != 1:
        raise ValueError(f"slots has shape {list(slots.shape)}, expected [T]")
    T = slots.shape[0]
    shape = (T, desc.heads, desc.d)
    for name, t in (("K", K), ("V", V)):
        if t is not None:
            _expect(t, name, shape, torch.bfloat16, slots.device)
    if K is None and V is None:
        both = (slots.new_empty((2, *shape), dtype=torch.bfloat16) if stream is None
                else _empty(slots, (2, *shape), stream, torch.bfloat16))
        K, V = both.unbind()
    elif K is None:
        K = _empty(V, shape, stream)
    elif V is None:
        V = _empty(K, shape, stream)
    st = _lib.kv_cache_read(cache.ref, _int32(slots, "slots", (T,), slots), T, DN_BF16, _dev(K, "K"), _dev(V, "V"),
                            _stream_of(stream, slots))
    if st:
        raise DNError("kv_cache_read", st)
    return K, V


def attention_cache_workspace_bytes(T: int, B: int, q_heads: int, heads: int, d: int, table_width: int,
                                    prefix_len: int = 0) -> int:
    return int(_lib.attention_cache_workspace_bytes(T, B, q_heads, heads, d, table_width, prefix_len))


def _attention_cache_args(Q, cache, block_table, q_start, kv_len, prefix_len, scale, workspace, out, stream):
    """The call's arguments before and after the prefix's, and the output and scratch, which the caller holds
    until the kernels are launched."""
    desc = _check_cache(cache, Q)
    if Q.dim() != 3 or Q.shape[2] != desc.d or Q.shape[1] % desc.heads:
        raise ValueError(f"Q has shape {list(Q.shape)}, expected [T, a multiple of {desc.heads}, {desc.d}]")
    if block_table.dim() != 2:
        raise ValueError(f"block_table has shape {list(block_table.shape)}, expected [B, pages]")
    T, q_heads, d = Q.shape
    B, width = block_table.shape
    qp, qs = _rows(Q, "Q")
    if out is None:
        out = Q.new_empty((T, q_heads, d)) if stream is None else _empty(Q, (T, q_heads, d), stream)
        op = out.data_ptr()
    else:
        if not _like(out, Q.shape, Q):
            _expect(out, "out", (T, q_heads, d), Q.dtype, Q.device)
        op = _dev(out, "out")
    if workspace is None:
        n = attention_cache_workspace_bytes(T, B, q_heads, desc.heads, d, width, prefix_len)
        workspace = _empty(Q, max(n, 16), stream, torch.uint8)
    elif workspace.dtype is not torch.uint8 or workspace.get_device() != Q.get_device() or not workspace.is_contiguous():
        _expect(workspace, "workspace", None, torch.uint8, Q.device)
        _dev(workspace, "workspace")
    head = (qp, qs, T, q_heads, cache.ref)
    tail = (_int32(block_table, "block_table", (B, width), Q), width, _int32(q_start, "q_start", (B + 1,), Q),
            _int32(kv_len, "kv_len", (B,), Q), B, d ** -0.5 if scale is None else float(scale), _dt(Q),
            workspace.data_ptr(), workspace.numel(), op)
    return head, tail, out, workspace


def attention_cache_deferred(Q: torch.Tensor, cache: KVCache, block_table: torch.Tensor, q_start: torch.Tensor,
                             kv_len: torch.Tensor, scale: Optional[float] = None,
                             workspace: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                             stream=None) -> torch.Tensor:
    """Attention of ragged sequences over the cache: rows q_start[b] .. q_start[b + 1] - 1 of
    Q[T, q_heads, d] are sequence b's new tokens, the last of its kv_len[b] cached ones, which lie in
    pages block_table[b]; each sees the keys up to its own.  scale defaults to 1/sqrt(d)."""
    head, tail, out, held = _attention_cache_args(Q, cache, block_table, q_start, kv_len, 0, scale, workspace, out, stream)
    st = _lib.attention_cache_deferred(*head, *tail, _stream_of(stream, Q))
    if st:
        raise DNError("attention_cache_deferred", st)
    return out


def attention_shared_prefix_deferred(Q: torch.Tensor, cache: KVCache, prefix_table: torch.Tensor, prefix_len: int,
                                     block_table: torch.Tensor, q_start: torch.Tensor, kv_len: torch.Tensor,
                                     scale: Optional[float] = None, workspace: Optional[torch.Tensor] = None,
                                     out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """attention_cache_deferred of sequences that share their first prefix_len tokens, in pages
    prefix_table: read once for all of them.  kv_len counts each sequence's own tokens."""
    prefix_len = int(prefix_len)
    pages = (prefix_len + DN_KV_PAGE - 1) // DN_KV_PAGE
    if prefix_table.dim() != 1 or prefix_table.shape[0] < pages:
        raise ValueError(f"prefix_table has shape {list(prefix_table.shape)}, expected [at least {pages}]")
    head, tail, out, held = _attention_cache_args(Q, cache, block_table, q_start, kv_len, prefix_len, scale, workspace, out,
                                                  stream)
    pp = _int32(prefix_table, "prefix_table", tuple(prefix_table.shape), Q)
    st = _lib.attention_shared_prefix_deferred(*head, pp, prefix_len, *tail, _stream_of(stream, Q))
    if st:
        raise DNError("attention_shared_prefix_deferred", st)
    return out


# ------------------------------------------------------------------------------- products in 8 bits
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _launch(f, dev: int, *args):
    """f(*args), called on device dev.  Raises if it refuses."""
    if _current_device() == dev:
        st = f(*args)
    else:
        with torch.cuda.device(dev):
            st = f(*args)
    if st:
        raise DNError(f.__name__, st)


def _ptr(t: Optional[torch.Tensor], name: str, shape, dtype, device: int):
    """Pointer of a contiguous GPU tensor of this shape and type; None for None."""
    if t is None:
        return None
    if not (isinstance(t, torch.Tensor) and t.shape == shape and t.dtype is dtype and t.get_device() == device
            and t.is_contiguous()):
        _expect(t, name, shape, dtype, torch.device("cuda", device))
        return _dev(t, name)
    return t.data_ptr()


def _rows_of(x: torch.Tensor):
    """Pointer and sizes of x[M, K], and its device."""
    if not isinstance(x, torch.Tensor) or x.dim() != 2:
        raise ValueError(f"x has shape {list(x.shape)}, expected [M, K]")
    M, K = x.shape
    return _dev(x, "x"), M, K, x.get_device()


def _made(x, t, name, shape, dtype, dev, stream):
    """(tensor, pointer) of an output: the one given, or one made for the call."""
    if t is None:
        if stream is not None:
            t = _empty(x, shape, stream, dtype)
        elif shape == x.shape and x.is_contiguous():  # the quickest of torch's ways
            t = torch.empty_like(x, dtype=dtype)
        else:
            t = x.new_empty(shape, dtype=dtype)
        return t, t.data_ptr()
    return t, _ptr(t, name, shape, dtype, dev)


def _norm_args(x, residual, gamma, total, stream):
    """What both norms take: pointer and sizes of x, pointers of the residual, gamma and the sum, the sum."""
    xp, M, K, dev = _rows_of(x)
    rp = sp = None
    if residual is not None:
        rp = _ptr(residual, "residual", (M, K), x.dtype, dev)
        total, sp = _made(x, total, "total", (M, K), x.dtype, dev, stream)
    elif total is not None:
        raise ValueError("there is no residual to sum")
    return xp, M, K, dev, rp, _ptr(gamma, "gamma", (K,), x.dtype, dev), sp, total


def residual_rmsnorm(x: torch.Tensor, residual: Optional[torch.Tensor] = None, gamma: Optional[torch.Tensor] = None,
                     eps: float = 1e-5, total: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                     stream=None):
    """(RMSNorm(x + residual) * gamma, x + residual) of x[M, K] and residual[M, K]; without a residual the
    second is None.  total may be x or residual: the stream updated in place."""
    xp, M, K, dev, rp, gp, sp, total = _norm_args(x, residual, gamma, total, stream)
    out, op = _made(x, out, "out", (M, K), x.dtype, dev, stream)
    _launch(_lib.residual_rmsnorm, dev, xp, rp, gp, M, K, eps, _dt(x), sp, op, _stream_of(stream, x))
    return out, total


def residual_rmsnorm_fp8(x: torch.Tensor, residual: Optional[torch.Tensor] = None, gamma: Optional[torch.Tensor] = None,
                         eps: float = 1e-5, total: Optional[torch.Tensor] = None, codes: Optional[torch.Tensor] = None,
                         scales: Optional[torch.Tensor] = None, stream=None):
    """(codes, scales, x + residual): residual_rmsnorm with its rows as e4m3 codes [M, K] and one scale a row."""
    xp, M, K, dev, rp, gp, sp, total = _norm_args(x, residual, gamma, total, stream)
    codes, cp = _made(x, codes, "codes", (M, K), torch.float8_e4m3fn, dev, stream)
    scales, scp = _made(x, scales, "scales", (M,), torch.float32, dev, stream)
    _launch(_lib.residual_rmsnorm_fp8, dev, xp, rp, gp, M, K, eps, _dt(x), sp, cp, scp, _stream_of(stream, x))
    return codes, scales, total


def rows_fp8(x: torch.Tensor, codes: Optional[torch.Tensor] = None, scales: Optional[torch.Tensor] = None, stream=None):
    """(codes, scales): the rows of x[M, K] as e4m3 codes and one scale each, x = codes * scales[:, None]."""
    xp, M, K, dev = _rows_of(x)
    codes, cp = _made(x, codes, "codes", (M, K), torch.float8_e4m3fn, dev, stream)
    scales, scp = _made(x, scales, "scales", (M,), torch.float32, dev, stream)
    _launch(_lib.rows_fp8, dev, xp, M, K, _dt(x), cp, scp, _stream_of(stream, x))
    return codes, scales


@dataclasses.dataclass
class PreparedFp8:
    """Weights of linear_fp8: the packed device buffer and its descriptor."""
    packed: torch.Tensor
    desc: LinearFp8Weights

    def __post_init__(self):
        self.ref = ctypes.byref(self.desc)

    @property
    def K(self):
        return self.desc.K

    @property
    def N(self):
        return self.desc.N

    @property
    def gated(self):
        return bool(self.desc.gated)


def linear_fp8_packed_bytes(K: int, N: int, gated: bool = False) -> int:
    return int(_lib.linear_fp8_packed_bytes(K, N, int(gated)))


def linear_fp8_prepare(W: torch.Tensor, scales: Optional[torch.Tensor] = None, gamma: Optional[torch.Tensor] = None,
                       bias: Optional[torch.Tensor] = None, up: Optional[torch.Tensor] = None,
                       up_scales: Optional[torch.Tensor] = None, up_bias: Optional[torch.Tensor] = None,
                       stream=None) -> PreparedFp8:
    """Weights of linear_fp8 from W[K, N]: float8_e4m3fn codes with one fp32 scale per column, or fp32 or
    bf16 values that are quantised here (with gamma[K]: Diag(gamma) W).  bias[N] is fp32.  up[K, N], with its own
    scales and bias, makes the weights gated: act(x W + bias) * (x up + up_bias)."""
    if W.dim() != 2:
        raise ValueError(f"W has shape {list(W.shape)}, expected [K, N]")
    K, N = W.shape
    dt = DN_E4M3 if W.dtype is torch.float8_e4m3fn else _dt(W)
    _expect(gamma, "gamma", (K,), W.dtype, W.device)
    _expect(up, "up", (K, N), W.dtype, W.device)
    for name, t in (("scales", scales), ("bias", bias), ("up_scales", up_scales), ("up_bias", up_bias)):
        _expect(t, name, (N,), torch.float32, W.device)
    nbytes = linear_fp8_packed_bytes(K, N, up is not None)
    if nbytes == 0:
        raise DNError("linear_fp8_packed_bytes", 2)
    packed = _empty(W, nbytes, stream, torch.uint8)
    desc = LinearFp8Weights()
    _launch(_lib.linear_fp8_prepare, W.get_device(), _dev(W, "W"), _dev(scales, "scales"), _dev(gamma, "gamma"),
            _dev(bias, "bias"), _dev(up, "up"), _dev(up_scales, "up_scales"), _dev(up_bias, "up_bias"), K, N, dt,
            packed.data_ptr(), nbytes, ctypes.byref(desc), _stream_of(stream, W))
    return PreparedFp8(packed, desc)


def linear_fp8_workspace_bytes(M: int, w: PreparedFp8) -> int:
    return int(_lib.linear_fp8_workspace_bytes(M, w.ref))


def _scratch(x: torch.Tensor, workspace: Optional[torch.Tensor], need, sizes, stream):
    """Pointer and bytes of the workspace given, or of one of need(*sizes) bytes (None for 0), and what holds it."""
    if workspace is None:
        n = need(*sizes)
        if not n:
            return None, 0, None
        workspace = _empty(x, n, stream, torch.uint8)
    elif workspace.dtype is not torch.uint8 or workspace.get_device() != x.get_device() or not workspace.is_contiguous():
        _expect(workspace, "workspace", None, torch.uint8, x.device)
        _dev(workspace, "workspace")
    return workspace.data_ptr(), workspace.numel(), workspace


def linear_fp8(x: torch.Tensor, x_scales: torch.Tensor, w: PreparedFp8, activation: str = "none",
               residual: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
               out_dtype: Optional[torch.dtype] = None, workspace: Optional[torch.Tensor] = None,
               stream=None) -> torch.Tensor:
    """act(x W + bias) + residual of e4m3 rows x[M, K] with scales x_scales[M] (gated weights: times x up + up_bias
    before the residual).  activation: "none", "relu", "silu", "gelu" or "gelu_tanh".  The result has out_dtype
    (fp32 or bf16; by default out's or residual's type, else bf16); residual may be out."""
    if not isinstance(w, PreparedFp8):
        raise TypeError("w must come from linear_fp8_prepare")
    act = ACTIVATIONS.get(activation)
    if act is None:
        raise ValueError(f"unknown activation {activation!r}")
    desc = w.desc
    K, N, dev = desc.K, desc.N, w.packed.get_device()
    if x.dim() != 2:
        raise ValueError(f"x has shape {list(x.shape)}, expected [M, {K}]")
    M = x.shape[0]
    xp = _ptr(x, "x", (M, K), torch.float8_e4m3fn, dev)
    sp = _ptr(x_scales, "x_scales", (M,), torch.float32, dev)
    if sp is None:
        raise ValueError("x_scales is required")
    if out_dtype is None:
        like = out if out is not None else residual
        out_dtype = torch.bfloat16 if like is None else like.dtype
    if out_dtype is not torch.bfloat16 and out_dtype is not torch.float32:
        raise TypeError(f"unsupported out_dtype {out_dtype}")
    rp = _ptr(residual, "residual", (M, N), out_dtype, dev)
    out, op = _made(x, out, "out", (M, N), out_dtype, dev, stream)
    wp, wn, held = _scratch(x, workspace, _lib.linear_fp8_workspace_bytes, (M, w.ref), stream)
    _launch(_lib.linear_fp8, dev, xp, sp, w.ref, M, act, rp, DN_BF16 if out_dtype is torch.bfloat16 else DN_F32, wp, wn, op,
            _stream_of(stream, x))
    return out


# ------------------------------------------------------------------------------- log probabilities
def token_logprobs_workspace_bytes(T: int, V: int, top: int = 0) -> int:
    return int(_lib.token_logprobs_workspace_bytes(T, V, top))


def token_logprobs(logits: torch.Tensor, targets: Optional[torch.Tensor] = None, top: int = 0, scale: float = 1.0,
                   entropy: bool = True, workspace: Optional[torch.Tensor] = None, stream=None):
    """{"logprobs", "entropy", "top_logprobs", "top_ids"} of softmax(scale * logits), scale >= 2^-96, for logits[T, V] (rows may be
    strided, V and the stride odd): ln p of targets[T, n] (int32; 0 for a negative one), the entropy [T], and the
    `top` likeliest tokens (the lowest id first among equals) with their ln p.  What was not asked for is None."""
    if logits.dim() != 2:
        raise ValueError(f"logits has shape {list(logits.shape)}, expected [T, V]")
    if not logits.is_cuda:
        raise ValueError("logits must be a GPU tensor")
    T, V = logits.shape
    if logits.stride(1) != 1 and V != 1:
        raise ValueError("logits must be contiguous within a row")
    stride = logits.stride(0) if T != 1 else V
    dev = logits.get_device()
    n, tp, lp, ep, kp, ip = 0, None, None, None, None, None
    given = spread = likely = ids = None
    if targets is not None:
        if targets.dim() != 2:
            raise ValueError(f"targets has shape {list(targets.shape)}, expected [T, n]")
        n = targets.shape[1]
        tp = _int32(targets, "targets", (T, n), logits)
        if n == 0:
            tp = None
    new = logits.new_empty if stream is None else lambda shape, dtype: _empty(logits, shape, stream, dtype)
    if n:
        given = new((T, n), dtype=torch.float32)
        lp = given.data_ptr()
    if entropy:
        spread = new((T,), dtype=torch.float32)
        ep = spread.data_ptr()
    if top > 0:
        likely, ids = new((T, top), dtype=torch.float32), new((T, top), dtype=torch.int32)
        kp, ip = likely.data_ptr(), ids.data_ptr()
    wp, wn, held = _scratch(logits, workspace, _lib.token_logprobs_workspace_bytes, (T, V, top), stream)
    _launch(_lib.token_logprobs, dev, logits.data_ptr(), stride, T, V, _dt(logits), scale, tp, n, top, lp, ep, kp, ip, wp, wn,
            _stream_of(stream, logits))
    return {"logprobs": given, "entropy": spread, "top_logprobs": likely, "top_ids": ids}
