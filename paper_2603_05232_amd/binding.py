"""Thin binding of libslidesparse.so: argument marshalling only, by ctypes and, for the calls of a forward pass, by the
extension module _calls (csrc/py_calls.cpp).

Every function has the name and argument order of its C entry point in
include/slidesparse.h; tensors are torch CUDA tensors used purely as device
memory, and work is enqueued on torch's current stream.  There is no CPU
fallback: if the library is missing, loading raises."""
from __future__ import annotations

import ctypes
import functools
import math
import os
import sysconfig
import types
import warnings

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libslidesparse.so")
CALLS_PATH = os.path.join(_PKG, "_calls" + sysconfig.get_config_var("EXT_SUFFIX"))

SS_I8, SS_FP8_E4M3, SS_BF16, SS_FP16 = 0, 1, 2, 3
SS_IN_F32, SS_IN_BF16 = 0, 1
DTYPE_CODE = {"i8": SS_I8, "fp8": SS_FP8_E4M3, "bf16": SS_BF16, "fp16": SS_FP16}
EXPORTS = ("slide_lifted_k", "slide_lifted_ld", "slide_packed_sizes", "slide_prune_quant", "slide_decompose",
           "slide_decompose_canonical", "act_lift_quant", "slide_sparse_gemm", "dense_gemm",
           "slide_gemm_workspace_bytes", "slide_sparse_gemm_ws", "dense_gemm_ws",
           "slide_packed_sizes_fused", "slide_decompose_fused", "slide_sparse_gemm_fused", "slide_sparse_gemm_fused_ws",
           "slide_static_scratch_bytes", "slide_sparse_gemm_static",
           "mx4_row_bytes", "mx4_row_scales", "mx4_quant", "mx4_dequant", "mx4_packed_sizes", "mx4_pack", "mx4_gemm_workspace_bytes", "mx4_gemm",
           "mx4_grouped_gemm", "expert_route_workspace_bytes", "expert_route", "expert_combine",
           "kv_page_bytes", "kv_tables_workspace_bytes", "kv_tables", "kv_write", "kv_read", "kv_attention_workspace_bytes", "kv_attention",
           "ss_status_string", "slide_format_version")
# entry points that the extension module calls, at the addresses of the library loaded here (order of its bind())
_CALLED = ("slide_lifted_ld", "act_lift_quant", "slide_sparse_gemm_ws", "slide_sparse_gemm_fused_ws")
_CALLED_MX4 = ("mx4_row_bytes", "mx4_quant", "mx4_dequant", "mx4_packed_sizes", "mx4_gemm", "mx4_grouped_gemm", "expert_route_workspace_bytes", "expert_route",
               "expert_combine")                          # of its bind_mx4()
_CALLED_KV = ("kv_page_bytes", "kv_tables_workspace_bytes", "kv_tables", "kv_write", "kv_read", "kv_attention")      # of its bind_kv()

# the calls that it does
_MODULE_CALLS = ("act_lift_quant", "slide_sparse_gemm", "slide_sparse_gemm_fused", "mx4_quant", "mx4_dequant", "mx4_product", "expert_route", "expert_combine", "kv_tables", "kv_write", "kv_read",
                 "kv_attention")

_lib = None
_calls = None
_mx4_calls = None                                         # the module again, for the 4-bit expert layer's calls
_kv_calls = None                                          # and for those on a cache


class SlideSparseError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {status_string(code)} (status {code})")


def load():
    """Load the shared library (raises if it has not been built)."""
    global _lib, _calls, _mx4_calls, _kv_calls
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} not found: build it first (python -m paper_2603_05232_amd.build)")
    lib = ctypes.CDLL(LIB_PATH)
    i64, i32, vp, sz = ctypes.c_int64, ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t
    lib.slide_lifted_k.argtypes = [i64, i32]
    lib.slide_lifted_k.restype = i64
    lib.slide_lifted_ld.argtypes = [i64, i32, i32]
    lib.slide_lifted_ld.restype = i64
    lib.slide_packed_sizes.argtypes = [i64, i64, i32, i32, ctypes.POINTER(sz), ctypes.POINTER(sz)]
    lib.slide_prune_quant.argtypes = [vp, i32, i64, i64, i32, i32, vp, vp, vp]
    lib.slide_decompose.argtypes = [vp, i64, i64, i32, i32, vp, vp, vp, vp]
    lib.slide_decompose_canonical.argtypes = [vp, i64, i64, i32, i32, vp, vp, vp, vp]
    lib.act_lift_quant.argtypes = [vp, i32, i64, i64, i64, i32, i32, vp, vp, vp]
    lib.slide_sparse_gemm.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, i32, vp, i64, vp]
    lib.dense_gemm.argtypes = [vp, vp, vp, vp, i64, i64, i64, i32, vp, i64, vp]
    lib.slide_sparse_gemm_ws.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, i32, vp, i64, vp, sz, vp]
    lib.dense_gemm_ws.argtypes = [vp, vp, vp, vp, i64, i64, i64, i32, vp, i64, vp, sz, vp]
    lib.slide_packed_sizes_fused.argtypes = [i64, i64, i32, i32, ctypes.POINTER(sz), ctypes.POINTER(sz)]
    lib.slide_decompose_fused.argtypes = [vp, i64, i64, i32, i32, vp, vp, vp, vp]
    lib.slide_sparse_gemm_fused.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, i64, i32, i32, vp, i64, vp]
    lib.slide_sparse_gemm_fused_ws.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, i64, i32, i32, vp, i64, vp, sz, vp]
    lib.slide_static_scratch_bytes.argtypes = []
    lib.slide_static_scratch_bytes.restype = sz
    lib.slide_sparse_gemm_static.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, i32, vp, i64, vp]
    lib.slide_sparse_gemm_static.restype = i32
    lib.slide_gemm_workspace_bytes.argtypes = [i64, i64, i64, i32]
    lib.slide_gemm_workspace_bytes.restype = sz
    for name in ("slide_packed_sizes", "slide_prune_quant", "slide_decompose", "slide_decompose_canonical",
                 "act_lift_quant", "slide_sparse_gemm", "dense_gemm", "slide_sparse_gemm_ws", "dense_gemm_ws",
                 "slide_packed_sizes_fused", "slide_decompose_fused", "slide_sparse_gemm_fused"):
        getattr(lib, name).restype = i32
    for name, args, res in (("mx4_row_bytes", [i64], i64), ("mx4_row_scales", [i64], i64),
                            ("mx4_quant", [vp, i32, i64, i64, i64, vp, i64, vp, vp, vp], i32),
                            ("mx4_dequant", [vp, vp, i64, i64, i32, vp, i64, vp], i32),
                            ("mx4_packed_sizes", [i64, i64, i64, i32, ctypes.POINTER(sz), ctypes.POINTER(sz)], i32),
                            ("mx4_pack", [vp, vp, i64, i64, i64, i32, vp, vp, vp], i32),
                            ("mx4_gemm_workspace_bytes", [i64, i64, i64, i64, i32], sz),
                            ("mx4_gemm", [vp, vp, vp, vp, i64, i64, i64, i32, vp, i64, vp, sz, vp], i32),
                            ("mx4_grouped_gemm", [vp, vp, vp, vp, vp, i64, i64, i64, i64, i32, vp, i64, vp, sz, vp], i32),
                            ("expert_route_workspace_bytes", [i64, i64, i64], sz),
                            ("expert_route", [vp, i32, i64, i64, i64, i32, i32, vp, vp, vp, vp, vp, vp, sz, vp], i32),
                            ("expert_combine", [vp, i64, i64, i64, vp, vp, i64, i32, vp, i64, vp, i64, vp], i32),
                            ("kv_page_bytes", [i64, i64, i64, i32], i64),
                            ("kv_tables_workspace_bytes", [i64, i64], sz),
                            ("kv_tables", [vp, vp, i64, vp, i64, i64, i64, vp, i64, vp, i64, vp, vp, vp, vp, vp, sz, vp], i32),
                            ("kv_write", [vp, i64, i64, vp, i64, i64, i32, i64, i64, i64, vp, vp, i64, i64, i32, vp], i32),
                            ("kv_read", [vp, i64, i64, i32, vp, i64, i64, i64, i32, vp, i64, i64, vp, i64, i64, vp], i32),
                            ("kv_attention_workspace_bytes", [i64, i64, i64, i64], sz),
                            ("kv_attention", [vp, i32, i64, i64, vp, i64, i64, i32, vp, i64, i64, vp, i64, i64, i64, i64, ctypes.c_float, i64, vp, i64, i64, vp, sz, vp], i32)):
        fn = getattr(lib, name)
        fn.argtypes, fn.restype = args, res
    lib.ss_status_string.argtypes = [i32]
    lib.ss_status_string.restype = ctypes.c_char_p
    lib.slide_format_version.restype = i32
    calls = _load_calls(lib)
    _lib, _calls, _mx4_calls, _kv_calls = lib, calls, calls, calls
    return lib


def _load_calls(lib):
    """The extension module, told which library to call; without one that was built for this torch and from these sources, as far as its names tell, a stand-in
    that leaves every call to the general path, which needs the library alone."""
    try:
        from . import _calls as calls
        if calls.torch_version != str(torch.__version__):
            raise ImportError(f"built for torch {calls.torch_version}, not {torch.__version__}")
        missing = [name for name in (*_MODULE_CALLS, "bind", "bind_mx4", "bind_kv") if not hasattr(calls, name)]
        if missing:
            raise ImportError(f"an older build, without {', '.join(missing)}")
    except (ImportError, AttributeError) as e:
        warnings.warn(f"{CALLS_PATH} cannot be used ({e}): calls go through ctypes, 6 us more on the host for each layer", RuntimeWarning, stacklevel=3)
        return types.SimpleNamespace(**dict.fromkeys(_MODULE_CALLS, lambda *args: None))
    calls.bind(SlideSparseError, *(ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in _CALLED))
    calls.bind_mx4(*(ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in _CALLED_MX4))
    calls.bind_kv(*(ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in _CALLED_KV))
    return calls


def status_string(code: int) -> str:
    return load().ss_status_string(int(code)).decode()


def _check(code: int, where: str) -> None:
    if code != 0:
        raise SlideSparseError(code, where)


# Few-token calls are bound by the time between launches, most of which is spent here.  The calls of a forward pass
# (act_lift_quant and the sparse GEMMs) therefore go to the extension module first, which does plain calls (exact torch
# tensors on the GPU, no active mode, nothing to refuse) and answers None to any other; what follows is the general path,
# which refuses what has to be.  It does no more than the call needs either: addresses go to ctypes as plain integers (None is NULL), and
# the stream handle is read without building a torch.cuda.Stream object (0.2 instead of 2.8 us; a launch itself is 2.8 us).
# Quantisation + GEMM of 16 x 512 x 512 on the host: 15.3 us by the general path, 9.1 by the module.
_STORAGE_DTYPE = {"i8": torch.int8, "fp8": torch.uint8, "bf16": torch.bfloat16, "fp16": torch.float16}
_IN_CODE = {torch.float32: SS_IN_F32, torch.bfloat16: SS_IN_BF16}
_UNSCALED = ("bf16", "fp16")


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream():
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _in_code(t: torch.Tensor) -> int:
    code = _IN_CODE.get(t.dtype)
    if code is None:
        raise TypeError(f"activations/weights must be float32 or bfloat16, got {t.dtype}")
    return code


def _storage_dtype(dtype: str) -> torch.dtype:
    return _STORAGE_DTYPE[dtype]


def slide_lifted_k(K: int, N: int) -> int:
    return int(load().slide_lifted_k(K, N))


@functools.lru_cache(maxsize=4096, typed=True)       # typed: 512.0 equals 512 but is refused
def slide_lifted_ld(K: int, N: int, dtype: str) -> int:
    return int(load().slide_lifted_ld(K, N, DTYPE_CODE[dtype]))


def slide_packed_sizes(O: int, K: int, N: int, dtype: str):
    v, m = ctypes.c_size_t(), ctypes.c_size_t()
    _check(load().slide_packed_sizes(O, K, N, DTYPE_CODE[dtype], ctypes.byref(v), ctypes.byref(m)), "slide_packed_sizes")
    return int(v.value), int(m.value)


def slide_prune_quant(W: torch.Tensor, N: int, dtype: str):
    """W[O,K] fp32/bf16 on the GPU -> (Wq[O,K], s_w[O] or None)."""
    O, K = W.shape
    assert W.is_cuda and W.is_contiguous()
    Wq = torch.empty((O, K), dtype=_storage_dtype(dtype), device=W.device)
    s_w = None if dtype in ("bf16", "fp16") else torch.empty((O,), dtype=torch.float32, device=W.device)
    _check(load().slide_prune_quant(_ptr(W), _in_code(W), O, K, N, DTYPE_CODE[dtype], _ptr(Wq), _ptr(s_w), _stream()),
           "slide_prune_quant")
    return Wq, s_w


def slide_decompose(Wq: torch.Tensor, N: int, dtype: str, count_violations: bool = False):
    """Wq[O,K] -> (w_vals, w_meta[, violations]) in the packed layout."""
    O, K = Wq.shape
    assert Wq.is_cuda and Wq.is_contiguous()
    vb, mb = slide_packed_sizes(O, K, N, dtype)
    w_vals = torch.empty((vb,), dtype=torch.uint8, device=Wq.device)
    w_meta = torch.empty((mb,), dtype=torch.uint8, device=Wq.device)
    viol = torch.zeros((1,), dtype=torch.int32, device=Wq.device) if count_violations else None
    _check(load().slide_decompose(_ptr(Wq), O, K, N, DTYPE_CODE[dtype], _ptr(w_vals), _ptr(w_meta), _ptr(viol), _stream()),
           "slide_decompose")
    return (w_vals, w_meta, viol) if count_violations else (w_vals, w_meta)


def slide_decompose_canonical(Wq: torch.Tensor, N: int, dtype: str):
    """Wq[O,K] -> (vals[O,K'/2], idx[O,K'/4] uint8, violations[1] int32)."""
    O, K = Wq.shape
    assert Wq.is_cuda and Wq.is_contiguous()
    Kp = slide_lifted_k(K, N)
    if Kp < 0:
        raise SlideSparseError(3 if 2 <= N <= 8 else 2, "slide_decompose_canonical")
    vals = torch.empty((O, Kp // 2), dtype=Wq.dtype, device=Wq.device)
    idx = torch.empty((O, Kp // 4), dtype=torch.uint8, device=Wq.device)
    viol = torch.zeros((1,), dtype=torch.int32, device=Wq.device)
    _check(load().slide_decompose_canonical(_ptr(Wq), O, K, N, DTYPE_CODE[dtype], _ptr(vals), _ptr(idx), _ptr(viol), _stream()),
           "slide_decompose_canonical")
    return vals, idx, viol


def act_lift_quant(X: torch.Tensor, N: int, dtype: str, out=None, s_x=None):
    """X[M,K] fp32/bf16 (row stride allowed) -> (X_lifted[M,Kld], s_x[M] or None)."""
    if _calls is None:
        load()
    done = _calls.act_lift_quant(X, N, dtype, out, s_x)
    if done is not None:
        return done
    M, K = X.shape
    ldx, inner = X.stride()
    assert X.is_cuda and inner == 1
    Kp = slide_lifted_ld(K, N, dtype)
    if Kp < 0:
        raise SlideSparseError(3 if 2 <= N <= 8 else 2, "act_lift_quant")
    if out is None:
        out = X.new_empty((M, Kp), dtype=_STORAGE_DTYPE[dtype])
    if s_x is None and dtype not in _UNSCALED:
        s_x = X.new_empty((M,), dtype=torch.float32)
    code = load().act_lift_quant(X.data_ptr(), _in_code(X), M, K, ldx if M > 1 else K, N, DTYPE_CODE[dtype], out.data_ptr(), _ptr(s_x), _stream())
    if code:
        _check(code, "act_lift_quant")
    return out, s_x


def slide_gemm_workspace_bytes(M: int, O: int, K: int, dtype: str) -> int:
    return int(load().slide_gemm_workspace_bytes(M, O, K, DTYPE_CODE[dtype]))


def slide_sparse_gemm(X_lifted, s_x, w_vals, w_meta, s_w, O: int, dtype: str, out=None, workspace=None):
    """Y[M,O] bf16 = epilogue(X_lifted[M,Kld] . W'^T); workspace: optional uint8 device tensor (slide_sparse_gemm_ws)."""
    if _calls is None:
        load()
    done = _calls.slide_sparse_gemm(X_lifted, s_x, w_vals, w_meta, s_w, O, dtype, out, workspace)
    if done is not None:
        return done
    M, Kp = X_lifted.shape
    assert X_lifted.is_contiguous()
    if out is None:
        out = X_lifted.new_empty((M, O), dtype=torch.bfloat16)
    args = (X_lifted.data_ptr(), _ptr(s_x), _ptr(w_vals), _ptr(w_meta), _ptr(s_w), M, O, Kp, DTYPE_CODE[dtype], out.data_ptr(), out.stride(0))
    if workspace is None:
        code = load().slide_sparse_gemm(*args, _stream())
    else:
        code = load().slide_sparse_gemm_ws(*args, workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream())
    if code:
        _check(code, "slide_sparse_gemm" if workspace is None else "slide_sparse_gemm_ws")
    return out


def dense_gemm(Xq, s_x, Wq, s_w, dtype: str, out=None, workspace=None):
    """Y[M,O] bf16 = epilogue(Xq[M,K] . Wq[O,K]^T); workspace: optional uint8 device tensor (dense_gemm_ws)."""
    M, K = Xq.shape
    O = Wq.shape[0]
    assert Xq.is_contiguous() and Wq.is_contiguous() and Wq.shape[1] == K
    if out is None:
        out = torch.empty((M, O), dtype=torch.bfloat16, device=Xq.device)
    if workspace is None:
        _check(load().dense_gemm(_ptr(Xq), _ptr(s_x), _ptr(Wq), _ptr(s_w), M, O, K, DTYPE_CODE[dtype], _ptr(out),
                                 out.stride(0), _stream()), "dense_gemm")
    else:
        _check(load().dense_gemm_ws(_ptr(Xq), _ptr(s_x), _ptr(Wq), _ptr(s_w), M, O, K, DTYPE_CODE[dtype], _ptr(out),
                                    out.stride(0), _ptr(workspace), workspace.numel() * workspace.element_size(), _stream()),
               "dense_gemm_ws")
    return out


def slide_packed_sizes_fused(O: int, K: int, N: int, dtype: str):
    v, m = ctypes.c_size_t(), ctypes.c_size_t()
    _check(load().slide_packed_sizes_fused(O, K, N, DTYPE_CODE[dtype], ctypes.byref(v), ctypes.byref(m)), "slide_packed_sizes_fused")
    return int(v.value), int(m.value)


def slide_decompose_fused(Wq: torch.Tensor, N: int, dtype: str, count_violations: bool = False):
    """Wq[O,K] -> (w_vals, w_meta[, violations]) in the window order of slide_sparse_gemm_fused."""
    O, K = Wq.shape
    assert Wq.is_cuda and Wq.is_contiguous()
    vb, mb = slide_packed_sizes_fused(O, K, N, dtype)
    w_vals = torch.empty((vb,), dtype=torch.uint8, device=Wq.device)
    w_meta = torch.empty((mb,), dtype=torch.uint8, device=Wq.device)
    viol = torch.zeros((1,), dtype=torch.int32, device=Wq.device) if count_violations else None
    _check(load().slide_decompose_fused(_ptr(Wq), O, K, N, DTYPE_CODE[dtype], _ptr(w_vals), _ptr(w_meta), _ptr(viol), _stream()),
           "slide_decompose_fused")
    return (w_vals, w_meta, viol) if count_violations else (w_vals, w_meta)


def slide_sparse_gemm_fused(Xq, s_x, w_vals, w_meta, s_w, O: int, K: int, N: int, dtype: str, out=None, workspace=None):
    """Y[M,O] bf16 = epilogue(Psi(Xq[M, :K]) . W'^T) from unlifted quantised activations (row stride = Xq.stride(0)).
    workspace: optional uint8 device tensor (slide_gemm_workspace_bytes(M, O, K, dtype) bytes) that lets the kernels for
    small and medium M split the k range."""
    if _calls is None:
        load()
    done = _calls.slide_sparse_gemm_fused(Xq, s_x, w_vals, w_meta, s_w, O, K, N, dtype, out, workspace)
    if done is not None:
        return done
    M, width = Xq.shape
    ldx, inner = Xq.stride()
    assert Xq.is_cuda and inner == 1 and width >= K
    if out is None:
        out = Xq.new_empty((M, O), dtype=torch.bfloat16)
    args = (Xq.data_ptr(), _ptr(s_x), _ptr(w_vals), _ptr(w_meta), _ptr(s_w), M, O, K, ldx if M > 1 else width, N, DTYPE_CODE[dtype], out.data_ptr(),
            out.stride(0))
    if workspace is None:
        code = load().slide_sparse_gemm_fused(*args, _stream())
    else:
        code = load().slide_sparse_gemm_fused_ws(*args, workspace.data_ptr(), workspace.numel(), _stream())
    if code:
        _check(code, "slide_sparse_gemm_fused" if workspace is None else "slide_sparse_gemm_fused_ws")
    return out


def slide_static_scratch_bytes() -> int:
    return int(load().slide_static_scratch_bytes())


def slide_sparse_gemm_static(X_lifted, s_x, w_vals, w_meta, s_w, O: int, dtype: str, out):
    """slide_sparse_gemm with the split-k scratch in the library's static device array; `out` is required: this call
    path allocates nothing."""
    M, Kp = X_lifted.shape
    assert X_lifted.is_contiguous() and out is not None
    _check(load().slide_sparse_gemm_static(_ptr(X_lifted), _ptr(s_x), _ptr(w_vals), _ptr(w_meta), _ptr(s_w), M, O, Kp,
                                           DTYPE_CODE[dtype], _ptr(out), out.stride(0), _stream()), "slide_sparse_gemm_static")
    return out


# ---- microscaled 4-bit operands and layers of experts -------------------------------------------------------------------------

# A kernel reads and writes through every address that it is given, so each of them has to lie on the GPU of the operator's first tensor.

def _beside(t: torch.Tensor, first: torch.Tensor) -> bool:
    return first.is_cuda and t.is_cuda and t.get_device() == first.get_device()


def _row_stride(t: torch.Tensor, first: torch.Tensor) -> int:
    """Elements between the rows of a matrix whose rows are dense (of a single row: its width)."""
    rows, width = t.shape
    assert _beside(t, first) and (width < 2 or t.stride(1) == 1)
    return t.stride(0) if rows > 1 else width


def _dense_i32(t: torch.Tensor, what: str, first: torch.Tensor, dims: int = 1) -> int:
    if t.dtype != torch.int32:
        raise TypeError(f"{what} must be int32, got {t.dtype}")
    assert _beside(t, first) and t.is_contiguous() and t.dim() == dims
    return t.data_ptr()


def _workspace(t, first: torch.Tensor):
    """(address, bytes) of an optional workspace."""
    if t is None:
        return None, 0
    assert _beside(t, first) and t.is_contiguous()
    return t.data_ptr(), t.numel() * t.element_size()


def _mx4_operand(codes: torch.Tensor, scales: torch.Tensor, K: int, first: torch.Tensor):
    """Checks that codes[R, 128 U] and scales[U, R, 8] are rows of K values."""
    assert _beside(codes, first) and _beside(scales, first) and codes.is_contiguous() and scales.is_contiguous() and codes.dtype == scales.dtype == torch.uint8
    assert codes.shape[1] == mx4_row_bytes(K) and scales.shape == (codes.shape[1] // 128, codes.shape[0], 8)


@functools.lru_cache(maxsize=4096, typed=True)
def mx4_row_bytes(K: int) -> int:
    return int(load().mx4_row_bytes(K))


def mx4_row_scales(K: int) -> int:
    return int(load().mx4_row_scales(K))


def mx4_quant(X: torch.Tensor, rows=None, codes=None, scales=None):
    """X[M,K] fp32/bf16 (row stride allowed) -> (codes[R, 128 U] uint8, scales[U, R, 8] uint8); rows: int32 [R], the row of X that each
    row of codes is made of."""
    if _mx4_calls is None:
        load()
    done = _mx4_calls.mx4_quant(X, rows, codes, scales)
    if done is not None:
        return done
    M, K = X.shape
    R = M if rows is None else rows.shape[0]
    width = mx4_row_bytes(K)
    if width < 0:
        raise SlideSparseError(3, "mx4_quant")
    if codes is None:
        codes = X.new_empty((R, width), dtype=torch.uint8)
    if scales is None:
        scales = X.new_empty((width // 128, R, 8), dtype=torch.uint8)
    assert codes.shape[0] == R
    _mx4_operand(codes, scales, K, X)
    code = load().mx4_quant(X.data_ptr(), _in_code(X), M, K, _row_stride(X, X), None if rows is None else _dense_i32(rows, "rows", X), R, codes.data_ptr(),
                            scales.data_ptr(), _stream())
    if code:
        _check(code, "mx4_quant")
    return codes, scales


def mx4_dequant(codes: torch.Tensor, scales: torch.Tensor, K: int, dtype: torch.dtype = torch.float32, out=None):
    """codes, scales of mx4_quant -> their values [R,K] as fp32 or bf16."""
    if _mx4_calls is None:
        load()
    done = _mx4_calls.mx4_dequant(codes, scales, K, _IN_CODE.get(dtype), out)
    if done is not None:
        return done
    _mx4_operand(codes, scales, K, codes)
    if out is None:
        out = codes.new_empty((codes.shape[0], K), dtype=dtype)
    assert out.shape == (codes.shape[0], K)
    code = load().mx4_dequant(codes.data_ptr(), scales.data_ptr(), codes.shape[0], K, _in_code(out), out.data_ptr(), _row_stride(out, codes), _stream())
    if code:
        _check(code, "mx4_dequant")
    return out


def mx4_packed_sizes(O: int, K: int, experts: int = 1, gated: bool = False):
    v, m = ctypes.c_size_t(), ctypes.c_size_t()
    _check(load().mx4_packed_sizes(experts, O, K, int(gated), ctypes.byref(v), ctypes.byref(m)), "mx4_packed_sizes")
    return int(v.value), int(m.value)


def mx4_pack(codes: torch.Tensor, scales: torch.Tensor, K: int, experts: int = 1, gated: bool = False):
    """Codes of experts x [O,K] weights (gated: of experts x [2 O,K], gate's rows before up's) -> (w_vals, w_meta)."""
    _mx4_operand(codes, scales, K, codes)
    O, rest = divmod(codes.shape[0], experts * (2 if gated else 1))
    if rest:
        raise SlideSparseError(3, "mx4_pack")
    vb, mb = mx4_packed_sizes(O, K, experts, gated)
    w_vals = codes.new_empty((vb,))
    w_meta = codes.new_empty((mb,))
    _check(load().mx4_pack(codes.data_ptr(), scales.data_ptr(), experts, O, K, int(gated), w_vals.data_ptr(), w_meta.data_ptr(), _stream()), "mx4_pack")
    return w_vals, w_meta


def mx4_gemm_workspace_bytes(R: int, O: int, K: int, experts: int = 1, gated: bool = False) -> int:
    return int(load().mx4_gemm_workspace_bytes(R, experts, O, K, int(gated)))


def _mx4_product(name, offsets, codes, scales, w_vals, w_meta, experts, O, K, gated, out, workspace):
    _mx4_operand(codes, scales, K, codes)
    sizes = _mx4_sizes(O, K, experts, gated)
    assert _beside(w_vals, codes) and _beside(w_meta, codes) and w_vals.dtype == w_meta.dtype == torch.uint8
    assert w_vals.is_contiguous() and w_meta.is_contiguous() and (w_vals.numel(), w_meta.numel()) == sizes
    R = codes.shape[0]
    if out is None:
        out = codes.new_empty((R, O), dtype=torch.bfloat16)
    assert out.dtype == torch.bfloat16 and out.shape == (R, O)
    tail = (O, K, int(gated), out.data_ptr(), _row_stride(out, codes), *_workspace(workspace, codes), _stream())
    if offsets is None:
        code = load().mx4_gemm(codes.data_ptr(), scales.data_ptr(), w_vals.data_ptr(), w_meta.data_ptr(), R, *tail)
    else:
        code = load().mx4_grouped_gemm(codes.data_ptr(), scales.data_ptr(), offsets, w_vals.data_ptr(), w_meta.data_ptr(), R, experts, *tail)
    if code:
        _check(code, name)
    return out


_mx4_sizes = functools.lru_cache(maxsize=4096, typed=True)(mx4_packed_sizes)


def mx4_gemm(codes, scales, w_vals, w_meta, O: int, K: int, gated: bool = False, out=None, workspace=None):
    """Y[M,O] bf16 = X . W^T of 4-bit operands (gated: silu(X . Wg^T) * (X . Wu^T)); workspace: optional uint8 device tensor."""
    if _mx4_calls is None:
        load()
    done = _mx4_calls.mx4_product(None, codes, scales, w_vals, w_meta, O, K, gated, out, workspace)
    if done is not None:
        return done
    return _mx4_product("mx4_gemm", None, codes, scales, w_vals, w_meta, 1, O, K, gated, out, workspace)


def mx4_grouped_gemm(codes, scales, offsets, w_vals, w_meta, O: int, K: int, gated: bool = False, out=None, workspace=None):
    """The same with the weights of expert e for the rows offsets[e] .. offsets[e + 1] - 1 (int32, on the device); the others give zeros."""
    if _mx4_calls is None:
        load()
    done = _mx4_calls.mx4_product(offsets, codes, scales, w_vals, w_meta, O, K, gated, out, workspace)
    if done is not None:
        return done
    return _mx4_product("mx4_grouped_gemm", _dense_i32(offsets, "offsets", codes), codes, scales, w_vals, w_meta, offsets.shape[0] - 1, O, K, gated, out, workspace)


def expert_route_workspace_bytes(M: int, E: int, k: int) -> int:
    return int(load().expert_route_workspace_bytes(M, E, k))


def expert_route(logits: torch.Tensor, k: int, renormalise: bool = True, workspace=None):
    """logits[M,E] fp32/bf16 -> (ids[M,k], weights[M,k], slots[M,k], rows[M k], offsets[E + 1]): the k experts of largest score, their softmax
    weights, and the order of the rows by expert."""
    if _mx4_calls is None:
        load()
    done = _mx4_calls.expert_route(logits, k, renormalise, workspace)
    if done is not None:
        return done
    M, E = logits.shape
    if workspace is None:
        n = expert_route_workspace_bytes(M, E, k)
        workspace = logits.new_empty((n,), dtype=torch.uint8) if n else None
    ids, slots = logits.new_empty((2, M, max(k, 0)), dtype=torch.int32)
    weights = logits.new_empty((M, max(k, 0)), dtype=torch.float32)
    rows = logits.new_empty((M * max(k, 0),), dtype=torch.int32)
    offsets = logits.new_empty((E + 1,), dtype=torch.int32)
    code = load().expert_route(logits.data_ptr(), _in_code(logits), M, E, _row_stride(logits, logits), k, int(renormalise), ids.data_ptr(), weights.data_ptr(),
                               slots.data_ptr(), rows.data_ptr(), offsets.data_ptr(), *_workspace(workspace, logits), _stream())
    if code:
        _check(code, "expert_route")
    return ids, weights, slots, rows, offsets


def expert_combine(Y: torch.Tensor, slots: torch.Tensor, weights: torch.Tensor, base=None, out=None):
    """out[M,O] bf16 = sum over j of weights[m,j] Y[slots[m,j]] (+ base[m]); Y bf16 [R,O], slots int32 [M,k], weights fp32 [M,k]."""
    if _mx4_calls is None:
        load()
    done = _mx4_calls.expert_combine(Y, slots, weights, base, out)
    if done is not None:
        return done
    R, O = Y.shape
    M, k = slots.shape
    assert _beside(weights, Y) and weights.shape == (M, k) and weights.is_contiguous() and weights.dtype == torch.float32 and Y.dtype == torch.bfloat16
    assert base is None or (base.shape == (M, O) and base.dtype == torch.bfloat16)
    if out is None:
        out = Y.new_empty((M, O))
    assert out.shape == (M, O) and out.dtype == torch.bfloat16
    code = load().expert_combine(Y.data_ptr(), R, O, _row_stride(Y, Y), _dense_i32(slots, "slots", Y, dims=2), weights.data_ptr(), M, k, _ptr(base),
                                 0 if base is None else _row_stride(base, Y), out.data_ptr(), _row_stride(out, Y), _stream())
    if code:
        _check(code, "expert_combine")
    return out


# ---- a paged cache of keys and values --------------------------------------------------------------------------------------------

# The stream is the current device's, so the tensors have to be there too.  Results that a call makes itself may share one allocation, which lives as long as any of them.

def _current_device() -> int:
    return torch._C._cuda_getDevice()


def _here(first: torch.Tensor) -> None:
    assert first.is_cuda and first.get_device() == _current_device()


@functools.lru_cache(maxsize=4096, typed=True)
def kv_page_bytes(heads: int, page: int, D: int, dtype: str) -> int:
    return int(load().kv_page_bytes(heads, page, D, DTYPE_CODE[dtype]))


def _kv_heads(t: torch.Tensor, first: torch.Tensor):
    """(elements between tokens, between heads) of [N, H, D] whose heads are dense."""
    N, H, D = t.shape
    assert _beside(t, first) and (D < 2 or t.stride(2) == 1)
    return t.stride(0) if N > 1 else H * D, t.stride(1) if H > 1 else D


def _kv_pages(pages: torch.Tensor, heads: int, page: int, D: int, dtype: str, first: torch.Tensor):
    """(address, number) of pages[P, kv_page_bytes]."""
    n = kv_page_bytes(heads, page, D, dtype)
    if n < 0:
        raise SlideSparseError(3, "kv_page_bytes")
    assert _beside(pages, first) and pages.dtype == torch.uint8 and pages.is_contiguous() and pages.dim() == 2 and pages.shape[1] == n
    return pages.data_ptr(), pages.shape[0]


def kv_tables_workspace_bytes(B: int, N: int) -> int:
    return int(load().kv_tables_workspace_bytes(B, N))


def kv_tables(lens: torch.Tensor, want: torch.Tensor, table: torch.Tensor, pool: torch.Tensor, left: torch.Tensor, page: int, N: int, new_lens=None, new_left=None, workspace=None):
    """Pages for B requests that go from lens[B] to want[B] tokens (int32): table[B,W] and the stack of free pages pool[0 .. left[0] - 1] are brought up to date in place
    -> (new_lens[B], new_left[1], slots[N], offsets[B + 1]); new_lens may be lens and new_left may be left, or lie in the memory of want."""
    if _kv_calls is None:
        load()
    done = _kv_calls.kv_tables(lens, want, table, pool, left, page, N, new_lens, new_left, workspace)
    if done is not None:
        return done
    _here(lens)
    B, W = table.shape
    if workspace is None:
        n = kv_tables_workspace_bytes(B, N)
        workspace = lens.new_empty((n,), dtype=torch.uint8) if n else None
    if new_lens is None:
        new_lens = torch.empty_like(lens)
    if new_left is None:
        new_left = torch.empty_like(left)
    assert lens.shape == want.shape == new_lens.shape == (B,) and left.shape == new_left.shape == (1,)
    if table.dtype != torch.int32:
        raise TypeError(f"table must be int32, got {table.dtype}")
    slots, offsets = lens.new_empty((max(N, 0),)), lens.new_empty((B + 1,))
    code = load().kv_tables(_dense_i32(lens, "lens", lens), _dense_i32(want, "want", lens), B, table.data_ptr(), _row_stride(table, lens), W, page, _dense_i32(pool, "pool", lens), pool.shape[0],
                            _dense_i32(left, "left", lens), N, _dense_i32(new_lens, "new_lens", lens), _dense_i32(new_left, "new_left", lens), slots.data_ptr(), offsets.data_ptr(),
                            *_workspace(workspace, lens), _stream())
    if code:
        _check(code, "kv_tables")
    return new_lens, new_left, slots, offsets


def kv_write(K: torch.Tensor, V: torch.Tensor, slots: torch.Tensor, pages: torch.Tensor, page: int, dtype: str):
    """K, V [N,H,D] fp32/bf16 (strides between tokens and heads allowed) into slots[N] (int32) of pages[P, kv_page_bytes(H, page, D, dtype)] uint8."""
    if _kv_calls is None:
        load()
    done = _kv_calls.kv_write(K, V, slots, pages, page, dtype)
    if done is not None:
        return
    _here(K)
    N, H, D = K.shape
    assert V.shape == K.shape and V.dtype == K.dtype and slots.shape == (N,)
    at, P = _kv_pages(pages, H, page, D, dtype, K)
    code = load().kv_write(K.data_ptr(), *_kv_heads(K, K), V.data_ptr(), *_kv_heads(V, K), _in_code(K), N, H, D, _dense_i32(slots, "slots", K), at, P, page, DTYPE_CODE[dtype], _stream())
    if code:
        _check(code, "kv_write")


def kv_read(pages: torch.Tensor, slots: torch.Tensor, heads: int, D: int, page: int, dtype: str, out_dtype: torch.dtype = torch.bfloat16, K=None, V=None):
    """What pages hold of slots[N] -> (K, V) [N,heads,D] fp32 or bf16."""
    if _kv_calls is None:
        load()
    done = _kv_calls.kv_read(pages, slots, heads, D, page, dtype, _IN_CODE.get(out_dtype), K, V)
    if done is not None:
        return done
    _here(pages)
    at, P = _kv_pages(pages, heads, page, D, dtype, pages)
    N = slots.shape[0]
    if K is None:
        K = pages.new_empty((N, heads, D), dtype=out_dtype)
    if V is None:
        V = torch.empty_like(K)
    assert K.shape == V.shape == (N, heads, D) and K.dtype == V.dtype
    code = load().kv_read(at, P, page, DTYPE_CODE[dtype], _dense_i32(slots, "slots", pages), N, heads, D, _in_code(K), K.data_ptr(), *_kv_heads(K, pages), V.data_ptr(),
                          *_kv_heads(V, pages), _stream())
    if code:
        _check(code, "kv_read")
    return K, V


def kv_attention_workspace_bytes(B: int, Hq: int, heads: int, D: int) -> int:
    return int(load().kv_attention_workspace_bytes(B, Hq, heads, D))


def kv_attention(q: torch.Tensor, pages: torch.Tensor, table: torch.Tensor, lens: torch.Tensor, heads: int, page: int, dtype: str, scale=None, window: int = 0, out=None, workspace=None):
    """out[B,Hq,D] bf16: attention of q[B,Hq,D] (fp32/bf16), one new token of each request, over the lens[B] cached tokens (with a window, the last `window` of them) that lie in
    the pages of table[B,W].  scale: D^-0.5 if None; workspace: optional uint8 device tensor (kv_attention_workspace_bytes) that lets long requests use the whole chip."""
    if _kv_calls is None:
        load()
    done = _kv_calls.kv_attention(q, pages, table, lens, heads, page, dtype, scale, window, out, workspace)
    if done is not None:
        return done
    _here(q)
    B, Hq, D = q.shape
    at, P = _kv_pages(pages, heads, page, D, dtype, q)
    if table.dtype != torch.int32:
        raise TypeError(f"table must be int32, got {table.dtype}")
    assert table.shape[0] == B and lens.shape == (B,)
    if out is None:
        out = q.new_empty((B, Hq, D), dtype=torch.bfloat16)
    assert out.shape == (B, Hq, D) and out.dtype == torch.bfloat16
    code = load().kv_attention(q.data_ptr(), _in_code(q), *_kv_heads(q, q), at, P, page, DTYPE_CODE[dtype], table.data_ptr(), _row_stride(table, q), table.shape[1],
                               _dense_i32(lens, "lens", q), B, Hq, heads, D, 1 / math.sqrt(D) if scale is None else scale, window, out.data_ptr(), *_kv_heads(out, q),
                               *_workspace(workspace, q), _stream())
    if code:
        _check(code, "kv_attention")
    return out
