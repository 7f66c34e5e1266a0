"""Binding of libcoda.so -- argument marshalling only.

Every function here has the name of the C entry point it forwards to (include/coda.h)
and does nothing but turn torch tensors into raw device pointers, sizes and pitches: the
calls that a program makes for every layer in C (csrc/binding.cpp), the others by ctypes.
All arithmetic happens in the HIP kernels.  If the library has not been built the
import of this module fails loudly; there is no fallback path of any kind.
The measurement-only entry points (include/coda_unfused.h, include/coda_calib.h) live in
a second library, libcoda_bench.so, loaded here as well.
"""
import ctypes
import os
import sysconfig

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcoda.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(
        "libcoda.so is not built (%s). Build it with `python -m paper_2605_19269_amd.build`; "
        "there is no fallback implementation." % LIB_PATH)

LIB_BENCH_PATH = os.path.join(_HERE, "libcoda_bench.so")
if not os.path.exists(LIB_BENCH_PATH):
    raise ImportError("libcoda_bench.so is not built (%s). Build it with `python -m paper_2605_19269_amd.build`." % LIB_BENCH_PATH)

_BINDING_PATH = os.path.join(_HERE, "_binding" + sysconfig.get_config_var("EXT_SUFFIX"))
if not os.path.exists(_BINDING_PATH):
    raise ImportError("the C half of the binding is not built for this interpreter (%s). Build it with `python -m paper_2605_19269_amd.build`." % _BINDING_PATH)

_lib = ctypes.CDLL(LIB_PATH)
_blib = ctypes.CDLL(LIB_BENCH_PATH)

# status codes / enums (mirrors of include/coda.h)
CODA_OK, CODA_ERR_NULL, CODA_ERR_SHAPE, CODA_ERR_ALIGN, CODA_ERR_DTYPE, CODA_ERR_PROGRAM, \
    CODA_ERR_WORKSPACE, CODA_ERR_LAUNCH = range(8)
CODA_BF16, CODA_F32, CODA_F8E4M3 = 0, 1, 2
(CODA_EPI_ROW_SCALE, CODA_EPI_COL_SCALE_SIDE, CODA_EPI_ADD_TILE, CODA_EPI_SWIGLU_FWD, CODA_EPI_SWIGLU_BWD,
 CODA_EPI_ROW_SUMSQ, CODA_EPI_STORE, CODA_EPI_ACCUM_F32, CODA_EPI_ROPE, CODA_EPI_RMSNORM_BWD, CODA_EPI_LSE_PARTIAL,
 CODA_EPI_STORE_Q8, CODA_EPI_SWIGLU_FWD_Q8, CODA_EPI_SWIGLU_BWD_Q8) = range(14)
CODA_REDUCE_PARTIALS, CODA_REDUCE_ATOMIC, CODA_STORE_F32 = 0, 1, 2

EXPORTS = ["coda_gemm", "coda_gemm_static_ws", "coda_gemm_workspace_bytes", "coda_row_partial_blocks", "coda_row_finalize",
           "coda_col_partial_blocks", "coda_col_finalize", "coda_lse_finalize",
           "coda_row_sumsq", "coda_fold_gamma", "coda_interleave_pairs", "coda_quantize", "coda_dequantize",
           "coda_gemm_scaled", "coda_gemm_scaled_workspace_bytes", "coda_grad_scaled", "coda_grad_scaled_workspace_bytes",
           "coda_attention", "coda_attention_bwd", "coda_attention_bwd_workspace_bytes", "coda_cache_store", "coda_attention_cached",
           "coda_attention_cached_workspace_bytes", "coda_status_string", "coda_last_hip_error"]
EXPORTS_UNFUSED = ["coda_unfused_rmsnorm_apply", "coda_unfused_swiglu_fwd", "coda_unfused_swiglu_bwd",
                   "coda_unfused_add_sumsq", "coda_unfused_accumulate"]
EXPORTS_CALIB = ["coda_calib_mfma_loop", "coda_calib_mfma_loop16"]


class coda_mat(ctypes.Structure):
    _fields_ = [("ptr", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("ld", ctypes.c_int64), ("trans", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class coda_epi_op(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("flags", ctypes.c_uint32), ("in_", ctypes.c_void_p),
                ("out", ctypes.c_void_p), ("out2", ctypes.c_void_p), ("ld_in", ctypes.c_int64),
                ("ld_out", ctypes.c_int64), ("in2", ctypes.c_void_p), ("in3", ctypes.c_void_p),
                ("in4", ctypes.c_void_p), ("out3", ctypes.c_void_p), ("i0", ctypes.c_int64), ("i1", ctypes.c_int64)]


class coda_rope(ctypes.Structure):
    _fields_ = [("cos", ctypes.c_void_p), ("sin", ctypes.c_void_p), ("pos_q", ctypes.c_void_p), ("pos_k", ctypes.c_void_p), ("rows", ctypes.c_int64)]


class coda_cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("pages", ctypes.c_int64), ("page", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32)]


_vp, _i64, _i32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32
_lib.coda_gemm.restype = ctypes.c_int
_lib.coda_gemm.argtypes = [_vp, _i64, _i64, _i64, _vp, _vp, _vp, _i32, _vp, ctypes.c_size_t]     # structures: a pointer to one, or its bytes
_lib.coda_gemm_static_ws.restype = ctypes.c_int
_lib.coda_gemm_static_ws.argtypes = [_vp, _i64, _i64, _i64, ctypes.POINTER(coda_mat), ctypes.POINTER(coda_mat),
                                     ctypes.POINTER(coda_epi_op), _i32]
_lib.coda_gemm_workspace_bytes.restype = ctypes.c_size_t
_lib.coda_gemm_workspace_bytes.argtypes = [_i64, _i64, _i64, ctypes.POINTER(coda_epi_op), _i32]
_lib.coda_row_partial_blocks.restype = _i64
_lib.coda_row_partial_blocks.argtypes = [_i64, ctypes.POINTER(coda_epi_op), _i32]
_lib.coda_row_finalize.restype = ctypes.c_int
_lib.coda_row_finalize.argtypes = [_vp, _vp, _i64, _i64, _vp, _vp, _i64, ctypes.c_float]
_lib.coda_col_partial_blocks.restype = _i64
_lib.coda_col_partial_blocks.argtypes = [_i64]
_lib.coda_col_finalize.restype = ctypes.c_int
_lib.coda_col_finalize.argtypes = [_vp, _vp, _i64, _i64, _vp]
_lib.coda_lse_finalize.restype = ctypes.c_int
_lib.coda_lse_finalize.argtypes = [_vp, _vp, _vp, _i64, _i64, _vp, _vp, _vp]
_lib.coda_row_sumsq.restype = ctypes.c_int
_lib.coda_row_sumsq.argtypes = [_vp, _vp, _vp]
_lib.coda_fold_gamma.restype = ctypes.c_int
_lib.coda_fold_gamma.argtypes = [_vp, ctypes.POINTER(coda_mat), _vp, _vp, _i64]
_lib.coda_interleave_pairs.restype = ctypes.c_int
_lib.coda_interleave_pairs.argtypes = [_vp, ctypes.POINTER(coda_mat), ctypes.POINTER(coda_mat), _vp, _i64]
_lib.coda_quantize.restype = ctypes.c_int
_lib.coda_quantize.argtypes = [_vp, _vp, _i32, _vp, _i64, _vp, _i64, _vp, _i64]
_lib.coda_dequantize.restype = ctypes.c_int
_lib.coda_dequantize.argtypes = [_vp, _vp, _vp, _i64, _vp, _i64]
_lib.coda_gemm_scaled.restype = ctypes.c_int
_lib.coda_gemm_scaled.argtypes = [_vp, _i64, _i64, _i64, _vp, _vp, _i64, _vp, _vp, _i64, _vp, _i32, _vp, ctypes.c_size_t]
_lib.coda_gemm_scaled_workspace_bytes.restype = ctypes.c_size_t
_lib.coda_gemm_scaled_workspace_bytes.argtypes = [_i64, _i64, _i64]
_lib.coda_grad_scaled.restype = ctypes.c_int
_lib.coda_grad_scaled.argtypes = [_vp, _i64, _i64, _i64, _vp, _vp, _i64, _vp, _vp, _i64, _vp, _i64, _vp, ctypes.c_size_t]
_lib.coda_grad_scaled_workspace_bytes.restype = ctypes.c_size_t
_lib.coda_grad_scaled_workspace_bytes.argtypes = [_i64, _i64, _i64]
_f32, _size = ctypes.c_float, ctypes.c_size_t
_lib.coda_attention.restype = ctypes.c_int
_lib.coda_attention.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _i32, _i32, _i32, _f32, _i32, _vp, _i64, _vp]
_lib.coda_attention_bwd.restype = ctypes.c_int
_lib.coda_attention_bwd.argtypes = [_vp] * 9 + [_i32, _i32, _i32, _f32, _i32, _vp, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _size]
_lib.coda_attention_bwd_workspace_bytes.restype = _size
_lib.coda_attention_bwd_workspace_bytes.argtypes = [_i64, _i64, _i32, _i32, _i32, _i32]
_lib.coda_cache_store.restype = ctypes.c_int
_lib.coda_cache_store.argtypes = [_vp] * 5
_lib.coda_attention_cached.restype = ctypes.c_int
_lib.coda_attention_cached.argtypes = [_vp, _vp, _vp, _vp, _i64, _i64, _vp, _vp, _i32, _i32, _f32, _vp, _vp, _i64, _vp, _vp, _size]
_lib.coda_attention_cached_workspace_bytes.restype = _size
_lib.coda_attention_cached_workspace_bytes.argtypes = [_i64, _i32, _i32, _i32, _i32]
_lib.coda_status_string.restype = ctypes.c_char_p
_lib.coda_status_string.argtypes = [ctypes.c_int]
_lib.coda_last_hip_error.restype = ctypes.c_int
_lib.coda_last_hip_error.argtypes = []
_blib.coda_unfused_rmsnorm_apply.restype = ctypes.c_int
_blib.coda_unfused_rmsnorm_apply.argtypes = [_vp, _vp, _i64, _vp, _vp, _i64, _i64, _vp, _i64]
_blib.coda_unfused_swiglu_fwd.restype = ctypes.c_int
_blib.coda_unfused_swiglu_fwd.argtypes = [_vp, _vp, _i64, _i64, _i64, _vp, _i64]
_blib.coda_unfused_swiglu_bwd.restype = ctypes.c_int
_blib.coda_unfused_swiglu_bwd.argtypes = [_vp, _vp, _i64, _vp, _i64, _i64, _i64, _vp, _i64]
_blib.coda_unfused_add_sumsq.restype = ctypes.c_int
_blib.coda_unfused_add_sumsq.argtypes = [_vp, _vp, _i64, _vp, _i64, _i64, _i64, _vp, _i64, _vp]
_blib.coda_unfused_accumulate.restype = ctypes.c_int
_blib.coda_unfused_accumulate.argtypes = [_vp, _vp, _i64, _i64, _i64, _vp, _i64]
_blib.coda_calib_mfma_loop.restype = ctypes.c_int
_blib.coda_calib_mfma_loop.argtypes = [_vp, _vp, _vp, _i64, _i64, _vp]
_blib.coda_calib_mfma_loop16.restype = ctypes.c_int
_blib.coda_calib_mfma_loop16.argtypes = [_vp, _vp, _vp, _i64, _i64, _vp]

# The calls of every layer: the C functions take their place, and hand unusual arguments on to them.
from . import _binding  # noqa: E402  (links libcoda.so)

_NATIVE = ("coda_gemm", "coda_row_finalize", "coda_row_sumsq", "coda_col_finalize", "coda_lse_finalize", "coda_quantize", "coda_dequantize",
           "coda_gemm_scaled", "coda_grad_scaled", "coda_attention_bwd")
_binding.ctypes_calls(*(getattr(_lib, _n) for _n in _NATIVE))
for _n in _NATIVE:
    setattr(_lib, _n, getattr(_binding, _n))


class CodaError(RuntimeError):
    def __init__(self, status):
        self.status = status
        msg = _lib.coda_status_string(status).decode()
        if status == CODA_ERR_LAUNCH:
            msg += " (hipError %d)" % _lib.coda_last_hip_error()
        super().__init__("coda status %d: %s" % (status, msg))


def _check(status):
    if status != CODA_OK:
        raise CodaError(status)


_torch = None


def _import_torch():
    global _torch, _DTYPES, _TYPES
    import torch
    # raw OCP E4M3 bytes come as either 8-bit type
    _DTYPES = {torch.bfloat16: CODA_BF16, torch.uint8: CODA_F8E4M3, torch.float8_e4m3fn: CODA_F8E4M3}
    _TYPES = (_DTYPES, torch.bfloat16, torch.float32, torch.int32)
    _torch = torch
    return torch


def _stream(stream):
    if stream is None:
        torch = _torch or _import_torch()
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return getattr(stream, "cuda_stream", stream)


def _ptr(t):
    return None if t is None else t.data_ptr()


def mat(t, trans=False):
    """coda_mat describing a 2-D torch tensor as stored (row-major, unit column stride)."""
    _torch or _import_torch()
    assert t.dim() == 2, "row-major 2-D tensor expected"
    rows, cols = t.shape
    ld, step = t.stride()
    assert cols <= 1 or step == 1, "row-major 2-D tensor expected"
    return coda_mat(t.data_ptr(), rows, cols, ld, 1 if trans else 0, _DTYPES.get(t.dtype, CODA_F32))


# --- epilogue op constructors (each op holds its tensors for as long as the op object lives) ---
# _op(type, kind, flags, in_, out, out2, in2, in3, in4, out3, i0, i1); the pitches are those of a 2-D in_ and out
_op = _binding.op


def row_scale(r):
    return _op(coda_epi_op, CODA_EPI_ROW_SCALE, 0, r, None, None, None, None, None, None, 0, 0)


def col_scale_side(gamma, out):
    return _op(coda_epi_op, CODA_EPI_COL_SCALE_SIDE, 0, gamma, out, None, None, None, None, None, 0, 0)


def rope(cos, sin, pos, head_dim, rope_cols):
    """cos / sin: f32 [T x head_dim/2] dense tables; pos: int32 [M]."""
    op = _op(coda_epi_op, CODA_EPI_ROPE, 0, cos, None, None, sin, pos, None, None, head_dim, rope_cols)
    op.ld_in = cos.shape[0]     # T: rows of the tables
    return op


def rmsnorm_bwd(C, r, z, gamma, c_out=None, dgamma_out=None, atomic=False, z_sum_over=0):
    """z: f32 [M] row statistic; with z_sum_over = d > 0 it holds the raw row sums and the kernel divides by d."""
    return _op(coda_epi_op, CODA_EPI_RMSNORM_BWD, CODA_REDUCE_ATOMIC if atomic else CODA_REDUCE_PARTIALS, C, c_out, dgamma_out, r, z, gamma, None,
               z_sum_over, 0)


def lse_partial(y, pmax, psum, ztgt):
    """y: int32 [M] targets; pmax, psum: f32 [nblk x M]; ztgt: f32 [M]."""
    op = coda_epi_op(CODA_EPI_LSE_PARTIAL, 0, None, _ptr(pmax), _ptr(psum), 0, 0, None, _ptr(y), None, _ptr(ztgt), 0, 0)
    op._keep = (y, pmax, psum, ztgt)
    return op


def add_tile(C):
    return _op(coda_epi_op, CODA_EPI_ADD_TILE, 0, C, None, None, None, None, None, None, 0, 0)


def swiglu_fwd(preact_out=None):
    return _op(coda_epi_op, CODA_EPI_SWIGLU_FWD, 0, None, preact_out, None, None, None, None, None, 0, 0)


def swiglu_bwd(Z, act_out=None, stat_out=None, atomic=False):
    return _op(coda_epi_op, CODA_EPI_SWIGLU_BWD, CODA_REDUCE_ATOMIC if atomic else CODA_REDUCE_PARTIALS, Z, act_out, stat_out, None, None, None, None,
               0, 0)


def row_sumsq(out, atomic=False):
    return _op(coda_epi_op, CODA_EPI_ROW_SUMSQ, CODA_REDUCE_ATOMIC if atomic else CODA_REDUCE_PARTIALS, None, out, None, None, None, None, None, 0, 0)


def store(out, f32=False):
    return _op(coda_epi_op, CODA_EPI_STORE, CODA_STORE_F32 if f32 else 0, None, out, None, None, None, None, None, 0, 0)


def _q8(t, scales, what):
    """The pitch of the scales of a 2-D tensor of codes; both are tensors of bytes."""
    return _binding.q8_pitch(t, scales, 0, 0, what)


def _scales(scales, blocks, rows, what):
    """The pitch of scale bytes [blocks x rows]."""
    return _binding.q8_pitch(None, scales, blocks, rows, what)


def store_q8(out, scales):
    """out: codes [M x W]; scales: bytes [ceil(W / 128) x M], pitch a multiple of 16.  coda_gemm_scaled only, like the next two."""
    return _op(coda_epi_op, CODA_EPI_STORE_Q8, 0, None, out, scales, None, None, None, None, _q8(out, scales, "store_q8"), 0)


def swiglu_fwd_q8(preact_out=None, preact_scales=None):
    """preact_out, preact_scales: codes [M x N] and scale bytes [ceil(N / 128) x M] of the pre-activation, or None."""
    pitch = 0 if preact_out is None else _q8(preact_out, preact_scales, "swiglu_fwd_q8")
    return _op(coda_epi_op, CODA_EPI_SWIGLU_FWD_Q8, 0, None, preact_out, preact_scales, None, None, None, None, pitch, 0)


def swiglu_bwd_q8(Z, Z_scales, stat_out=None, atomic=False):
    """Z, Z_scales: what swiglu_fwd_q8 left, codes [M x 2N] and scale bytes [ceil(2N / 128) x M]."""
    return _op(coda_epi_op, CODA_EPI_SWIGLU_BWD_Q8, CODA_REDUCE_ATOMIC if atomic else CODA_REDUCE_PARTIALS, Z, None, stat_out, Z_scales, None, None, None,
               _q8(Z, Z_scales, "swiglu_bwd_q8"), 0)


def accum_f32(G):
    return _op(coda_epi_op, CODA_EPI_ACCUM_F32, 0, None, G, None, None, None, None, None, 0, 0)


_PROG = [coda_epi_op * max(1, n) for n in range(9)]


def _prog(ops):
    n = len(ops)
    return (_PROG[n] if n < 9 else coda_epi_op * n)(*ops), n


# --- entry points -------------------------------------------------------------------------------
def coda_gemm_raw(stream, M, N, K, A, B, ops, workspace=None, workspace_bytes=0):
    """Forward coda_mat / coda_epi_op values unchanged; returns the status code."""
    arr, n = _prog(ops)
    return _lib.coda_gemm(stream, M, N, K, ctypes.byref(A) if A is not None else None,
                          ctypes.byref(B) if B is not None else None, arr if ops is not None else None, n,
                          workspace, workspace_bytes)


def coda_gemm(A, B, ops, transA=False, transB=False, stream=None, workspace=None):
    """D = op(A) op(B), then the epilogue ops in order.  A, B: 2-D bf16 CUDA tensors as stored.
    workspace: optional device tensor of at least coda_gemm_workspace_bytes(...) bytes (enables split-K)."""
    _torch or _import_torch()
    M, N, K, a, b = _binding.gemm_mats(A, B, transA, transB, _DTYPES)
    ops = list(ops)      # of a generator too: the ops own the tensors, and stay until the call returns
    arr = _binding.prog(ops, coda_epi_op)
    if arr is None:
        arr = _prog(ops)[0]
    _check(_lib.coda_gemm(_stream(stream), M, N, K, a, b, arr, len(ops),
                          None if workspace is None else workspace.data_ptr(),
                          0 if workspace is None else workspace.numel() * workspace.element_size()))


def coda_gemm_static_ws_raw(stream, M, N, K, A, B, ops):
    arr, n = _prog(ops)
    return _lib.coda_gemm_static_ws(stream, M, N, K, ctypes.byref(A) if A is not None else None,
                                    ctypes.byref(B) if B is not None else None, arr if ops is not None else None, n)


def coda_gemm_static_ws(A, B, ops, transA=False, transB=False, stream=None):
    """coda_gemm with the library's static split-K scratch instead of a caller workspace (allocates nothing)."""
    a, b = mat(A, transA), mat(B, transB)
    M, K = (A.shape[1], A.shape[0]) if transA else (A.shape[0], A.shape[1])
    N = B.shape[0] if transB else B.shape[1]
    _check(coda_gemm_static_ws_raw(_stream(stream), M, N, K, a, b, list(ops)))


CODA_STATIC_WS_BYTES = 32 * 1024 * 1024 + 1024


def coda_gemm_workspace_bytes(M, N, K, ops):
    arr, n = _prog(list(ops))
    return _lib.coda_gemm_workspace_bytes(M, N, K, arr, n)


def coda_row_partial_blocks(N, ops=None):
    if ops is None:
        return _lib.coda_row_partial_blocks(N, None, 0)
    arr, n = _prog(list(ops))
    return _lib.coda_row_partial_blocks(N, arr, n)


def coda_row_finalize(partials, M, nblk, sum_out=None, rstd_out=None, d=1, eps=0.0, stream=None):
    _check(_lib.coda_row_finalize(_stream(stream), _ptr(partials), M, nblk, _ptr(sum_out), _ptr(rstd_out), d, eps))


def coda_lse_finalize(pmax, psum, M, nblk, ztgt=None, lse_out=None, loss_out=None, stream=None):
    _check(_lib.coda_lse_finalize(_stream(stream), _ptr(pmax), _ptr(psum), M, nblk, _ptr(ztgt), _ptr(lse_out), _ptr(loss_out)))


def coda_col_partial_blocks(M):
    return _lib.coda_col_partial_blocks(M)


def coda_col_finalize(partials, N, nblk, out, stream=None):
    _check(_lib.coda_col_finalize(_stream(stream), _ptr(partials), N, nblk, _ptr(out)))


def coda_row_sumsq(X, sum_out, stream=None):
    _torch or _import_torch()
    _check(_lib.coda_row_sumsq(_stream(stream), _binding.mat(X, False, _DTYPES), _ptr(sum_out)))


def coda_fold_gamma(W, gamma, W_out, stream=None):
    m = mat(W)
    _check(_lib.coda_fold_gamma(_stream(stream), ctypes.byref(m), _ptr(gamma), _ptr(W_out), W_out.stride(0)))


def coda_interleave_pairs(Wa, Wb, W_out, stream=None):
    a, b = mat(Wa), mat(Wb)
    _check(_lib.coda_interleave_pairs(_stream(stream), ctypes.byref(a), ctypes.byref(b), _ptr(W_out), W_out.stride(0)))


# --- 8 bits with a scale for each block of 128: codes and scales are uint8 (or float8_e4m3fn, float8_e8m0fnu) tensors -------
def _at(workspace):
    return (None, 0) if workspace is None else (workspace.data_ptr(), workspace.numel() * workspace.element_size())


def coda_quantize(X, codes, scales, scales_t=None, square=False, stream=None):
    """X: bf16 [R x C]; codes: [R x C]; scales: bytes [ceil(C / 128) x R]; with square blocks optionally scales_t: [ceil(R / 128) x C]."""
    _torch or _import_torch()
    m = _binding.mat(X, False, _DTYPES)
    assert codes.shape == X.shape, "codes of X's shape expected"
    pitch = _q8(codes, scales, "coda_quantize")
    pitch_t = 0 if scales_t is None else _scales(scales_t, (X.shape[0] + 127) // 128, X.shape[1], "coda_quantize")
    _check(_lib.coda_quantize(_stream(stream), m, 1 if square else 0, codes.data_ptr(), codes.stride(0), scales.data_ptr(), pitch, _ptr(scales_t), pitch_t))


def coda_dequantize(codes, scales, out, stream=None):
    """codes, scales -> out: bf16 [R x C]."""
    torch = _torch or _import_torch()
    m = _binding.mat(codes, False, _DTYPES)
    assert out.shape == codes.shape and out.dtype == torch.bfloat16 and (out.shape[1] <= 1 or out.stride(1) == 1), "a bf16 output of the codes' shape expected"
    _check(_lib.coda_dequantize(_stream(stream), m, scales.data_ptr(), _q8(codes, scales, "coda_dequantize"), out.data_ptr(), out.stride(0)))


def coda_gemm_scaled(A, scales_a, B, scales_b, ops, transB=False, stream=None, workspace=None):
    """D = A op(B), then the epilogue ops.  A: codes [M x K], scales_a: bytes [ceil(K / 128) x M]; B: codes [K x N], or [N x K] with transB,
    scales_b: bytes [ceil(K / 128) x N].  workspace: optional, coda_gemm_scaled_workspace_bytes(M, N, K) bytes."""
    _torch or _import_torch()
    M, N, K, a, b = _binding.gemm_mats(A, B, False, transB, _DTYPES)
    blocks = (K + 127) // 128
    ops = list(ops)      # as in coda_gemm
    arr = _binding.prog(ops, coda_epi_op)
    if arr is None:
        arr = _prog(ops)[0]
    _check(_lib.coda_gemm_scaled(_stream(stream), M, N, K, a, scales_a.data_ptr(), _scales(scales_a, blocks, M, "scales_a"), b, scales_b.data_ptr(),
                                 _scales(scales_b, blocks, N, "scales_b"), arr, len(ops), *_at(workspace)))


def coda_gemm_scaled_workspace_bytes(M, N, K):
    return _lib.coda_gemm_scaled_workspace_bytes(M, N, K)


def coda_grad_scaled(A, scales_a, B, scales_b, G, stream=None, workspace=None):
    """G [M x N] f32 += A^T B over the K rows of both.  A: codes [K x M], scales_a: bytes [ceil(M / 128) x K]; B: codes [K x N] with scales_b, or
    bf16 [K x N] with scales_b None.  workspace: optional, coda_grad_scaled_workspace_bytes(M, N, K) bytes."""
    torch = _torch or _import_torch()
    M, N, K, a, b = _binding.gemm_mats(A, B, True, False, _DTYPES)
    assert G.shape == (M, N) and G.dtype == torch.float32 and (N <= 1 or G.stride(1) == 1), "a row-major f32 [M x N] gradient expected"
    pitch_b = 0 if scales_b is None else _scales(scales_b, (N + 127) // 128, K, "scales_b")
    _check(_lib.coda_grad_scaled(_stream(stream), M, N, K, a, scales_a.data_ptr(), _scales(scales_a, (M + 127) // 128, K, "scales_a"), b, _ptr(scales_b),
                                 pitch_b, G.data_ptr(), G.stride(0), *_at(workspace)))


def coda_grad_scaled_workspace_bytes(M, N, K):
    return _lib.coda_grad_scaled_workspace_bytes(M, N, K)


# --- attention: Q, K, V and their gradients are bf16 [tokens x heads * dim] (column blocks of a QKV matrix too), seq_q, seq_k int32 [sequences + 1] ---
def _sequences(seq_q, seq_k):
    n = seq_q.shape[0] - 1
    assert n >= 0, "seq_q: sequences + 1 offsets expected"
    return _binding.vec(seq_q, _torch.int32, n + 1, None, "seq_q"), _binding.vec(seq_k, _torch.int32, n + 1, None, "seq_k"), n


def coda_attention(Q, K, V, seq_q, out, heads, kv_heads, scale, lse=None, seq_k=None, causal=True, stream=None):
    """out: bf16 [Tq x heads * dim]; lse: f32 [heads x Tq] or None; seq_k: None where K and V are packed as Q is."""
    _torch or _import_torch()
    _check(_binding.attention(_TYPES, _stream(stream), Q, K, V, seq_q, seq_k, out, lse, heads, kv_heads, scale, causal))


def coda_attention_bwd(Q, K, V, out, dout, lse, seq_q, dQ, dK, dV, heads, kv_heads, scale, workspace, seq_k=None, causal=True, rope=None, stream=None):
    """out, lse: what coda_attention left; dout: the gradient of out.  rope: (cos, sin, pos_q, pos_k) to turn dQ and dK back, pos_k None for pos_q;
    cos / sin: f32 [rows x dim / 2] dense tables, pos_q: int32 [Tq], pos_k: int32 [Tk].  workspace: coda_attention_bwd_workspace_bytes(...) bytes."""
    torch = _torch or _import_torch()
    mats = [_binding.mat(x, False, _DTYPES) for x in (Q, K, V, out, dout)]
    bf16, T, Tk = torch.bfloat16, Q.shape[0], K.shape[0]
    turn = None
    if rope is not None:
        cos, sin, pos_q, pos_k = tuple(rope) if len(rope) == 4 else tuple(rope) + (None,)
        n, half = cos.shape[0], Q.shape[1] // max(heads, 1) // 2
        turn = bytes(coda_rope(_binding.vec(cos, torch.float32, n, half, "cos"), _binding.vec(sin, torch.float32, n, half, "sin"),
                               _binding.vec(pos_q, torch.int32, T, None, "pos_q"), _binding.vec(pos_q if pos_k is None else pos_k, torch.int32, Tk, None, "pos_k"), n))
    _check(_lib.coda_attention_bwd(_stream(stream), *mats, _binding.vec(lse, torch.float32, heads, T, "lse"), *_sequences(seq_q, seq_k), heads, kv_heads, float(scale),
                                   1 if causal else 0, turn, *_binding.rows(dQ, Q, bf16, "dQ"), *_binding.rows(dK, K, bf16, "dK"), *_binding.rows(dV, V, bf16, "dV"),
                                   *_at(workspace)))


def coda_attention_bwd_workspace_bytes(Tq, Tk, n_seqs, heads, kv_heads, head_dim):
    return _lib.coda_attention_bwd_workspace_bytes(Tq, Tk, n_seqs, heads, kv_heads, head_dim)


def coda_cache_store(K, V, slots, cache_k, cache_v, stream=None):
    """Rows of K, V: bf16 [T x kv_heads * dim] to slots: int32 [T] (page * places + place, or -1 to leave a row out) of the caches
    [pages x kv_heads x places x dim]."""
    _torch or _import_torch()
    _check(_binding.cache_store(_TYPES, _stream(stream), K, V, slots, cache_k, cache_v))


def coda_attention_cached(Q, cache_k, cache_v, table, lens, seq_q, out, heads, scale, workspace, tree=None, lse=None, stream=None):
    """Q: bf16 [Tq x heads * dim], rows seq_q[s] .. of sequence s; table: int32 [sequences x pages], row-major; lens: int32 [sequences], keys in the cache with
    those of the rows; tree: int64 or uint64 [Tq] bits of the sequence's rows that each row sees, None for a chain; workspace:
    coda_attention_cached_workspace_bytes(...) bytes."""
    torch = _torch or _import_torch()
    kind = None if tree is None else tree.dtype
    assert kind in (None, torch.int64, torch.uint64), "tree: a 64-bit integer for each row expected"
    _check(_binding.attention_cached(_TYPES, _stream(stream), Q, cache_k, cache_v, table, lens, seq_q, out, lse, heads, scale, tree, kind, workspace))


def coda_attention_cached_workspace_bytes(Tq, n_seqs, heads, kv_heads, head_dim):
    return _lib.coda_attention_cached_workspace_bytes(Tq, n_seqs, heads, kv_heads, head_dim)


def coda_status_string(status):
    return _lib.coda_status_string(status).decode()


def coda_last_hip_error():
    return _lib.coda_last_hip_error()


# --- unfused baseline kernels (include/coda_unfused.h) -----------------------------------------
def coda_unfused_rmsnorm_apply(X, r, gamma, Xn, stream=None):
    _check(_blib.coda_unfused_rmsnorm_apply(_stream(stream), _ptr(X), X.stride(0), _ptr(r), _ptr(gamma),
                                           X.shape[0], X.shape[1], _ptr(Xn), Xn.stride(0)))


def coda_unfused_swiglu_fwd(Z, H, stream=None):
    _check(_blib.coda_unfused_swiglu_fwd(_stream(stream), _ptr(Z), Z.stride(0), H.shape[0], H.shape[1],
                                        _ptr(H), H.stride(0)))


def coda_unfused_swiglu_bwd(dH, Z, dZ, stream=None):
    _check(_blib.coda_unfused_swiglu_bwd(_stream(stream), _ptr(dH), dH.stride(0), _ptr(Z), Z.stride(0),
                                        dH.shape[0], dH.shape[1], _ptr(dZ), dZ.stride(0)))


def coda_unfused_add_sumsq(D, R, Y, ss=None, stream=None):
    _check(_blib.coda_unfused_add_sumsq(_stream(stream), _ptr(D), D.stride(0), _ptr(R), R.stride(0),
                                       D.shape[0], D.shape[1], _ptr(Y), Y.stride(0), _ptr(ss)))


def coda_unfused_accumulate(T, G, stream=None):
    _check(_blib.coda_unfused_accumulate(_stream(stream), _ptr(T), T.stride(0), T.shape[0], T.shape[1],
                                        _ptr(G), G.stride(0)))


# --- measurement calibration (include/coda_calib.h) ----------------------------------------------
def _calib(fn, out_elems, a_frags, b_frags, n_blocks, iters, out, stream):
    need_a, need_b = n_blocks * 4 * 512 * 8, n_blocks * 2 * 512 * 8
    if a_frags.numel() < need_a or b_frags.numel() < need_b or a_frags.element_size() != 2 or b_frags.element_size() != 2:
        raise ValueError("fragment buffers too small: need %d and %d 16-bit elements" % (need_a, need_b))
    if out is not None and (out.numel() < out_elems or out.element_size() != 4):
        raise ValueError("out must hold %d fp32 values" % out_elems)
    _check(fn(_stream(stream), _ptr(a_frags), _ptr(b_frags), n_blocks, iters, _ptr(out)))


def coda_calib_mfma_loop(a_frags, b_frags, n_blocks, iters, out=None, stream=None):
    _calib(_blib.coda_calib_mfma_loop, 8 * 8 * 16 * 64, a_frags, b_frags, n_blocks, iters, out, stream)


def coda_calib_mfma_loop16(a_frags, b_frags, n_blocks, iters, out=None, stream=None):
    _calib(_blib.coda_calib_mfma_loop16, 8 * 8 * 4 * 64, a_frags, b_frags, n_blocks, iters, out, stream)
