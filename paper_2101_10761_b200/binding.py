"""ctypes binding of libsidco.so: argument marshalling only.

Every function has the name and the meaning of the C entry point declared in
``include/sidco.h``; tensors are passed as raw device (or host) pointers and
nothing is computed here.  Loading fails loudly if the library has not been
built (``python -m paper_2101_10761_b200.build``): there is no fallback path.
"""
from __future__ import annotations

import ctypes as C
import operator
import os
from typing import Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
# SIDCO_LIB_VARIANT=profile|check selects a build of the same sources with device timestamps or with
# device-side bounds checks (see build.py); the default is the product library.
_VARIANT = os.environ.get("SIDCO_LIB_VARIANT", "")
LIB_PATH = os.path.join(_HERE, "libsidco%s.so" % ("_" + _VARIANT if _VARIANT else ""))

SID_EXP, SID_GAMMA, SID_GPD = 0, 1, 2
MAX_STAGES = 8

ST_NONFINITE, ST_DEGENERATE, ST_ALL_ZERO, ST_TIMEOUT, ST_BOUNDS = 1, 2, 4, 8, 16
BUILD_PROFILE, BUILD_BOUNDS_CHECK = 1, 2


class SegDebug(C.Structure):
    _fields_ = [
        ("M_used", C.c_int32),
        ("M_next", C.c_int32),
        ("status", C.c_int32),
        ("calls", C.c_int32),
        ("k_sum", C.c_int64),
        ("eta", C.c_double * MAX_STAGES),
        ("k_stage", C.c_int32 * MAX_STAGES),
    ]


EXPORTS = [
    "sidco_compress", "sidco_compress_host", "sidco_workspace_bytes", "sidco_set_workspace",
    "sidco_set_params", "sidco_reset_state", "sidco_get_debug", "sidco_state_save", "sidco_state_load",
    "sidco_release", "sidco_release_all", "sidco_launch_count", "sidco_error_string", "sidco_version",
    "sidco_get_phase_times", "sidco_get_cta_sweep_times", "sidco_compress_static",
    "sidco_reset_state_async", "sidco_set_test_hooks", "sidco_build_flags", "sidco_aggregate", "sidco_compress_bf16", "sidco_get_cta_selection_info",
    "sidco_reference_workspace_bytes", "sidco_topk", "sidco_dgc", "sidco_set_policy",
    "sidco_mx4_code_bytes", "sidco_mx4_scale_bytes", "sidco_mx4_quantize", "sidco_mx4_dequantize", "sidco_mx4_matmul",
    "sidco_mx4_compress", "sidco_mx4_mean", "sidco_orthogonalize_workspace_bytes", "sidco_orthogonalize",
    "sidco_wait_timeouts", "sidco_set_product_test_hooks",
    "sidco_dropout", "sidco_embedding", "sidco_embedding_grad_workspace_bytes", "sidco_embedding_grad",
    "sidco_linear_cross_entropy_workspace_bytes", "sidco_linear_cross_entropy", "sidco_linear_cross_entropy_typed",
    "sidco_scale_gradient", "sidco_round_gradient",
]

_lib = None


class SidcoError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        msg = lib().sidco_error_string(code).decode()
        super().__init__(f"{where} failed with code {code}: {msg}")


def lib() -> C.CDLL:
    """Load libsidco.so once.  Raises if it is missing: the CUDA path is the only path."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} not found: build it with `python -m paper_2101_10761_b200.build` "
            "(there is no CPU fallback)")
    L = C.CDLL(LIB_PATH)
    vp, i32, f32, i64, dbl = C.c_void_p, C.c_int, C.c_float, C.c_int64, C.c_double
    compress_sig = [vp, vp, C.POINTER(i64), i32, f32, i32, i32, vp, vp, vp, vp]
    L.sidco_compress.argtypes = compress_sig
    L.sidco_compress.restype = i32
    L.sidco_compress_host.argtypes = compress_sig
    L.sidco_compress_host.restype = i32
    L.sidco_compress_static.argtypes = compress_sig
    L.sidco_compress_static.restype = i32
    L.sidco_compress_bf16.argtypes = compress_sig
    L.sidco_compress_bf16.restype = i32
    L.sidco_workspace_bytes.argtypes = [i64, i32]
    L.sidco_workspace_bytes.restype = C.c_size_t
    L.sidco_set_workspace.argtypes = [vp, vp, C.c_size_t]
    L.sidco_set_workspace.restype = i32
    L.sidco_set_params.argtypes = [dbl, dbl, dbl, i32]
    L.sidco_set_params.restype = i32
    L.sidco_reset_state.argtypes = [vp]
    L.sidco_reset_state.restype = i32
    L.sidco_reset_state_async.argtypes = [vp, vp]
    L.sidco_reset_state_async.restype = i32
    L.sidco_get_debug.argtypes = [vp, C.POINTER(SegDebug), i32]
    L.sidco_get_debug.restype = i32
    L.sidco_get_phase_times.argtypes = [vp, C.POINTER(dbl)]
    L.sidco_get_phase_times.restype = i32
    L.sidco_get_cta_sweep_times.argtypes = [vp, C.POINTER(dbl), i32]
    L.sidco_get_cta_sweep_times.restype = i32
    L.sidco_state_save.argtypes = [vp, C.POINTER(i64), i32]
    L.sidco_state_save.restype = i32
    L.sidco_state_load.argtypes = [vp, C.POINTER(i64), i32]
    L.sidco_state_load.restype = i32
    L.sidco_release.argtypes = [vp]
    L.sidco_release.restype = i32
    L.sidco_release_all.argtypes = []
    L.sidco_release_all.restype = i32
    L.sidco_launch_count.argtypes = []
    L.sidco_launch_count.restype = i64
    L.sidco_error_string.argtypes = [i32]
    L.sidco_error_string.restype = C.c_char_p
    L.sidco_version.argtypes = []
    L.sidco_version.restype = i32
    L.sidco_set_test_hooks.argtypes = [i32, i32, C.c_longlong, i32]
    L.sidco_set_test_hooks.restype = i32
    L.sidco_build_flags.argtypes = []
    L.sidco_build_flags.restype = i32
    L.sidco_get_cta_selection_info.argtypes = [vp, C.POINTER(C.c_int32), i32]
    L.sidco_get_cta_selection_info.restype = i32
    L.sidco_reference_workspace_bytes.argtypes = [i64, i64]
    L.sidco_reference_workspace_bytes.restype = C.c_size_t
    L.sidco_topk.argtypes = [vp, vp, i64, i64, vp, vp, vp, vp, C.c_size_t, vp]
    L.sidco_topk.restype = i32
    L.sidco_dgc.argtypes = [vp, vp, i64, f32, vp, i64, vp, vp, vp, vp, C.c_size_t, vp]
    L.sidco_dgc.restype = i32
    L.sidco_set_policy.argtypes = [i32, i32, i32]
    L.sidco_set_policy.restype = i32
    L.sidco_aggregate.argtypes = [vp, vp, vp, i32, i64, i64, vp, vp, vp]
    L.sidco_aggregate.restype = i32
    pi64 = C.POINTER(i64)
    L.sidco_mx4_code_bytes.argtypes = L.sidco_mx4_scale_bytes.argtypes = [i64, i64]
    L.sidco_mx4_code_bytes.restype = L.sidco_mx4_scale_bytes.restype = i64
    L.sidco_mx4_quantize.argtypes = [vp, i32, i64, i64, i64, vp, vp, vp, vp, vp]
    L.sidco_mx4_quantize.restype = i32
    L.sidco_mx4_dequantize.argtypes = [vp, vp, i64, i64, vp, i32, i64, vp]
    L.sidco_mx4_dequantize.restype = i32
    L.sidco_mx4_matmul.argtypes = [vp, vp, vp, vp, i64, i64, i64, vp, i32, i64, i32, vp]
    L.sidco_mx4_matmul.restype = i32
    L.sidco_mx4_compress.argtypes = [vp, i32, vp, i64, vp, vp, vp]
    L.sidco_mx4_compress.restype = i32
    L.sidco_mx4_mean.argtypes = [vp, vp, i32, i64, vp, vp]
    L.sidco_mx4_mean.restype = i32
    L.sidco_orthogonalize_workspace_bytes.argtypes = [pi64, pi64, i32]
    L.sidco_orthogonalize_workspace_bytes.restype = i64
    L.sidco_orthogonalize.argtypes = [vp, i32, vp, f32, i32, pi64, pi64, pi64, i32, i32, f32, vp, vp, C.c_size_t, vp]
    L.sidco_orthogonalize.restype = i32
    L.sidco_wait_timeouts.argtypes = []
    L.sidco_wait_timeouts.restype = i32
    L.sidco_set_product_test_hooks.argtypes = [C.c_longlong, i32]
    L.sidco_set_product_test_hooks.restype = i32
    u64, sz = C.c_uint64, C.c_size_t
    L.sidco_dropout.argtypes = [vp, i32, i64, f32, u64, u64, vp, vp, vp, vp]
    L.sidco_dropout.restype = i32
    L.sidco_embedding.argtypes = [vp, i32, i64, i64, i64, vp, i32, i64, f32, f32, u64, u64, vp, vp, i32, i64, vp, vp]
    L.sidco_embedding.restype = i32
    L.sidco_embedding_grad_workspace_bytes.argtypes = [i64, i64, i64]
    L.sidco_embedding_grad_workspace_bytes.restype = i64
    L.sidco_embedding_grad.argtypes = [vp, i32, i64, vp, i32, i64, i64, i64, f32, f32, u64, u64, vp, vp, i32, i64, i32, vp,
                                       sz, vp]
    L.sidco_embedding_grad.restype = i32
    L.sidco_linear_cross_entropy_workspace_bytes.argtypes = [vp, i32, i32, i64, i64, i64, i64, i32, i64]
    L.sidco_linear_cross_entropy_workspace_bytes.restype = i64
    L.sidco_linear_cross_entropy.argtypes = [vp, i32, i64, vp, i32, i64, vp, i32, vp, f32, i64, i64, i64, vp, vp, vp, i64, vp,
                                             i32, i64, i32, i64, vp, vp, sz, vp]
    L.sidco_linear_cross_entropy.restype = i32
    L.sidco_linear_cross_entropy_typed.argtypes = [vp, i32, i64, vp, i32, i64, vp, i32, vp, f32, i64, i64, i64, vp, vp, vp,
                                                   i32, i64, vp, i32, i64, i32, i64, vp, vp, sz, vp]
    L.sidco_linear_cross_entropy_typed.restype = i32
    L.sidco_round_gradient.argtypes = [vp, i64, vp, vp, i32, vp]
    L.sidco_round_gradient.restype = i32
    L.sidco_scale_gradient.argtypes = [vp, i32, i64, vp, vp]
    L.sidco_scale_gradient.restype = i32
    _lib = L
    return L


def _ptr(x) -> Optional[int]:
    """Raw address of a torch tensor, a numpy array or an int; None stays NULL."""
    if x is None:
        return None
    try:
        return x.data_ptr()
    except AttributeError:
        return x.ctypes.data if isinstance(x, np.ndarray) else operator.index(x)


def _offsets(seg_offsets: Sequence[int]):
    arr = np.ascontiguousarray(np.asarray(seg_offsets, dtype=np.int64))
    return arr, arr.ctypes.data_as(C.POINTER(C.c_int64)), int(arr.size - 1)


_current = None


def _current_stream() -> int:
    """torch's current stream as a raw handle (looked up without building a Stream object where torch allows it)."""
    global _current
    if _current is None:
        import torch
        raw, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
        if raw is None or device is None:
            return torch.cuda.current_stream().cuda_stream
        torch.cuda.current_stream()                          # initialises CUDA
        _current = lambda: raw(device())                     # noqa: E731
    return _current()


def _stream(stream) -> Optional[int]:
    if stream is None:
        return _current_stream()
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def sidco_compress(grad, residual, seg_offsets, delta: float, sid_type: int, max_stages: int,
                   out_idx, out_val, out_k, stream=None) -> None:
    """Device buffers (torch CUDA tensors or raw addresses); enqueues on `stream`
    (default: torch's current stream) and returns without synchronising."""
    arr, p, n = _offsets(seg_offsets)
    rc = lib().sidco_compress(_ptr(grad), _ptr(residual), p, n, delta, sid_type, max_stages,
                              _ptr(out_idx), _ptr(out_val), _ptr(out_k), _stream(stream))
    if rc:
        raise SidcoError(rc, "sidco_compress")


def sidco_compress_bf16(grad_bf16, residual, seg_offsets, delta: float, sid_type: int, max_stages: int,
                        out_idx, out_val, out_k, stream=None) -> None:
    """sidco_compress with a bf16 gradient (torch.bfloat16 tensor, or uint16 bit patterns); fp32 residual."""
    arr, p, n = _offsets(seg_offsets)
    rc = lib().sidco_compress_bf16(_ptr(grad_bf16), _ptr(residual), p, n, delta, sid_type, max_stages,
                                   _ptr(out_idx), _ptr(out_val), _ptr(out_k), _stream(stream))
    if rc:
        raise SidcoError(rc, "sidco_compress_bf16")


def sidco_compress_host(grad, residual, seg_offsets, delta: float, sid_type: int, max_stages: int,
                        out_idx, out_val, out_k, stream=None) -> None:
    """Host buffers (numpy arrays or pinned torch CPU tensors); copies in, compresses,
    copies back and synchronises."""
    arr, p, n = _offsets(seg_offsets)
    rc = lib().sidco_compress_host(_ptr(grad), _ptr(residual), p, n, delta, sid_type, max_stages,
                                   _ptr(out_idx), _ptr(out_val), _ptr(out_k), _stream(stream))
    if rc:
        raise SidcoError(rc, "sidco_compress_host")


def sidco_workspace_bytes(d: int, n_segs: int) -> int:
    return int(lib().sidco_workspace_bytes(d, n_segs))


def sidco_set_workspace(residual, device_ptr, nbytes: int) -> None:
    rc = lib().sidco_set_workspace(_ptr(residual), _ptr(device_ptr), nbytes)
    if rc:
        raise SidcoError(rc, "sidco_set_workspace")


def sidco_set_params(delta1: float = 0.25, eps_H: float = 0.2, eps_L: float = 0.2, Q: int = 5) -> None:
    rc = lib().sidco_set_params(delta1, eps_H, eps_L, Q)
    if rc:
        raise SidcoError(rc, "sidco_set_params")


def sidco_set_policy(gamma_exact: bool = False, ratio_from_counts: bool = False, adapt_reversed: bool = False) -> None:
    """Variants the paper describes and replaces (see sidco.h); the defaults restore the method as evaluated."""
    rc = lib().sidco_set_policy(int(gamma_exact), int(ratio_from_counts), int(adapt_reversed))
    if rc:
        raise SidcoError(rc, "sidco_set_policy")


def sidco_reset_state(residual) -> None:
    rc = lib().sidco_reset_state(_ptr(residual))
    if rc:
        raise SidcoError(rc, "sidco_reset_state")


def sidco_get_debug(residual, n_segs: int):
    buf = (SegDebug * n_segs)()
    rc = lib().sidco_get_debug(_ptr(residual), buf, n_segs)
    if rc:
        raise SidcoError(rc, "sidco_get_debug")
    return list(buf)


def sidco_state_save(residual, n_segs: int) -> np.ndarray:
    blob = np.zeros(3 * n_segs, dtype=np.int64)
    rc = lib().sidco_state_save(_ptr(residual), blob.ctypes.data_as(C.POINTER(C.c_int64)), n_segs)
    if rc:
        raise SidcoError(rc, "sidco_state_save")
    return blob


def sidco_state_load(residual, blob: np.ndarray) -> None:
    blob = np.ascontiguousarray(blob, dtype=np.int64)
    rc = lib().sidco_state_load(_ptr(residual), blob.ctypes.data_as(C.POINTER(C.c_int64)), blob.size // 3)
    if rc:
        raise SidcoError(rc, "sidco_state_load")


def sidco_release(residual) -> None:
    rc = lib().sidco_release(_ptr(residual))
    if rc:
        raise SidcoError(rc, "sidco_release")


def sidco_release_all() -> None:
    lib().sidco_release_all()


def sidco_launch_count() -> int:
    return int(lib().sidco_launch_count())


def sidco_version() -> int:
    return int(lib().sidco_version())


AGG_MAX_WORKERS = 64
AGG_ST_COUNT, AGG_ST_ORDER = 1, 2


def sidco_aggregate(idx_all, val_all, counts, n_workers: int, stride: int, d: int, out_dense, status=None,
                    stream=None) -> None:
    """Dense mean of n_workers gathered sparse lists (device buffers; see sidco.h)."""
    rc = lib().sidco_aggregate(_ptr(idx_all), _ptr(val_all), _ptr(counts), n_workers, stride, d,
                               _ptr(out_dense), _ptr(status), _stream(stream))
    if rc:
        raise SidcoError(rc, "sidco_aggregate")


def sidco_reference_workspace_bytes(d: int, n_sample: int = 0) -> int:
    return int(lib().sidco_reference_workspace_bytes(d, n_sample))


def sidco_topk(grad, residual, d: int, k: int, out_idx, out_val, out_k, workspace, workspace_bytes: int,
               stream=None) -> None:
    """Exact Top-k reference point (device buffers; see sidco.h)."""
    rc = lib().sidco_topk(_ptr(grad), _ptr(residual), d, k, _ptr(out_idx), _ptr(out_val), _ptr(out_k),
                          _ptr(workspace), workspace_bytes, _stream(stream))
    if rc:
        raise SidcoError(rc, "sidco_topk")


def sidco_dgc(grad, residual, d: int, delta: float, sample_idx, n_sample: int, out_idx, out_val, out_k,
              workspace, workspace_bytes: int, stream=None) -> None:
    """Sampled-threshold reference point (device buffers; see sidco.h)."""
    rc = lib().sidco_dgc(_ptr(grad), _ptr(residual), d, delta, _ptr(sample_idx), n_sample, _ptr(out_idx),
                         _ptr(out_val), _ptr(out_k), _ptr(workspace), workspace_bytes, _stream(stream))
    if rc:
        raise SidcoError(rc, "sidco_dgc")


def sidco_set_test_hooks(grid: int = 0, spec_enable: int = 1, spin_limit: int = 0,
                         drop_publication_seg: int = -1) -> None:
    """Test switches (see sidco.h); the defaults restore normal operation."""
    rc = lib().sidco_set_test_hooks(grid, spec_enable, spin_limit, drop_publication_seg)
    if rc:
        raise SidcoError(rc, "sidco_set_test_hooks")


def sidco_build_flags() -> int:
    return int(lib().sidco_build_flags())


def sidco_error_string(code: int) -> str:
    return lib().sidco_error_string(code).decode()


def sidco_get_phase_times(residual):
    """Microseconds of the last call: [P1, stage 2, stages 3..M, staging, placement, total] followed by
    six finer marks of CTA 0 (see sidco.h)."""
    buf = (C.c_double * 12)()
    rc = lib().sidco_get_phase_times(_ptr(residual), buf)
    if rc:
        raise SidcoError(rc, "sidco_get_phase_times")
    return list(buf)


def sidco_get_cta_sweep_times(residual, max_ctas: int = 1024) -> np.ndarray:
    """(n_ctas, 4) array: microseconds after kernel start at which each CTA finished its sweeps."""
    buf = (C.c_double * (4 * max_ctas))()
    rc = lib().sidco_get_cta_sweep_times(_ptr(residual), buf, max_ctas)
    if rc < 0:
        raise SidcoError(rc, "sidco_get_cta_sweep_times")
    return np.ctypeslib.as_array(buf)[: 4 * rc].reshape(rc, 4).copy()


def sidco_get_cta_selection_info(residual, max_ctas: int = 1024) -> np.ndarray:
    """(n_ctas, 8) int array, profile builds only: see sidco.h."""
    buf = (C.c_int32 * (8 * max_ctas))()
    rc = lib().sidco_get_cta_selection_info(_ptr(residual), buf, max_ctas)
    if rc < 0:
        raise SidcoError(rc, "sidco_get_cta_selection_info")
    return np.ctypeslib.as_array(buf)[: 8 * rc].reshape(rc, 8).copy()


STATIC_MAX_ELEMS = 1048576
STATIC_MAX_SEGS = 256


def sidco_compress_static(grad, residual, seg_offsets, delta: float, sid_type: int, max_stages: int,
                          out_idx, out_val, out_k, stream=None) -> None:
    """sidco_compress without any device allocation: the workspace is a fixed 18 MiB array inside the
    library, one per GPU, shared by all calls (do not overlap calls on one GPU).  For callers that
    cannot call cudaMalloc, e.g. under stream capture or inside a pool-managed allocator.  Limits:
    STATIC_MAX_ELEMS elements, STATIC_MAX_SEGS segments."""
    arr, p, n = _offsets(seg_offsets)
    rc = lib().sidco_compress_static(_ptr(grad), _ptr(residual), p, n, delta, sid_type, max_stages,
                                     _ptr(out_idx), _ptr(out_val), _ptr(out_k), _stream(stream))
    if rc:
        raise SidcoError(rc, "sidco_compress_static")


def sidco_reset_state_async(residual, stream=None) -> None:
    """Reset the stage adaptation of `residual` on `stream` without synchronising."""
    rc = lib().sidco_reset_state_async(_ptr(residual), _stream(stream))
    if rc:
        raise SidcoError(rc, "sidco_reset_state_async")


# ---- microscaled 4-bit numbers and the orthogonalised update (formats and arguments: see sidco.h)

T_F32, T_BF16, T_F16 = 0, 1, 2
ORTHO_MAX_DIM, ORTHO_MAX_SHORT, ORTHO_MAX_STEPS = 4194304, 16384, 32
_TYPES = {"torch.float32": T_F32, "torch.bfloat16": T_BF16, "torch.float16": T_F16, "float32": T_F32, "float16": T_F16}
_seen_types = {}


def _type(x, given: Optional[int]) -> int:
    """The SIDCO_T_* code of a tensor or array; raw addresses need `given`."""
    if given is not None:
        return given
    dtype = getattr(x, "dtype", None)
    code = _seen_types.get(dtype)
    if code is None:
        code = _TYPES.get(str(dtype))
        if code is None:
            raise SidcoError(-13, "element type %s:" % ("of a raw address" if dtype is None else dtype))
        _seen_types[dtype] = code
    return code


def _sizes(values):
    arr = np.ascontiguousarray(values, dtype=np.int64)
    return arr, arr.ctypes.data_as(C.POINTER(C.c_int64))


def sidco_mx4_code_bytes(rows: int, cols: int) -> int:
    n = int(lib().sidco_mx4_code_bytes(rows, cols))
    if n < 0:
        raise SidcoError(n, "sidco_mx4_code_bytes")
    return n


def sidco_mx4_scale_bytes(rows: int, cols: int) -> int:
    n = int(lib().sidco_mx4_scale_bytes(rows, cols))
    if n < 0:
        raise SidcoError(n, "sidco_mx4_scale_bytes")
    return n


def sidco_mx4_quantize(x, rows: int, cols: int, ld: int, codes, scales, codes_t=None, scales_t=None, x_type=None,
                       stream=None) -> None:
    """Quantise x[rows][ld] along its rows (codes, scales) and / or its columns (codes_t, scales_t); see sidco.h."""
    rc = lib().sidco_mx4_quantize(_ptr(x), _type(x, x_type), rows, cols, ld, _ptr(codes), _ptr(scales), _ptr(codes_t),
                                  _ptr(scales_t), _stream(stream))
    if rc:
        raise SidcoError(rc, "sidco_mx4_quantize")


def sidco_mx4_dequantize(codes, scales, rows: int, cols: int, out, ld: int, out_type=None, stream=None) -> None:
    """The values of a quantised matrix."""
    rc = lib().sidco_mx4_dequantize(_ptr(codes), _ptr(scales), rows, cols, _ptr(out), _type(out, out_type), ld,
                                    _stream(stream))
    if rc:
        raise SidcoError(rc, "sidco_mx4_dequantize")


def sidco_mx4_matmul(a_codes, a_scales, b_codes, b_scales, m: int, n: int, k: int, c, ldc: int, add: bool = False,
                     c_type=None, stream=None) -> None:
    """C[m][ldc] = A[m, k] B[n, k]^T of quantised matrices; `add`: C += A B^T."""
    rc = lib().sidco_mx4_matmul(_ptr(a_codes), _ptr(a_scales), _ptr(b_codes), _ptr(b_scales), m, n, k, _ptr(c),
                                _type(c, c_type), ldc, int(add), _stream(stream))
    if rc:
        raise SidcoError(rc, "sidco_mx4_matmul")


def sidco_mx4_compress(grad, residual, d: int, codes, scales, grad_type=None, stream=None) -> None:
    """Error-compensated 4-bit quantisation of a flat gradient (dense counterpart of sidco_compress)."""
    rc = lib().sidco_mx4_compress(_ptr(grad), _type(grad, grad_type), _ptr(residual), d, _ptr(codes), _ptr(scales),
                                  _stream(stream))
    if rc:
        raise SidcoError(rc, "sidco_mx4_compress")


def sidco_mx4_mean(codes_all, scales_all, n_workers: int, d: int, out_dense, stream=None) -> None:
    """Dense mean of n_workers gathered 4-bit gradients (counterpart of sidco_aggregate)."""
    rc = lib().sidco_mx4_mean(_ptr(codes_all), _ptr(scales_all), n_workers, d, _ptr(out_dense), _stream(stream))
    if rc:
        raise SidcoError(rc, "sidco_mx4_mean")


def sidco_orthogonalize_workspace_bytes(rows: Sequence[int], cols: Sequence[int]) -> int:
    (r, rp), (c, cp) = _sizes(rows), _sizes(cols)
    if r.size != c.size:
        raise ValueError("rows and cols have different lengths")
    n = int(lib().sidco_orthogonalize_workspace_bytes(rp, cp, r.size))
    if n < 0:
        raise SidcoError(n, "sidco_orthogonalize_workspace_bytes")
    return n


def sidco_orthogonalize(grad, momentum, mu: float, nesterov: bool, offsets: Sequence[int], rows: Sequence[int],
                        cols: Sequence[int], steps: int, out_bf16, workspace, workspace_bytes: int, eps: float = 1e-7,
                        grad_type=None, stream=None) -> None:
    """Momentum and orthogonalised update of the matrices at `offsets` of a flat vector (device buffers; see sidco.h)."""
    (o, op), (r, rp), (c, cp) = _sizes(offsets), _sizes(rows), _sizes(cols)
    if not o.size == r.size == c.size:
        raise ValueError("offsets, rows and cols have different lengths")
    rc = lib().sidco_orthogonalize(_ptr(grad), _type(grad, grad_type), _ptr(momentum), mu, int(nesterov), op, rp, cp,
                                   o.size, steps, eps, _ptr(out_bf16), _ptr(workspace), workspace_bytes,
                                   _stream(stream))
    if rc:
        raise SidcoError(rc, "sidco_orthogonalize")


def sidco_wait_timeouts() -> int:
    n = int(lib().sidco_wait_timeouts())
    if n < 0:
        raise SidcoError(-n, "sidco_wait_timeouts")
    return n


def sidco_set_product_test_hooks(wait_us: int = 0, drop_phase: int = -1) -> None:
    """Test switches of sidco_orthogonalize (see sidco.h); the defaults restore normal operation."""
    rc = lib().sidco_set_product_test_hooks(wait_us, drop_phase)
    if rc:
        raise SidcoError(rc, "sidco_set_product_test_hooks")


# ---- the ends of a language model's training step: lookup, dropout, cross entropy (see sidco.h)

T_I32, T_I64 = 3, 4
EMBEDDING_ST_TOKEN = 1
_TOKEN_TYPES = {"torch.int32": T_I32, "torch.int64": T_I64, "int32": T_I32, "int64": T_I64}
_seen_token_types = {}


def _token_type(x, given: Optional[int]) -> int:
    """The SIDCO_T_I* code of a tensor or array of tokens or labels; raw addresses need `given`."""
    if given is not None:
        return given
    dtype = getattr(x, "dtype", None)
    code = _seen_token_types.get(dtype)
    if code is None:
        code = _TOKEN_TYPES.get(str(dtype))
        if code is None:
            raise SidcoError(-13, "type of tokens %s:" % ("of a raw address" if dtype is None else dtype))
        _seen_token_types[dtype] = code
    return code


def sidco_dropout(x, n: int, p: float, seed: int, call: int, out, residual=None, step=None, x_type=None,
                  stream=None) -> None:
    """out = dropout(x) (+ residual) of n elements; the mask is a function of seed, call and position."""
    rc = lib().sidco_dropout(_ptr(x), _type(x, x_type), n, p, seed, call, _ptr(step), _ptr(residual), _ptr(out),
                             _stream(stream))
    if rc:
        raise SidcoError(rc, "sidco_dropout")


def sidco_embedding(table, vocab: int, cols: int, ld: int, tokens, n: int, scale: float, out, ldo: int, p: float = 0.0,
                    seed: int = 0, call: int = 0, step=None, status=None, table_type=None, token_type=None,
                    out_type=None, stream=None) -> None:
    """out[i] = scale * dropout(table[tokens[i]])."""
    rc = lib().sidco_embedding(_ptr(table), _type(table, table_type), vocab, cols, ld, _ptr(tokens),
                               _token_type(tokens, token_type), n, scale, p, seed, call, _ptr(step), _ptr(out),
                               _type(out, out_type), ldo, _ptr(status), _stream(stream))
    if rc:
        raise SidcoError(rc, "sidco_embedding")


def sidco_embedding_grad_workspace_bytes(n: int, vocab: int, cols: int) -> int:
    size = int(lib().sidco_embedding_grad_workspace_bytes(n, vocab, cols))
    if size < 0:
        raise SidcoError(size, "sidco_embedding_grad_workspace_bytes")
    return size


def sidco_embedding_grad(dy, ld_dy: int, tokens, n: int, vocab: int, cols: int, scale: float, dtable, ldd: int, workspace,
                         workspace_bytes: int, add: bool = False, p: float = 0.0, seed: int = 0, call: int = 0, step=None,
                         dy_type=None, token_type=None, dtable_type=None, stream=None) -> None:
    """Gradient of the table of sidco_embedding, written (all rows) or added (the rows of tokens that occur)."""
    rc = lib().sidco_embedding_grad(_ptr(dy), _type(dy, dy_type), ld_dy, _ptr(tokens), _token_type(tokens, token_type), n,
                                    vocab, cols, scale, p, seed, call, _ptr(step), _ptr(dtable),
                                    _type(dtable, dtable_type), ldd, int(add), _ptr(workspace), workspace_bytes,
                                    _stream(stream))
    if rc:
        raise SidcoError(rc, "sidco_embedding_grad")


CROSS_ENTROPY_ST_LABEL = 1


def sidco_linear_cross_entropy_workspace_bytes(x, w, ldw: int, rows: int, vocab: int, hidden: int, grads=True,
                                               piece_rows: int = 0, x_type=None, w_type=None) -> int:
    """`grads`: True (dx and dw), False, or 1 for dx and 2 for dw alone."""
    size = int(lib().sidco_linear_cross_entropy_workspace_bytes(
        _ptr(w), _type(x, x_type), _type(w, w_type), ldw, rows, vocab, hidden, 3 if grads is True else int(grads),
        piece_rows))
    if size < 0:
        raise SidcoError(size, "sidco_linear_cross_entropy_workspace_bytes")
    return size


def sidco_linear_cross_entropy(x, ldx: int, w, ldw: int, labels, rows: int, vocab: int, hidden: int, row_losses, loss, dx,
                               lddx: int, dw, lddw: int, workspace, workspace_bytes: int, row_weights=None,
                               scale: float = 1.0, add: bool = False, piece_rows: int = 0, status=None, x_type=None,
                               w_type=None, label_type=None, dw_type=None, dx_type=None, stream=None) -> None:
    """Cross entropy of scale * x w^T against labels: losses and, where dx / dw are given, the gradients.  A dx without a type
    of its own has that of x."""
    t = _type(x, x_type)
    if dx_type is None:
        dx_type = _type(dx, None) if hasattr(dx, "dtype") else t
    rc = lib().sidco_linear_cross_entropy_typed(
        _ptr(x), t, ldx, _ptr(w), _type(w, w_type), ldw, _ptr(labels), _token_type(labels, label_type),
        _ptr(row_weights), scale, rows, vocab, hidden, _ptr(row_losses), _ptr(loss), _ptr(dx), dx_type, lddx, _ptr(dw),
        0 if dw is None else _type(dw, dw_type), lddw, int(add), piece_rows, _ptr(status), _ptr(workspace),
        workspace_bytes, _stream(stream))
    if rc:
        raise SidcoError(rc, "sidco_linear_cross_entropy")


sidco_linear_cross_entropy_typed = sidco_linear_cross_entropy       # (its dx may have a type of its own here too)


def sidco_scale_gradient(x, n: int, factor, x_type=None, stream=None) -> None:
    """x *= *factor (a float on the device); a factor of one costs nothing."""
    rc = lib().sidco_scale_gradient(_ptr(x), _type(x, x_type), n, _ptr(factor), _stream(stream))
    if rc:
        raise SidcoError(rc, "sidco_scale_gradient")


def sidco_round_gradient(x, n: int, factor, out, out_type=None, stream=None) -> None:
    """out = *factor * x, rounded once; x in fp32."""
    rc = lib().sidco_round_gradient(_ptr(x), n, _ptr(factor), _ptr(out), _type(out, out_type), _stream(stream))
    if rc:
        raise SidcoError(rc, "sidco_round_gradient")
