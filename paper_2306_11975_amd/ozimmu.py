"""Thin binding over the C ABI of libozimmu (include/ozimmu.h): argument marshalling only.

Every function has the name of the C entry point it calls; tensors are torch CUDA tensors used
purely as device memory, and the stream is torch's current HIP stream unless one is given.
There is no fallback: if the library has not been built, loading raises.
"""
from __future__ import annotations

import ctypes
from pathlib import Path

_LIB_PATH = Path(__file__).resolve().parent / "libozimmu.so"

(OK, ERR_BAD_DIM, ERR_BAD_LD, ERR_BAD_SLICES, ERR_NULL, ERR_WORKSPACE, ERR_HIP, ERR_NOT_IMPLEMENTED,
 ERR_TOO_LARGE, ERR_BAD_TYPE, ERR_BAD_POLYNOMIAL, ERR_MISALIGNED) = range(12)
F32, BF16, F16, E4M3, E8M0 = range(5)            # ozimmu_type_t
SOFTMAX, SIGMOID = range(2)          # ozimmu_score_t
MAX_SLICES = 16
ROW_ALIGN = 128
K_ALIGN = 32
FRAG_ROWS = 32
INT32_BLOCK = 131072
WORKSPACE_ALIGN = 256
STATIC_SCRATCH_BYTES = 64 << 20

EXPORTS = (
    "ozimmu_status_string", "ozimmu_slice_geometry", "ozimmu_slice_offset", "ozimmu_split_rows", "ozimmu_split_cols",
    "ozimmu_slice_gemm", "ozimmu_workspace_bytes", "ozimmu_dgemm", "ozimmu_zgemm", "ozimmu_dgemm_static", "ozimmu_dgemm_stage",
    "ozimmu_launch_plan", "ozimmu_dgemm_dd", "ozimmu_dgemm_blas", "ozimmu_zgemm_blas_workspace_bytes", "ozimmu_zgemm_blas",
    "ozimmu_auto_scratch_bytes", "ozimmu_auto_num_slices", "ozimmu_auto_num_slices_blas", "ozimmu_zgemm_auto",
    "ozimmu_dgemm_auto", "ozimmu_dgemm_blas_auto", "ozimmu_zgemm_blas_auto",
    "ozimmu_q4_geometry", "ozimmu_q4_split", "ozimmu_q4_expand", "ozimmu_q4_workspace_bytes", "ozimmu_q4_gemm", "ozimmu_q4_gemm_grad",
    "ozimmu_orthogonalize_workspace_bytes", "ozimmu_orthogonalize",
    "ozimmu_f8_geometry", "ozimmu_f8_split", "ozimmu_f8_expand", "ozimmu_f8_workspace_bytes", "ozimmu_f8_gemm", "ozimmu_f8_gemm_grad",
    "ozimmu_f8_weight_grad", "ozimmu_route", "ozimmu_route_grad", "ozimmu_expert_order_workspace_bytes", "ozimmu_expert_order",
    "ozimmu_expert_combine", "ozimmu_expert_combine_grad",
)
PROBE_EXPORTS = ("ozimmu_probe_int8_mfma",)      # include/ozimmu_probe.h: measurement utility, not the product path


class OzimmuError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"ozimmu error {code}: {what}")
        self.code = code


class Plan(ctypes.Structure):
    """ozimmu_plan_t of include/ozimmu.h."""
    _fields_ = [("tile_rows", ctypes.c_int), ("tile_cols", ctypes.c_int), ("workgroups", ctypes.c_int64),
                ("bands", ctypes.c_int), ("int32_block_steps", ctypes.c_int)]


_lib = None


def lib() -> ctypes.CDLL:
    """Load libozimmu.so (built by ``python -m paper_2306_11975_amd.build``)."""
    global _lib
    if _lib is None:
        if not _LIB_PATH.exists():
            raise RuntimeError(f"{_LIB_PATH} is missing: build it with `python -m paper_2306_11975_amd.build` "
                               "(there is no CPU fallback)")
        L = ctypes.CDLL(str(_LIB_PATH))
        i64, i32, vp, sz = ctypes.c_int64, ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t
        L.ozimmu_status_string.restype = ctypes.c_char_p
        L.ozimmu_status_string.argtypes = [i32]
        L.ozimmu_slice_geometry.restype = i32
        L.ozimmu_slice_geometry.argtypes = [i64, i64, ctypes.POINTER(i64), ctypes.POINTER(i64)]
        L.ozimmu_slice_offset.restype = i64
        L.ozimmu_slice_offset.argtypes = [i64, i64, i32, i64, i64]
        L.ozimmu_split_rows.restype = i32
        L.ozimmu_split_rows.argtypes = [i64, i64, vp, i64, i32, vp, vp, vp]
        L.ozimmu_split_cols.restype = i32
        L.ozimmu_split_cols.argtypes = [i64, i64, vp, i64, i32, vp, vp, vp, vp]
        L.ozimmu_slice_gemm.restype = i32
        L.ozimmu_slice_gemm.argtypes = [i64, i64, i64, vp, vp, i32, i32, i64, i64, vp, i64, vp]
        L.ozimmu_workspace_bytes.restype = i32
        L.ozimmu_workspace_bytes.argtypes = [i64, i64, i64, i32, i32, ctypes.POINTER(sz)]
        for name in ("ozimmu_dgemm", "ozimmu_zgemm"):
            f = getattr(L, name)
            f.restype = i32
            f.argtypes = [i64, i64, i64, vp, i64, vp, i64, vp, i64, i32, vp, sz, vp]
        L.ozimmu_dgemm_static.restype = i32
        L.ozimmu_dgemm_static.argtypes = [i64, i64, i64, vp, i64, vp, i64, vp, i64, i32, vp]
        L.ozimmu_dgemm_stage.restype = i32
        L.ozimmu_dgemm_stage.argtypes = [i32, i64, i64, i64, vp, i64, vp, i64, vp, i64, i32, vp, sz, vp]
        L.ozimmu_launch_plan.restype = i32
        L.ozimmu_launch_plan.argtypes = [i64, i64, i64, i32, ctypes.POINTER(Plan)]
        L.ozimmu_dgemm_dd.restype = i32
        L.ozimmu_dgemm_dd.argtypes = [i64, i64, i64, vp, i64, vp, i64, vp, vp, i64, i32, vp, sz, vp]
        L.ozimmu_dgemm_blas.restype = i32
        L.ozimmu_dgemm_blas.argtypes = [ctypes.c_char, ctypes.c_char, i64, i64, i64, ctypes.c_double, vp, i64, vp, i64,
                                        ctypes.c_double, vp, i64, i32, vp, sz, vp]
        L.ozimmu_zgemm_blas_workspace_bytes.restype = i32
        L.ozimmu_zgemm_blas_workspace_bytes.argtypes = [i64, i64, i64, i32, i32, ctypes.POINTER(sz)]
        L.ozimmu_zgemm_blas.restype = i32
        L.ozimmu_zgemm_blas.argtypes = [ctypes.c_char, ctypes.c_char, i64, i64, i64, vp, vp, i64, vp, i64, vp, vp, i64,
                                        i32, vp, sz, vp]
        L.ozimmu_auto_scratch_bytes.restype = i32
        L.ozimmu_auto_scratch_bytes.argtypes = [i64, ctypes.POINTER(sz)]
        L.ozimmu_auto_num_slices.restype = i32
        L.ozimmu_auto_num_slices.argtypes = [i64, i64, i64, vp, i64, vp, i64, i32, ctypes.c_double, i32, vp, sz,
                                             ctypes.POINTER(i32), vp, vp]
        L.ozimmu_auto_num_slices_blas.restype = i32
        L.ozimmu_auto_num_slices_blas.argtypes = [ctypes.c_char, ctypes.c_char, i64, i64, i64, vp, i64, vp, i64, i32,
                                                  ctypes.c_double, i32, vp, sz, ctypes.POINTER(i32), vp, vp]
        L.ozimmu_zgemm_auto.restype = i32
        L.ozimmu_zgemm_auto.argtypes = [i64, i64, i64, vp, i64, vp, i64, vp, i64, ctypes.c_double, i32, i32, vp, sz, vp, sz,
                                        ctypes.POINTER(i32), ctypes.POINTER(i32), vp]
        L.ozimmu_dgemm_auto.restype = i32
        L.ozimmu_dgemm_auto.argtypes = [i64, i64, i64, vp, i64, vp, i64, vp, i64, ctypes.c_double, i32, i32, vp, sz, vp, sz,
                                        ctypes.POINTER(i32), ctypes.POINTER(i32), vp]
        L.ozimmu_dgemm_blas_auto.restype = i32
        L.ozimmu_dgemm_blas_auto.argtypes = [ctypes.c_char, ctypes.c_char, i64, i64, i64, ctypes.c_double, vp, i64, vp, i64,
                                             ctypes.c_double, vp, i64, ctypes.c_double, i32, i32, vp, sz, vp, sz,
                                             ctypes.POINTER(i32), ctypes.POINTER(i32), vp]
        L.ozimmu_zgemm_blas_auto.restype = i32
        L.ozimmu_zgemm_blas_auto.argtypes = [ctypes.c_char, ctypes.c_char, i64, i64, i64, vp, vp, i64, vp, i64, vp, vp, i64,
                                             ctypes.c_double, i32, i32, vp, sz, vp, sz, ctypes.POINTER(i32),
                                             ctypes.POINTER(i32), vp]
        L.ozimmu_q4_geometry.restype = i32
        L.ozimmu_q4_geometry.argtypes = [i64, i32, ctypes.POINTER(i64), ctypes.POINTER(i64)]
        L.ozimmu_q4_split.restype = i32
        L.ozimmu_q4_split.argtypes = [i64, i64, i32, i32, vp, i64, vp, i64, i32, vp, i64, vp]
        L.ozimmu_q4_expand.restype = i32
        L.ozimmu_q4_expand.argtypes = [i64, i64, i32, i32, vp, i64, vp, i64, vp, i64, vp]
        L.ozimmu_q4_workspace_bytes.restype = i32
        L.ozimmu_q4_workspace_bytes.argtypes = [i64, i64, i64, i32, i32, i32, ctypes.POINTER(sz)]
        for name in ("ozimmu_q4_gemm", "ozimmu_q4_gemm_grad"):
            f = getattr(L, name)
            f.restype = i32
            f.argtypes = [i64, i64, i64, i32, i32, vp, i64, vp, i64, vp, i64, vp, i64, vp, sz, vp]
        L.ozimmu_orthogonalize_workspace_bytes.restype = i32
        L.ozimmu_orthogonalize_workspace_bytes.argtypes = [i64, i64, i64, ctypes.POINTER(sz)]
        L.ozimmu_orthogonalize.restype = i32
        L.ozimmu_orthogonalize.argtypes = [i64, i64, i64, i32, vp, i64, i64, vp, i64, i64, i32] + [ctypes.c_double] * 4 + [vp, sz, vp]
        for name, args in {
            "f8_geometry": [i64, ctypes.POINTER(i64), ctypes.POINTER(i64)],
            "f8_split": [i64, i64, i32, i32, vp, i64, vp, i64, vp, i64, vp],
            "f8_expand": [i64, i64, i32, vp, i64, i32, vp, i64, i32, vp, i64, vp],
            "f8_workspace_bytes": [i32, i64, i64, i64, i64, i64, i32, ctypes.POINTER(sz)],
            "f8_gemm": [i64, i64, i64, i64, i64, i32, vp, i64, vp, i64, vp, i64, i32, vp, i64, vp, vp, i32, vp, i64, vp, sz, vp],
            "f8_gemm_grad": [i64, i64, i64, i64, i32, vp, i64, vp, i64, vp, i64, i32, vp, i64, vp, i32, vp, i64, vp, sz, vp],
            "f8_weight_grad": [i64, i64, i64, i64, i64, i32, vp, i64, vp, i64, vp, vp, i32, vp, i64, vp, sz, vp],
            "route": [i64, i64, i32, i32, vp, i64, vp, i32, i32, i32, i32, ctypes.c_double, vp, vp, vp],
            "route_grad": [i64, i64, i32, i32, vp, i64, vp, vp, i32, i32, ctypes.c_double, vp, i64, vp],
            "expert_order_workspace_bytes": [i64, i32, i64, ctypes.POINTER(sz)],
            "expert_order": [i64, i32, i64, vp, vp, vp, vp, vp, sz, vp],
            "expert_combine": [i64, i32, i64, i64, i32, vp, i64, vp, vp, vp, i64, vp],
            "expert_combine_grad": [i64, i32, i64, i64, i32, vp, i64, vp, i64, vp, vp, vp, i64, vp, vp],
        }.items():
            f = getattr(L, "ozimmu_" + name)
            f.restype = i32
            f.argtypes = args
        dp = ctypes.POINTER(ctypes.c_double)
        L.ozimmu_probe_int8_mfma.restype = i32
        L.ozimmu_probe_int8_mfma.argtypes = [i32, i32, i32, dp, dp]
        _lib = L
    return _lib


def status_string(code: int) -> str:
    return lib().ozimmu_status_string(int(code)).decode()


def _check(code: int) -> None:
    if code != OK:
        raise OzimmuError(code, status_string(code))


def _ptr(t) -> int:
    return 0 if t is None else t.data_ptr()


def _stream(stream) -> int:
    import torch

    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


def _ld(t, cols):
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError("expected a 2-D row-major tensor (unit stride along the second dimension)")
    return t.stride(0) if t.shape[0] > 1 else max(cols, 1)


def slice_geometry(rows: int, k: int):
    rp, kp = ctypes.c_int64(), ctypes.c_int64()
    _check(lib().ozimmu_slice_geometry(rows, k, ctypes.byref(rp), ctypes.byref(kp)))
    return rp.value, kp.value


def slice_offset(rows_padded: int, k_padded: int, slice_: int, row: int, l: int) -> int:
    return int(lib().ozimmu_slice_offset(rows_padded, k_padded, slice_, row, l))


def unpack_slices(raw, num_slices: int, rows: int, k: int):
    """Re-order the bytes of a slice tensor (as the library stores it, any 1-D or N-D int8 numpy
    array of num_slices * rows_padded * k_padded elements) into a plain [slice][row][l] numpy
    array of the padded shape. Pure index permutation: the block geometry is queried from the
    library through ozimmu_slice_offset, no arithmetic of the method happens here."""
    import numpy as np

    rp, kp = slice_geometry(rows, k)
    flat = np.ascontiguousarray(raw).reshape(-1)
    assert flat.size == num_slices * rp * kp
    if flat.size == 0:
        return flat.reshape(num_slices, rp, kp)
    # offsets are separable: offset(s, r, l) = s * rp * kp + f(r - r % 32, 0) + g(r % 32, l % 32) + h(0, l - l % 32)
    row_part = np.array([slice_offset(rp, kp, 0, r, 0) for r in range(0, rp, FRAG_ROWS)], dtype=np.int64)
    in_frag = np.array([[slice_offset(rp, kp, 0, rr, l) for l in range(K_ALIGN)] for rr in range(FRAG_ROWS)],
                       dtype=np.int64)                       # [32][32], fragment 0
    slab_part = np.array([slice_offset(rp, kp, 0, 0, l) for l in range(0, kp, K_ALIGN)], dtype=np.int64)
    idx = (row_part[:, None, None, None] + in_frag[None, :, None, :] + slab_part[None, None, :, None])
    idx = idx.reshape(rp, kp)                                # [row][l]
    out = np.empty((num_slices, rp, kp), dtype=flat.dtype)
    for s_ in range(num_slices):
        out[s_] = flat[s_ * rp * kp + idx]
    return out


def workspace_bytes(m: int, n: int, k: int, num_slices: int, is_complex: bool = False) -> int:
    out = ctypes.c_size_t()
    _check(lib().ozimmu_workspace_bytes(m, n, k, num_slices, int(is_complex), ctypes.byref(out)))
    return out.value


def split_rows(A, num_slices: int, slices, exps, stream=None) -> None:
    """A: (m, k) float64 device tensor with unit column stride; slices: int8 device buffer of
    num_slices * rows_padded * k_padded bytes; exps: int32 device tensor of m entries."""
    m, k = A.shape
    _check(lib().ozimmu_split_rows(m, k, _ptr(A), _ld(A, k), num_slices,
                                   _ptr(slices), _ptr(exps), _stream(stream)))


def split_cols(B, num_slices: int, slices, exps, col_scratch, stream=None) -> None:
    k, n = B.shape
    _check(lib().ozimmu_split_cols(k, n, _ptr(B), _ld(B, n), num_slices,
                                   _ptr(slices), _ptr(exps), _ptr(col_scratch), _stream(stream)))


def slice_gemm(m: int, n: int, k: int, SA, SB, p: int, q: int, k0: int, klen: int, P, stream=None) -> None:
    _check(lib().ozimmu_slice_gemm(m, n, k, _ptr(SA), _ptr(SB), p, q, k0, klen, _ptr(P),
                                   _ld(P, n), _stream(stream)))


def dgemm(A, B, C, num_slices: int, workspace, stream=None) -> None:
    """C = A . B by the Ozaki scheme on the INT8 matrix cores (A: m x k, B: k x n, C: m x n,
    float64 device tensors with unit column stride; workspace: uint8 device tensor)."""
    m, k = A.shape
    n = B.shape[1]
    _check(lib().ozimmu_dgemm(m, n, k, _ptr(A), _ld(A, k), _ptr(B), _ld(B, n), _ptr(C), _ld(C, n), num_slices,
                              _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream(stream)))


def dgemm_static(A, B, C, num_slices: int, stream=None) -> None:
    """ozimmu_dgemm without a workspace argument: the library's built-in scratch is used (see ozimmu.h)."""
    m, k = A.shape
    n = B.shape[1]
    _check(lib().ozimmu_dgemm_static(m, n, k, _ptr(A), _ld(A, k), _ptr(B), _ld(B, n), _ptr(C), _ld(C, n),
                                     num_slices, _stream(stream)))


def dgemm_stage(stage: int, A, B, C, num_slices: int, workspace, stream=None) -> None:
    m, k = A.shape
    n = B.shape[1]
    _check(lib().ozimmu_dgemm_stage(stage, m, n, k, _ptr(A), _ld(A, k), _ptr(B), _ld(B, n), _ptr(C), _ld(C, n),
                                    num_slices, _ptr(workspace), 0 if workspace is None else workspace.numel(),
                                    _stream(stream)))


def zgemm(A, B, C, num_slices: int, workspace, stream=None) -> None:
    """Complex128 device tensors (interleaved re, im), otherwise as dgemm."""
    m, k = A.shape
    n = B.shape[1]
    _check(lib().ozimmu_zgemm(m, n, k, _ptr(A), _ld(A, k), _ptr(B), _ld(B, n), _ptr(C), _ld(C, n), num_slices,
                              _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream(stream)))


def launch_plan(m: int, n: int, k: int, num_slices: int) -> dict:
    """How ozimmu_dgemm runs a shape with a workspace of the reported size (ozimmu_plan_t as a dict; see ozimmu.h)."""
    plan = Plan()
    _check(lib().ozimmu_launch_plan(m, n, k, num_slices, ctypes.byref(plan)))
    return {name: getattr(plan, name) for name, _ in Plan._fields_}


def dgemm_dd(A, B, C_hi, C_lo, num_slices: int, workspace, stream=None) -> None:
    """C_hi + C_lo = A . B with the diagonal sums added in double-double (see ozimmu.h)."""
    m, k = A.shape
    n = B.shape[1]
    ldc = _ld(C_hi, n)
    if _ld(C_lo, n) != ldc:
        raise ValueError("C_hi and C_lo must have the same leading dimension")
    _check(lib().ozimmu_dgemm_dd(m, n, k, _ptr(A), _ld(A, k), _ptr(B), _ld(B, n), _ptr(C_hi), _ptr(C_lo), ldc,
                                 num_slices, _ptr(workspace), 0 if workspace is None else workspace.numel(),
                                 _stream(stream)))


def dgemm_blas(transa: str, transb: str, m: int, n: int, k: int, alpha: float, A, lda: int, B, ldb: int,
               beta: float, C, ldc: int, num_slices: int, workspace, stream=None) -> None:
    """Column-major C = alpha op(A) op(B) + beta C; A, B, C are device tensors used as raw
    column-major storage with the given leading dimensions (see ozimmu.h)."""
    _check(lib().ozimmu_dgemm_blas(transa.encode()[:1], transb.encode()[:1], m, n, k, float(alpha), _ptr(A), lda,
                                   _ptr(B), ldb, float(beta), _ptr(C), ldc, num_slices, _ptr(workspace),
                                   0 if workspace is None else workspace.numel(), _stream(stream)))


def zgemm_blas_workspace_bytes(m: int, n: int, k: int, num_slices: int, beta_is_zero: bool) -> int:
    out = ctypes.c_size_t()
    _check(lib().ozimmu_zgemm_blas_workspace_bytes(m, n, k, num_slices, int(bool(beta_is_zero)), ctypes.byref(out)))
    return out.value


def zgemm_blas(transa: str, transb: str, m: int, n: int, k: int, alpha: complex, A, lda: int, B, ldb: int,
               beta: complex, C, ldc: int, num_slices: int, workspace, stream=None) -> None:
    """Column-major complex C = alpha op(A) op(B) + beta C; A, B, C are complex128 device tensors used as
    raw column-major storage with the given leading dimensions in complex elements (see ozimmu.h)."""
    al = (ctypes.c_double * 2)(complex(alpha).real, complex(alpha).imag)
    be = (ctypes.c_double * 2)(complex(beta).real, complex(beta).imag)
    _check(lib().ozimmu_zgemm_blas(transa.encode()[:1], transb.encode()[:1], m, n, k, ctypes.addressof(al), _ptr(A), lda,
                                   _ptr(B), ldb, ctypes.addressof(be), _ptr(C), ldc, num_slices, _ptr(workspace),
                                   0 if workspace is None else workspace.numel(), _stream(stream)))


def auto_scratch_bytes(n: int) -> int:
    out = ctypes.c_size_t()
    _check(lib().ozimmu_auto_scratch_bytes(n, ctypes.byref(out)))
    return out.value


def auto_num_slices(A, B, threshold: float, max_slices: int = MAX_SLICES, scratch=None, stream=None):
    """Number of slices whose average mantissa loss is within `threshold` (see ozimmu.h) for the
    float64 or complex128 device tensors A (m x k) and B (k x n). Returns (s, sums) with sums a
    numpy uint64 array [planes][16]. Waits for the stream."""
    import numpy as np
    import torch

    m, k = A.shape
    n = B.shape[1]
    cplx = A.is_complex()
    assert cplx == B.is_complex()
    if scratch is None:
        scratch = torch.empty(max(auto_scratch_bytes(n), WORKSPACE_ALIGN), dtype=torch.uint8, device=A.device)
    planes = 4 if cplx else 2
    sums = np.zeros((planes, MAX_SLICES), dtype=np.uint64)
    s = ctypes.c_int()
    _check(lib().ozimmu_auto_num_slices(m, n, k, _ptr(A), _ld(A, k), _ptr(B), _ld(B, n), int(cplx), float(threshold),
                                        int(max_slices), _ptr(scratch), scratch.numel(), ctypes.byref(s),
                                        sums.ctypes.data, _stream(stream)))
    return s.value, sums


def _gemm_auto(cplx, A, B, C, threshold, guess, max_slices, workspace, scratch, stream):
    import torch

    m, k = A.shape
    n = B.shape[1]
    if workspace is None:
        need = max(workspace_bytes(m, n, k, s, cplx) for s in range(1, max_slices + 1))
        workspace = torch.empty(max(need, WORKSPACE_ALIGN), dtype=torch.uint8, device=A.device)
    if scratch is None:
        scratch = torch.empty(max(auto_scratch_bytes(n), WORKSPACE_ALIGN), dtype=torch.uint8, device=A.device)
    s, confirmed = ctypes.c_int(), ctypes.c_int()
    f = lib().ozimmu_zgemm_auto if cplx else lib().ozimmu_dgemm_auto
    _check(f(m, n, k, _ptr(A), _ld(A, k), _ptr(B), _ld(B, n), _ptr(C), _ld(C, n), float(threshold), int(max_slices),
             int(guess), _ptr(workspace), workspace.numel(), _ptr(scratch), scratch.numel(), ctypes.byref(s),
             ctypes.byref(confirmed), _stream(stream)))
    return s.value, bool(confirmed.value)


def dgemm_auto(A, B, C, threshold: float, guess: int = 0, max_slices: int = MAX_SLICES, workspace=None, scratch=None,
               stream=None):
    """C = A . B (float64 device tensors) with the slice count ozimmu_auto_num_slices would choose, in one call (see
    ozimmu.h); `guess` is the expected count (0: none). Returns (s, guess_confirmed). Waits for the stream."""
    return _gemm_auto(False, A, B, C, threshold, guess, max_slices, workspace, scratch, stream)


def zgemm_auto(A, B, C, threshold: float, guess: int = 0, max_slices: int = MAX_SLICES, workspace=None, scratch=None,
               stream=None):
    """The same for complex128 device tensors."""
    return _gemm_auto(True, A, B, C, threshold, guess, max_slices, workspace, scratch, stream)


def gemm_blas_auto(transa: str, transb: str, m: int, n: int, k: int, alpha, A, lda: int, B, ldb: int, beta, C, ldc: int,
                   is_complex: bool, threshold: float, guess: int = 0, max_slices: int = MAX_SLICES, stream=None):
    """The BLAS-style call with the slice count chosen inside it (see ozimmu.h); A, B, C are device tensors used as raw
    column-major storage. Returns (s, guess_confirmed). Waits for the stream."""
    import torch

    beta_zero = complex(beta) == 0
    if is_complex:
        need = max(zgemm_blas_workspace_bytes(m, n, k, s, beta_zero) for s in range(1, max_slices + 1))
    else:
        need = max(workspace_bytes(n, m, k, s) for s in range(1, max_slices + 1))
    workspace = torch.empty(max(need, WORKSPACE_ALIGN), dtype=torch.uint8, device=C.device)
    scratch = torch.empty(max(auto_scratch_bytes(max(m, n)), WORKSPACE_ALIGN), dtype=torch.uint8, device=C.device)
    s, confirmed = ctypes.c_int(), ctypes.c_int()
    common = (float(threshold), int(max_slices), int(guess), _ptr(workspace), workspace.numel(), _ptr(scratch),
              scratch.numel(), ctypes.byref(s), ctypes.byref(confirmed), _stream(stream))
    if is_complex:
        al = (ctypes.c_double * 2)(complex(alpha).real, complex(alpha).imag)
        be = (ctypes.c_double * 2)(complex(beta).real, complex(beta).imag)
        _check(lib().ozimmu_zgemm_blas_auto(transa.encode()[:1], transb.encode()[:1], m, n, k, ctypes.addressof(al), _ptr(A),
                                            lda, _ptr(B), ldb, ctypes.addressof(be), _ptr(C), ldc, *common))
    else:
        _check(lib().ozimmu_dgemm_blas_auto(transa.encode()[:1], transb.encode()[:1], m, n, k, float(alpha), _ptr(A), lda,
                                            _ptr(B), ldb, float(beta), _ptr(C), ldc, *common))
    return s.value, bool(confirmed.value)


def auto_num_slices_blas(transa: str, transb: str, m: int, n: int, k: int, A, lda: int, B, ldb: int, is_complex: bool,
                         threshold: float, max_slices: int = MAX_SLICES, scratch=None, stream=None):
    """The same choice for column-major operands with transposes (see ozimmu.h); A and B are device
    tensors used as raw storage. Returns (s, sums). Waits for the stream."""
    import numpy as np
    import torch

    if scratch is None:
        scratch = torch.empty(max(auto_scratch_bytes(max(m, n)), WORKSPACE_ALIGN), dtype=torch.uint8, device=A.device)
    planes = 4 if is_complex else 2
    sums = np.zeros((planes, MAX_SLICES), dtype=np.uint64)
    s = ctypes.c_int()
    _check(lib().ozimmu_auto_num_slices_blas(transa.encode()[:1], transb.encode()[:1], m, n, k, _ptr(A), lda, _ptr(B), ldb,
                                             int(bool(is_complex)), float(threshold), int(max_slices), _ptr(scratch),
                                             scratch.numel(), ctypes.byref(s), sums.ctypes.data, _stream(stream)))
    return s.value, sums


_torch = _uint8 = None
_types = {}      # torch's types as ozimmu_type_t, once torch is there


def _load_torch():
    global _torch, _uint8
    import torch

    _types.update({torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16})
    _torch, _uint8 = torch, torch.uint8


def _type_of(dtype) -> int:
    if _torch is None:
        _load_torch()
    t = _types.get(dtype)
    if t is None:
        raise ValueError(f"expected float32, bfloat16 or float16, got {dtype}")
    return t


def _expect(condition, what: str) -> None:
    if not condition:
        raise ValueError(what)


def _call(f, stream, tensors, *args) -> None:
    """f(*args, stream) with the tensors' device current: all must be on one GPU. Without a stream, torch's current one of that
    device is taken. (One token's call is a few microseconds of GPU time: what happens here is kept short.)"""
    if _torch is None:
        _load_torch()
    index = tensors[0].get_device()
    for t in tensors[1:]:
        if t is not None and t.get_device() != index:
            raise ValueError("all tensors must be on one device")
    if index < 0:
        raise ValueError("expected tensors on a GPU")
    if stream is None:
        raw = _torch._C._cuda_getCurrentRawStream(index)
    elif stream.device.index != index:
        raise ValueError("the stream belongs to another device than the tensors")
    else:
        raw = stream.cuda_stream
    if index == _torch._C._cuda_getDevice():
        code = f(*args, raw)
    else:
        with _torch.cuda.device(index):
            code = f(*args, raw)
    if code:
        _check(code)


def _rows(t):
    """Rows, columns and row stride of a 2-D tensor with unit stride along its rows."""
    try:
        rows, cols = t.shape
    except ValueError:
        raise ValueError("expected a 2-D tensor") from None
    ld, step = t.stride()
    if step != 1 and cols > 1:
        raise ValueError("expected a row-major tensor (unit stride along the second dimension)")
    return rows, cols, ld if rows > 1 else cols or 1


def q4_geometry(k: int, group: int):
    """(bytes of a row of codes, scales of a row) for weights of k inputs (see ozimmu.h)."""
    row_bytes_, groups = ctypes.c_int64(), ctypes.c_int64()
    _check(lib().ozimmu_q4_geometry(k, group, ctypes.byref(row_bytes_), ctypes.byref(groups)))
    return row_bytes_.value, groups.value


def q4_row_bytes(k: int) -> int:
    return q4_geometry(k, 32)[0]


_GROUPS = (32, 64, 128)


def _q4_weights(n: int, k: int, codes, scales, group: int):
    """Checks the codes and scales of an n x k weight matrix; (codes' row stride in bytes, scales' row stride)."""
    if _torch is None:
        _load_torch()
    if group not in _GROUPS:
        q4_geometry(k, group)       # raises
    row_bytes_, groups = (k + 31) // 32 * 16, -(-k // group)
    rows, cols, ldq = _rows(codes)
    if rows != n or cols < row_bytes_ or codes.dtype is not _uint8:
        raise ValueError(f"codes: expected {n} rows of at least {row_bytes_} bytes (uint8)")
    rows, cols, lds = _rows(scales)
    if rows != n or cols != groups:
        raise ValueError(f"scales: expected the shape {(n, groups)}")
    return (ldq if n > 1 else row_bytes_), lds


def q4_split(W, group: int, codes, scales, stream=None) -> None:
    """W (n x k; float32, bfloat16 or float16) into four-bit codes (uint8, n x q4_row_bytes(k)) and scales (n x ceil(k / group), any of
    the three types)."""
    n, k, ldw = _rows(W)
    ldq, lds = _q4_weights(n, k, codes, scales, group)
    _call(lib().ozimmu_q4_split, stream, (W, codes, scales), n, k, group, _type_of(W.dtype), W.data_ptr(), ldw, codes.data_ptr(), ldq,
          _type_of(scales.dtype), scales.data_ptr(), lds)


def q4_expand(codes, scales, group: int, W, stream=None) -> None:
    """The weights that codes and scales stand for, into W (n x k, of the scales' type)."""
    n, k, ldw = _rows(W)
    ldq, lds = _q4_weights(n, k, codes, scales, group)
    _expect(W.dtype == scales.dtype, "W and the scales must have one type")
    _call(lib().ozimmu_q4_expand, stream, (W, codes, scales), n, k, group, _type_of(W.dtype), codes.data_ptr(), ldq, scales.data_ptr(), lds, W.data_ptr(),
          ldw)


def q4_workspace_bytes(t: int, n: int, k: int, group: int, dtype, gradient: bool = False) -> int:
    out = ctypes.c_size_t()
    _check(lib().ozimmu_q4_workspace_bytes(t, n, k, group, _type_of(dtype), int(bool(gradient)), ctypes.byref(out)))
    return out.value


def alloc_q4_workspace(t: int, n: int, k: int, group: int, dtype, gradient: bool = False, device="cuda"):
    """A uint8 tensor of the size that q4_gemm (gradient: q4_gemm_grad) asks for; it serves fewer tokens too."""
    import torch

    return torch.empty(max(q4_workspace_bytes(t, n, k, group, dtype, gradient), WORKSPACE_ALIGN), dtype=torch.uint8, device=device)


def _size(workspace) -> int:
    if workspace is None:
        return 0
    if not workspace.is_contiguous():
        raise ValueError("expected a contiguous workspace")
    return workspace.numel() * workspace.element_size()


def _q4_product(f, gradient, V, codes, scales, group, R, workspace, stream):
    # (The checks of _rows and _q4_weights in one place: a token's call waits for every microsecond spent here.)
    if _torch is None:
        _load_torch()
    dtype = V.dtype
    kind = _types.get(dtype)
    if kind is None:
        _type_of(dtype)             # raises
    if dtype is not scales.dtype or dtype is not R.dtype:
        raise ValueError("tokens, scales and result must have one type")
    try:
        t, inner = V.shape
        rows, outer = R.shape
        code_rows, code_bytes = codes.shape
        scale_rows, groups = scales.shape
    except ValueError:
        raise ValueError("expected 2-D tensors") from None
    ldv, step_v = V.stride()
    ldr, step_r = R.stride()
    ldq, step_q = codes.stride()
    lds, step_s = scales.stride()
    if step_v != 1 and inner > 1 or step_r != 1 and outer > 1 or step_q != 1 and code_bytes > 1 or step_s != 1 and groups > 1:
        raise ValueError("expected row-major tensors (unit stride along the second dimension)")
    if rows != t:
        raise ValueError("tokens and result must have the same number of rows")
    n, k = (inner, outer) if gradient else (outer, inner)
    if group not in _GROUPS:
        q4_geometry(k, group)       # raises
    row_bytes_ = (k + 31) // 32 * 16
    if code_rows != n or code_bytes < row_bytes_ or codes.dtype is not _uint8:
        raise ValueError(f"codes: expected {n} rows of at least {row_bytes_} bytes (uint8)")
    if scale_rows != n or groups != -(-k // group):
        raise ValueError(f"scales: expected the shape {(n, -(-k // group))}")
    if t <= 1:
        ldv, ldr = inner or 1, outer or 1
    if n <= 1:
        ldq, lds = row_bytes_, groups or 1
    _call(f, stream, (V, codes, scales, R, workspace), t, n, k, group, kind, V.data_ptr(), ldv, codes.data_ptr(), ldq, scales.data_ptr(), lds, R.data_ptr(),
          ldr, None if workspace is None else workspace.data_ptr(), _size(workspace))


def q4_gemm(X, codes, scales, group: int, Y, workspace=None, stream=None) -> None:
    """Y = X W^T for weights in four bits (X: t x k, Y: t x n; X, Y and the scales of one type). The workspace may be None
    where q4_workspace_bytes gives 0 (up to 16 tokens always, often for many more)."""
    _q4_product(lib().ozimmu_q4_gemm, False, X, codes, scales, group, Y, workspace, stream)


def q4_gemm_grad(dY, codes, scales, group: int, dX, workspace, stream=None) -> None:
    """dX = dY W for weights in four bits (dY: t x n, dX: t x k): the gradient of q4_gemm's result, on its way to X."""
    _q4_product(lib().ozimmu_q4_gemm_grad, True, dY, codes, scales, group, dX, workspace, stream)


def orthogonalize_workspace_bytes(batch: int, m: int, n: int) -> int:
    out = ctypes.c_size_t()
    _check(lib().ozimmu_orthogonalize_workspace_bytes(batch, m, n, ctypes.byref(out)))
    return out.value


def alloc_orthogonalize_workspace(batch: int, m: int, n: int, dtype=None, device="cuda"):
    """A uint8 tensor of the size that orthogonalize asks for. (`dtype`, the matrices' type, does not change it; it may be given as to alloc_q4_workspace.)"""
    import torch

    return torch.empty(max(orthogonalize_workspace_bytes(batch, m, n), WORKSPACE_ALIGN), dtype=torch.uint8, device=device)


def orthogonalize(G, X, workspace, steps: int = 5, coefficients=(3.4445, -4.7750, 2.0315), eps: float = 1e-7, stream=None) -> None:
    """X = the orthogonal update of G by `steps` Newton-Schulz steps (see ozimmu.h). G and X: m x n, or a batch of such, of one
    type (float32, bfloat16, float16), rows with unit stride; X may be G itself."""
    _expect(G.dim() in (2, 3) and G.shape == X.shape and G.dtype == X.dtype, "G and X must have one shape (two or three dimensions) and type")
    m, n = G.shape[-2:]
    batch = G.shape[0] if G.dim() == 3 else 1
    ld = {}
    for name, t in (("g", G), ("x", X)):
        _expect(n <= 1 or t.stride(-1) == 1, "expected rows with unit stride")
        ld[name] = (t.stride(-2) if m > 1 else max(n, 1), t.stride(0) if t.dim() == 3 else 0)
    a, b, c = coefficients
    _call(lib().ozimmu_orthogonalize, stream, (G, X, workspace), batch, m, n, _type_of(G.dtype), G.data_ptr(), *ld["g"], X.data_ptr(), *ld["x"], int(steps),
          float(a), float(b), float(c), float(eps), _ptr(workspace), _size(workspace))


def f8_geometry(k: int):
    """(bytes of a row of codes, bytes of a row of scales) of a matrix of k columns in 8-bit floating point (see ozimmu.h)."""
    row_bytes_, scale_bytes_ = ctypes.c_int64(), ctypes.c_int64()
    _check(lib().ozimmu_f8_geometry(k, ctypes.byref(row_bytes_), ctypes.byref(scale_bytes_)))
    return row_bytes_.value, scale_bytes_.value


def f8_row_bytes(k: int) -> int:
    return f8_geometry(k)[0]


def f8_scale_bytes(k: int) -> int:
    return f8_geometry(k)[1]


_native = None


def _calls():
    """The module whose functions check tensors and call the library in one step (csrc/calls.cpp): a token's call waits for every microsecond spent
    on the host."""
    global _native
    if _native is None:
        lib()
        if _torch is None:
            _load_torch()
        try:
            from . import _calls as module
        except ImportError as e:
            raise RuntimeError(f"{Path(__file__).parent / '_calls.so'} is missing or was built for another torch: build it with "
                               "`python -m paper_2306_11975_amd.build`") from e
        _native = module
    return _native


def f8_split(W, codes, scales, block_rows: int = 128, stream=None) -> None:
    """W (n x k; float32, bfloat16 or float16) into codes (n x f8_row_bytes(k); uint8 or float8_e4m3fn) and scales (ceil(n / block_rows) x
    f8_scale_bytes(k); uint8 or float8_e8m0fnu), in blocks of block_rows (1: tokens, 128: weights) x 128."""
    code = (_native or _calls()).f8_split(W, codes, scales, block_rows, stream)
    if code:
        _check(code)


def f8_expand(codes, scales, W, block_rows: int = 128, stream=None) -> None:
    """The values that codes and scales stand for, into W (n x k; float32, bfloat16 or float16)."""
    code = (_native or _calls()).f8_expand(codes, scales, W, block_rows, stream)
    if code:
        _check(code)


_F8_OPS = {"gemm": 0, "grad": 1, "weight_grad": 2}


def f8_workspace_bytes(op: str, t: int, n: int, k: int, dtype, rows=None, experts: int = 0) -> int:
    """Workspace of f8_gemm ("gemm"), f8_gemm_grad ("grad") or f8_weight_grad ("weight_grad"): t tokens, rows of Y and dY (experts; t without
    them), and the type of X and dY."""
    if _torch is None:
        _load_torch()
    _expect(op in _F8_OPS, "op: expected gemm, grad or weight_grad")
    out = ctypes.c_size_t()
    kind = E4M3 if dtype in (_torch.uint8, _torch.float8_e4m3fn) else _type_of(dtype)
    _check(lib().ozimmu_f8_workspace_bytes(_F8_OPS[op], t, t if rows is None else rows, n, k, experts, kind, ctypes.byref(out)))
    return out.value


def alloc_f8_workspace(op: str, t: int, n: int, k: int, dtype, rows=None, experts: int = 0, device="cuda"):
    """A uint8 tensor of the size that the operator asks for; it serves fewer tokens and rows too."""
    import torch

    return torch.empty(max(f8_workspace_bytes(op, t, n, k, dtype, rows, experts), WORKSPACE_ALIGN), dtype=torch.uint8, device=device)


def f8_gemm(X, codes, scales, Y, workspace=None, x_scales=None, offsets=None, source=None, stream=None) -> None:
    """Y = X W^T for weights in 8-bit floating point (X: t x k, Y: rows x n, each float32, bfloat16 or float16). X is cut in the call, or given
    as codes with x_scales (f8_split with block_rows 1). Over experts: codes and scales with a first dimension of experts, offsets (experts + 1,
    int32): the rows of Y of each, and source (rows, int32): the row of X for each row of Y (without it X has the rows of Y)."""
    code = (_native or _calls()).f8_gemm(X, codes, scales, Y, workspace, x_scales, offsets, source, stream)
    if code:
        _check(code)


def f8_gemm_grad(dY, codes, scales, dX, workspace, dy_scales=None, offsets=None, stream=None) -> None:
    """dX = dY W for weights in 8-bit floating point (dY: rows x n, dX: rows x k): the gradient of f8_gemm's result, on its way to X. Over
    experts dX has the rows of dY: expert_combine without weights adds those of a token."""
    code = (_native or _calls()).f8_gemm_grad(dY, codes, scales, dX, workspace, dy_scales, offsets, stream)
    if code:
        _check(code)


def f8_weight_grad(dY, X, dW, workspace, offsets=None, source=None, stream=None) -> None:
    """dW = dY^T X in 8-bit floating point, cut along the tokens (dY: rows x n, X: t x k of one type, dW: n x k). Over experts: dW with a
    first dimension of experts, offsets and source as for f8_gemm."""
    code = (_native or _calls()).f8_weight_grad(dY, X, dW, workspace, offsets, source, stream)
    if code:
        _check(code)


_SCORES = {"softmax": SOFTMAX, "sigmoid": SIGMOID}


def _score(name: str) -> int:
    score = _SCORES.get(name)
    if score is None:
        raise ValueError("score: expected softmax or sigmoid")
    return score


def route(logits, indices, weights, bias=None, score: str = "softmax", groups: int = 1, top_groups: int = 1, renormalize: bool = True, scale: float = 1.0,
          stream=None) -> None:
    """The best experts of each token and their weights (see ozimmu.h). logits: t x experts (float32, bfloat16 or float16); indices (int32)
    and weights (float32): t x top, contiguous; bias: experts, float32, for the choice alone."""
    code = (_native or _calls()).route(logits, indices, weights, bias, _score(score), groups, top_groups, renormalize, scale, stream)
    if code:
        _check(code)


def route_grad(logits, indices, dweights, dlogits, score: str = "softmax", renormalize: bool = True, scale: float = 1.0, stream=None) -> None:
    """The gradient of the logits (dlogits: their shape and type) from that of route's weights; the choice counts as constant."""
    code = (_native or _calls()).route_grad(logits, indices, dweights, dlogits, _score(score), renormalize, scale, stream)
    if code:
        _check(code)


def expert_order_workspace_bytes(t: int, top: int, experts: int) -> int:
    out = ctypes.c_size_t()
    _check(lib().ozimmu_expert_order_workspace_bytes(t, top, experts, ctypes.byref(out)))
    return out.value


def alloc_expert_order_workspace(t: int, top: int, experts: int, device="cuda"):
    """A uint8 tensor of the size that expert_order asks for; it serves fewer tokens too."""
    import torch

    return torch.empty(max(expert_order_workspace_bytes(t, top, experts), WORKSPACE_ALIGN), dtype=torch.uint8, device=device)


def expert_order(indices, experts: int, offsets, source, place, workspace=None, stream=None) -> None:
    """The (token, choice) pairs of indices (t x top) sorted by expert: offsets (experts + 1), source (t top: the token of each row) and
    place (t x top: the row of each pair, -1 for an index that is no expert). All int32."""
    code = (_native or _calls()).expert_order(indices, experts, offsets, source, place, workspace, stream)
    if code:
        _check(code)


def expert_combine(O, place, weights, Y, stream=None) -> None:
    """Y[i] = sum over j of weights[i, j] O[place[i, j]] (O: rows x n, Y: t x n of one type; place, weights: t x top; weights None: ones, which
    gives the gradient of taking rows by `source`)."""
    code = (_native or _calls()).expert_combine(O, place, weights, Y, stream)
    if code:
        _check(code)


def expert_combine_grad(dY, O, place, weights, dO, dweights, stream=None) -> None:
    """The gradients of expert_combine: dO (rows x n; rows without a pair are left alone) and dweights (t x top, float32)."""
    code = (_native or _calls()).expert_combine_grad(dY, O, place, weights, dO, dweights, stream)
    if code:
        _check(code)


def probe_int8_mfma(pattern: int, shape: int = 0, iters: int = 200000):
    """(10^12 INT8 ops/s, shader MHz) of a register-only MFMA issue loop; see ozimmu_probe.h."""
    tops, mhz = ctypes.c_double(), ctypes.c_double()
    _check(lib().ozimmu_probe_int8_mfma(pattern, shape, iters, ctypes.byref(tops), ctypes.byref(mhz)))
    return tops.value, mhz.value


def alloc_workspace(m: int, n: int, k: int, num_slices: int, is_complex: bool = False, device="cuda"):
    """Convenience for callers that use torch for device memory: a uint8 tensor of the right size
    (torch's caching allocator returns 512-byte aligned blocks)."""
    import torch

    nbytes = max(workspace_bytes(m, n, k, num_slices, is_complex), WORKSPACE_ALIGN)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    assert ws.data_ptr() % WORKSPACE_ALIGN == 0
    return ws
