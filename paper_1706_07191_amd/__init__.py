"""Thin ctypes binding of libbrsvd (hand-written HIP for MI355X / gfx950).

Only argument marshalling lives here: torch provides device memory and streams, every step of
the block randomized SVD runs inside the shared library.  The functions carry the same names
as the C entry points declared in include/brsvd.h.  There is no CPU fallback: if the shared
library has not been built (python -m paper_1706_07191_amd.build) importing `lib()` raises.
"""
from __future__ import annotations

import ctypes as C
import operator
import os
from typing import Optional

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libbrsvd.so")

BRSVD_OK = 0
BRSVD_ERR_ARG = -1
BRSVD_ERR_BUDGET = -2
BRSVD_ERR_ALLOC = -3
BRSVD_ERR_HIP = -4
BRSVD_ERR_ORTH_BREAKDOWN = -5
BRSVD_ERR_SVD_NOCONV = -6
BRSVD_A_DEVICE = 0
BRSVD_A_HOST_PINNED = 1
BRSVD_ORTH_AUTO = 0
BRSVD_ORTH_CHOLQR2 = 1
BRSVD_ORTH_TSQR = 2
BRSVD_PASSES_SEPARATE = 0
BRSVD_PASSES_FUSED = 1
BRSVD_DTYPE_F32 = 0
BRSVD_DTYPE_F64 = 1
BRSVD_DTYPE_BF16 = 2
BRSVD_DTYPE_F16 = 3
BRSVD_ACT_SILU = 0
BRSVD_ACT_GELU = 1
BRSVD_ACT_GELU_TANH = 2


class brsvd_params(C.Structure):
    _fields_ = [("m", C.c_int64), ("n", C.c_int64),
                ("k", C.c_int32), ("p", C.c_int32), ("q", C.c_int32), ("a_location", C.c_int32),
                ("row_block", C.c_int64), ("device_budget_bytes", C.c_uint64),
                ("orth_method", C.c_int32), ("pass_mode", C.c_int32),
                ("compute_stream", C.c_void_p), ("copy_stream", C.c_void_p),
                ("dtype", C.c_int32), ("timing_level", C.c_int32),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_uint64)]


class brsvd_tensor(C.Structure):
    _fields_ = [("data", C.c_void_p), ("rows", C.c_int64), ("cols", C.c_int64), ("ld", C.c_int64), ("dtype", C.c_int64)]


class brsvd_stats(C.Structure):
    _fields_ = [("total_seconds", C.c_double), ("gemm_an_seconds", C.c_double),
                ("gemm_at_seconds", C.c_double), ("orth_seconds", C.c_double),
                ("svd_seconds", C.c_double), ("lift_seconds", C.c_double),
                ("copy_seconds", C.c_double), ("elementwise_seconds", C.c_double),
                ("gemm_an_launches", C.c_int64), ("gemm_at_launches", C.c_int64),
                ("passes_over_A", C.c_int64), ("bytes_A_streamed", C.c_int64),
                ("orth_fallbacks", C.c_int32), ("jacobi_sweeps", C.c_int32),
                ("row_block", C.c_int32), ("n_blocks", C.c_int32),
                ("split_sum_seconds", C.c_double), ("rpca_update_seconds", C.c_double),
                ("rpca_update_launches", C.c_int64), ("bytes_A_read_by_kernels", C.c_int64),
                ("fused_fallbacks", C.c_int32), ("reserved_", C.c_int32)]

    def as_dict(self):
        return {f: getattr(self, f) for f, _ in self._fields_}


# entry points declared in include/brsvd.h (the product calls) and include/brsvd_steps.h (the steps)
EXPORTS = ["brsvd_workspace_bytes", "brsvd_create", "brsvd_run", "brsvd_run_f64", "brsvd_rpca_ialm",
           "brsvd_rpca_ialm_tol", "brsvd_rpca_ialm_tol_f64", "brsvd_norm2_power", "brsvd_norm2_power_f64",
           "brsvd_run_alg2", "brsvd_run_alg2_f64", "brsvd_philox_normal", "brsvd_philox_normal_f64",
           "brsvd_quantize_e4m3", "brsvd_dequantize_e4m3", "brsvd_gemm_e4m3", "brsvd_gemm_e4m3_scratch_bytes",
           "brsvd_linear_e4m3", "brsvd_linear_e4m3_scratch_bytes", "brsvd_quantize_e2m1", "brsvd_dequantize_e2m1",
           "brsvd_linear_e2m1", "brsvd_linear_e2m1_backward", "brsvd_linear_e2m1_scratch_bytes", "brsvd_glu_forward",
           "brsvd_glu_backward", "brsvd_glu_workspace_bytes", "brsvd_grad_norm", "brsvd_grad_norm_workspace_bytes", "brsvd_grad_clip",
           "brsvd_xent_forward", "brsvd_xent_backward",
           "brsvd_distill_forward", "brsvd_distill_backward", "brsvd_head_workspace_bytes",
           "brsvd_destroy", "brsvd_status_string"]
STEP_EXPORTS = ["brsvd_gemm_an", "brsvd_gemm_at", "brsvd_gemm_scratch_bytes", "brsvd_gemm_an_f64",
                "brsvd_gemm_at_f64", "brsvd_gemm_scratch_bytes_f64", "brsvd_orth", "brsvd_orth_scratch_bytes",
                "brsvd_small_svd", "brsvd_small_svd_scratch_bytes", "brsvd_small_svd_static", "brsvd_gemm_plan", "brsvd_linear_e2m1_plan", "brsvd_glu_plan",
                "brsvd_gemm_is_split", "brsvd_gemm_split_parts", "brsvd_probe"]

_lib = None


class BrsvdError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where} failed: {status} ({brsvd_status_string(status)})")


def lib() -> C.CDLL:
    """Loads libbrsvd.so (raises if it was not built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_1706_07191_amd.build`; "
                          "there is no fallback implementation")
    L = C.CDLL(LIB_PATH)
    vp, i32, i64, u64, dbl, flt = C.c_void_p, C.c_int32, C.c_int64, C.c_uint64, C.c_double, C.c_float
    L.brsvd_workspace_bytes.argtypes = [C.POINTER(brsvd_params), C.POINTER(u64)]
    L.brsvd_create.argtypes = [C.POINTER(brsvd_params), C.POINTER(vp)]
    L.brsvd_run.argtypes = [vp, vp, i64, vp, vp, vp, vp, C.POINTER(brsvd_stats)]
    L.brsvd_run_f64.argtypes = L.brsvd_run.argtypes
    L.brsvd_rpca_ialm.argtypes = [vp, vp, vp, i32, flt, flt, flt, dbl, vp, vp, vp, C.POINTER(dbl),
                                  C.POINTER(brsvd_stats)]
    L.brsvd_rpca_ialm_tol.argtypes = [vp, vp, vp, i32, dbl, flt, flt, flt, dbl, vp, vp, vp, C.POINTER(dbl),
                                      C.POINTER(i32), C.POINTER(brsvd_stats)]
    L.brsvd_rpca_ialm_tol_f64.argtypes = [vp, vp, vp, i32, dbl, dbl, dbl, dbl, dbl, vp, vp, vp, C.POINTER(dbl),
                                          C.POINTER(i32), C.POINTER(brsvd_stats)]
    L.brsvd_norm2_power.argtypes = [vp, vp, i64, vp, i32, C.POINTER(dbl)]
    L.brsvd_norm2_power_f64.argtypes = L.brsvd_norm2_power.argtypes
    L.brsvd_run_alg2.argtypes = [vp, vp, i64, u64, vp, vp, vp, vp, C.POINTER(brsvd_stats)]
    L.brsvd_philox_normal.argtypes = [u64, i64, i64, i32, vp, vp]
    L.brsvd_run_alg2_f64.argtypes = L.brsvd_run_alg2.argtypes
    L.brsvd_philox_normal_f64.argtypes = L.brsvd_philox_normal.argtypes
    L.brsvd_probe.argtypes = [i32, vp, u64, C.POINTER(dbl), C.POINTER(dbl), vp]
    L.brsvd_gemm_plan.argtypes = [i32, i64, i64, i32, i64, i32, C.POINTER(i32)]
    L.brsvd_linear_e2m1_plan.argtypes = [i64, i64, i64, i32, C.POINTER(i32)]
    L.brsvd_glu_plan.argtypes = [i32, i64, i64, i64, C.POINTER(i32)]
    L.brsvd_gemm_is_split.argtypes = [i32, vp, i64, i64, i64, i32, i32]
    L.brsvd_gemm_split_parts.argtypes = [i32, i64, i64, i32]
    L.brsvd_destroy.argtypes = [vp]
    L.brsvd_status_string.argtypes = [C.c_int]
    L.brsvd_status_string.restype = C.c_char_p
    L.brsvd_gemm_an.argtypes = [vp, i64, i64, i64, vp, i32, vp, vp, u64, vp]
    L.brsvd_gemm_at.argtypes = [vp, i64, i64, i64, vp, i32, vp, i32, vp, u64, vp]
    L.brsvd_gemm_scratch_bytes.argtypes = [i64, i64, i32]
    L.brsvd_gemm_an_f64.argtypes = L.brsvd_gemm_an.argtypes
    L.brsvd_gemm_at_f64.argtypes = L.brsvd_gemm_at.argtypes
    L.brsvd_gemm_scratch_bytes_f64.argtypes = [i64, i64, i32]
    L.brsvd_orth.argtypes = [vp, i64, i32, i32, vp, C.POINTER(i32), vp, u64, vp]
    L.brsvd_orth_scratch_bytes.argtypes = [i64, i32]
    L.brsvd_small_svd.argtypes = [vp, i32, vp, vp, vp, C.POINTER(i32), vp, u64, vp]
    L.brsvd_small_svd_scratch_bytes.argtypes = [i32]
    L.brsvd_small_svd_static.argtypes = [vp, i32, vp, vp, vp, C.POINTER(i32), vp]
    L.brsvd_quantize_e4m3.argtypes = [vp, i64, i64, i64, i32, i32, vp, i64, vp, vp, i64, vp, vp]
    L.brsvd_dequantize_e4m3.argtypes = [vp, i64, vp, i64, i64, i32, i32, vp, i64, vp]
    L.brsvd_gemm_e4m3.argtypes = [vp, i64, vp, vp, i64, vp, i32, i64, i64, i64, i32, vp, i64, vp, u64, vp]
    L.brsvd_gemm_e4m3_scratch_bytes.argtypes = [i64, i64, i64, i32, i32]
    L.brsvd_linear_e4m3.argtypes = [vp, i64, i32, vp, i64, vp, i64, i64, i64, vp, i64, vp, u64, vp]
    L.brsvd_linear_e4m3_scratch_bytes.argtypes = [i64, i64, i64, i32]
    L.brsvd_quantize_e2m1.argtypes = [vp, i64, i64, i64, i32, vp, i64, vp, vp]
    L.brsvd_dequantize_e2m1.argtypes = [vp, i64, vp, i64, i64, i32, vp, i64, vp]
    L.brsvd_linear_e2m1.argtypes = [vp, i64, i32, vp, i64, vp, i64, i64, i64, vp, i64, vp, u64, vp]
    L.brsvd_linear_e2m1_backward.argtypes = L.brsvd_linear_e2m1.argtypes
    L.brsvd_linear_e2m1_scratch_bytes.argtypes = [i64, i64, i64, i32, i32]
    L.brsvd_glu_forward.argtypes = [vp, i64, vp, i64, vp, i64, i64, i64, i64, i32, i32, vp, i64, vp, i64, vp, i64, vp, u64, vp]
    L.brsvd_glu_backward.argtypes = [vp, i64, vp, i64, vp, i64, vp, i64, vp, i64, vp, i64, i64, i64, i64, i32, i32, vp, i64, vp, i64, vp, i64,
                                     vp, u64, vp]
    L.brsvd_glu_workspace_bytes.argtypes = [i64, i64, i64, i32, i32]
    L.brsvd_grad_norm.argtypes = [vp, i64, flt, vp, vp, u64, vp]
    L.brsvd_grad_norm_workspace_bytes.argtypes = [vp, i64]
    L.brsvd_grad_clip.argtypes = [vp, vp, i64, flt, flt, vp, vp]
    L.brsvd_xent_forward.argtypes = [vp, i64, vp, i64, vp, i64, i64, i64, i32, vp, vp, vp, u64, vp]
    L.brsvd_xent_backward.argtypes = [vp, i64, vp, i64, vp, vp, vp, i64, i64, i64, i64, i64, i32, vp, i64, vp, i64, vp, u64, vp]
    L.brsvd_distill_forward.argtypes = [vp, i64, vp, i64, vp, vp, i32, flt, i64, i64, i64, i32, vp, vp, vp, vp, u64, vp]
    L.brsvd_distill_backward.argtypes = [vp, i64, vp, i64, vp, vp, i32, flt, vp, vp, vp, i64, i64, i64, i64, i64, i32, vp, i64,
                                         vp, i64, vp, u64, vp]
    L.brsvd_head_workspace_bytes.argtypes = [i64, i64, i64, i64, i32, i32]
    sizes = ("brsvd_gemm_scratch_bytes", "brsvd_gemm_scratch_bytes_f64", "brsvd_orth_scratch_bytes",
             "brsvd_small_svd_scratch_bytes", "brsvd_gemm_e4m3_scratch_bytes", "brsvd_linear_e4m3_scratch_bytes",
             "brsvd_linear_e2m1_scratch_bytes", "brsvd_glu_workspace_bytes", "brsvd_grad_norm_workspace_bytes",
             "brsvd_head_workspace_bytes")
    for name in EXPORTS + STEP_EXPORTS:
        if name in sizes:
            getattr(L, name).restype = u64
        elif name != "brsvd_status_string":
            getattr(L, name).restype = C.c_int
    _lib = L
    return L


def brsvd_status_string(status: int) -> str:
    return lib().brsvd_status_string(int(status)).decode()


def _check(status: int, where: str):
    if status != BRSVD_OK:
        raise BrsvdError(status, where)


def _stream_ptr(stream) -> Optional[int]:
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream or None
    if isinstance(stream, int):
        return stream or None
    return stream.cuda_stream or None


def _dev(t, dtype, name):
    import torch
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == dtype and t.is_contiguous()):
        raise TypeError(f"{name} must be a contiguous CUDA tensor of dtype {dtype}")
    return t.data_ptr()


def make_params(m, n, k, p, q, row_block=0, device_budget_bytes=0, a_location=BRSVD_A_DEVICE,
                orth_method=BRSVD_ORTH_AUTO, compute_stream=None, copy_stream=None,
                pass_mode=BRSVD_PASSES_SEPARATE, dtype=BRSVD_DTYPE_F32, timing_level=0,
                workspace=None) -> brsvd_params:
    """workspace: optional CUDA uint8 tensor the handle uses instead of allocating (keep it alive)."""
    return brsvd_params(workspace=workspace.data_ptr() if workspace is not None else None,
                        workspace_bytes=workspace.numel() * workspace.element_size() if workspace is not None else 0,
                        m=m, n=n, k=k, p=p, q=q, a_location=a_location, row_block=row_block,
                        device_budget_bytes=device_budget_bytes, orth_method=orth_method, pass_mode=pass_mode,
                        compute_stream=_stream_ptr(compute_stream),
                        copy_stream=_stream_ptr(copy_stream) if copy_stream is not None else None,
                        dtype=dtype, timing_level=timing_level)


def brsvd_workspace_bytes(params: brsvd_params) -> int:
    out = C.c_uint64(0)
    _check(lib().brsvd_workspace_bytes(C.byref(params), C.byref(out)), "brsvd_workspace_bytes")
    return out.value


def brsvd_create(params: brsvd_params) -> C.c_void_p:
    h = C.c_void_p()
    _check(lib().brsvd_create(C.byref(params), C.byref(h)), "brsvd_create")
    return h


def brsvd_destroy(handle) -> None:
    _check(lib().brsvd_destroy(handle), "brsvd_destroy")


def brsvd_run(handle, A, Omega, U=None, S=None, Vt=None, lda: Optional[int] = None, want_stats=True,
              pinned=False):
    """A: (m, n) CUDA tensor (or pinned host tensor for a host-resident handle), row stride lda, fp32 -- or
    fp64 for a handle created with dtype=BRSVD_DTYPE_F64 (brsvd_run_f64); Omega: (n, l) CUDA, same dtype.
    pinned=True vouches for a host A that torch did not allocate itself (see PinnedMatrix).
    Returns (U, S, Vt, stats) as CUDA tensors m x l, l, l x n."""
    import torch
    m, n = A.shape
    l = Omega.shape[1]
    dt = A.dtype
    if dt not in (torch.float32, torch.float64) or A.stride(1) != 1:
        raise TypeError("A must be fp32 or fp64 with unit column stride")
    if not A.is_cuda and not (pinned or A.is_pinned()):
        raise TypeError("a host-resident A must be pinned")
    lda = lda if lda is not None else A.stride(0)
    dev = Omega.device
    U = torch.empty(m, l, device=dev, dtype=dt) if U is None else U
    S = torch.empty(l, device=dev, dtype=dt) if S is None else S
    Vt = torch.empty(l, n, device=dev, dtype=dt) if Vt is None else Vt
    st = brsvd_stats()
    fn = lib().brsvd_run_f64 if dt == torch.float64 else lib().brsvd_run
    status = fn(handle, A.data_ptr(), lda, _dev(Omega, dt, "Omega"), _dev(U, dt, "U"), _dev(S, dt, "S"),
                _dev(Vt, dt, "Vt"), C.byref(st) if want_stats else None)
    _check(status, "brsvd_run")
    return U, S, Vt, (st.as_dict() if want_stats else None)


def brsvd_run_alg2(handle, A, l, seed=0, Omega=None, lda: Optional[int] = None, want_stats=True, pinned=False,
                   device=None):
    """Block-local scheme of Alg. 2.  A as for brsvd_run (fp32, or fp64 on a BRSVD_DTYPE_F64 handle); Omega
    (m, l) CUDA of the same dtype or None (then the library draws it from `seed`).  Returns (U, S, Vt, stats)."""
    import torch
    m, n = A.shape
    dt = A.dtype
    if dt not in (torch.float32, torch.float64) or A.stride(1) != 1:
        raise TypeError("A must be fp32 or fp64 with unit column stride")
    if not A.is_cuda and not (pinned or A.is_pinned()):
        raise TypeError("a host-resident A must be pinned")
    lda = lda if lda is not None else A.stride(0)
    dev = device or (Omega.device if Omega is not None else (A.device if A.is_cuda else torch.device("cuda:0")))
    U = torch.empty(m, l, device=dev, dtype=dt)
    S = torch.empty(l, device=dev, dtype=dt)
    Vt = torch.empty(l, n, device=dev, dtype=dt)
    st = brsvd_stats()
    fn = lib().brsvd_run_alg2_f64 if dt == torch.float64 else lib().brsvd_run_alg2
    status = fn(handle, A.data_ptr(), lda, int(seed), _dev(Omega, dt, "Omega") if Omega is not None else None,
                U.data_ptr(), S.data_ptr(), Vt.data_ptr(), C.byref(st) if want_stats else None)
    _check(status, "brsvd_run_alg2")
    return U, S, Vt, (st.as_dict() if want_stats else None)


def brsvd_gemm_plan(which, rows, n, l, block_rows=0, dtype=BRSVD_DTYPE_F32):
    """The launch plan of gemm_an (which = 0) or gemm_at (which = 1) as a list of 12 ints (see brsvd.h)."""
    out = (C.c_int32 * 12)()
    _check(lib().brsvd_gemm_plan(which, rows, n, l, block_rows, dtype, out), "brsvd_gemm_plan")
    return list(out)


def brsvd_linear_e2m1_plan(m, n, k, backward=False):
    """How X W^T (or its gradient) with X m x k and W n x k in 4 bits goes to the GPU, as a list of 8 ints (see brsvd_steps.h)."""
    out = (C.c_int32 * 8)()
    _check(lib().brsvd_linear_e2m1_plan(m, n, k, backward, out), "brsvd_linear_e2m1_plan")
    return list(out)


def brsvd_glu_plan(which, tokens, dim, width):
    """How a gated block's products (which = 0: forward, 1: dX, 2: dWg and dWu) go to the GPU, as a list of 8 ints (see brsvd_steps.h)."""
    out = (C.c_int32 * 8)()
    _check(lib().brsvd_glu_plan(which, tokens, dim, width, out), "brsvd_glu_plan")
    return list(out)


def brsvd_gemm_is_split(which, rows, n, l, lda=None, address=0, dtype=BRSVD_DTYPE_F32) -> bool:
    """Whether A X (which = 0) or A^T Q (which = 1) takes the split kernels; `address`: where A begins (its alignment counts)."""
    r = lib().brsvd_gemm_is_split(which, address, n if lda is None else lda, rows, n, l, dtype)
    if r < 0:
        _check(r, "brsvd_gemm_is_split")
    return bool(r)


def brsvd_gemm_split_parts(which, rows, n, l) -> int:
    """How many 16-bit numbers a split product's operands are made of: 3 (bf16, six matrix products) or 2 (fp16, three)."""
    r = lib().brsvd_gemm_split_parts(which, rows, n, l)
    if r < 0:
        _check(r, "brsvd_gemm_split_parts")
    return r


def brsvd_probe(kind, buf, amount):
    """Measured device peaks: kind 0 streaming read of `amount` bytes of buf, kind 1 an fp32 MFMA loop.
    Returns (seconds, work) with work in bytes or flops."""
    sec, work = C.c_double(0.0), C.c_double(0.0)
    _check(lib().brsvd_probe(kind, buf.data_ptr(), int(amount), C.byref(sec), C.byref(work), None), "brsvd_probe")
    return sec.value, work.value


def brsvd_philox_normal(seed, rows, cols, row0=0, device="cuda:0", stream=None, f64=False):
    """Rows [row0, row0 + rows) of the Gaussian matrix brsvd_run_alg2 draws from `seed` (fp32, or fp64)."""
    import torch
    out = torch.empty(rows, cols, device=device, dtype=torch.float64 if f64 else torch.float32)
    fn = lib().brsvd_philox_normal_f64 if f64 else lib().brsvd_philox_normal
    _check(fn(int(seed), row0, rows, cols, out.data_ptr(), _stream_ptr(stream)), "brsvd_philox_normal")
    return out


def brsvd_rpca_ialm(handle, M, Omegas, iters, lam, mu0, rho, norm2_M=0.0, L=None, S=None, work=None):
    import torch
    m, n = M.shape
    L = torch.empty_like(M) if L is None else L
    S = torch.empty_like(M) if S is None else S
    work = torch.empty(2 * m * n, device=M.device) if work is None else work
    res = (C.c_double * iters)()
    st = brsvd_stats()
    status = lib().brsvd_rpca_ialm(handle, _dev(M, torch.float32, "M"), _dev(Omegas, torch.float32, "Omegas"),
                                   iters, lam, mu0, rho, norm2_M, _dev(L, torch.float32, "L"),
                                   _dev(S, torch.float32, "S"), _dev(work, torch.float32, "work"), res,
                                   C.byref(st))
    _check(status, "brsvd_rpca_ialm")
    return L, S, list(res), st.as_dict()


def brsvd_rpca_ialm_tol(handle, M, Omegas, max_iters, tol, lam, mu0, rho, norm2_M=0.0, L=None, S=None, work=None):
    """Returns L, S, the residuals of the iterations run, their number, and the statistics.  fp32, or fp64 when M
    is a float64 tensor (handle created with dtype=BRSVD_DTYPE_F64)."""
    import torch
    m, n = M.shape
    dt = M.dtype
    L = torch.empty_like(M) if L is None else L
    S = torch.empty_like(M) if S is None else S
    work = torch.empty(2 * m * n, device=M.device, dtype=dt) if work is None else work
    res = (C.c_double * max_iters)()
    done = C.c_int32(0)
    st = brsvd_stats()
    fn = lib().brsvd_rpca_ialm_tol_f64 if dt == torch.float64 else lib().brsvd_rpca_ialm_tol
    status = fn(handle, _dev(M, dt, "M"), _dev(Omegas, dt, "Omegas"), max_iters, tol, lam, mu0, rho, norm2_M,
                _dev(L, dt, "L"), _dev(S, dt, "S"), _dev(work, dt, "work"), res, C.byref(done), C.byref(st))
    _check(status, "brsvd_rpca_ialm_tol")
    return L, S, list(res)[:done.value], done.value, st.as_dict()


def brsvd_norm2_power(handle, A, x0, iters, lda=None) -> float:
    import torch
    out = C.c_double(0.0)
    lda = A.stride(0) if lda is None else lda
    fn = lib().brsvd_norm2_power_f64 if A.dtype == torch.float64 else lib().brsvd_norm2_power
    _check(fn(handle, A.data_ptr(), lda, _dev(x0, A.dtype, "x0"), iters, C.byref(out)), "brsvd_norm2_power")
    return out.value


def brsvd_gemm_scratch_bytes(rows, n, l, f64=False) -> int:
    L = lib()
    return (L.brsvd_gemm_scratch_bytes_f64 if f64 else L.brsvd_gemm_scratch_bytes)(rows, n, l)


def _scratch(rows, n, l, device, f64=False):
    import torch
    nbytes = brsvd_gemm_scratch_bytes(rows, n, l, f64)
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device), nbytes


def brsvd_gemm_an(A, X, Y=None, rows=None, lda=None, stream=None):
    """Y = A[:rows] @ X on the HIP path.  A (rows, n) CUDA (row stride lda), X (n, l); fp32, or fp64 when
    A is a float64 tensor (brsvd_gemm_an_f64)."""
    import torch
    rows = A.shape[0] if rows is None else rows
    n = A.shape[1]
    l = X.shape[1]
    f64 = A.dtype == torch.float64
    dt = A.dtype
    lda = A.stride(0) if lda is None else lda
    Y = torch.empty(rows, l, device=X.device, dtype=dt) if Y is None else Y
    scr, nbytes = _scratch(rows, n, l, X.device, f64)
    fn = lib().brsvd_gemm_an_f64 if f64 else lib().brsvd_gemm_an
    _check(fn(A.data_ptr(), lda, rows, n, _dev(X, dt, "X"), l, _dev(Y, dt, "Y"), scr.data_ptr(), nbytes,
              _stream_ptr(stream)), "brsvd_gemm_an")
    return Y


def brsvd_gemm_at(A, Q, Z=None, accumulate=False, lda=None, stream=None):
    """Z (+)= A^T @ Q on the HIP path.  A (rows, n), Q (rows, l), Z (n, l); fp32 or fp64 by A's dtype."""
    import torch
    rows, n = A.shape
    l = Q.shape[1]
    f64 = A.dtype == torch.float64
    dt = A.dtype
    lda = A.stride(0) if lda is None else lda
    Z = torch.zeros(n, l, device=Q.device, dtype=dt) if Z is None else Z
    scr, nbytes = _scratch(rows, n, l, Q.device, f64)
    fn = lib().brsvd_gemm_at_f64 if f64 else lib().brsvd_gemm_at
    _check(fn(A.data_ptr(), lda, rows, n, _dev(Q, dt, "Q"), l, _dev(Z, dt, "Z"), 1 if accumulate else 0,
              scr.data_ptr(), nbytes, _stream_ptr(stream)), "brsvd_gemm_at")
    return Z


def _byte_scratch(nbytes, device):
    import torch
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def brsvd_orth(P, method=BRSVD_ORTH_AUTO, want_R=False, stream=None):
    """In-place orthonormalisation of the columns of P (rows, l).  Returns (P, R or None, fallback)."""
    import torch
    rows, l = P.shape
    R = torch.empty(l, l, dtype=torch.float64, device=P.device) if want_R else None
    fb = C.c_int32(0)
    nbytes = lib().brsvd_orth_scratch_bytes(rows, l)
    scr = _byte_scratch(nbytes, P.device)
    _check(lib().brsvd_orth(_dev(P, torch.float32, "P"), rows, l, method, R.data_ptr() if want_R else None,
                            C.byref(fb), scr.data_ptr(), nbytes, _stream_ptr(stream)), "brsvd_orth")
    return P, R, bool(fb.value)


def brsvd_small_svd(R, stream=None, out=None, static=False):
    """One-sided Jacobi SVD of an l x l fp64 CUDA matrix: returns (S, Ur, Vr, sweeps).  out = (S, Ur, Vr)
    reuses the caller's tensors; static=True calls brsvd_small_svd_static (scratch inside the library)."""
    import torch
    l = R.shape[0]
    if out is None:
        out = (torch.empty(l, dtype=torch.float64, device=R.device),
               torch.empty(l, l, dtype=torch.float64, device=R.device),
               torch.empty(l, l, dtype=torch.float64, device=R.device))
    S, Ur, Vr = out
    sw = C.c_int32(0)
    args = (_dev(R, torch.float64, "R"), l, _dev(S, torch.float64, "S"), _dev(Ur, torch.float64, "Ur"),
            _dev(Vr, torch.float64, "Vr"), C.byref(sw))
    if static:
        _check(lib().brsvd_small_svd_static(*args, _stream_ptr(stream)), "brsvd_small_svd_static")
    else:
        nbytes = lib().brsvd_small_svd_scratch_bytes(l)
        scr = _byte_scratch(nbytes, R.device)
        _check(lib().brsvd_small_svd(*args, scr.data_ptr(), nbytes, _stream_ptr(stream)), "brsvd_small_svd")
    return S, Ur, Vr, sw.value


def brsvd_small_svd_static(R, stream=None, out=None):
    return brsvd_small_svd(R, stream=stream, out=out, static=True)


# ---- a model's matrices: 8-bit products and losses over a large vocabulary -----------------------------------------
# Looking torch up in every one of a call's helpers takes longer than what they do: the first call leaves it here, and the number of
# devices that the process sees.
torch = None
_devices = 0

# Every call takes stream= (a torch stream of the operands' device or its address; default: torch's current stream there), on which it
# runs and allocates; operands have to stay until that stream has passed the call, and out= must not overlap them.  Results carry no
# autograd graph, whatever an operand's requires_grad says: gradients are what the *_backward calls return.

def _model_dtype(dtype, name, half=False):
    if dtype is torch.bfloat16:
        return BRSVD_DTYPE_BF16
    if dtype is torch.float16:
        return BRSVD_DTYPE_F16
    if dtype is torch.float32 and not half:
        return BRSVD_DTYPE_F32
    raise TypeError(f"{name} must be of dtype torch.bfloat16, torch.float16{'' if half else ' or torch.float32'}, not {dtype}")


def _rows(t, dtype, cols, name, rows=None):
    """(address, leading dimension) of a CUDA matrix with neighbouring elements in a row; cols, rows: None where any number will do."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is dtype and t.dim() == 2):
        raise TypeError(f"{name} must be a 2-d CUDA tensor of dtype {dtype}")
    r, c = t.shape
    if (cols is not None and c != cols) or (rows is not None and r != rows):
        raise TypeError(f"{name} has shape {(r, c)}, expected {tuple('any' if s is None else s for s in (rows, cols))}")
    ld, step = t.stride()
    if r <= 1 or not c:
        ld = -(-c // 16) * 16 or 1        # of one row any pitch is right, and whole 16 bytes are read fastest
    elif ld < c:
        raise TypeError(f"{name} must have rows that do not overlap")
    if step != 1 and c > 1 and r:
        raise TypeError(f"{name} must have unit column stride")
    return t.data_ptr(), ld


def _device_of(operands):
    """Index of the one CUDA device that the tensors among the operands lie on, -1 where none does."""
    index = -1
    for t in operands:
        if isinstance(t, torch.Tensor):
            at = t.get_device()
        elif isinstance(t, (list, tuple)):
            try:
                found = set(map(operator.methodcaller("get_device"), t))      # lists are long
                at = found.pop() if len(found) == 1 else _device_of(t)
            except AttributeError:
                at = _device_of(t)
        else:
            continue
        if at >= 0 and at != index:
            if index >= 0:
                raise TypeError(f"the operands must be on one device, not on cuda:{index} and cuda:{at}")
            index = at
    return index


def _scope(stream, index):
    """Memory taken inside belongs to the stream that the call runs on: what a call frees at its end, or the caller later, is not handed out
    to work of another stream before the call is through with it."""
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream) if stream else torch.cuda.default_stream()
    elif index >= 0 and stream.device_index != index:
        raise ValueError(f"stream belongs to cuda:{stream.device_index}, the operands are on cuda:{index}")
    return torch.cuda.stream(stream)


def _scoped(call):
    """Runs a binding with the device of its operands as the current one, to which launches go, and `stream` as torch's current stream."""
    import functools

    @functools.wraps(call)
    def wrapped(*args, stream=None, **kw):
        global torch, _devices
        if torch is None:
            import torch
            _devices = torch.cuda.device_count()
        index = -1
        if _devices > 1:                   # with one device there is nothing to tell apart
            index = _device_of((*args, *kw.values()))
            if index >= 0 and index != torch.cuda.current_device():
                with torch.cuda.device(index):
                    return wrapped(*args, stream=stream, **kw)
        if stream is None:
            return call(*args, **kw)
        with _scope(stream, index):
            return call(*args, **kw)
    return wrapped


def _current(device):
    """torch's current stream on a device, as an address (torch.cuda.current_stream() makes an object of it, at several times the cost)."""
    return torch._C._cuda_getCurrentRawStream(device.index) or None


def _scales(S, rows, cols, block_rows, name):
    shape = (rows if block_rows == 1 else -(-rows // 128), -(-cols // 128))
    if S.shape != shape:
        raise TypeError(f"{name} has shape {tuple(S.shape)}, expected {shape}")
    return _dev(S, torch.float32, name)


def _eight_bit(rows, cols, device):
    """rows x cols numbers of 8 bits in rows of whole 16 bytes, long ones of whole 128 (lines of the caches), which the products
    read fastest."""
    whole = 16 if cols < 1024 else 128
    return torch.empty_strided((rows, cols), (-(-cols // whole) * whole, 1), dtype=torch.float8_e4m3fn, device=device)


@_scoped
def brsvd_quantize_e4m3(X, block_rows=1, transpose=False):
    """X (rows, cols) CUDA, fp32, bf16 or fp16, as e4m3 numbers Q (float8_e4m3fn, rows 16- or 128-byte aligned) and power-of-two
    scales S, one for each 128 numbers of a row (block_rows=1) or each 128 x 128 block (block_rows=128).  Returns (Q, S), with
    transpose=True (Q, S, Qt, St), the last two those of X^T."""
    if block_rows not in (1, 128):
        raise ValueError("block_rows must be 1 or 128")
    dt = _model_dtype(X.dtype, "X")
    x, ldx = _rows(X, X.dtype, None, "X")
    rows, cols = X.shape
    dev = X.device

    def result(r, c):
        return _eight_bit(r, c, dev), torch.empty(r if block_rows == 1 else -(-r // 128), -(-c // 128), dtype=torch.float32, device=dev)
    Q, S = result(rows, cols)
    Qt, St = result(cols, rows) if transpose else (None, None)
    _check(lib().brsvd_quantize_e4m3(x, ldx, rows, cols, dt, block_rows, Q.data_ptr(), Q.stride(0), S.data_ptr(),
                                     Qt.data_ptr() if transpose else None, Qt.stride(0) if transpose else 0,
                                     St.data_ptr() if transpose else None, _current(X.device)), "brsvd_quantize_e4m3")
    return (Q, S, Qt, St) if transpose else (Q, S)


@_scoped
def brsvd_dequantize_e4m3(Q, S, block_rows=1, dtype=None):
    """What Q with its scales stands for, as fp32 (or bf16, fp16: dtype)."""
    if block_rows not in (1, 128):
        raise ValueError("block_rows must be 1 or 128")
    dtype = dtype or torch.float32
    dt = _model_dtype(dtype, "the result")
    q, ldq = _rows(Q, torch.float8_e4m3fn, None, "Q")
    rows, cols = Q.shape
    X = torch.empty(rows, cols, dtype=dtype, device=Q.device)
    _check(lib().brsvd_dequantize_e4m3(q, ldq, _scales(S, rows, cols, block_rows, "S"), rows, cols, block_rows, dt,
                                       X.data_ptr(), max(cols, 1), _current(Q.device)), "brsvd_dequantize_e4m3")
    return X


@_scoped
def brsvd_gemm_e4m3(A, SA, Bm, SB, block_rows=128, dtype=None, out=None):
    """A Bm^T of 8-bit matrices A (m, k) with a scale per row and 128 numbers and Bm (n, k) with one per 128 x 128 block, or
    with block_rows=1 like A's.  The result is bf16 unless dtype says fp32 or fp16; out: write it there."""
    if block_rows not in (1, 128):
        raise ValueError("block_rows must be 1 or 128")
    a, lda = _rows(A, torch.float8_e4m3fn, None, "A")
    m, k = A.shape
    b, ldb = _rows(Bm, torch.float8_e4m3fn, k, "Bm")
    n = Bm.shape[0]
    sa, sb = _scales(SA, m, k, 1, "SA"), _scales(SB, n, k, block_rows, "SB")
    dtype = dtype or (torch.bfloat16 if out is None else out.dtype)
    dt = _model_dtype(dtype, "the result")
    if out is None:
        Cm = torch.empty(m, n, dtype=dtype, device=A.device)
        c, ldc = Cm.data_ptr(), n or 1
    else:
        Cm = out
        c, ldc = _rows(Cm, dtype, n, "out", m)
    nbytes = lib().brsvd_gemm_e4m3_scratch_bytes(m, n, k, block_rows, dt)
    scr = _byte_scratch(nbytes, A.device) if nbytes else None
    _check(lib().brsvd_gemm_e4m3(a, lda, sa, b, ldb, sb, block_rows, m, n, k, dt, c, ldc,
                                 scr.data_ptr() if nbytes else None, nbytes, _current(A.device)), "brsvd_gemm_e4m3")
    return Cm


@_scoped
def brsvd_linear_e4m3(X, W, SW, out=None):
    """X W^T: X (m, k) fp32, bf16 or fp16 is cast into 8 bits by rows of 128 on the way, W (n, k) is in 8 bits with a scale
    for each 128 x 128 block.  The result has X's type."""
    dt = _model_dtype(X.dtype, "X")
    x, ldx = _rows(X, X.dtype, None, "X")
    m, k = X.shape
    w, ldw = _rows(W, torch.float8_e4m3fn, k, "W")
    n = W.shape[0]
    sw = _scales(SW, n, k, 128, "SW")
    if out is None:
        Y = torch.empty(m, n, dtype=X.dtype, device=X.device)
        y, ldy = Y.data_ptr(), n or 1
    else:
        Y = out
        y, ldy = _rows(Y, X.dtype, n, "out", m)
    nbytes = lib().brsvd_linear_e4m3_scratch_bytes(m, n, k, dt)
    scr = _byte_scratch(nbytes, X.device) if nbytes else None
    _check(lib().brsvd_linear_e4m3(x, ldx, dt, w, ldw, sw, m, n, k, y, ldy, scr.data_ptr() if nbytes else None, nbytes,
                                   _current(X.device)), "brsvd_linear_e4m3")
    return Y


def _four_bit(W, S, cols, name, scales):
    """Address and leading dimension of a matrix in 4 bits with `cols` numbers a row, and the address of its scales."""
    w, ldw = _rows(W, torch.float4_e2m1fn_x2, (cols + 1) // 2, name)
    shape = (W.shape[0], -(-cols // 32))
    if S.shape != shape:
        raise TypeError(f"{scales} has shape {tuple(S.shape)}, expected {shape}")
    return w, ldw, _dev(S, torch.float8_e8m0fnu, scales)


def _columns(Q, cols):
    """Numbers of a row: two for each byte, or one less where cols says so."""
    if cols is None:
        return 2 * Q.shape[1]
    if not isinstance(cols, int) or (cols + 1) // 2 != Q.shape[1]:
        raise ValueError(f"cols must be {max(2 * Q.shape[1] - 1, 0)} or {2 * Q.shape[1]} for rows of {Q.shape[1]} bytes, not {cols}")
    return cols


@_scoped
def brsvd_quantize_e2m1(X):
    """X (rows, cols) CUDA, fp32, bf16 or fp16, as e2m1 numbers Q (float4_e2m1fn_x2, (rows, ceil(cols/2)): two in a byte, the first in its
    lower half; rows 16- or 128-byte aligned) and power-of-two scales S (float8_e8m0fnu), one for each 32 numbers of a row.  A group with an
    infinity or a NaN becomes NaN; finite numbers from 3.5 * 2^126 on stand for 2^128 and come back infinite.  Returns (Q, S)."""
    dt = _model_dtype(X.dtype, "X")
    x, ldx = _rows(X, X.dtype, None, "X")
    rows, cols = X.shape
    width = (cols + 1) // 2
    whole = 16 if width < 1024 else 128
    Q = torch.empty_strided((rows, width), (-(-width // whole) * whole, 1), dtype=torch.float4_e2m1fn_x2, device=X.device)
    S = torch.empty(rows, -(-cols // 32), dtype=torch.float8_e8m0fnu, device=X.device)
    _check(lib().brsvd_quantize_e2m1(x, ldx, rows, cols, dt, Q.data_ptr(), Q.stride(0), S.data_ptr(), _current(X.device)), "brsvd_quantize_e2m1")
    return Q, S


@_scoped
def brsvd_dequantize_e2m1(Q, S, cols=None, dtype=None):
    """What Q with its scales stands for, as fp32 (or bf16, fp16: dtype).  cols: numbers of a row where they are odd."""
    dtype = dtype or torch.float32
    dt = _model_dtype(dtype, "the result")
    cols = _columns(Q, cols)
    q, ldq, s = _four_bit(Q, S, cols, "Q", "S")
    X = torch.empty(Q.shape[0], cols, dtype=dtype, device=Q.device)
    _check(lib().brsvd_dequantize_e2m1(q, ldq, s, Q.shape[0], cols, dt, X.data_ptr(), max(cols, 1), _current(Q.device)), "brsvd_dequantize_e2m1")
    return X


def _linear_e2m1(name, X, x_name, W, SW, k, backward, out):
    dt = _model_dtype(X.dtype, x_name, half=True)
    w, ldw, sw = _four_bit(W, SW, k, "W", "SW")
    n = W.shape[0]
    x, ldx = _rows(X, X.dtype, n if backward else k, x_name)
    m, width = X.shape[0], k if backward else n
    if out is None:
        Y = torch.empty(m, width, dtype=X.dtype, device=X.device)
        y, ldy = Y.data_ptr(), width or 1
    else:
        Y = out
        y, ldy = _rows(Y, X.dtype, width, "out", m)
    L = lib()
    # up to 16 rows of X take none
    nbytes = L.brsvd_linear_e2m1_scratch_bytes(m, n, k, not ((x | w | ldw) & 15 or ldx & 7), backward) if m > 16 or backward else 0
    scr = _byte_scratch(nbytes, X.device) if nbytes else None
    _check((L.brsvd_linear_e2m1_backward if backward else L.brsvd_linear_e2m1)(x, ldx, dt, w, ldw, sw, m, n, k, y, ldy, scr.data_ptr() if nbytes else None, nbytes, _current(X.device)), name)
    return Y


@_scoped
def brsvd_linear_e2m1(X, W, SW, out=None):
    """X W^T: X (m, k) bf16 or fp16, W (n, k) in 4 bits with a scale for each 32 numbers of a row (brsvd_quantize_e2m1).  The result has X's type."""
    return _linear_e2m1("brsvd_linear_e2m1", X, "X", W, SW, X.shape[1] if X.dim() == 2 else 0, 0, out)


@_scoped
def brsvd_linear_e2m1_backward(dY, W, SW, cols=None, out=None):
    """The gradient dY W of brsvd_linear_e2m1's X from dY (m, n), the gradient of its result.  cols: numbers of a row of W where they are odd."""
    return _linear_e2m1("brsvd_linear_e2m1_backward", dY, "dY", W, SW, _columns(W, cols), 1, out)


_ACTIVATIONS = {"silu": BRSVD_ACT_SILU, "gelu": BRSVD_ACT_GELU, "gelu_tanh": BRSVD_ACT_GELU_TANH}


def _glu(X, Wg, Wu, act):
    dt = _model_dtype(X.dtype, "X", half=True)
    if act not in _ACTIVATIONS:
        raise ValueError(f"act must be one of {', '.join(_ACTIVATIONS)}, not {act!r}")
    x, ldx = _rows(X, X.dtype, None, "X")
    wg, ldwg = _rows(Wg, X.dtype, X.shape[1], "Wg")
    wu, ldwu = _rows(Wu, X.dtype, X.shape[1], "Wu", Wg.shape[0])
    sizes = (X.shape[0], X.shape[1], Wg.shape[0])
    aligned = ldwg == ldwu and not ((x | wg | wu) & 15 or (ldx | ldwg | ldwu) & 7)
    return (x, ldx, wg, ldwg, wu, ldwu), sizes, dt, _ACTIVATIONS[act], aligned


def _glu_workspace(sizes, aligned, backward, device):
    nbytes = lib().brsvd_glu_workspace_bytes(*sizes, aligned, backward)
    if not nbytes:
        return None, None, 0
    ws = _byte_scratch(nbytes, device)
    return ws, ws.data_ptr(), nbytes


@_scoped
def brsvd_glu_forward(X, Wg, Wu, act="silu", keep=False):
    """H = a(X Wg^T) * (X Wu^T), the first half of a gated feed-forward block: X (tokens, dim), Wg and Wu (width, dim; they may be halves of
    one matrix), bf16 or fp16.  act: silu, gelu or gelu_tanh.  keep=True returns (H, G, U) with G = X Wg^T and U = X Wu^T, which
    brsvd_glu_backward wants.  No autograd graph."""
    ops, (tokens, dim, width), dt, a, aligned = _glu(X, Wg, Wu, act)
    n = 3 if keep else 1
    outs = [torch.empty(tokens, width, dtype=X.dtype, device=X.device) for _ in range(n)]
    ld = width or 1
    at = [t.data_ptr() for t in outs] + [None] * (3 - n)
    ws, w, nbytes = _glu_workspace((tokens, dim, width), aligned, 0, X.device)
    _check(lib().brsvd_glu_forward(*ops, tokens, dim, width, dt, a, at[0], ld, at[1], ld, at[2], ld, w, nbytes, _current(X.device)),
           "brsvd_glu_forward")
    return tuple(outs) if keep else outs[0]


@_scoped
def brsvd_glu_backward(X, Wg, Wu, G, U, dH, act="silu", need_dX=True, need_dW=True):
    """Gradients (dX, dWg, dWu) from dH, the gradient of H, and the G and U that the forward call kept; None for those that are not needed.
    dWg and dWu are halves of one (2 width, dim) matrix."""
    ops, (tokens, dim, width), dt, a, aligned = _glu(X, Wg, Wu, act)
    kept = sum((_rows(t, X.dtype, width, name, tokens) for t, name in ((G, "G"), (U, "U"), (dH, "dH"))), ())
    if not (need_dX or need_dW):
        raise ValueError("neither gradient is wanted")
    dX = torch.empty(tokens, dim, dtype=X.dtype, device=X.device) if need_dX else None
    dWg, dWu = torch.empty(2, width, dim, dtype=X.dtype, device=X.device).unbind(0) if need_dW else (None, None)
    d = dim or 1
    ws, w, nbytes = _glu_workspace((tokens, dim, width), aligned, 1, X.device)
    at = [None if t is None else t.data_ptr() for t in (dX, dWg, dWu)]
    _check(lib().brsvd_glu_backward(*ops, *kept, tokens, dim, width, dt, a, at[0], d, at[1], d, at[2], d, w, nbytes, _current(X.device)),
           "brsvd_glu_backward")
    return dX, dWg, dWu


_tables = None


def _tensors(*lists):
    """A list of tensors as an array of brsvd_tensor; two lists, whose numbers have to be in the same order, as two."""
    global _tables
    if _tables is None:
        import torch

        from . import _lists               # needs torch
        if _lists.torch_version != torch.__version__:
            raise ImportError(f"_lists.so was built for torch {_lists.torch_version}, this is {torch.__version__}: python -m paper_1706_07191_amd.build")
        _tables = _lists.tables
    return _tables(*lists)


@_scoped
def brsvd_grad_norm(tensors, scale=1.0):
    """|scale| times the 2-norm over all numbers of a list of CUDA tensors (fp32, bf16 or fp16, mixed; dense or matrices with strided rows), as a
    tensor of one fp32 number.  Sums are fp64.  scale: what the gradients are to be multiplied by, such as one over a loss's factor."""
    table, = _tensors(tensors)
    count = len(tensors)
    device = tensors[0].device if count else torch.device("cuda", torch.cuda.current_device())
    norm = torch.empty(1, dtype=torch.float32, device=device)
    nbytes = lib().brsvd_grad_norm_workspace_bytes(table, count)
    ws = _byte_scratch(nbytes, device)
    _check(lib().brsvd_grad_norm(table, count, scale, norm.data_ptr(), ws.data_ptr(), nbytes, _current(device)), "brsvd_grad_norm")
    return norm


@_scoped
def brsvd_grad_clip(tensors, norm, max_norm, scale=1.0, out=None):
    """Multiplies every tensor of a list by scale min(1, max_norm / norm), norm being that of brsvd_grad_norm with the same scale (one fp32 number on
    the device).  out: tensors of the same shapes, of any of the three types, that the results are written to instead of the tensors
    themselves.  A norm that is infinite or NaN clips nothing.  Results that share memory with each other, with another
    tensor or with norm are refused.  Returns the tensors written."""
    if not isinstance(norm, torch.Tensor) or norm.numel() != 1:
        raise TypeError("norm must be a CUDA tensor of one fp32 number")
    n = _dev(norm, torch.float32, "norm")
    tables = _tensors(tensors) if out is None or out is tensors else _tensors(tensors, out)
    _check(lib().brsvd_grad_clip(tables[0], tables[-1], len(tensors), scale, max_norm, n, _current(norm.device)), "brsvd_grad_clip")
    return tensors if out is None else out


def _head(H, W):
    dt = _model_dtype(H.dtype, "H", half=True)
    h, ldh = _rows(H, H.dtype, None, "H")
    w, ldw = _rows(W, H.dtype, H.shape[1], "W")
    return (h, ldh, w, ldw), (H.shape[0], W.shape[0], H.shape[1]), dt


def _vector(t, dtype, n, name):
    if t.shape != (n,):
        raise TypeError(f"{name} has shape {tuple(t.shape)}, expected {(n,)}")
    return _dev(t, dtype, name)


def _factors(grad, tokens):
    """(tensor, address, stride) of a factor for each token: a number, a tensor with one for all (also expanded) or one for each."""
    if not isinstance(grad, torch.Tensor):
        raise TypeError("grad must be a CUDA tensor of dtype torch.float32")
    if grad.dtype != torch.float32 or not grad.is_cuda:
        raise TypeError("grad must be a CUDA tensor of dtype torch.float32")
    if grad.numel() != 1 and tuple(grad.shape) != (tokens,):
        raise TypeError(f"grad has shape {tuple(grad.shape)}, expected one number or {(tokens,)}")
    if grad.numel() == 1:
        return grad, grad.data_ptr(), 0
    if grad.stride(0) < 0:
        grad = grad.contiguous()
    return grad, grad.data_ptr(), grad.stride(0)


def _head_workspace(sizes, piece, top, backward, device):
    nbytes = lib().brsvd_head_workspace_bytes(*sizes, piece, top, backward)
    return _byte_scratch(nbytes, device), nbytes


@_scoped
def brsvd_xent_forward(H, W, labels):
    """Softmax cross entropy of the logits H W^T (H (tokens, dim), W (vocab, dim), bf16 or fp16) per token, without the
    logits: returns (loss, lse), fp32.  labels: int64, one outside [0, vocab) marks a token that does not count (loss 0).
    No autograd graph: brsvd_xent_backward gives the gradients."""
    ops, sizes, dt = _head(H, W)
    y = _vector(labels, torch.int64, sizes[0], "labels")
    loss, lse = torch.empty(2, sizes[0], dtype=torch.float32, device=H.device).unbind(0)
    ws, nbytes = _head_workspace(sizes, 0, 0, 0, H.device)
    _check(lib().brsvd_xent_forward(*ops, y, *sizes, dt, loss.data_ptr(), lse.data_ptr(), ws.data_ptr(), nbytes,
                                    _current(H.device)), "brsvd_xent_forward")
    return loss, lse


def _gradients(H, W, need_dH, need_dW):
    if not (need_dH or need_dW):
        raise ValueError("neither gradient is wanted")
    dH = torch.empty(H.shape, dtype=H.dtype, device=H.device) if need_dH else None
    dW = torch.empty(W.shape, dtype=W.dtype, device=W.device) if need_dW else None
    d = max(H.shape[1], 1)
    return dH, dW, (dH.data_ptr() if need_dH else None, d, dW.data_ptr() if need_dW else None, d)


@_scoped
def brsvd_xent_backward(H, W, labels, lse, grad, need_dH=True, need_dW=True, piece=0):
    """Gradients (dH, dW) of sum_t grad_t loss_t, from the lse of the forward call; None for one that is not needed.  grad:
    fp32 tensor with a factor for each token or one for all.  piece: rows of W taken at a time (0: by the memory they need)."""
    ops, sizes, dt = _head(H, W)
    y, l = _vector(labels, torch.int64, sizes[0], "labels"), _vector(lse, torch.float32, sizes[0], "lse")
    keep, g, stride = _factors(grad, sizes[0])
    dH, dW, outs = _gradients(H, W, need_dH, need_dW)
    ws, nbytes = _head_workspace(sizes, piece, 0, 1, H.device)
    _check(lib().brsvd_xent_backward(*ops, y, l, g, stride, *sizes, piece, dt, *outs, ws.data_ptr(), nbytes,
                                     _current(H.device)), "brsvd_xent_backward")
    return dH, dW


def _teacher(ids, logits, tokens):
    if ids.dim() != 2 or ids.shape[0] != tokens or ids.shape[1] < 1 or ids.shape != logits.shape:
        raise TypeError(f"ids and logits must have shape (tokens, top), not {tuple(ids.shape)} and {tuple(logits.shape)}")
    return (_dev(ids, torch.int64, "ids"), _dev(logits, torch.float32, "logits"), ids.shape[1])


@_scoped
def brsvd_distill_forward(H, W, ids, logits, temperature=1.0):
    """tau^2 KL(q || p) per token of the student's p = softmax(H W^T / tau) against the teacher's q, the softmax of its `top`
    kept logits / tau: ids int64, logits fp32, both (tokens, top); an entry with an id outside [0, vocab) or a logit of -inf
    does not count.  Returns (loss, lse, z), fp32: z (tokens, top) holds the student's logits of those words.  No autograd
    graph: brsvd_distill_backward gives the gradients."""
    ops, sizes, dt = _head(H, W)
    te = _teacher(ids, logits, sizes[0])
    loss, lse = torch.empty(2, sizes[0], dtype=torch.float32, device=H.device).unbind(0)
    z = torch.empty(ids.shape, dtype=torch.float32, device=H.device)
    ws, nbytes = _head_workspace(sizes, 0, te[2], 0, H.device)
    _check(lib().brsvd_distill_forward(*ops, *te, temperature, *sizes, dt, loss.data_ptr(), lse.data_ptr(), z.data_ptr(),
                                       ws.data_ptr(), nbytes, _current(H.device)), "brsvd_distill_forward")
    return loss, lse, z


@_scoped
def brsvd_distill_backward(H, W, ids, logits, temperature, lse, z, grad, need_dH=True, need_dW=True, piece=0):
    """Gradients (dH, dW) of sum_t grad_t loss_t from the lse and z of the forward call; the rest as brsvd_xent_backward."""
    ops, sizes, dt = _head(H, W)
    te = _teacher(ids, logits, sizes[0])
    l = _vector(lse, torch.float32, sizes[0], "lse")
    if z.shape != ids.shape:
        raise TypeError(f"z has shape {tuple(z.shape)}, expected {tuple(ids.shape)}")
    keep, g, stride = _factors(grad, sizes[0])
    dH, dW, outs = _gradients(H, W, need_dH, need_dW)
    ws, nbytes = _head_workspace(sizes, piece, te[2], 1, H.device)
    _check(lib().brsvd_distill_backward(*ops, *te, temperature, l, _dev(z, torch.float32, "z"), g, stride, *sizes, piece, dt,
                                        *outs, ws.data_ptr(), nbytes, _current(H.device)), "brsvd_distill_backward")
    return dH, dW


class PinnedMatrix:
    """rows x cols fp32 matrix in pinned host memory obtained with one hipHostMalloc of the exact size
    (torch's pinned allocator rounds requests up to a power of two, which fails for very large A).
    `.tensor` is a torch view of the memory; call `.free()` when done."""

    def __init__(self, rows: int, cols: int):
        import numpy as np
        import torch
        self._hip = C.CDLL("libamdhip64.so")
        self._hip.hipHostMalloc.argtypes = [C.POINTER(C.c_void_p), C.c_size_t, C.c_uint]
        self._hip.hipHostFree.argtypes = [C.c_void_p]
        ptr = C.c_void_p()
        err = self._hip.hipHostMalloc(C.byref(ptr), rows * cols * 4, 0)
        if err != 0 or not ptr.value:
            self._hip.hipGetLastError()          # the failure is reported here; do not leave it for the next HIP call
            raise MemoryError(f"hipHostMalloc of {rows * cols * 4} bytes failed (hip error {err})")
        self.ptr = ptr.value
        buf = (C.c_float * (rows * cols)).from_address(self.ptr)
        self.tensor = torch.from_numpy(np.ctypeslib.as_array(buf)).view(rows, cols)

    def free(self):
        if self.ptr:
            self.tensor = None
            self._hip.hipHostFree(C.c_void_p(self.ptr))
            self.ptr = None
