"""MI355X (gfx950) fused SDDMM->SpMM: Python binding of libsparselnr.so.

The binding only marshals arguments: it checks tensor devices, dtypes and
shapes, passes raw device pointers and the stream to the C ABI declared in
include/sparselnr.h, and raises on a non-zero status.  Every step of the
computation runs in the library's HIP kernels; there is no fallback.

    A = sparselnr_fused_sddmm_spmm(rowptr, colidx, vals, C, D, E)

computes A(i,l) = sum_{j,k} B(i,j) C(i,k) D(j,k) E(j,l) for B in CSR form
(rowptr int32[N+1], colidx int32[nnz], vals float32[nnz]) and dense
row-major float32 C (N x K), D (M x K), E (M x L).

The calls of the paged cache (bf16, fp16 or fp32) serve a language model's
attention, one step of a batch of requests after the other:

    qptr, seq, slots, counts = sparselnr_page_tables(ctx, new, table, free, T, P)
    sparselnr_cache_append(k, v, slots, kcache, vcache, kq, kscale)
    out = sparselnr_paged_attention(q, kcache, vcache, table, seq, qptr)

or, over the pages that a cheap score selects for each token and KV head,

    sel = sparselnr_block_select(q, kq, kscale, table, seq, qptr, P, top)
    out = sparselnr_block_attention(q, kcache, vcache, table, seq, qptr, sel)
"""
from __future__ import annotations

import ctypes
import os

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libsparselnr.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_HIP, ERR_NO_MEMORY, ERR_INVALID_CSR = range(6)

__all__ = [
    "sparselnr_fused_sddmm_spmm", "sparselnr_fused_sddmm_spmm_noalloc",
    "sparselnr_unfused_sddmm_spmm", "sparselnr_sddmm",
    "sparselnr_spmm", "sparselnr_fused_sddmm_spmm_gemm", "sparselnr_spmm_gemm",
    "sparselnr_spmmh_gemm", "sparselnr_fused_sddmm_spmm_dt", "sparselnr_validate_csr", "sparselnr_release", "sparselnr_status_string",
    "sparselnr_last_hip_error", "sparselnr_abi_version", "sparselnr_set_grid_factor",
    "sparselnr_get_grid_factor", "sparselnr_page_tables", "sparselnr_cache_append",
    "sparselnr_paged_attention", "sparselnr_block_select", "sparselnr_block_attention",
    "SparseLNRError", "lib", "LIB_PATH",
]


class SparseLNRError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib().sparselnr_status_string(status).decode()
        if status == ERR_HIP:
            msg += " (hipError_t %d)" % lib().sparselnr_last_hip_error()
        super().__init__("%s: %s [status %d]" % (where, msg, status))


class _KvCache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p)] + [
        (n, ctypes.c_int64) for n in ("pages", "page_size", "heads", "dim", "k_page", "k_slot", "k_head",
                                      "v_page", "v_slot", "v_head")] + [("dtype", ctypes.c_int32)]


class _Requests(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("table_stride", ctypes.c_int64), ("seq_len", ctypes.c_void_p),
                ("qptr", ctypes.c_void_p), ("R", ctypes.c_int64), ("W", ctypes.c_int64), ("T", ctypes.c_int64)]


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded C library (built in place by __graft_entry__.build())."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError("libsparselnr.so is not built (%s); run `python -c "
                              "'import __graft_entry__ as g; g.build()'`" % LIB_PATH)
        L = ctypes.CDLL(LIB_PATH)
        vp, i64, ci = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int
        L.sparselnr_fused_sddmm_spmm.argtypes = [vp] * 7 + [i64] * 4 + [vp]
        L.sparselnr_fused_sddmm_spmm.restype = ci
        L.sparselnr_fused_sddmm_spmm_noalloc.argtypes = [vp] * 7 + [i64] * 4 + [vp]
        L.sparselnr_fused_sddmm_spmm_noalloc.restype = ci
        L.sparselnr_unfused_sddmm_spmm.argtypes = [vp] * 8 + [i64] * 4 + [vp]
        L.sparselnr_unfused_sddmm_spmm.restype = ci
        L.sparselnr_sddmm.argtypes = [vp] * 6 + [i64] * 3 + [vp]
        L.sparselnr_sddmm.restype = ci
        L.sparselnr_spmm.argtypes = [vp] * 5 + [i64] * 3 + [vp]
        L.sparselnr_spmm.restype = ci
        L.sparselnr_fused_sddmm_spmm_gemm.argtypes = [vp] * 8 + [i64] * 5 + [vp]
        L.sparselnr_fused_sddmm_spmm_gemm.restype = ci
        L.sparselnr_spmm_gemm.argtypes = [vp] * 6 + [i64] * 4 + [vp]
        L.sparselnr_spmm_gemm.restype = ci
        L.sparselnr_spmmh_gemm.argtypes = [vp] * 7 + [i64] * 4 + [vp]
        L.sparselnr_spmmh_gemm.restype = ci
        L.sparselnr_fused_sddmm_spmm_dt.argtypes = [vp] * 7 + [i64] * 4 + [vp]
        L.sparselnr_fused_sddmm_spmm_dt.restype = ci
        L.sparselnr_validate_csr.argtypes = [vp, vp, i64, i64, i64, ctypes.POINTER(i64), vp]
        L.sparselnr_validate_csr.restype = ci
        L.sparselnr_status_string.argtypes = [ci]
        L.sparselnr_status_string.restype = ctypes.c_char_p
        L.sparselnr_last_hip_error.argtypes = []
        L.sparselnr_last_hip_error.restype = ci
        L.sparselnr_release.argtypes = []
        L.sparselnr_release.restype = ci
        L.sparselnr_abi_version.argtypes = []
        L.sparselnr_abi_version.restype = ci
        L.sparselnr_set_grid_factor.argtypes = [ci]
        L.sparselnr_set_grid_factor.restype = ci
        L.sparselnr_get_grid_factor.argtypes = []
        L.sparselnr_get_grid_factor.restype = ci
        i32, cache, requests = ctypes.c_int32, ctypes.POINTER(_KvCache), ctypes.POINTER(_Requests)
        L.sparselnr_page_tables.argtypes = [vp, vp, vp, i64] + [vp] * 5 + [i64] * 5 + [vp]
        L.sparselnr_page_tables.restype = ci
        L.sparselnr_cache_append.argtypes = [vp, i64, i64, vp, i64, i64, vp, cache, vp, vp, i64, vp]
        L.sparselnr_cache_append.restype = ci
        L.sparselnr_paged_attention.argtypes = [vp, i64, i64, i64, cache, requests, ctypes.c_double,
                                                i64, i64, vp, vp, vp]
        L.sparselnr_paged_attention.restype = ci
        L.sparselnr_block_select.argtypes = [vp, i64, i64, i64, i32, vp, vp, i64, i64, i64, i64, requests,
                                             i64, i64, i64, vp, vp]
        L.sparselnr_block_select.restype = ci
        L.sparselnr_block_attention.argtypes = [vp, i64, i64, i64, cache, requests, vp, i64,
                                                ctypes.c_double, vp, vp, vp]
        L.sparselnr_block_attention.restype = ci
        _lib = L
    return _lib


def sparselnr_abi_version() -> int:
    return int(lib().sparselnr_abi_version())


def sparselnr_status_string(status: int) -> str:
    return lib().sparselnr_status_string(status).decode()


def sparselnr_last_hip_error() -> int:
    return int(lib().sparselnr_last_hip_error())


def sparselnr_set_grid_factor(factor: int) -> None:
    """Resident grids per walk launch: 0 automatic, 1..64 fixed (process-wide)."""
    rc = lib().sparselnr_set_grid_factor(int(factor))
    if rc != OK:
        raise SparseLNRError(rc, "sparselnr_set_grid_factor")


def sparselnr_get_grid_factor() -> int:
    return int(lib().sparselnr_get_grid_factor())


def sparselnr_release() -> None:
    rc = lib().sparselnr_release()
    if rc != OK:
        raise SparseLNRError(rc, "sparselnr_release")


# ------------------------------------------------------------ marshalling

def _torch():
    import torch
    return torch


def _check(t, name, dtype, device, ndim=None):
    torch = _torch()
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if t.device != device:
        raise ValueError("%s is on %s, expected %s" % (name, t.device, device))
    if t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if ndim is not None and t.dim() != ndim:
        raise ValueError("%s must have %d dimensions" % (name, ndim))


_dummy = {}


def _ptr(t, device):
    """Device address of t; a 16-byte dummy allocation when t is empty, so that
    the library never sees NULL for an empty array."""
    if t.numel() > 0:
        return t.data_ptr()
    torch = _torch()
    d = _dummy.get(device)
    if d is None:
        d = _dummy[device] = torch.zeros(4, dtype=torch.float32, device=device)
    return d.data_ptr()


def _stream(stream, device):
    if stream is None:
        return _torch().cuda.current_stream(device).cuda_stream
    return getattr(stream, "cuda_stream", stream)


def _csr(rowptr, colidx, vals, vals_name="vals"):
    torch = _torch()
    device = rowptr.device
    if device.type != "cuda":
        raise ValueError("inputs must be on a GPU device")
    _check(rowptr, "rowptr", torch.int32, device, 1)
    _check(colidx, "colidx", torch.int32, device, 1)
    _check(vals, vals_name, torch.float32, device, 1)
    if rowptr.numel() < 1:
        raise ValueError("rowptr needs N+1 >= 1 entries")
    if colidx.numel() != vals.numel():
        raise ValueError("colidx and %s differ in length" % vals_name)
    return device, rowptr.numel() - 1


def _dense(t, name, rows, device):
    torch = _torch()
    _check(t, name, torch.float32, device, 2)
    if t.shape[0] != rows:
        raise ValueError("%s has %d rows, expected %d" % (name, t.shape[0], rows))
    return t.shape[1]


def sparselnr_fused_sddmm_spmm(rowptr, colidx, vals, C, D, E, A=None, stream=None):
    """Fused SDDMM->SpMM (the paper's Figure 2d schedule).  Returns A (N x L).

    A, if given, is overwritten.  Asynchronous on `stream` (default: the
    current torch stream of the inputs' device)."""
    torch = _torch()
    device, N = _csr(rowptr, colidx, vals)
    K = _dense(C, "C", N, device)
    M = D.shape[0] if isinstance(D, torch.Tensor) and D.dim() == 2 else -1
    if _dense(D, "D", M, device) != K:
        raise ValueError("C and D differ in width K")
    L = _dense(E, "E", M, device)
    if A is None:
        A = torch.empty((N, L), dtype=torch.float32, device=device)
    elif _dense(A, "A", N, device) != L:
        raise ValueError("A must be N x L")
    rc = lib().sparselnr_fused_sddmm_spmm(
        _ptr(rowptr, device), _ptr(colidx, device), _ptr(vals, device), _ptr(C, device),
        _ptr(D, device), _ptr(E, device), _ptr(A, device), N, M, K, L, _stream(stream, device))
    if rc != OK:
        raise SparseLNRError(rc, "sparselnr_fused_sddmm_spmm")
    return A


def sparselnr_fused_sddmm_spmm_noalloc(rowptr, colidx, vals, C, D, E, A, stream=None):
    """The fused call for callers that cannot allocate: A (N x L) must be
    given; the library uses a fixed device array for split rows.  Calls that
    overlap on one GPU race (see include/sparselnr.h)."""
    torch = _torch()
    device, N = _csr(rowptr, colidx, vals)
    K = _dense(C, "C", N, device)
    M = D.shape[0] if isinstance(D, torch.Tensor) and D.dim() == 2 else -1
    if _dense(D, "D", M, device) != K:
        raise ValueError("C and D differ in width K")
    L = _dense(E, "E", M, device)
    if A is None or _dense(A, "A", N, device) != L:
        raise ValueError("A must be given, N x L")
    rc = lib().sparselnr_fused_sddmm_spmm_noalloc(
        _ptr(rowptr, device), _ptr(colidx, device), _ptr(vals, device), _ptr(C, device),
        _ptr(D, device), _ptr(E, device), _ptr(A, device), N, M, K, L, _stream(stream, device))
    if rc != OK:
        raise SparseLNRError(rc, "sparselnr_fused_sddmm_spmm_noalloc")
    return A


def sparselnr_sddmm(rowptr, colidx, vals, C, D, Y=None, stream=None):
    """SDDMM (Figure 2a): Y[p] = vals[p] * dot(C[i], D[colidx[p]]).  Returns Y."""
    torch = _torch()
    device, N = _csr(rowptr, colidx, vals)
    K = _dense(C, "C", N, device)
    M = D.shape[0] if isinstance(D, torch.Tensor) and D.dim() == 2 else -1
    if _dense(D, "D", M, device) != K:
        raise ValueError("C and D differ in width K")
    if Y is None:
        Y = torch.empty(colidx.numel(), dtype=torch.float32, device=device)
    else:
        _check(Y, "Y", torch.float32, device, 1)
        if Y.numel() != colidx.numel():
            raise ValueError("Y must have nnz entries")
    rc = lib().sparselnr_sddmm(_ptr(rowptr, device), _ptr(colidx, device), _ptr(vals, device),
                               _ptr(C, device), _ptr(D, device), _ptr(Y, device), N, M, K,
                               _stream(stream, device))
    if rc != OK:
        raise SparseLNRError(rc, "sparselnr_sddmm")
    return Y


def sparselnr_spmm(rowptr, colidx, Y, E, A=None, stream=None):
    """SpMM (Figure 2b): A[i] = sum_p Y[p] * E[colidx[p]].  Returns A."""
    torch = _torch()
    device, N = _csr(rowptr, colidx, Y, "Y")
    M = E.shape[0] if isinstance(E, torch.Tensor) and E.dim() == 2 else -1
    L = _dense(E, "E", M, device)
    if A is None:
        A = torch.empty((N, L), dtype=torch.float32, device=device)
    elif _dense(A, "A", N, device) != L:
        raise ValueError("A must be N x L")
    rc = lib().sparselnr_spmm(_ptr(rowptr, device), _ptr(colidx, device), _ptr(Y, device),
                              _ptr(E, device), _ptr(A, device), N, M, L, _stream(stream, device))
    if rc != OK:
        raise SparseLNRError(rc, "sparselnr_spmm")
    return A


def sparselnr_unfused_sddmm_spmm(rowptr, colidx, vals, C, D, E, Y=None, A=None, stream=None):
    """Unfused comparison (Figure 2a then 2b) through an nnz-sized Y.  Returns (Y, A)."""
    torch = _torch()
    device, N = _csr(rowptr, colidx, vals)
    K = _dense(C, "C", N, device)
    M = D.shape[0] if isinstance(D, torch.Tensor) and D.dim() == 2 else -1
    if _dense(D, "D", M, device) != K:
        raise ValueError("C and D differ in width K")
    L = _dense(E, "E", M, device)
    if Y is None:
        Y = torch.empty(colidx.numel(), dtype=torch.float32, device=device)
    else:
        _check(Y, "Y", torch.float32, device, 1)
        if Y.numel() != colidx.numel():
            raise ValueError("Y must have nnz entries")
    if A is None:
        A = torch.empty((N, L), dtype=torch.float32, device=device)
    elif _dense(A, "A", N, device) != L:
        raise ValueError("A must be N x L")
    rc = lib().sparselnr_unfused_sddmm_spmm(
        _ptr(rowptr, device), _ptr(colidx, device), _ptr(vals, device), _ptr(C, device),
        _ptr(D, device), _ptr(E, device), _ptr(Y, device), _ptr(A, device), N, M, K, L,
        _stream(stream, device))
    if rc != OK:
        raise SparseLNRError(rc, "sparselnr_unfused_sddmm_spmm")
    return Y, A


def _out(A, rows, cols, device, name="A"):
    torch = _torch()
    if A is None:
        return torch.empty((rows, cols), dtype=torch.float32, device=device)
    if _dense(A, name, rows, device) != cols:
        raise ValueError("%s must be %d x %d" % (name, rows, cols))
    return A


def sparselnr_fused_sddmm_spmm_gemm(rowptr, colidx, vals, C, D, F, W, A=None, stream=None):
    """<SDDMM, SpMM, GEMM>: A = ((B .* C D^T) F) W, one pass (Section 6.2).
    C: N x K, D: M x K, F: M x L, W: L x Mo.  Returns A (N x Mo)."""
    torch = _torch()
    device, N = _csr(rowptr, colidx, vals)
    K = _dense(C, "C", N, device)
    M = D.shape[0] if isinstance(D, torch.Tensor) and D.dim() == 2 else -1
    if _dense(D, "D", M, device) != K:
        raise ValueError("C and D differ in width K")
    L = _dense(F, "F", M, device)
    Mo = _dense(W, "W", L, device)
    A = _out(A, N, Mo, device)
    rc = lib().sparselnr_fused_sddmm_spmm_gemm(
        _ptr(rowptr, device), _ptr(colidx, device), _ptr(vals, device), _ptr(C, device),
        _ptr(D, device), _ptr(F, device), _ptr(W, device), _ptr(A, device), N, M, K, L, Mo,
        _stream(stream, device))
    if rc != OK:
        raise SparseLNRError(rc, "sparselnr_fused_sddmm_spmm_gemm")
    return A


def sparselnr_spmm_gemm(rowptr, colidx, vals, C, D, A=None, stream=None):
    """<SpMM, GEMM>: A = (B C) D (Section 6.2).  C: M x K, D: K x L.  Returns A (N x L)."""
    torch = _torch()
    device, N = _csr(rowptr, colidx, vals)
    M = C.shape[0] if isinstance(C, torch.Tensor) and C.dim() == 2 else -1
    K = _dense(C, "C", M, device)
    L = _dense(D, "D", K, device)
    A = _out(A, N, L, device)
    rc = lib().sparselnr_spmm_gemm(_ptr(rowptr, device), _ptr(colidx, device),
                                   _ptr(vals, device), _ptr(C, device), _ptr(D, device),
                                   _ptr(A, device), N, M, K, L, _stream(stream, device))
    if rc != OK:
        raise SparseLNRError(rc, "sparselnr_spmm_gemm")
    return A


def sparselnr_spmmh_gemm(rowptr, colidx, vals, C, D, E, A=None, stream=None):
    """<SpMMH, GEMM>: A = (B (C .* D)) E (Section 6.2).  C, D: M x J, E: J x L."""
    torch = _torch()
    device, N = _csr(rowptr, colidx, vals)
    M = C.shape[0] if isinstance(C, torch.Tensor) and C.dim() == 2 else -1
    J = _dense(C, "C", M, device)
    if _dense(D, "D", M, device) != J:
        raise ValueError("C and D must have the same shape")
    L = _dense(E, "E", J, device)
    A = _out(A, N, L, device)
    rc = lib().sparselnr_spmmh_gemm(_ptr(rowptr, device), _ptr(colidx, device),
                                    _ptr(vals, device), _ptr(C, device), _ptr(D, device),
                                    _ptr(E, device), _ptr(A, device), N, M, J, L,
                                    _stream(stream, device))
    if rc != OK:
        raise SparseLNRError(rc, "sparselnr_spmmh_gemm")
    return A


def sparselnr_fused_sddmm_spmm_dt(rowptr, colidx, vals, C, Dt, E, A=None, stream=None):
    """<SDDMM, SpMM> with D stored transposed (Dt: K x M, Section 4.3.1)."""
    torch = _torch()
    device, N = _csr(rowptr, colidx, vals)
    K = _dense(C, "C", N, device)
    M = E.shape[0] if isinstance(E, torch.Tensor) and E.dim() == 2 else -1
    if _dense(Dt, "Dt", K, device) != M:
        raise ValueError("Dt must be K x M")
    L = _dense(E, "E", M, device)
    A = _out(A, N, L, device)
    rc = lib().sparselnr_fused_sddmm_spmm_dt(
        _ptr(rowptr, device), _ptr(colidx, device), _ptr(vals, device), _ptr(C, device),
        _ptr(Dt, device), _ptr(E, device), _ptr(A, device), N, M, K, L, _stream(stream, device))
    if rc != OK:
        raise SparseLNRError(rc, "sparselnr_fused_sddmm_spmm_dt")
    return A


def sparselnr_validate_csr(rowptr, colidx, M, stream=None) -> int:
    """Checks the CSR preconditions on the device (synchronous).  Returns nnz;
    raises SparseLNRError(ERR_INVALID_CSR) on a violation."""
    torch = _torch()
    device = rowptr.device
    _check(rowptr, "rowptr", torch.int32, device, 1)
    _check(colidx, "colidx", torch.int32, device, 1)
    nnz = ctypes.c_int64(-1)
    rc = lib().sparselnr_validate_csr(_ptr(rowptr, device), _ptr(colidx, device),
                                      rowptr.numel() - 1, M, colidx.numel(), ctypes.byref(nnz),
                                      _stream(stream, device))
    if rc != OK:
        raise SparseLNRError(rc, "sparselnr_validate_csr")
    return int(nnz.value)


# ------------------------------------------------------------ paged cache

_DTYPES = {}


def _dtype_code(t, name):
    if not _DTYPES:
        torch = _torch()
        _DTYPES.update({torch.bfloat16: 0, torch.float16: 1, torch.float32: 2})
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise TypeError("%s must be bfloat16, float16 or float32, got %s" % (name, t.dtype))
    return code


def _rows(t, name, dims, dtype, device):
    """t of rows of adjacent values, any other strides."""
    if not isinstance(t, _torch().Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if t.dim() != dims:
        raise ValueError("%s must have %d dimensions" % (name, dims))
    if t.device != device:
        raise ValueError("%s is on %s, expected %s" % (name, t.device, device))
    if t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    s = t.stride()
    if s[-1] != 1 and t.shape[-1] > 1:
        raise ValueError("the last dimension of %s must be contiguous" % name)
    return s


def _gpu(t, name):
    if not isinstance(t, _torch().Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if t.device.type != "cuda":
        raise ValueError("inputs must be on a GPU device")
    return t.device


def _table(table, device):
    """Row stride and width of a block table; its rows need not be adjacent."""
    stride, _ = _rows(table, "table", 2, _torch().int32, device)
    R, W = table.shape
    return (stride if R > 1 else max(stride, W)), R, W


def _cache(kcache, vcache):
    device = _gpu(kcache, "kcache")
    code = _dtype_code(kcache, "kcache")
    ks = _rows(kcache, "kcache", 4, kcache.dtype, device)
    vs = _rows(vcache, "vcache", 4, kcache.dtype, device)
    shape = kcache.shape
    if vcache.shape != shape:
        raise ValueError("kcache and vcache differ in shape")
    return device, shape, _KvCache(kcache.data_ptr(), vcache.data_ptr(), *shape, *ks[:3], *vs[:3], code)


def _requests(table, seq_len, qptr, T, device):
    torch = _torch()
    stride, R, W = _table(table, device)
    _check(seq_len, "seq_len", torch.int32, device, 1)
    _check(qptr, "qptr", torch.int32, device, 1)
    if seq_len.numel() != R or qptr.numel() != R + 1:
        raise ValueError("seq_len and qptr must have R and R + 1 entries for R = %d rows of table" % R)
    return _Requests(table.data_ptr(), stride, seq_len.data_ptr(), qptr.data_ptr(), R, W, T)


def _page_size(page_size):
    if not isinstance(page_size, int) or page_size < 1:
        raise ValueError("page_size must be a positive integer")
    return page_size


def sparselnr_page_tables(ctx_len, new_len, table, free_pages, tokens, page_size, qptr=None, seq_len=None,
                          slots=None, counts=None, stream=None):
    """Block tables and slots of `tokens` new tokens from the request lengths.

    ctx_len, new_len: int32[R]; table: int32[R, W], changed in place;
    free_pages: int32[F].  Returns (qptr int32[R + 1], seq_len int32[R], slots
    int64[tokens], counts int32[3]), in the tensors given for them if any."""
    torch = _torch()
    device = _gpu(ctx_len, "ctx_len")
    _check(ctx_len, "ctx_len", torch.int32, device, 1)
    _check(new_len, "new_len", torch.int32, device, 1)
    _check(free_pages, "free_pages", torch.int32, device, 1)
    stride, R, W = _table(table, device)
    if ctx_len.numel() != R or new_len.numel() != R:
        raise ValueError("ctx_len and new_len must have one entry per row of table")
    if tokens < 0:
        raise ValueError("tokens must not be negative")
    if qptr is None and seq_len is None and counts is None:
        # one allocation for the three
        ints = torch.empty(2 * R + 4, dtype=torch.int32, device=device)
        qptr, seq_len, counts = ints[:R + 1], ints[R + 1:2 * R + 1], ints[2 * R + 1:]
    else:
        qptr = _given(qptr, "qptr", R + 1, torch.int32, device)
        seq_len = _given(seq_len, "seq_len", R, torch.int32, device)
        counts = _given(counts, "counts", 3, torch.int32, device)
    slots = _given(slots, "slots", tokens, torch.int64, device)
    rc = lib().sparselnr_page_tables(
        ctx_len.data_ptr(), new_len.data_ptr(), table.data_ptr(), stride, free_pages.data_ptr(), qptr.data_ptr(),
        seq_len.data_ptr(), slots.data_ptr(), counts.data_ptr(), R, W, free_pages.numel(), tokens,
        _page_size(page_size), _stream(stream, device))
    if rc != OK:
        raise SparseLNRError(rc, "sparselnr_page_tables")
    return qptr, seq_len, slots, counts


def _given(t, name, n, dtype, device):
    if t is None:
        return _torch().empty(n, dtype=dtype, device=device)
    _check(t, name, dtype, device, 1)
    if t.numel() != n:
        raise ValueError("%s must have %d entries" % (name, n))
    return t


def _summaries(kq, kscale, device):
    torch = _torch()
    _check(kq, "kq", torch.int8, device, 3)
    _check(kscale, "kscale", torch.float32, device, 2)
    if kscale.shape != kq.shape[:2]:
        raise ValueError("kscale must be pages x Hkv, as kq")
    return kq.shape


def sparselnr_cache_append(k, v, slots, kcache, vcache, kq=None, kscale=None, stream=None):
    """Writes k and v (T x Hkv x D) into the slots (int64[T]; -1: left out) of
    kcache and vcache (pages x page_size x Hkv x D, any order of memory), and renews
    the written pages' summaries kq (int8 pages x Hkv x D), kscale (float32 pages x Hkv)."""
    torch = _torch()
    device, shape, cache = _cache(kcache, vcache)
    ks = _rows(k, "k", 3, kcache.dtype, device)
    vs = _rows(v, "v", 3, kcache.dtype, device)
    T = k.shape[0]
    if k.shape != v.shape or k.shape[1:] != shape[2:]:
        raise ValueError("k and v must be T x Hkv x D, as the cache's rows")
    _check(slots, "slots", torch.int64, device, 1)
    if slots.numel() != T:
        raise ValueError("slots must have one entry per token")
    if (kq is None) != (kscale is None):
        raise ValueError("kq and kscale go together")
    if kq is not None and _summaries(kq, kscale, device) != (shape[0], shape[2], shape[3]):
        raise ValueError("kq must be pages x Hkv x D")
    rc = lib().sparselnr_cache_append(
        k.data_ptr(), ks[0], ks[1], v.data_ptr(), vs[0], vs[1], slots.data_ptr(), cache,
        kq.data_ptr() if kq is not None else None, kscale.data_ptr() if kq is not None else None, T,
        _stream(stream, device))
    if rc != OK:
        raise SparseLNRError(rc, "sparselnr_cache_append")


def _attention(q, kcache, vcache, table, seq_len, qptr, scale, out, lse):
    torch = _torch()
    device, shape, cache = _cache(kcache, vcache)
    qs = _rows(q, "q", 3, kcache.dtype, device)
    T, Hq, D = q.shape
    if D != shape[3]:
        raise ValueError("q and the cache differ in head dimension")
    if shape[2] == 0 or Hq % shape[2]:
        raise ValueError("query heads must be a multiple of the cache's heads")
    requests = _requests(table, seq_len, qptr, T, device)
    if out is None:
        out = torch.empty((T, Hq, D), dtype=q.dtype, device=device)
    else:
        _check(out, "out", q.dtype, device, 3)
        if out.shape != q.shape:
            raise ValueError("out must have the shape of q")
    if lse is not None:
        _check(lse, "lse", torch.float32, device, 2)
        if lse.shape != q.shape[:2]:
            raise ValueError("lse must be T x Hq")
    if scale is None:
        scale = D ** -0.5
    return (device, out, (q.data_ptr(), qs[0], qs[1], Hq, cache, requests), scale,
            lse.data_ptr() if lse is not None else None)


def sparselnr_paged_attention(q, kcache, vcache, table, seq_len, qptr, scale=None, window=0, max_new=0, out=None,
                              lse=None, stream=None):
    """Causal attention of the new tokens q (T x Hq x D, packed by qptr) over the
    cached rows of their requests.  scale defaults to D ** -0.5; window > 0 bounds
    how far back a token sees; max_new > 0 says that no request has more new
    tokens.  lse (float32 T x Hq), if given, is filled.  Returns out (T x Hq x D)."""
    device, out, head, scale, lse = _attention(q, kcache, vcache, table, seq_len, qptr, scale, out, lse)
    rc = lib().sparselnr_paged_attention(*head, scale, window, max_new, out.data_ptr(), lse,
                                         _stream(stream, device))
    if rc != OK:
        raise SparseLNRError(rc, "sparselnr_paged_attention")
    return out


def sparselnr_block_select(q, kq, kscale, table, seq_len, qptr, page_size, top, first=1, local=1, sel=None,
                           stream=None):
    """The `top` pages that each new token attends, per KV head: the first `first`
    and last `local` ones and the best by the 8-bit score.  Returns sel (int32
    T x Hkv x top): indices into the table row, ascending, -1 behind them."""
    torch = _torch()
    device = _gpu(q, "q")
    code = _dtype_code(q, "q")
    qs = _rows(q, "q", 3, q.dtype, device)
    T, Hq, D = q.shape
    pages, Hkv, Dk = _summaries(kq, kscale, device)
    if Dk != D:
        raise ValueError("q and kq differ in head dimension")
    if Hkv == 0 or Hq % Hkv:
        raise ValueError("query heads must be a multiple of the summaries' heads")
    requests = _requests(table, seq_len, qptr, T, device)
    if sel is None:
        sel = torch.empty((T, Hkv, top), dtype=torch.int32, device=device)
    else:
        _check(sel, "sel", torch.int32, device, 3)
        if sel.shape != (T, Hkv, top):
            raise ValueError("sel must be T x Hkv x top")
    rc = lib().sparselnr_block_select(
        q.data_ptr(), qs[0], qs[1], Hq, code, kq.data_ptr(), kscale.data_ptr(), pages, _page_size(page_size), Hkv,
        D, requests, top, first, local, sel.data_ptr(), _stream(stream, device))
    if rc != OK:
        raise SparseLNRError(rc, "sparselnr_block_select")
    return sel


def sparselnr_block_attention(q, kcache, vcache, table, seq_len, qptr, sel, scale=None, out=None, lse=None,
                              stream=None):
    """As sparselnr_paged_attention, over the pages sel (int32 T x Hkv x top) of each
    token and KV head only.  Returns out (T x Hq x D)."""
    device, out, head, scale, lse = _attention(q, kcache, vcache, table, seq_len, qptr, scale, out, lse)
    _check(sel, "sel", _torch().int32, device, 3)
    T, Hkv, top = sel.shape
    if T != q.shape[0] or Hkv != kcache.shape[2]:
        raise ValueError("sel must be T x Hkv x top")
    rc = lib().sparselnr_block_attention(*head, sel.data_ptr(), top, scale, out.data_ptr(), lse,
                                         _stream(stream, device))
    if rc != OK:
        raise SparseLNRError(rc, "sparselnr_block_attention")
    return out
