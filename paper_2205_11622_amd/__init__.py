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

_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


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


_get_device = None


def _on(index, entry, *args):
    """entry(*args) with GPU `index` current: the library launches and allocates there."""
    global _get_device
    if _get_device is None:
        torch = _torch()
        _get_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
    if _get_device() == index:
        return entry(*args)
    with _torch().cuda.device(index):
        return entry(*args)


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
    rc = _on(device.index, lib().sparselnr_fused_sddmm_spmm,
             _ptr(rowptr, device), _ptr(colidx, device), _ptr(vals, device), _ptr(C, device), _ptr(D, device),
             _ptr(E, device), _ptr(A, device), N, M, K, L, _stream(stream, device))
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
    rc = _on(device.index, lib().sparselnr_fused_sddmm_spmm_noalloc,
             _ptr(rowptr, device), _ptr(colidx, device), _ptr(vals, device), _ptr(C, device), _ptr(D, device),
             _ptr(E, device), _ptr(A, device), N, M, K, L, _stream(stream, device))
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
    rc = _on(device.index, lib().sparselnr_sddmm,
             _ptr(rowptr, device), _ptr(colidx, device), _ptr(vals, device), _ptr(C, device), _ptr(D, device),
             _ptr(Y, device), N, M, K, _stream(stream, device))
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
    rc = _on(device.index, lib().sparselnr_spmm,
             _ptr(rowptr, device), _ptr(colidx, device), _ptr(Y, device), _ptr(E, device), _ptr(A, device), N, M, L,
             _stream(stream, device))
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
    rc = _on(device.index, lib().sparselnr_unfused_sddmm_spmm,
             _ptr(rowptr, device), _ptr(colidx, device), _ptr(vals, device), _ptr(C, device), _ptr(D, device),
             _ptr(E, device), _ptr(Y, device), _ptr(A, device), N, M, K, L, _stream(stream, device))
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
    rc = _on(device.index, lib().sparselnr_fused_sddmm_spmm_gemm,
             _ptr(rowptr, device), _ptr(colidx, device), _ptr(vals, device), _ptr(C, device), _ptr(D, device),
             _ptr(F, device), _ptr(W, device), _ptr(A, device), N, M, K, L, Mo, _stream(stream, device))
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
    rc = _on(device.index, lib().sparselnr_spmm_gemm,
             _ptr(rowptr, device), _ptr(colidx, device), _ptr(vals, device), _ptr(C, device), _ptr(D, device),
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
    rc = _on(device.index, lib().sparselnr_spmmh_gemm,
             _ptr(rowptr, device), _ptr(colidx, device), _ptr(vals, device), _ptr(C, device), _ptr(D, device),
             _ptr(E, device), _ptr(A, device), N, M, J, L, _stream(stream, device))
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
    rc = _on(device.index, lib().sparselnr_fused_sddmm_spmm_dt,
             _ptr(rowptr, device), _ptr(colidx, device), _ptr(vals, device), _ptr(C, device), _ptr(Dt, device),
             _ptr(E, device), _ptr(A, device), N, M, K, L, _stream(stream, device))
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
    rc = _on(device.index, lib().sparselnr_validate_csr,
             _ptr(rowptr, device), _ptr(colidx, device), rowptr.numel() - 1, M, colidx.numel(), ctypes.byref(nnz),
             _stream(stream, device))
    if rc != OK:
        raise SparseLNRError(rc, "sparselnr_validate_csr")
    return int(nnz.value)


# ------------------------------------------------------------ paged cache
#
# These calls run once per layer and decode step, where the GPU is done in a few
# microseconds: arguments are looked at in one expression first, and one by one, for the
# message, only if that fails.

_DTYPES = {}
_raw_stream = None


def _launch_stream(stream, index):
    """The raw stream: the one given, or the current one of GPU `index`."""
    global _raw_stream
    if stream is not None:
        return getattr(stream, "cuda_stream", stream)
    if _raw_stream is None:
        torch = _torch()
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream",
                              lambda i: torch.cuda.current_stream(i).cuda_stream)
    return _raw_stream(index)


def _dtype_code(t, name):
    if not _DTYPES:
        torch = _torch()
        _DTYPES.update({torch.bfloat16: 0, torch.float16: 1, torch.float32: 2})
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise TypeError("%s must be bfloat16, float16 or float32, got %s" % (name, t.dtype))
    return code


def _gpu(t, name):
    """Index of the GPU that tensor t is on."""
    try:
        index = t.get_device()
    except AttributeError:
        raise TypeError("%s must be a torch.Tensor" % name) from None
    if index < 0 or not t.is_cuda:
        raise ValueError("inputs must be on a GPU device")
    return index


def _rows(t, name, dims, dtype, index):
    """Strides of t, whose rows (the last dimension) are adjacent values."""
    try:
        s = t.stride()
        if len(s) == dims and t.dtype is dtype and t.get_device() == index and (s[-1] == 1 or t.shape[-1] <= 1):
            return s
    except AttributeError:
        raise TypeError("%s must be a torch.Tensor" % name) from None
    if t.dim() != dims:
        raise ValueError("%s must have %d dimensions" % (name, dims))
    if t.get_device() != index:
        raise ValueError("%s is on %s, expected GPU %d" % (name, t.device, index))
    if t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    raise ValueError("the last dimension of %s must be contiguous" % name)


def _packed(t, name, dtype, index, shape):
    """Address of t, densely packed and of that shape."""
    try:
        if t.dtype is dtype and t.shape == shape and t.get_device() == index and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        raise TypeError("%s must be a torch.Tensor" % name) from None
    if t.get_device() != index:
        raise ValueError("%s is on %s, expected GPU %d" % (name, t.device, index))
    if t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if t.shape != shape:
        raise ValueError("%s must be %s, got %s" % (name, " x ".join(map(str, shape)), tuple(t.shape)))
    raise ValueError("%s must be contiguous" % name)


def _table(table, index):
    """Row stride, rows and width of a block table; its rows need not be adjacent."""
    stride = _rows(table, "table", 2, _torch().int32, index)[0]
    R, W = table.shape
    return (stride if R > 1 else max(stride, W)), R, W


def _cache(kcache, vcache):
    index = _gpu(kcache, "kcache")
    code = _dtype_code(kcache, "kcache")
    dtype = kcache.dtype
    ks = _rows(kcache, "kcache", 4, dtype, index)
    vs = _rows(vcache, "vcache", 4, dtype, index)
    shape = kcache.shape
    if vcache.shape != shape:
        raise ValueError("kcache and vcache differ in shape")
    return index, shape, _KvCache(kcache.data_ptr(), vcache.data_ptr(), *shape, ks[0], ks[1], ks[2], vs[0], vs[1],
                                  vs[2], code)


def _requests(table, seq_len, qptr, T, index):
    int32 = _torch().int32
    stride, R, W = _table(table, index)
    return _Requests(table.data_ptr(), stride, _packed(seq_len, "seq_len", int32, index, (R,)),
                     _packed(qptr, "qptr", int32, index, (R + 1,)), R, W, T)


def sparselnr_page_tables(ctx_len, new_len, table, free_pages, tokens, page_size, qptr=None, seq_len=None,
                          slots=None, counts=None, stream=None):
    """Block tables and slots of `tokens` new tokens from the request lengths.

    ctx_len, new_len: int32[R]; table: int32[R, W], changed in place;
    free_pages: int32[F].  Returns (qptr int32[R + 1], seq_len int32[R], slots
    int64[tokens], counts int32[3]), in the tensors given for them if any."""
    torch = _torch()
    int32 = torch.int32
    index = _gpu(ctx_len, "ctx_len")
    stride, R, W = _table(table, index)
    F = free_pages.numel() if isinstance(free_pages, torch.Tensor) else 0
    args = (_packed(ctx_len, "ctx_len", int32, index, (R,)), _packed(new_len, "new_len", int32, index, (R,)),
            table.data_ptr(), stride, _packed(free_pages, "free_pages", int32, index, (F,)))
    if tokens < 0:
        raise ValueError("tokens must not be negative")
    device = ctx_len.device
    if qptr is None and seq_len is None and counts is None:
        # one allocation for the three
        qptr, seq_len, counts = torch.empty(2 * R + 4, dtype=int32, device=device).split_with_sizes((R + 1, R, 3))
    qptr = torch.empty(R + 1, dtype=int32, device=device) if qptr is None else qptr
    seq_len = torch.empty(R, dtype=int32, device=device) if seq_len is None else seq_len
    counts = torch.empty(3, dtype=int32, device=device) if counts is None else counts
    slots = torch.empty(tokens, dtype=torch.int64, device=device) if slots is None else slots
    rc = _on(index, lib().sparselnr_page_tables,
             *args, _packed(qptr, "qptr", int32, index, (R + 1,)), _packed(seq_len, "seq_len", int32, index, (R,)),
             _packed(slots, "slots", torch.int64, index, (tokens,)), _packed(counts, "counts", int32, index, (3,)),
             R, W, F, tokens, page_size, _launch_stream(stream, index))
    if rc != OK:
        raise SparseLNRError(rc, "sparselnr_page_tables")
    return qptr, seq_len, slots, counts


def sparselnr_cache_append(k, v, slots, kcache, vcache, kq=None, kscale=None, stream=None):
    """Writes k and v (T x Hkv x D) into the slots (int64[T]; -1: left out) of
    kcache and vcache (pages x page_size x Hkv x D, any order of memory), and renews
    the written pages' summaries kq (int8 pages x Hkv x D), kscale (float32 pages x Hkv)."""
    torch = _torch()
    index, shape, cache = _cache(kcache, vcache)
    ks = _rows(k, "k", 3, kcache.dtype, index)
    vs = _rows(v, "v", 3, kcache.dtype, index)
    T = k.shape[0]
    if k.shape != v.shape or k.shape[1:] != shape[2:]:
        raise ValueError("k and v must be T x Hkv x D, as the cache's rows")
    if (kq is None) != (kscale is None):
        raise ValueError("kq and kscale go together")
    kq_at = ks_at = None
    if kq is not None:
        kq_at = _packed(kq, "kq", torch.int8, index, (shape[0], shape[2], shape[3]))
        ks_at = _packed(kscale, "kscale", torch.float32, index, (shape[0], shape[2]))
    rc = _on(index, lib().sparselnr_cache_append,
             k.data_ptr(), ks[0], ks[1], v.data_ptr(), vs[0], vs[1],
             _packed(slots, "slots", torch.int64, index, (T,)), cache, kq_at, ks_at, T,
             _launch_stream(stream, index))
    if rc != OK:
        raise SparseLNRError(rc, "sparselnr_cache_append")


def _attention(q, kcache, vcache, table, seq_len, qptr, scale, out, lse):
    torch = _torch()
    index, shape, cache = _cache(kcache, vcache)
    dtype = kcache.dtype
    qs = _rows(q, "q", 3, dtype, index)
    T, Hq, D = q.shape
    if D != shape[3]:
        raise ValueError("q and the cache differ in head dimension")
    if shape[2] == 0 or Hq % shape[2]:
        raise ValueError("query heads must be a multiple of the cache's heads")
    requests = _requests(table, seq_len, qptr, T, index)
    if out is None:
        out = torch.empty((T, Hq, D), dtype=dtype, device=q.device)
    else:
        _packed(out, "out", dtype, index, (T, Hq, D))
    lse_at = None if lse is None else _packed(lse, "lse", torch.float32, index, (T, Hq))
    return (index, out, (q.data_ptr(), qs[0], qs[1], Hq, cache, requests), D ** -0.5 if scale is None else scale,
            lse_at)


def sparselnr_paged_attention(q, kcache, vcache, table, seq_len, qptr, scale=None, window=0, max_new=0, out=None,
                              lse=None, stream=None):
    """Causal attention of the new tokens q (T x Hq x D, packed by qptr) over the
    cached rows of their requests.  scale defaults to D ** -0.5; window > 0 bounds
    how far back a token sees; max_new > 0 says that no request has more new
    tokens.  lse (float32 T x Hq), if given, is filled.  Returns out (T x Hq x D)."""
    index, out, head, scale, lse = _attention(q, kcache, vcache, table, seq_len, qptr, scale, out, lse)
    rc = _on(index, lib().sparselnr_paged_attention,
             *head, scale, window, max_new, out.data_ptr(), lse, _launch_stream(stream, index))
    if rc != OK:
        raise SparseLNRError(rc, "sparselnr_paged_attention")
    return out


def sparselnr_block_select(q, kq, kscale, table, seq_len, qptr, page_size, top, first=1, local=1, sel=None,
                           stream=None):
    """The `top` pages that each new token attends, per KV head: the first `first`
    and last `local` ones and the best by the 8-bit score.  Returns sel (int32
    T x Hkv x top): indices into the table row, ascending, -1 behind them."""
    torch = _torch()
    index = _gpu(q, "q")
    code = _dtype_code(q, "q")
    qs = _rows(q, "q", 3, q.dtype, index)
    T, Hq, D = q.shape
    if not isinstance(kq, torch.Tensor) or kq.dim() != 3:
        raise ValueError("kq must have 3 dimensions")
    pages, Hkv, Dk = kq.shape
    if Dk != D:
        raise ValueError("q and kq differ in head dimension")
    if Hkv == 0 or Hq % Hkv:
        raise ValueError("query heads must be a multiple of the summaries' heads")
    kq_at = _packed(kq, "kq", torch.int8, index, (pages, Hkv, D))
    ks_at = _packed(kscale, "kscale", torch.float32, index, (pages, Hkv))
    requests = _requests(table, seq_len, qptr, T, index)
    if sel is None:
        sel = torch.empty((T, Hkv, max(top, 0)), dtype=torch.int32, device=q.device)
    else:
        _packed(sel, "sel", torch.int32, index, (T, Hkv, top))
    rc = _on(index, lib().sparselnr_block_select,
             q.data_ptr(), qs[0], qs[1], Hq, code, kq_at, ks_at, pages, page_size, Hkv, D, requests, top, first,
             local, sel.data_ptr(), _launch_stream(stream, index))
    if rc != OK:
        raise SparseLNRError(rc, "sparselnr_block_select")
    return sel


def sparselnr_block_attention(q, kcache, vcache, table, seq_len, qptr, sel, scale=None, out=None, lse=None,
                              stream=None):
    """As sparselnr_paged_attention, over the pages sel (int32 T x Hkv x top) of each
    token and KV head only.  Returns out (T x Hq x D)."""
    index, out, head, scale, lse = _attention(q, kcache, vcache, table, seq_len, qptr, scale, out, lse)
    if not isinstance(sel, _torch().Tensor) or sel.dim() != 3:
        raise ValueError("sel must have 3 dimensions")
    top = sel.shape[2]
    sel_at = _packed(sel, "sel", _torch().int32, index, (q.shape[0], kcache.shape[2], top))
    rc = _on(index, lib().sparselnr_block_attention,
             *head, sel_at, top, scale, out.data_ptr(), lse, _launch_stream(stream, index))
    if rc != OK:
        raise SparseLNRError(rc, "sparselnr_block_attention")
    return out
