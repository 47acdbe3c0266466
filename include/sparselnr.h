/*
 * sparselnr.h -- C ABI of the MI355X (gfx950) fused SDDMM->SpMM library.
 *
 * Computes, for a sparse matrix B in CSR form and dense C, D, E,
 *
 *     A(i,l) = sum_{j,k} B(i,j) * C(i,k) * D(j,k) * E(j,l)
 *
 * the <SDDMM, SpMM> computation of Dias et al., "SparseLNR: Accelerating
 * Sparse Tensor Computations Using Loop Nest Restructuring" (ICS 2022),
 * Section 3.1 and Figure 2.  The fused entry point runs the paper's
 * loop-fused, kernel-distributed schedule (Figure 2d; Section 3.1.3): one
 * pass over the rows of B in which, for every nonzero, a scalar SDDMM value
 * is produced and immediately consumed by the SpMM update of the row, so no
 * nnz-sized intermediate exists (Section 4.2: the temporary of this
 * expression is a scalar because no index below the nest boundary is shared
 * by producer and consumer).  The unfused entry points are the paper's
 * separate-kernel schedule (Figures 2a and 2b, Section 3.1.2), kept as the
 * in-library comparison.
 *
 * Layouts (all row-major, densely packed, fp32 values, int32 indices):
 *   rowptr  int32[N+1]   CSR row offsets; rowptr[0] = 0, non-decreasing
 *   colidx  int32[nnz]   column of every nonzero, 0 <= colidx[p] < M
 *   vals    float[nnz]   value of every nonzero
 *   C       float[N*K]   C(i,k) at C[i*K + k]
 *   D       float[M*K]   D(j,k) at D[j*K + k]
 *   E       float[M*L]   E(j,l) at E[j*L + l]
 *   A       float[N*L]   A(i,l) at A[i*L + l]   (output, overwritten)
 *   Y       float[nnz]   SDDMM values with the structure of B (unfused only)
 * where nnz = rowptr[N] (read on the device; never passed in).
 *
 * Conventions shared by every compute entry point:
 *   - All array pointers are DEVICE pointers owned by the caller; the library
 *     never frees or retains them.  The base pointers must be 4-byte aligned;
 *     16-byte alignment of all of them enables the kernels of fixed width.
 *   - Calls are asynchronous on `stream` (a hipStream_t; NULL is the null
 *     stream).  No call synchronises with the host.  The arrays and the stream are
 *     of the calling thread's current device.
 *   - Columns within a row may be unsorted and may repeat (repeats add).
 *     Preconditions on the CSR arrays are not checked on the device; use
 *     sparselnr_validate_csr in tests.  nnz and N + nnz must be < 2^31.
 *   - N = 0 or L = 0 is a no-op.  K = 0 makes every SDDMM value zero.  Rows
 *     without nonzeros produce zero rows of A.
 *   - rowptr must be non-NULL when N > 0.  colidx and vals (Y for SpMM) must
 *     be non-NULL when N > 0; pass any valid device address when nnz = 0.
 *     C must be non-NULL when N > 0 and K > 0; D when N, M, K > 0; E when
 *     N, M, L > 0; A when N > 0 and L > 0; Y (unfused/SDDMM) when N > 0.
 *   - Argument errors are reported BEFORE any HIP call, with no side effect.
 *   - The fused, unfused and SpMM calls use a workspace per (device, stream)
 *     for rows whose nonzeros are split between workers (2 partial rows per
 *     worker: tens of MB for matrices of millions of rows); it is allocated
 *     on first use, grown when a call needs more, reused, and freed by
 *     sparselnr_release().
 *     Calls on different streams use different workspaces; calls on one
 *     stream are ordered by the stream.  A call of the sparse products is several
 *     launches over its workspace: host threads that share a stream have to
 *     make them one after the other (the calls of the paged cache, below, hold their
 *     workspace until their last launch is queued and need no such care).
 *   - HIP graph capture: once a stream's workspace is large enough (after
 *     one uncaptured call of the same size, width and grid factor on that
 *     stream), a call launches kernels only, with no allocation,
 *     synchronisation or memset, and can be captured on that stream.  The
 *     graph records the workspace address: while it may still be replayed,
 *     do not call sparselnr_release() and make no call on that stream that
 *     needs a larger workspace (more rows, a larger grid factor, other widths
 *     K and L or another entry point, which may take more workers), since
 *     either frees the workspace.  Calls made once before the capture do not.
 *   - Results are deterministic: the same inputs give bit-identical outputs
 *     on the same device model (no floating-point atomics).
 *   - No C++ exception crosses this interface.
 */
#ifndef SPARSELNR_H
#define SPARSELNR_H

#include <stddef.h>
#include <stdint.h>

#if defined(__GNUC__)
#define SPARSELNR_API __attribute__((visibility("default")))
#else
#define SPARSELNR_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

/* Status codes returned by every int-valued entry point. */
enum sparselnr_status_code {
  SPARSELNR_OK = 0,
  SPARSELNR_ERR_INVALID_ARG = 1, /* NULL pointer, negative size, misuse      */
  SPARSELNR_ERR_UNSUPPORTED = 2, /* K or L above SPARSELNR_MAX_WIDTH, or
                                    sizes beyond the int32 index range        */
  SPARSELNR_ERR_HIP = 3,         /* a HIP call failed; see last_hip_error      */
  SPARSELNR_ERR_NO_MEMORY = 4,   /* workspace allocation failed               */
  SPARSELNR_ERR_INVALID_CSR = 5  /* sparselnr_validate_csr found a violation  */
};

/* Largest accepted K and L. */
#define SPARSELNR_MAX_WIDTH 65536

/* Version of this interface (incremented on incompatible change). */
SPARSELNR_API int sparselnr_abi_version(void);

/*
 * Fused SDDMM->SpMM (Figure 2d; Section 3.1.3):
 *   A(i,:) = sum_{p in row i} vals[p] * dot(C(i,:), D(colidx[p],:)) * E(colidx[p],:)
 * A is overwritten.  Arithmetic is fp32 (fused multiply-add), with the
 * k-reduction done as a lane-parallel tree.  The nonzeros of a row are added
 * in an order fixed by its length, the widths and the grid: up to 16 partial
 * sums side by side, long rows in groups of four, then the sums of the pieces
 * of a split row in order.  Needs the per-(device, stream) workspace.
 */
SPARSELNR_API int sparselnr_fused_sddmm_spmm(const int32_t *rowptr, const int32_t *colidx,
                                             const float *vals, const float *C,
                                             const float *D, const float *E, float *A,
                                             int64_t N, int64_t M, int64_t K, int64_t L,
                                             void *stream);

/* Size in bytes of the device array of sparselnr_fused_sddmm_spmm_noalloc. */
#define SPARSELNR_NOALLOC_SCRATCH_BYTES (64u * 1024u * 1024u)

/*
 * For callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid allocation): the same
 * computation, arguments, layouts and argument errors as
 * sparselnr_fused_sddmm_spmm, with no allocation of any kind (no hipMalloc,
 * hipFree or allocating library routine).  The partial rows of rows split
 * between workers go to a fixed device array of
 * SPARSELNR_NOALLOC_SCRATCH_BYTES (64 MiB) inside the library, one per GPU,
 * held from the first call on that GPU until the process ends.  The call
 * runs at the grid factor the fused entry point would use, halved until the
 * partial rows fit the array (so results may differ from the fused entry
 * point's in rounding order, within its accuracy; they are bit-identical
 * when the same factor fits, as it does at the automatic factor for L up to
 * 256).  It returns SPARSELNR_ERR_UNSUPPORTED if they
 * do not fit even at one resident grid (not reached for K, L <= 512).
 * All calls on one GPU share that GPU's array and it keeps the last call's
 * contents: calls that overlap in time on one GPU (different streams, or
 * different host threads) RACE and corrupt each other's results; order them
 * on one stream.  Nothing in the array needs clearing between calls.
 */
SPARSELNR_API int sparselnr_fused_sddmm_spmm_noalloc(const int32_t *rowptr,
                                                     const int32_t *colidx, const float *vals,
                                                     const float *C, const float *D,
                                                     const float *E, float *A, int64_t N,
                                                     int64_t M, int64_t K, int64_t L,
                                                     void *stream);

/*
 * Unfused comparison (Figure 2a then Figure 2b, Section 3.1.2): the SDDMM
 * writes Y (nnz floats, structure of B, same order as colidx), then the SpMM
 * reads it.  Same result as the fused call up to rounding order.
 */
SPARSELNR_API int sparselnr_unfused_sddmm_spmm(const int32_t *rowptr, const int32_t *colidx,
                                               const float *vals, const float *C,
                                               const float *D, const float *E, float *Y,
                                               float *A, int64_t N, int64_t M, int64_t K,
                                               int64_t L, void *stream);

/* SDDMM alone (Figure 2a): Y[p] = vals[p] * dot(C(i,:), D(colidx[p],:)). */
SPARSELNR_API int sparselnr_sddmm(const int32_t *rowptr, const int32_t *colidx,
                                  const float *vals, const float *C, const float *D,
                                  float *Y, int64_t N, int64_t M, int64_t K, void *stream);

/* SpMM alone (Figure 2b): A(i,:) = sum_{p in row i} Y[p] * E(colidx[p],:).
 * A is overwritten.  Needs the per-(device, stream) workspace. */
SPARSELNR_API int sparselnr_spmm(const int32_t *rowptr, const int32_t *colidx,
                                 const float *Y, const float *E, float *A, int64_t N,
                                 int64_t M, int64_t L, void *stream);

/*
 * <SDDMM, SpMM, GEMM> (Section 6.2; the recursive application of the fusion
 * in Section 4.2):
 *   A(i,m) = sum_{j,k,l} B(i,j) C(i,k) D(j,k) F(j,l) W(l,m)
 * computed as the fused <SDDMM, SpMM> row t_i (Figure 2d) followed, in the
 * same pass, by the per-row product A_i = t_i W, so neither the nnz-sized
 * SDDMM values nor the N x L matrix t is ever stored.  The row products
 * run on the matrix cores over tiles of finished rows.
 *   C: N x K, D: M x K, F: M x L, W: L x Mo, A: N x Mo (overwritten).
 * Supported: K == L in {16, 32, 64, 128, 256, 512}, any Mo; C, D and F
 * 16-byte aligned.  Other shapes return SPARSELNR_ERR_UNSUPPORTED.
 */
SPARSELNR_API int sparselnr_fused_sddmm_spmm_gemm(const int32_t *rowptr, const int32_t *colidx,
                                                  const float *vals, const float *C,
                                                  const float *D, const float *F,
                                                  const float *W, float *A, int64_t N,
                                                  int64_t M, int64_t K, int64_t L, int64_t Mo,
                                                  void *stream);

/*
 * <SpMM, GEMM> (Section 6.2; the GNN hidden-state update):
 *   A(i,l) = sum_{j,k} B(i,j) C(j,k) D(k,l)
 * computed per row as the SpMM row t_i = sum_j B(i,j) C(j,:) (a vector
 * temporary of length K, Section 6.3) followed by A_i = t_i D.
 *   C: M x K, D: K x L, A: N x L (overwritten).
 * Supported: K in {16, 32, 64, 128, 256, 512}, any L; C 16-byte aligned.
 */
SPARSELNR_API int sparselnr_spmm_gemm(const int32_t *rowptr, const int32_t *colidx,
                                      const float *vals, const float *C, const float *D,
                                      float *A, int64_t N, int64_t M, int64_t K, int64_t L,
                                      void *stream);

/*
 * <SpMMH, GEMM> (Section 6.2):
 *   A(i,l) = sum_{k,j} B(i,k) C(k,j) D(k,j) E(j,l)
 * computed per row as t_i = sum_k B(i,k) (C(k,:) .* D(k,:)) (length J)
 * followed by A_i = t_i E.  B is N x M; C, D: M x J; E: J x L; A: N x L.
 * Supported: J in {16, 32, 64, 128, 256, 512}, any L; C and D 16-byte
 * aligned.
 * C .* D does not depend on the row i.  When nnz >= 3 M (decided on the
 * device, which alone knows nnz) it is formed once into a per-(device,
 * stream) workspace of M x J floats and gathered as one row per nonzero;
 * otherwise each nonzero multiplies its two gathered rows.  Both schedules
 * round the same products in the same order, so A is bit-identical either
 * way.  The workspace is allocated on the first call of a shape (failure:
 * SPARSELNR_ERR_NO_MEMORY) and freed by sparselnr_release().
 */
SPARSELNR_API int sparselnr_spmmh_gemm(const int32_t *rowptr, const int32_t *colidx,
                                       const float *vals, const float *C, const float *D,
                                       const float *E, float *A, int64_t N, int64_t M,
                                       int64_t J, int64_t L, void *stream);

/*
 * <SDDMM, SpMM> with D stored transposed (Section 4.3.1: the layout whose
 * temporary becomes a vector over j unless the loops are reordered):
 *   A(i,l) = sum_{j,k} B(i,j) C(i,k) Dt(k,j) E(j,l),   Dt: K x M.
 * On the GPU the reorder is done on the data: Dt is transposed once into a
 * per-(device, stream) workspace of M x K floats (coalesced tile transpose),
 * then the fused kernel runs.  Same result, shapes and errors as
 * sparselnr_fused_sddmm_spmm; the workspace is freed by sparselnr_release().
 */
SPARSELNR_API int sparselnr_fused_sddmm_spmm_dt(const int32_t *rowptr, const int32_t *colidx,
                                                const float *vals, const float *C,
                                                const float *Dt, const float *E, float *A,
                                                int64_t N, int64_t M, int64_t K, int64_t L,
                                                void *stream);

/*
 * Checks the CSR preconditions on the device: rowptr[0] == 0, rowptr
 * non-decreasing, 0 <= rowptr[N] <= colidx_len, N + rowptr[N] < 2^31, every
 * colidx in [0, M).  colidx_len is the number of int32 entries the caller
 * allocated for colidx; at most that many are read.  SYNCHRONOUS (waits for
 * `stream`); meant for tests and debugging, not the hot path.  Writes
 * nnz = rowptr[N] to *nnz_out (host pointer, may be NULL).
 * Returns SPARSELNR_OK or SPARSELNR_ERR_INVALID_CSR (or an error code).
 */
SPARSELNR_API int sparselnr_validate_csr(const int32_t *rowptr, const int32_t *colidx,
                                         int64_t N, int64_t M, int64_t colidx_len,
                                         int64_t *nnz_out, void *stream);

/* ------------------------------------------------------------------------
 * Attention over a paged cache.
 *
 * A serving program keeps the keys and values of its requests in pages of a
 * shared cache: request r's row of position j lies in page table[r][j / P] at
 * place j % P.  That table is the structure of a sparse matrix as B is above,
 * and attention is its SDDMM (q.k) and SpMM (p.v) with a softmax between them,
 * computed in one pass.  (No counterpart in the paper, whose <SDDMM, SpMM> has
 * no softmax.)
 *
 * Conventions, besides those above on pointers, streams, errors and
 * determinism (results are bit-identical for the same inputs):
 *   - Types: bf16, fp16 or fp32 values; products of 16-bit values accumulate in
 *     fp32, and so do the softmax' maximum, sum and the weighted sum.  The
 *     weights are rounded to the values' type for their product with V.
 *   - New tokens are packed: request r's n_r = qptr[r+1] - qptr[r] new tokens are
 *     the rows qptr[r] .. of q, k, v and out (as the rows of a CSR matrix); they
 *     are the last n_r of its seq_len[r] positions, and their own rows have to be
 *     in the cache.  n_r = 1 is a decode step; any mixture is fine.  Rows of out
 *     and sel that belong to no request are left as they were.
 *   - Heads: Hq is a multiple of Hkv; query head h reads KV head h / (Hq / Hkv).
 *   - A table entry outside [0, pages) is a page that is not there (not yet
 *     taken, or given back): its keys are not seen.  A query that sees no key
 *     gets zeros, and -inf as its lse.  Whatever the arrays on the device hold,
 *     no call reads or writes outside the arrays that it was given.
 *   - Keys that a query does not see have no part in its result, whatever their
 *     rows hold (NaN and infinities included).  NaN in what it sees gives NaN.
 *   - dim: a multiple of 8 up to 256.  page_size: a power of two up to
 *     SPARSELNR_MAX_PAGE.  Row, page and head strides are in values, may be any
 *     that keep each row of dim values at a multiple of 16 bytes (the stride of an
 *     extent of one does not count; so a slice of a fused q/k/v projection and caches
 *     of either order of slots and heads will do); the dim values of a row are
 *     adjacent.  Anything else is SPARSELNR_ERR_UNSUPPORTED.  R < 2^24, T < 2^28,
 *     T * Hq < 2^31, W * page_size <= 2^31 - 4096; a seq_len past that of its table's
 *     row ends there.
 *   - R = 0 or T = 0 is a no-op, but for sparselnr_page_tables.
 *   - The two attention calls use a workspace per (device, stream) for the results of
 *     contexts that are cut into pieces.  It has one size for all of them, whatever
 *     their tokens, lengths, heads, hint, type and dim are (130 MB on 256 compute
 *     units): a stream's first such call allocates it, later ones and captured graphs find it.
 *     sparselnr_block_attention of many tokens (four and more per page of
 *     the table, on average) goes by pages and has another workspace instead: its partial
 *     results, at most 144 MB, and lists, which grow with T, R, W, top and the heads.
 *     A capture of such a call needs one before, and while the graph may be
 *     replayed no call by pages on that stream may be larger.
 * ---------------------------------------------------------------------- */

enum sparselnr_dtype { SPARSELNR_BF16 = 0, SPARSELNR_FP16 = 1, SPARSELNR_FP32 = 2 };

#define SPARSELNR_MAX_PAGE 4096

/* The cache: K and V rows of dim values for every page, place and KV head. */
typedef struct sparselnr_kv_cache {
  void *k, *v;
  int64_t pages, page_size, heads, dim;
  int64_t k_page, k_slot, k_head; /* strides of K, in values */
  int64_t v_page, v_slot, v_head; /* strides of V */
  int32_t dtype;                  /* sparselnr_dtype, of q, k, v and out too */
} sparselnr_kv_cache;

/* The requests of a call. */
typedef struct sparselnr_requests {
  const int32_t *table; /* [R][W], rows table_stride apart */
  int64_t table_stride;
  const int32_t *seq_len; /* [R] positions, new tokens included */
  const int32_t *qptr;    /* [R + 1] */
  int64_t R, W, T;        /* T: rows of q */
} sparselnr_requests;

/*
 * Block tables and slots from the request lengths: request r has ctx_len[r]
 * cached and new_len[r] new tokens (negative lengths count as none).  Writes
 *   qptr[r]     = sum of new_len before r          (R + 1 entries)
 *   seq_len[r]  = ctx_len[r] + new_len[r]
 *   table[r][j] for the pages j that the new tokens begin, handed out of
 *               free_pages[0 .. F) in the order of requests and positions; -1 where
 *               the list is used up.  Entries from W on do not exist.  A negative entry
 *               of the list is no page (so a list of fixed length can be filled up).
 *   slots[t]    = page * page_size + place of new token t, -1 if it has no page;
 *               T >= qptr[R] entries, those from qptr[R] on -1
 *   counts      = { qptr[R], pages wanted, tokens without a page }
 * counts[1] is what the free list goes forward by (if it is at most F); a
 * counts[2] above zero tells that F or W was too small.  A counts[0] above T
 * tells that T was: tokens from T on get no slot and enter no page into the table, but
 * counts[1] holds their pages, and counts[2] only those of them that found none.
 * qptr and counts are written for R = 0 and T = 0 too.  The sums have to stay below 2^31.
 */
SPARSELNR_API int sparselnr_page_tables(const int32_t *ctx_len, const int32_t *new_len, int32_t *table,
                                        int64_t table_stride, const int32_t *free_pages, int32_t *qptr,
                                        int32_t *seq_len, int64_t *slots, int32_t *counts, int64_t R,
                                        int64_t W, int64_t F, int64_t T, int64_t page_size,
                                        void *stream);

/*
 * Writes the new tokens' K and V rows (T x Hkv x dim, strides in values) into
 * their slots; slots outside the cache are left out.  With kq (int8
 * [pages][Hkv][dim]) and kscale (float [pages][Hkv]), renews the summaries of the
 * pages written to: m = mean of the page's K rows up to the last one written (sum in
 * 64 bits, rounded once to 32), step = max|m| * s, s = 1/127 in 32 bits, kq = m / step rounded to the nearest
 * whole number (ties to even), kscale = step; 0 and 0 for a mean of zeros, 0 and
 * +inf if the mean is not finite.  Slots of one page have to be adjacent in `slots` and
 * ascending, without gaps, as sparselnr_page_tables gives them; no slot may occur twice.
 */
SPARSELNR_API int sparselnr_cache_append(const void *k, int64_t k_token, int64_t k_head,
                                         const void *v, int64_t v_token, int64_t v_head,
                                         const int64_t *slots, const sparselnr_kv_cache *cache,
                                         int8_t *kq, float *kscale, int64_t T, void *stream);

/*
 * Attention of the new tokens over their requests' cached rows, causal: the
 * query at position p sees the keys j <= p, and of those only j > p - window if
 * window > 0.
 *   out(t, h) = sum_j softmax_j(scale * q(t, h).k(j)) v(j),
 *   lse(t, h) = log sum_j exp(scale * q(t, h).k(j))
 * q: T x Hq x dim with strides; out: T x Hq x dim, packed; lse: float T x Hq or
 * NULL.  scale > 0.  max_new > 0 is a hint: no request has more new tokens (0:
 * not known); it chooses kernels, and results stay right if it is wrong.
 */
SPARSELNR_API int sparselnr_paged_attention(const void *q, int64_t q_token, int64_t q_head,
                                            int64_t Hq, const sparselnr_kv_cache *cache,
                                            const sparselnr_requests *requests, double scale,
                                            int64_t window, int64_t max_new, void *out, float *lse,
                                            void *stream);

/*
 * The `top` pages (at most 256) that each new token attends, per KV head, by a
 * cheap score of the pages b <= p / page_size of its request:
 *   u = sum of the group's query heads (in 64 bits, rounded once to 32),
 *   q8 = u / (max|u| * s) rounded to the nearest whole number (0 if u is zero or not finite),
 *   score(b) = float(sum_d q8(d) kq(page, d)) * kscale(page)
 * The sum is a whole number below 2^24, so scores are exact up to one rounding
 * and do not depend on any order.  The first `first` and the last `local` of those
 * pages are always taken (first + local <= top); the others by score, NaN before every
 * number, equal scores by the lower index.  Pages that are not there are never
 * taken.  sel: int32 [T][Hkv][top], indices into the request's table row, ascending,
 * with -1 behind them where there are fewer.
 */
SPARSELNR_API int sparselnr_block_select(const void *q, int64_t q_token, int64_t q_head, int64_t Hq,
                                         int32_t dtype, const int8_t *kq, const float *kscale,
                                         int64_t pages, int64_t page_size, int64_t Hkv, int64_t dim,
                                         const sparselnr_requests *requests, int64_t top,
                                         int64_t first, int64_t local, int32_t *sel, void *stream);

/*
 * Attention of each new token over its selected pages only: as
 * sparselnr_paged_attention, with the keys j <= p of the pages sel[t][h / (Hq / Hkv)][:].
 * Entries outside the table's row are skipped; a page that is named twice counts
 * twice.  top * page_size < 2^29.
 */
SPARSELNR_API int sparselnr_block_attention(const void *q, int64_t q_token, int64_t q_head,
                                            int64_t Hq, const sparselnr_kv_cache *cache,
                                            const sparselnr_requests *requests, const int32_t *sel,
                                            int64_t top, double scale, void *out, float *lse,
                                            void *stream);

/* ------------------------------------------------------------------------
 * A cache in 4 bits.
 *
 * The same pages, slots and block tables, with rows of 17 * NG bytes (17/64 of 16-bit rows where
 * dim is a multiple of 32): a row of dim values is NG = ceil(dim / 32) groups of 32, the last one filled up with
 * zeros.  A group has 16 bytes, two values each, the first in the low half: a sign
 * (8) and 0..7 for 0, 0.5, 1, 1.5, 2, 3, 4, 6.  It has one more byte e + 127 elsewhere: its values are
 * multiplied by 2^e.  255 stands for a group that is NaN.  (The public formats E2M1
 * and E8M0 of microscaled numbers.)
 *
 * Conventions as above, and:
 *   - e is the least whole number with max|x| <= 7 * 2^e of the group, at least -125 and at
 *     most 125 in bf16 and fp32, -23 and 13 in fp16, so that what a group stands for are values of
 *     the type it came from.  A value is rounded to the nearest, ties to an even code, and
 *     is off by at most 2^e (0.25, 0.5 or 1 times 2^e by its size), but for values above 7 times 2 to the
 *     largest e, which become 6 times that.  So in bf16 and fp32 a group of values up to 2^-127 becomes
 *     zeros.  A group with an infinity or a NaN is NaN.
 *   - Strides are in bytes; those of k and v keep rows at multiples of 16 bytes, those of the
 *     exponents may be any.  The 16 * NG bytes of a row, and its NG exponents, are adjacent.
 *     Heads before places in memory (a head's rows of a page adjacent) is the faster order.
 *   - dtype is that of the rows that are written and of q and out.  A cache is read in the type
 *     that it was written in: bf16 and fp32 have the same exponents, fp16 has fewer.
 *   - sparselnr_paged_attention_fp4 uses the workspace of sparselnr_paged_attention.
 * ---------------------------------------------------------------------- */

typedef struct sparselnr_fp4_cache {
  void *k, *v;             /* 16 * NG bytes for every page, place and KV head */
  void *k_scale, *v_scale; /* NG bytes for each */
  int64_t pages, page_size, heads, dim;
  int64_t k_page, k_slot, k_head; /* strides, in bytes */
  int64_t v_page, v_slot, v_head;
  int64_t ks_page, ks_slot, ks_head; /* of k_scale */
  int64_t vs_page, vs_slot, vs_head; /* of v_scale */
  int32_t dtype;                     /* sparselnr_dtype, of k, v, q and out outside the cache */
} sparselnr_fp4_cache;

/*
 * Writes the new tokens' K and V rows (T x Hkv x dim of dtype, strides in values) into
 * their slots in 4 bits; slots outside the cache are left out, and no slot may occur twice.
 */
SPARSELNR_API int sparselnr_cache_append_fp4(const void *k, int64_t k_token, int64_t k_head,
                                             const void *v, int64_t v_token, int64_t v_head,
                                             const int64_t *slots, const sparselnr_fp4_cache *cache,
                                             int64_t T, void *stream);

/*
 * What the rows of T slots stand for, as values of dtype: k and v are T x Hkv x dim, packed.
 * Zeros for slots outside the cache; a slot may occur any number of times.
 */
SPARSELNR_API int sparselnr_cache_read_fp4(const int64_t *slots, const sparselnr_fp4_cache *cache,
                                           void *k, void *v, int64_t T, void *stream);

/*
 * As sparselnr_paged_attention, over a cache in 4 bits.  q.k is computed on its bytes: a query's
 * groups of 32 values are written as sums of 6-bit pieces, exact to 2^-18 of the group's largest
 * value for fp16, to 2^-13 for bf16 (2^-18 if lse is asked for, and for requests of at most 64 tokens times query
 * heads to a KV head), to 2^-23 for fp32 (or to 2^-128 where that is more), and summed in fp32 (q * scale is taken
 * in fp32 and has to be finite there).  So what is left of small channels goes by the largest one of their group.
 * V is exact; the weights are rounded to the type of q, in fp32 to 24 bits.
 */
SPARSELNR_API int sparselnr_paged_attention_fp4(const void *q, int64_t q_token, int64_t q_head,
                                                int64_t Hq, const sparselnr_fp4_cache *cache,
                                                const sparselnr_requests *requests, double scale,
                                                int64_t window, int64_t max_new, void *out,
                                                float *lse, void *stream);

/* ------------------------------------------------------------------------
 * The pages' life: rows of the block table that share pages, rows given up, pages
 * moved to the front, and copies.
 *
 * shares (int32 [pages]) counts the rows that hold a page beyond the first: 0 for a
 * page of one row and for a free one.  So a program whose rows never share anything
 * passes zeros, and sparselnr_page_tables, which hands out pages, need not know of it.
 * Only pages that are full are ever shared, so rows that share pages never write to them (a program that makes
 * a row shorter has to leave it its shared pages).
 *
 * Conventions as above, and:
 *   - seq_len[r] (int32 [R]) is the length of row r; its pages are the first
 *     ceil(seq_len[r] / page_size) entries of its row of the table, at most W.  What
 *     lies behind them counts for nothing.  Entries outside [0, pages) are no pages.
 *   - Whatever the arrays on the device hold, no call reads or writes outside them, and
 *     results do not depend on the order in which the device works.
 *   - sparselnr_page_free and sparselnr_page_compact use a workspace per (device, stream) that
 *     grows with `pages` alone (256 KB and 12 bytes for 64 pages).  A capture of either needs one call
 *     of the same sizes before it, and while the graph may be replayed no such call on that stream may
 *     have more pages.
 * ---------------------------------------------------------------------- */

/*
 * Row children[i] of the table becomes a continuation of row parents[i], i < n: the
 * parent's full pages are shared (shares + 1 each), and where its last page is not full
 * the child gets a page of its own from free_pages, in the order of i; the rest of the child's
 * row is -1.  seq_len[child] becomes the parent's.  pairs[i] (int32 [n][2]) = { the
 * parent's last page, the child's }, which sparselnr_page_copy copies, or { -1, -1 }.
 *   counts = { pages taken from the list, forks among them that found none }
 * A fork that finds no page (the list is used up, or its entry is no page) has -1 there: its child
 * does not see those positions.  counts[0] is what the free list goes forward by, if it is at most F.
 * Forks whose parent or child is no row, or whose child is its parent, are left out.
 * A child's row must hold nothing (what it held is forgotten, not freed), may occur
 * once, and may not be a parent in the same call.
 */
SPARSELNR_API int sparselnr_page_fork(const int32_t *parents, const int32_t *children,
                                      int32_t *table, int64_t table_stride, int32_t *seq_len,
                                      int32_t *shares, const int32_t *free_pages, int32_t *pairs,
                                      int32_t *counts, int64_t n, int64_t R, int64_t W, int64_t F,
                                      int64_t pages, int64_t page_size, void *stream);

/*
 * Gives up the rows rows[i], i < n: their entries become -1 and their seq_len 0.  A
 * page that another row shares loses one of its shares; one that no other row holds is freed.
 *   freed (int32 [most]): the freed pages, ascending, -1 behind them
 *   counts = { pages freed, entries given up (2^31 - 1 if there are more) }
 * A row that occurs twice is given up once; numbers that are no rows are left out.  Pages
 * beyond `most` are freed but not listed (counts[0] tells).  min(pages, n * W) is always enough.
 */
SPARSELNR_API int sparselnr_page_free(const int32_t *rows, int32_t *table, int64_t table_stride,
                                      int32_t *seq_len, int32_t *shares, int32_t *freed,
                                      int32_t *counts, int64_t n, int64_t R, int64_t W, int64_t most,
                                      int64_t pages, int64_t page_size, void *stream);

/*
 * Moves the pages that rows hold to the front: of `used` pages in use the k-th one (ascending)
 * at or behind page `used` goes to the k-th free page before it.  Table and shares
 * follow at once; the contents do with sparselnr_page_copy on the pairs, before anything else
 * is written to the cache.  Afterwards the pages from `used` on are free, and all that are.
 *   pairs (int32 [pages / 2][2]): { from, to }, -1 behind them
 *   counts = { pages in use, pages moved }
 */
SPARSELNR_API int sparselnr_page_compact(int32_t *table, int64_t table_stride, const int32_t *seq_len,
                                         int32_t *shares, int32_t *pairs, int32_t *counts, int64_t R,
                                         int64_t W, int64_t pages, int64_t page_size, void *stream);

/* An array whose first dimension is the page.  Page p is outer * inner rows of `row` adjacent
 * bytes, row (i, j) at data + p * page + i * outer_stride + j * inner_stride.  All in bytes. */
typedef struct sparselnr_page_array {
  void *data;
  int64_t page, outer, outer_stride, inner, inner_stride, row;
} sparselnr_page_array;

/*
 * Copies page pairs[i][0] to page pairs[i][1], i < n, in each of `count` arrays (at most 8; a
 * host array): caches of any type and order, their summaries or exponents.  Pairs with an entry outside
 * [0, pages) are left out.  A page that is copied to may not occur in another pair.
 */
SPARSELNR_API int sparselnr_page_copy(const int32_t *pairs, int64_t n, const sparselnr_page_array *arrays,
                                      int64_t count, int64_t pages, void *stream);

/* Static text for a status code (never NULL). */
SPARSELNR_API const char *sparselnr_status_string(int status);

/* hipError_t of the last failing HIP call made by this library on the
 * calling thread (0 if none). */
SPARSELNR_API int sparselnr_last_hip_error(void);

/*
 * Launch tuning (no counterpart in the paper, which fixes no GPU launch).
 * Every walk launch runs `factor` resident grids of workers, each worker
 * taking one merge-path slice of rows + nonzeros, so a larger factor gives
 * more, shorter slices: the workers resident at one moment then cover a
 * narrower band of rows, which changes how D and E rows are shared in the
 * caches.  factor 0 restores the automatic choice (by the number of rows per
 * resident worker and the widths; 1 for small matrices; several waves may share
 * a slice of wide rows then).  Where rows have a few nonzeros the device makes
 * fewer, longer slices than there are workers.  1..64 fixes the factor for every
 * later call in the process, on every device and stream (the environment
 * variable SPARSELNR_GRID_FACTOR gives the first value).  Results are
 * deterministic for a fixed factor; another factor splits rows between slices
 * elsewhere and so changes the fp32 summation order (within the accuracy
 * stated for each entry point).  The carry workspace grows with the number
 * of workers: 2 * L floats per worker.  Launches already made are not
 * affected.  Returns SPARSELNR_OK, or SPARSELNR_ERR_INVALID_ARG for a factor
 * outside 0..64.
 */
SPARSELNR_API int sparselnr_set_grid_factor(int factor);

/* The factor fixed by sparselnr_set_grid_factor or SPARSELNR_GRID_FACTOR,
 * or 0 when it is chosen per call. */
SPARSELNR_API int sparselnr_get_grid_factor(void);

/* Waits for the device(s) and frees every workspace the library allocated.
 * Safe to call at any time that no other thread is inside a call of the sparse
 * products; later calls allocate again. */
SPARSELNR_API int sparselnr_release(void);

#ifdef __cplusplus
} /* extern "C" */
#endif

#endif /* SPARSELNR_H */
