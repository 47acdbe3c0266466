// Entry points of the pages' life: argument checks and launches.  The C ABI is declared in
// include/sparselnr.h.
#include "life.hpp"

#include "checks.hpp"

namespace {

using namespace slnr;
using namespace slnr::paged;


// Blocks for `n` things of a thread each, at most `most`.
unsigned blocks_for(int64_t n, int64_t most) {
  const int64_t b = (n + kLifeBlock - 1) / kLifeBlock;
  return (unsigned)(b < 1 ? 1 : b > most ? most : b);
}

int check_table(const int32_t *table, int64_t table_stride, const int32_t *seq_len, const int32_t *shares, int64_t R,
                int64_t W, int64_t pages, int64_t page_size) {
  if (R < 0 || W < 0 || pages < 0 || table_stride < 0) return SPARSELNR_ERR_INVALID_ARG;
  if ((R > 0 && !seq_len) || (R > 0 && W > 0 && !table) || (pages > 0 && !shares) || (R > 1 && table_stride < W))
    return SPARSELNR_ERR_INVALID_ARG;
  if (page_shift(page_size) < 0 || R >= ((int64_t)1 << 24) || pages > kMax31 || W > kMaxPositions / page_size)
    return SPARSELNR_ERR_UNSUPPORTED;
  return SPARSELNR_OK;
}

constexpr int64_t kMostRowBlocks = 8192, kMostRowParts = 8;

// The marks of the pages and, behind them, a number for each word or for each block of rows.  Its size goes by
// the pages alone: a captured graph holds its address, so a call of more rows may not have to grow it.
int life_workspace(const Launch &l, LifeArgs &a, HeldWorkspace *ws) {
  const size_t marks = (size_t)(a.words < 1 ? 1 : a.words) * sizeof(Word);
  const int64_t numbers = a.words > kMostRowBlocks * kMostRowParts ? a.words : kMostRowBlocks * kMostRowParts;
  const int rc = hold_workspace(l.dev, l.stream, marks + (size_t)numbers * sizeof(int32_t), kSlotLife, ws);
  if (rc != SPARSELNR_OK) return rc;
  a.marks = (Word *)ws->ptr;
  a.before = a.given = (int32_t *)((char *)ws->ptr + marks);
  return SPARSELNR_OK;
}

// One block does it all where the entries and an eighth of the pages are no more than 4096.  Time on the GPU in
// us, one block | several launches, free and compact, for entries of pages: 256 of 2048 4.0 | 8.6 and
// 4.3 | 9.5; 2048 of 4096 6.7 | 9.1 and 6.4 | 11.0; 4096 of 8192 11.1 | 9.7 and 9.7 | 11.9; 8192 of 16384 19.9 | 10.1
// and 17.2 | 12.4; 256 of 65536 10.9 | 9.5 and 16.4 | 11.2.
constexpr int64_t kOneMost = 4096;
static_assert(kOneMost * 8 <= kOneBlock * (int64_t)64, "a thread has a word of marks");

bool one_block(const LifeArgs &a, int64_t rows) { return rows * a.W + a.pages / 8 <= kOneMost; }

// Rows along x, up to eight blocks to a long one.
dim3 grid_of_rows(int64_t rows, int64_t W) {
  return dim3((unsigned)(rows < 1 ? 1 : rows > kMostRowBlocks ? kMostRowBlocks : rows), blocks_for(W, kMostRowParts));
}

// Blocks that go through the marks, 16 words each; each of them counts all marks before its own.  For 121796 pages 8.8 us,
// with 64 words a block 9.9.
unsigned grid_of_words(const LifeArgs &a) {
  const int64_t b = (a.words + 15) / 16;
  return (unsigned)(b < 1 ? 1 : b > 512 ? 512 : b);
}

}  // namespace

extern "C" {

int sparselnr_page_fork(const int32_t *parents, const int32_t *children, int32_t *table, int64_t table_stride,
                        int32_t *seq_len, int32_t *shares, const int32_t *free_pages, int32_t *pairs, int32_t *counts,
                        int64_t n, int64_t R, int64_t W, int64_t F, int64_t pages, int64_t page_size, void *stream) {
  if (n < 0 || F < 0) return SPARSELNR_ERR_INVALID_ARG;
  const int rc = check_table(table, table_stride, seq_len, shares, R, W, pages, page_size);
  if (rc != SPARSELNR_OK) return rc;
  if (!counts || (n > 0 && (!parents || !children || !pairs)) || (F > 0 && !free_pages)) return SPARSELNR_ERR_INVALID_ARG;
  if (n >= ((int64_t)1 << 24) || F > kMax31) return SPARSELNR_ERR_UNSUPPORTED;
  ForkArgs a{};
  a.parents = parents, a.children = children;
  a.table = table, a.table_row = table_stride;
  a.seq = seq_len, a.shares = shares;
  a.free_pages = free_pages;
  a.pairs = pairs, a.counts = counts;
  a.n = (int32_t)n, a.R = (int32_t)R, a.W = (int32_t)W, a.F = (int32_t)F, a.pages = (int32_t)pages;
  a.shift = page_shift(page_size);
  // every block counts the forks before its own
  const int64_t per = (n + 2047) / 2048 > 0 ? (n + 2047) / 2048 : 1;
  const unsigned blocks = (unsigned)(n > 0 ? (n + per - 1) / per : 1);
  // a long row is copied by several blocks, 1024 entries each: 8 forks of 8192 pages 5.2 us, by one block each 14.6, of
  // 65536 7.1 and 90; 2000 of 600 45 either way, with 256 entries a block 69
  const unsigned parts = blocks_for((W + 3) / 4, 32);
  hipLaunchKernelGGL(page_fork, dim3(blocks, parts), dim3(kLifeBlock), 0, (hipStream_t)stream, a, (int)per);
  return launched();
}

int sparselnr_page_free(const int32_t *rows, int32_t *table, int64_t table_stride, int32_t *seq_len, int32_t *shares,
                        int32_t *freed, int32_t *counts, int64_t n, int64_t R, int64_t W, int64_t most, int64_t pages,
                        int64_t page_size, void *stream) {
  if (n < 0 || most < 0) return SPARSELNR_ERR_INVALID_ARG;
  int rc = check_table(table, table_stride, seq_len, shares, R, W, pages, page_size);
  if (rc != SPARSELNR_OK) return rc;
  if (!counts || (n > 0 && !rows) || (most > 0 && !freed)) return SPARSELNR_ERR_INVALID_ARG;
  if (n >= ((int64_t)1 << 24) || most > kMax31) return SPARSELNR_ERR_UNSUPPORTED;
  LifeArgs a{};
  a.rows = rows;
  a.table = table, a.table_row = table_stride;
  a.seq = seq_len, a.shares = shares;
  a.out = freed, a.counts = counts;
  a.n = (int32_t)n, a.R = (int32_t)R, a.W = (int32_t)W, a.pages = (int32_t)pages, a.most = (int32_t)most;
  a.shift = page_shift(page_size);
  a.words = (pages + 63) / 64;
  if (one_block(a, n)) {
    hipLaunchKernelGGL(page_free_one, dim3(1), dim3(kOneBlock), 0, (hipStream_t)stream, a);
    return launched();
  }
  Launch l;
  if ((rc = current(&l, stream)) != SPARSELNR_OK) return rc;
  const dim3 block(kLifeBlock), rows_grid = grid_of_rows(n, W);
  const int blocks = (int)(rows_grid.x * rows_grid.y);
  HeldWorkspace ws;
  if ((rc = life_workspace(l, a, &ws)) != SPARSELNR_OK) return rc;
  hipLaunchKernelGGL(life_clear, dim3(blocks_for(most > a.words ? most : a.words, 1024)), block, 0, l.stream, a, most);
  if ((rc = launched()) != SPARSELNR_OK) return rc;
  hipLaunchKernelGGL(page_free_rows, rows_grid, block, 0, l.stream, a);
  if ((rc = launched()) != SPARSELNR_OK) return rc;
  hipLaunchKernelGGL(page_free_list, dim3(grid_of_words(a)), block, 0, l.stream, a, blocks);
  return launched();
}

int sparselnr_page_compact(int32_t *table, int64_t table_stride, const int32_t *seq_len, int32_t *shares,
                           int32_t *pairs, int32_t *counts, int64_t R, int64_t W, int64_t pages, int64_t page_size,
                           void *stream) {
  int rc = check_table(table, table_stride, seq_len, shares, R, W, pages, page_size);
  if (rc != SPARSELNR_OK) return rc;
  if (!counts || (pages > 1 && !pairs)) return SPARSELNR_ERR_INVALID_ARG;
  LifeArgs a{};
  a.table = table, a.table_row = table_stride;
  a.seq = const_cast<int32_t *>(seq_len), a.shares = shares;
  a.out = pairs, a.counts = counts;
  a.R = (int32_t)R, a.W = (int32_t)W, a.pages = (int32_t)pages, a.most = (int32_t)(pages / 2);
  a.shift = page_shift(page_size);
  a.words = (pages + 63) / 64;
  if (one_block(a, R)) {
    hipLaunchKernelGGL(page_compact_one, dim3(1), dim3(kOneBlock), 0, (hipStream_t)stream, a);
    return launched();
  }
  Launch l;
  if ((rc = current(&l, stream)) != SPARSELNR_OK) return rc;
  HeldWorkspace ws;
  if ((rc = life_workspace(l, a, &ws)) != SPARSELNR_OK) return rc;
  const dim3 block(kLifeBlock), rows = grid_of_rows(R, W);
  const int64_t outs = 2 * (int64_t)a.most;
  hipLaunchKernelGGL(life_clear, dim3(blocks_for(outs > a.words ? outs : a.words, 1024)), block, 0, l.stream, a, outs);
  if ((rc = launched()) != SPARSELNR_OK) return rc;
  hipLaunchKernelGGL(page_mark_used, rows, block, 0, l.stream, a);
  if ((rc = launched()) != SPARSELNR_OK) return rc;
  hipLaunchKernelGGL(page_compact_pairs, dim3(grid_of_words(a)), block, 0, l.stream, a);
  if ((rc = launched()) != SPARSELNR_OK) return rc;
  hipLaunchKernelGGL(page_compact_tables, rows, block, 0, l.stream, a);
  return launched();
}

int sparselnr_page_copy(const int32_t *pairs, int64_t n, const sparselnr_page_array *arrays, int64_t count,
                        int64_t pages, void *stream) {
  if (n < 0 || count < 0 || pages < 0 || (n > 0 && !pairs) || (count > 0 && !arrays)) return SPARSELNR_ERR_INVALID_ARG;
  if (count > kCopyArrays || n > kMax31 || pages > kMax31) return SPARSELNR_ERR_UNSUPPORTED;
  CopyArgs a{};
  int64_t steps = 0;
  for (int64_t k = 0; k < count; ++k) {
    const sparselnr_page_array &in = arrays[k];
    if (in.page < 0 || in.outer < 0 || in.inner < 0 || in.row < 0 || in.outer_stride < 0 || in.inner_stride < 0)
      return SPARSELNR_ERR_INVALID_ARG;
    if (in.outer == 0 || in.inner == 0 || in.row == 0 || pages == 0) continue;
    if (!in.data) return SPARSELNR_ERR_INVALID_ARG;
    if (in.outer > kMax31 || in.inner > kMax31 || in.row > kMax31 || in.outer * in.inner > (kMax31 << 10) / in.row)
      return SPARSELNR_ERR_UNSUPPORTED;
    CopyArray &x = a.array[a.arrays++];
    x.data = (uint8_t *)in.data;
    x.page = stride_of(in.page, pages);
    x.outer_stride = stride_of(in.outer_stride, in.outer), x.inner_stride = stride_of(in.inner_stride, in.inner);
    x.row = (unsigned)in.row, x.inner = (unsigned)in.inner;
    x.bytes = in.outer * in.inner * in.row;
    x.dense = (in.inner == 1 || x.inner_stride == in.row) && (in.outer == 1 || x.outer_stride == in.inner * in.row);
    const int64_t all = (int64_t)(uintptr_t)in.data | x.page | x.bytes |
                        (x.dense ? 0 : x.outer_stride | x.inner_stride | in.row);
    x.unit = all % 16 == 0 ? 16 : all % 4 == 0 ? 4 : 1;
    x.steps = (int)((x.bytes + kCopyBytes - 1) / kCopyBytes);
    steps += x.steps;
  }
  if (steps > kMax31) return SPARSELNR_ERR_UNSUPPORTED;
  if (n == 0 || a.arrays == 0) return SPARSELNR_OK;
  a.pairs = pairs;
  a.n = (int32_t)n, a.pages = (int32_t)pages, a.steps = (int32_t)steps;
  a.items = n * steps;
  Launch l;
  const int rc = current(&l, stream);
  if (rc != SPARSELNR_OK) return rc;
  const int64_t most = (int64_t)l.cus * 8;  // 697 MB: 136 us, with half as many 137, with twice as many 135
  hipLaunchKernelGGL(page_copy, dim3((unsigned)(a.items < most ? a.items : most)), dim3(kLifeBlock), 0, l.stream, a);
  return launched();
}

}  // extern "C"
