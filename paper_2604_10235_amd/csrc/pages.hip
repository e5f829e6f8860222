// Rows between dense caches and pages, and whole pages: copies of 16-byte pieces, bit for bit.  Bound by memory; K and V go together, since a
// row's two places are found once.  One piece of each in flight per thread and many threads are enough (two rows a thread: store 4.3 GB 742 -> 794
// us; whole pages, 350 MB, one piece 62, two 64, four 73), and stores go past the caches, which could not hold the rows until they are read (store 760 ->
// 740 us, pages 70 -> 64).
// Measured: 4.3 GB from dense rows into pages of 16 rows 750 us, 5.7 TB/s; 3.8 GB from pages into dense rows 647 us, 5.8; 236 MB of kept rows from pages to
// pages 44 us, 5.4; 350 MB of whole pages 63 us, 5.6.
#include "cache.h"

namespace codecomp {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kMoveThreads = 256;
constexpr int64_t kMostBlocks = (1 << 24) - 1;         // of 256 threads: an axis of a grid holds 2^32 threads

// Byte offset of a request's row; -1 where there is none.
template <bool PAGED>
__device__ __forceinline__ int64_t place(const RowSide& s, int r, int64_t row) {
  if constexpr (!PAGED) return ((int64_t)s.cu[r] + row) * s.s_tok;
  row += s.first ? s.first[r] : 0;
  if (row < 0 || (row >> s.page_log2) >= s.table_width) return -1;
  const int page = s.table[(int64_t)r * s.table_width + (row >> s.page_log2)];
  if (page < 0 || page >= s.n_pages) return -1;
  return page * s.s_page + (row & ((1 << s.page_log2) - 1)) * s.s_tok;
}

// blockIdx.x: rows of all requests, blockIdx.y: (layer, head).  Consecutive threads take the pieces of a row.
template <bool FROM_PAGES, bool TO_PAGES>
__global__ __launch_bounds__(kMoveThreads) void move_kernel(const MoveArgs a) {
  const int first = blockIdx.x * (kMoveThreads >> a.pieces_log2), row = first + (threadIdx.x >> a.pieces_log2);
  const int layer = blockIdx.y / a.Hkv, head = blockIdx.y - layer * a.Hkv;
  const int64_t in_row = (threadIdx.x & ((1 << a.pieces_log2) - 1)) * 16;
  int r = request_of(a.cu_rows, a.n_seqs, first);          // the rows of a workgroup walk forward from there
  if (row >= a.rows) return;
  while (r + 1 < a.n_seqs && a.cu_rows[r + 1] <= row) ++r;
  const int in_request = row - a.cu_rows[r];
  int64_t source = in_request;
  if (a.idx) source = min(max(a.idx[(int64_t)blockIdx.y * a.rows + row], 0), a.cu_source[r + 1] - a.cu_source[r] - 1);
  const int64_t from = place<FROM_PAGES>(a.from, r, source), to = place<TO_PAGES>(a.to, r, in_request);
  if (to < 0) return;
  u32x4 k = {0, 0, 0, 0}, v = {0, 0, 0, 0};
  if (from >= 0) {
    const int64_t at = layer * a.from.s_layer + head * a.from.s_head + in_row + from;
    k = *reinterpret_cast<const u32x4*>(a.from.k + at);
    v = *reinterpret_cast<const u32x4*>(a.from.v + at);
  }
  const int64_t at = layer * a.to.s_layer + head * a.to.s_head + in_row + to;
  __builtin_nontemporal_store(k, reinterpret_cast<u32x4*>(a.to.k + at));
  __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(a.to.v + at));
}

int launch_move(const MoveArgs& a, int problems, hipStream_t stream) {
  const int64_t per_block = kMoveThreads >> a.pieces_log2, blocks = (a.rows + per_block - 1) / per_block;
  if (blocks > kMostBlocks) return CODECOMP_EINVAL_SHAPE;
  const dim3 grid((unsigned)blocks, problems), block(kMoveThreads);
  if (a.from.table && a.to.table) move_kernel<true, true><<<grid, block, 0, stream>>>(a);
  else if (a.from.table) move_kernel<true, false><<<grid, block, 0, stream>>>(a);
  else move_kernel<false, true><<<grid, block, 0, stream>>>(a);
  return (int)hipGetLastError();
}

struct CopyArgs {
  PagePool pool;
  const int32_t* pairs;
  int blocks, pieces, row_log2, page_log2;      // workgroups per page, 16-byte pieces of a page, log2 of those of a row, of a head's rows
};

// blockIdx.x: pairs and shares of a page, blockIdx.y: layer.
__global__ __launch_bounds__(kMoveThreads) void copy_kernel(const CopyArgs a) {
  const int pair = blockIdx.x / a.blocks, share = blockIdx.x - pair * a.blocks;
  const int from = a.pairs[2 * (int64_t)pair], to = a.pairs[2 * (int64_t)pair + 1];
  if (from < 0 || from >= a.pool.n_pages || to < 0 || to >= a.pool.n_pages || from == to) return;
  const int64_t layer = blockIdx.y * a.pool.s_layer, source = layer + from * a.pool.s_page, target = layer + to * a.pool.s_page;
  const int piece = share * kMoveThreads + threadIdx.x;
  if (piece >= a.pieces) return;
  const int head = piece >> a.page_log2, row = (piece & ((1 << a.page_log2) - 1)) >> a.row_log2;
  const int64_t off = head * a.pool.s_head + row * a.pool.s_tok + (piece & ((1 << a.row_log2) - 1)) * 16;
  const u32x4 k = *reinterpret_cast<const u32x4*>(a.pool.k + source + off), v = *reinterpret_cast<const u32x4*>(a.pool.v + source + off);
  __builtin_nontemporal_store(k, reinterpret_cast<u32x4*>(a.pool.k + target + off));
  __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(a.pool.v + target + off));
}

int launch_pages_copy(const PagePool& pool, int L, int Hkv, int d, const int32_t* pairs, int n_pairs, hipStream_t stream) {
  CopyArgs a;
  a.pool = pool; a.pairs = pairs;
  a.row_log2 = (d == 128 ? 4 : 3) - (pool.fp8 ? 1 : 0);
  a.page_log2 = pool.page_log2 + a.row_log2;
  const int64_t pieces = (int64_t)Hkv << a.page_log2, per_block = kMoveThreads;
  if (pieces > INT32_MAX - per_block) return CODECOMP_EINVAL_SHAPE;
  a.pieces = (int)pieces;
  a.blocks = (int)((pieces + per_block - 1) / per_block);
  if ((int64_t)a.blocks * n_pairs > kMostBlocks) return CODECOMP_EINVAL_SHAPE;
  copy_kernel<<<dim3((unsigned)(a.blocks * n_pairs), L), dim3(kMoveThreads), 0, stream>>>(a);
  return (int)hipGetLastError();
}

}  // namespace codecomp
