// Eviction in place by summed attention weights (codecomp_evict): which rows stay, and their move together.
//
// Two kernels.  The first has a workgroup for each (layer, request, KV head): the sum that the last kept row has is found digit by digit from
// the top (counts of 8 bits of the ordered value at a time), then rows are gone through in order and their numbers written one behind the other, the sums along
// with them.  The second moves rows of K and V.  Row f + i comes from a row that is not before it, so a workgroup that goes through them in order, and has all
// rows of a batch in registers before it writes the first, needs no room elsewhere; K and V, and stretches of a row, do not meet and are different workgroups'.
#include "serve.h"

namespace codecomp {

constexpr int kMoveThreads = 256, kMoveDeep = 8;       // pieces of 16 bytes that a thread has in flight
constexpr int64_t kMostBlocks = (1 << 22) - 1;          // of up to 1024 threads: an axis of a grid holds 2^32 threads

struct Span { int f, n, m; };                            // rows [f, n) of a request, m of them kept
__device__ __forceinline__ Span span_of(const EvictArgs& a, int r) {
  Span s;
  s.n = min(max(a.kv_lens[r], 0), a.max_kv);
  s.f = a.first ? min(max(a.first[r], 0), s.n) : 0;
  s.m = min(s.n - s.f, min(max(a.budgets[r], a.recent), a.max_budget));
  return s;
}

// Floats as unsigned numbers of the same order; -0 as 0, NaN below all.
__device__ __forceinline__ unsigned ordered(float x) {
  const unsigned u = __float_as_uint(x + 0.0f);
  return x != x ? 0u : u & 0x80000000u ? ~u : u | 0x80000000u;
}

template <int THREADS>
__global__ __launch_bounds__(THREADS) void keep_kernel(const EvictArgs a) {
  constexpr int WAVES = THREADS / 64;
  __shared__ int counts[WAVES][256];
  __shared__ int found[2];
  __shared__ int2 strip[2][WAVES];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int problem = blockIdx.x, head = problem % a.Hkv, rest = problem / a.Hkv, r = rest % a.n_seqs, layer = rest / a.n_seqs;
  const Span s = span_of(a, r);
  if (tid == 0 && head == 0 && layer == 0) a.new_lens[r] = s.f + s.m;
  const float* sums = a.from.sums + layer * a.from.s_layer + r * a.from.s_seq + head * a.from.s_head;
  float* to = a.to.sums + layer * a.to.s_layer + r * a.to.s_seq + head * a.to.s_head + s.f;
  int32_t* kept = a.kept + (int64_t)problem * a.max_budget;
  const bool all = s.m == s.n - s.f;
  const int last = all ? s.f : s.n - a.recent;           // rows from there on stay
  unsigned border = all ? 0 : ~0u;                       // rows above it stay, and the first `equal` of those at it
  int equal = 0;
  if (!all && s.m > a.recent) {
    unsigned prefix = 0;
    int want = s.m - a.recent;
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = tid; i < WAVES * 256; i += THREADS) counts[i >> 8][i & 255] = 0;
      __syncthreads();
      for (int j = s.f + tid; j < last; j += THREADS) {
        const unsigned key = ordered(sums[j]);
        if (shift == 24 || key >> (shift + 8) == prefix) atomicAdd(&counts[wave][(key >> shift) & 255], 1);
      }
      __syncthreads();
      if (wave == 0) {                                   // four digits a lane, the largest first
        int of[4], mine = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          of[i] = 0;
#pragma unroll
          for (int w = 0; w < WAVES; ++w) of[i] += counts[w][255 - 4 * lane - i];
          mine += of[i];
        }
        int before = mine;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
          const int y = __shfl_up(before, off);
          if (lane >= off) before += y;
        }
        before -= mine;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (before < want && want <= before + of[i]) { found[0] = 255 - 4 * lane - i; found[1] = want - before; }
          before += of[i];
        }
      }
      __syncthreads();
      prefix = prefix << 8 | (unsigned)found[0];
      want = found[1];
    }
    border = prefix;
    equal = want;
  }
  int above = 0, at_border = 0;                          // rows before this strip
  for (int first = s.f, turn = 0; first < s.n; first += THREADS, turn ^= 1) {
    const int j = first + tid;
    const bool there = j < s.n;
    const float x = there ? sums[j] : 0.0f;
    const unsigned key = ordered(x);
    const bool more = there && (j >= last || key > border), same = there && j < last && key == border;
    const uint64_t more_mask = __ballot(more), same_mask = __ballot(same);
    if (lane == 0) strip[turn][wave] = make_int2(__popcll(more_mask), __popcll(same_mask));
    __syncthreads();                                     // all sums of the strip have been read
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    int m = above + __popcll(more_mask & below), e = at_border + __popcll(same_mask & below);
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const int2 c = strip[turn][w];
      if (w < wave) { m += c.x; e += c.y; }
      above += c.x; at_border += c.y;
    }
    if (more || (same && e < equal)) {
      const int i = m + min(e, equal);
      kept[i] = j;
      to[i] = x;
    }
  }
  for (int i = s.m + tid; i < a.max_budget; i += THREADS) kept[i] = -1;
}

// PIECES: 16-byte pieces of a row that a workgroup moves.
template <int PIECES>
__global__ __launch_bounds__(kMoveThreads) void close_up_kernel(const EvictArgs a, int slices) {
  constexpr int ROWS = kMoveThreads / PIECES;
  const int tid = threadIdx.x, part = blockIdx.x % (2 * slices), problem = blockIdx.x / (2 * slices);
  const int head = problem % a.Hkv, rest = problem / a.Hkv, r = rest % a.n_seqs, layer = rest / a.n_seqs;
  const Span s = span_of(a, r);
  if (s.m == s.n - s.f) return;
  unsigned char* base = (part & 1 ? a.pool.v : a.pool.k) + layer * a.pool.s_layer + head * a.pool.s_head + ((part >> 1) * PIECES + tid % PIECES) * 16;
  const int32_t* kept = a.kept + (int64_t)problem * a.max_budget;
  const int32_t* table = a.table + (int64_t)r * a.table_width;
  const int in_page = (1 << a.pool.page_log2) - 1;
  auto place = [&](int row) __attribute__((always_inline)) {
    const int page = table[row >> a.pool.page_log2];
    return page < 0 || page >= a.pool.n_pages ? (int64_t)-1 : page * a.pool.s_page + (row & in_page) * a.pool.s_tok;
  };
  for (int first = 0; first < s.m; first += ROWS * kMoveDeep) {
    u32x4 x[kMoveDeep];
    int64_t to[kMoveDeep];
#pragma unroll
    for (int u = 0; u < kMoveDeep; ++u) {
      const int i = first + u * ROWS + tid / PIECES;
      to[u] = -1;
      x[u] = u32x4{0, 0, 0, 0};
      if (i < s.m) {
        const int row = kept[i];
        if (row != s.f + i) {                            // else it stays where it is
          const int64_t from = place(row);
          to[u] = place(s.f + i);
          if (from >= 0) x[u] = *reinterpret_cast<const u32x4*>(base + from);
        }
      }
    }
    // All rows of the batch are in registers before one is overwritten; rows of later batches lie behind those that this one writes.
    asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
    for (int u = 0; u < kMoveDeep; ++u)
      if (to[u] >= 0) __builtin_nontemporal_store(x[u], reinterpret_cast<u32x4*>(base + to[u]));
  }
}

int launch_evict(const EvictArgs& a, int d, hipStream_t stream) {
  const int64_t problems = (int64_t)a.n_layers * a.n_seqs * a.Hkv;
  const int pieces = d * (a.pool.fp8 ? 1 : 2) / 16;
  int slices = 1;
  while (slices < pieces / 4 && problems * 2 * slices < 1024) slices *= 2;
  if (problems * 2 * slices > kMostBlocks) return CODECOMP_EINVAL_SHAPE;
  if (a.max_kv > 4096) keep_kernel<1024><<<dim3((unsigned)problems), dim3(1024), 0, stream>>>(a);
  else keep_kernel<256><<<dim3((unsigned)problems), dim3(256), 0, stream>>>(a);
  if (hipError_t e = hipGetLastError()) return (int)e;
  const dim3 grid((unsigned)(problems * 2 * slices)), block(kMoveThreads);
  switch (pieces / slices) {
    case 16: close_up_kernel<16><<<grid, block, 0, stream>>>(a, slices); break;
    case 8: close_up_kernel<8><<<grid, block, 0, stream>>>(a, slices); break;
    default: close_up_kernel<4><<<grid, block, 0, stream>>>(a, slices); break;
  }
  return (int)hipGetLastError();
}

}  // namespace codecomp
