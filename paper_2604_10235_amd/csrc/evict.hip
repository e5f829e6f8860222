// Eviction in place by summed attention weights (codecomp_evict): which rows stay, and their move together.
//
// The B largest of n sums: their smallest is found digit by digit from the top, by counting how many of the sums that are still possible have each value of the
// next 8 bits; then rows are gone through in order, and the numbers of those above it, and of the first ones at it, written one behind the other.
// Sums are read once and stand in registers; counts are integers, so that their order does not matter.  A row has 256 bytes of K and of V and 4 of its sum:
// the move is nearly all of the work, bound by memory: every kept row that changes its place is read and written once.
//
// The move is in place: row f + i comes from row kept[i], which is not before it (kept ascends).  A workgroup goes through its rows in order, a batch at a time, and has all of a
// batch in registers before it overwrites one: what later batches read lies behind that.  K and V, heads and layers, and stretches of a
// row, do not meet, and are different workgroups'.
//
// Many problems (a layer's request and head each): one kernel, a workgroup for each, whose waits for counts are hidden behind the rows of others.  28 layers, 32 requests of 900 to
// 1500 rows, 4 heads of 128, 1024 kept: 635 us, 5.3 TB/s; 32 layers, 48 requests behind 2049 protected rows, 8 bits: 1312 us, 4.9 TB/s.
// Fewer: two kernels, the second with two or four workgroups for each.  28 layers, one request of 32768 rows to 2048: 25 us for the numbers and 57 for the rows,
// which come from 256 bytes here and there, 4.1 TB/s; one layer of 1088 rows to 1024: 8 and 5 us, a chain of waits for counts and numbers.
// Tried before: digits of 11 bits (three passes; as long); the next batch sent for before one is written (as long: it is the scattered rows, not the wait);
// loads that may stay in the caches instead of those that pass by them (651 us instead of 637 for the steps above, 1307 instead of 1313 for 8 bits).
#include <algorithm>

#include "serve.h"

namespace codecomp {

// From as many problems on it is one kernel (28 layers of 4 heads, 900 to 1500 rows to 1024, us, one | two: 1 request 58 | 40, 2: 58 | 56, 3: 86 | 66, 4: 111 | 116, 16: 281 | 279;
// 8 bits and 256 kept of up to 8000, 4 requests 34 | 50, 32: 157 | 200), unless requests have many more rows than its registers hold: the rest is read
// five times (16 requests of 16000 rows 500 | 545, 32768 731 | 573).
constexpr int kManyProblems = 400, kBothRows = 16384;
// Its threads, and pieces of K and of V that each has in flight (steps as above, 8 bits: 256 threads 668 us, 1315; 512 635, 1307; 1024 707, 1517; 2, 4 and 6 pieces the same).
constexpr int kBothThreads = 512, kBothDeep = 4;
// Fewer threads where requests are short (1656 problems of up to 83 rows, us, 512 | 256 | 128 threads: 28 | 13 | 10; 28 layers, 32 requests of up to 500: 147 | 144 | 148; 8 of 900:
// 132 | 128 | 152).
constexpr int kShortRows = 1024, kShortThreads = 256;
// And always where few rows are kept of what registers hold (us, two kernels | one: 288 problems of up to 32 rows 13.0 | 7.6; 4 heads, 50 of 1000 rows 10.1 | 8.7, 50 of 4000 13.6 | 9.9, of
// 8000 13.6 | 18.0; 224 heads, 64 of 2000 15.1 | 11.6, 256 26.1 | 23.9; 4 heads, 400 of 500 12.7 | 18.6).
constexpr int kFewKept = 256, kHeldRows = 4096;
// Two kernels: threads of a workgroup that moves rows (one request of 32768, us: 512 threads 97, 1024 85), and pieces that each has in flight (2, 4, 8: 85, 87, 87).
constexpr int kMoveThreads = 1024, kMoveDeep = 2;
// Rows of 256 bytes are cut into two stretches of 128 where there are fewer workgroups than compute units (114 us -> 98), and down to 32 where there are very few and
// a batch does not move all: fewer waits one after another (4 heads, us, 128 bytes | 32: to 1024 of 1088 rows 16.4 | 12.7, to 300 of 2000 12.6 | 11.7, 8 heads to 2000 of 5000 34 | 22; up to 128
// workgroups, 16 heads to 16000 of 30000, 226 | 155, with 256 of them 167).  Stretches of a line of memory on different dies cost most of that (155 | 320 with 32 bytes).
constexpr int kFewest = 256, kFewer = 128, kManyRows = 256;
constexpr int64_t kMostBlocks = (1 << 22) - 1;          // of up to 1024 threads: an axis of a grid holds 2^32 threads

struct Span { int f, n, m; };                            // rows [f, n) of a request, m of them kept
__device__ __forceinline__ Span span_of(const EvictArgs& a, int r) {
  Span s;
  s.n = min(max(a.kv_lens[r], 0), a.max_kv);
  s.f = a.first ? min(max(a.first[r], 0), s.n) : 0;
  s.m = min(s.n - s.f, min(max(a.budgets[r], a.recent), a.max_budget));
  return s;
}

// Floats as unsigned numbers of the same order, from 1 on; -0 as 0, NaN below all.
__device__ __forceinline__ unsigned ordered(float x) {
  const unsigned u = __float_as_uint(x + 0.0f);
  return x != x ? 1u : u & 0x80000000u ? ~u : u | 0x80000000u;
}

// A thread has PER rows in registers, as numbers in the order in which rows stay: 0 for what is no row, the largest for the last `recent` ones.  A request that has
// more rows is read again for the rest of them, as often as they are looked at.
template <int THREADS, int PER>
__device__ __forceinline__ void keep_rows(const EvictArgs& a, const Span s, int layer, int r, int head) {
  constexpr int WAVES = THREADS / 64, ENTRIES = WAVES * PER;
  // Counts of a digit's values, for each of the four digits.  Of the first one, which mostly is one of a handful, every value has eight, side by side, which lanes
  // take in turn: additions of a wave to one of them wait for one another.
  __shared__ __attribute__((aligned(16))) int counts[(8 + 1 + 1 + 1) * 256];
  __shared__ int2 before[ENTRIES];                        // rows above the border and at it: of a wave's strip, then of all before it
  __shared__ int2 strip[2][WAVES];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (tid == 0 && head == 0 && layer == 0) a.new_lens[r] = s.f + s.m;
  const float* sums = a.from.sums + layer * a.from.s_layer + r * a.from.s_seq + head * a.from.s_head;
  float* to = a.to.sums + layer * a.to.s_layer + r * a.to.s_seq + head * a.to.s_head + s.f;
  int32_t* kept = a.kept + (((int64_t)layer * a.n_seqs + r) * a.Hkv + head) * a.max_budget;
  const bool all = s.m == s.n - s.f;
  const int last = s.n - a.recent;                       // rows from there on stay
  auto key_of = [&](int j) __attribute__((always_inline)) { return j >= s.n ? 0u : all || j >= last ? ~0u : ordered(sums[j]); };
  unsigned key[PER] = {};
  if (s.n > s.f) {
    float x[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) x[i] = sums[min(s.f + i * THREADS + tid, s.n - 1)];
    for (int i = tid; i < 11 * 64; i += THREADS) reinterpret_cast<int4*>(counts)[i] = int4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int j = s.f + i * THREADS + tid;
      key[i] = j >= s.n ? 0u : all || j >= last ? ~0u : ordered(x[i]);
    }
  }
  const int beyond = s.f + PER * THREADS;                // first row that is in no register
  unsigned border = 0;                                   // rows above it stay, and the first `equal` of those at it
  int equal = 0;
  __syncthreads();
  if (!all && s.m > 0) {
    int want = s.m;
#pragma unroll
    for (int digit = 0; digit < 4; ++digit) {
      const int shift = 24 - 8 * digit;
      constexpr int kAt[4] = {0, 8, 9, 10};
      int* count = counts + kAt[digit] * 256;
      auto look = [&](unsigned k) __attribute__((always_inline)) {
        const int value = (k >> shift) & 255;
        if (digit == 0) atomicAdd(&count[value * 8 + (lane & 7)], 1);
        else if (k >> ((shift + 8) & 31) == border) atomicAdd(&count[value], 1);
      };
#pragma unroll
      for (int i = 0; i < PER; ++i) look(key[i]);
      for (int j = beyond + tid; j < s.n; j += THREADS) look(key_of(j));
      __syncthreads();
      int4 of;                                           // four values a lane, the largest first; every wave for itself
      if (digit == 0) {
        int y[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const int4 lo = *reinterpret_cast<const int4*>(&count[(255 - 4 * lane - v) * 8]), hi = *reinterpret_cast<const int4*>(&count[(255 - 4 * lane - v) * 8 + 4]);
          y[v] = ((lo.x + lo.y) + (lo.z + lo.w)) + ((hi.x + hi.y) + (hi.z + hi.w));
        }
        of = int4{y[0], y[1], y[2], y[3]};
      } else {
        const int4 y = *reinterpret_cast<const int4*>(&count[252 - 4 * lane]);
        of = int4{y.w, y.z, y.y, y.x};
      }
      int above = of.x + of.y + of.z + of.w;
      const int mine = above;
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) {
        const int y = __shfl_up(above, off);
        if (lane >= off) above += y;
      }
      const int owner = __builtin_ctzll(__ballot(above >= want));       // the first lane up to which there are enough
      above -= mine;
      int at = 255 - 4 * lane, left = want - above;
      if (left > of.x) { left -= of.x; --at;
        if (left > of.y) { left -= of.y; --at;
          if (left > of.z) { left -= of.z; --at; } } }
      border = border << 8 | (unsigned)__shfl(at, owner);
      want = __shfl(left, owner);
    }
    equal = want;
  } else if (!all) {
    border = ~0u;
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const uint64_t m = __ballot(key[i] > border), e = __ballot(key[i] == border);
    if (lane == 0) before[i * WAVES + wave] = make_int2(__popcll(m), __popcll(e));
  }
  __syncthreads();
  if (wave == 0) {
    constexpr int EACH = (ENTRIES + 63) / 64;
    int2 own[EACH], sum = {0, 0};
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      own[i] = lane * EACH + i < ENTRIES ? before[lane * EACH + i] : make_int2(0, 0);
      sum.x += own[i].x; sum.y += own[i].y;
    }
    int2 upto = sum;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int px = __shfl_up(upto.x, off), py = __shfl_up(upto.y, off);
      if (lane >= off) { upto.x += px; upto.y += py; }
    }
    upto.x -= sum.x; upto.y -= sum.y;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      if (lane * EACH + i < ENTRIES) before[lane * EACH + i] = upto;
      upto.x += own[i].x; upto.y += own[i].y;
    }
    if (lane == 63) strip[0][0] = upto;
  }
  __syncthreads();
  auto keep = [&](int j, bool more, bool same, int m, int e) __attribute__((always_inline)) {
    if (more || (same && e < equal)) kept[m + min(e, equal)] = j;
  };
  const uint64_t below = ((uint64_t)1 << lane) - 1;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const bool more = key[i] > border, same = key[i] == border;
    const uint64_t m = __ballot(more), e = __ballot(same);
    const int2 b = before[i * WAVES + wave];
    keep(s.f + i * THREADS + tid, more, same, b.x + __popcll(m & below), b.y + __popcll(e & below));
  }
  if (beyond < s.n) {
    int above = strip[0][0].x, at_border = strip[0][0].y;
    __syncthreads();
    for (int first = beyond, turn = 0; first < s.n; first += THREADS, turn ^= 1) {
      const int j = first + tid;
      const unsigned k = key_of(j);
      const bool more = k > border, same = k == border;
      const uint64_t more_mask = __ballot(more), same_mask = __ballot(same);
      if (lane == 0) strip[turn][wave] = make_int2(__popcll(more_mask), __popcll(same_mask));
      __syncthreads();
      int m = above + __popcll(more_mask & below), e = at_border + __popcll(same_mask & below);
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        const int2 c = strip[turn][w];
        if (w < wave) { m += c.x; e += c.y; }
        above += c.x; at_border += c.y;
      }
      keep(j, more, same, m, e);
    }
  }
  for (int i = s.m + tid; i < a.max_budget; i += THREADS) kept[i] = -1;
  // The kept rows' sums, in lots: all of one have been read before any is written, and those of later ones stand behind what it writes.
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // the numbers of the kept rows are where the others read them
  __syncthreads();
  constexpr int LOT = 2;
  for (int first = 0; first < s.m; first += LOT * THREADS) {
    float v[LOT];
#pragma unroll
    for (int i = 0; i < LOT; ++i) {
      const int at = first + i * THREADS + tid;
      v[i] = at < s.m ? sums[kept[at]] : 0.0f;
    }
    asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
    for (int i = 0; i < LOT; ++i)
      if (first + i * THREADS + tid < s.m) to[first + i * THREADS + tid] = v[i];
  }
}

// Rows move together, DEEP pieces of 16 bytes of a pool a thread at a time.  PIECES: of a row that a workgroup moves; POOLS: one pool, or K and V.
template <int PIECES, int THREADS, int DEEP, int POOLS>
__device__ __forceinline__ void close_up(const EvictArgs& a, int layer, int r, int head, unsigned char* const (&pool)[POOLS], int slice) {
  constexpr int ROWS = THREADS / PIECES;
  const int tid = threadIdx.x;
  const int64_t base = layer * a.pool.s_layer + head * a.pool.s_head + (slice * PIECES + tid % PIECES) * 16;
  const int32_t* kept = a.kept + (((int64_t)layer * a.n_seqs + r) * a.Hkv + head) * a.max_budget;
  const int32_t* table = a.table + (int64_t)r * a.table_width;
  const int in_page = (1 << a.pool.page_log2) - 1;
  auto place = [&](int row) __attribute__((always_inline)) {
    const int page = table[row >> a.pool.page_log2];
    return page < 0 || page >= a.pool.n_pages ? (int64_t)-1 : page * a.pool.s_page + (row & in_page) * a.pool.s_tok;
  };
  // Numbers of the first batch's rows are sent for before it is known how many there are: one wait less; -1 where there is none.
  int row[DEEP];
  auto numbers = [&](int first) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < DEEP; ++u) row[u] = kept[min(first + u * ROWS + tid / PIECES, a.max_budget - 1)];
  };
  numbers(0);
  const Span s = span_of(a, r);
  if (s.m == s.n - s.f) return;
  for (int first = 0; first < s.m; first += ROWS * DEEP) {
    u32x4 x[DEEP][POOLS];
    int64_t to[DEEP];
#pragma unroll
    for (int u = 0; u < DEEP; ++u) {
      const int i = first + u * ROWS + tid / PIECES;
      to[u] = -1;
#pragma unroll
      for (int p = 0; p < POOLS; ++p) x[u][p] = u32x4{0, 0, 0, 0};
      if (i < s.m && row[u] != s.f + i) {                // else it stays where it is
        const int64_t from = place(row[u]);
        to[u] = place(s.f + i);
        if (from >= 0) {
#pragma unroll
          for (int p = 0; p < POOLS; ++p) x[u][p] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(pool[p] + base + from));
        }
      }
    }
    numbers(first + ROWS * DEEP);
    // All rows of the batch are in registers before one is overwritten; rows of later batches lie behind those that this one writes.
    asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
    for (int u = 0; u < DEEP; ++u)
      if (to[u] >= 0) {
#pragma unroll
        for (int p = 0; p < POOLS; ++p) __builtin_nontemporal_store(x[u][p], reinterpret_cast<u32x4*>(pool[p] + base + to[u]));
      }
  }
}

template <int THREADS, int PER>
__global__ __launch_bounds__(THREADS) void keep_kernel(const EvictArgs a) {
  const int head = blockIdx.x % a.Hkv, rest = blockIdx.x / a.Hkv, r = rest % a.n_seqs;
  keep_rows<THREADS, PER>(a, span_of(a, r), rest / a.n_seqs, r, head);
}

template <int PIECES, int THREADS>
__global__ __launch_bounds__(THREADS) void close_up_kernel(const EvictArgs a, int slices, int pools) {
  // Stretches of one row on one die, mostly (workgroups go to the eight dies in turn): they are parts of the same lines of memory.
  const int rows = gridDim.x / slices, slice = blockIdx.x / rows, part = blockIdx.x - slice * rows, problem = part / pools;
  const int head = problem % a.Hkv, rest = problem / a.Hkv, r = rest % a.n_seqs;
  unsigned char* const pool[1] = {part % pools ? a.pool.v : a.pool.k};
  close_up<PIECES, THREADS, kMoveDeep, 1>(a, rest / a.n_seqs, r, head, pool, slice);
}

// Both, for many problems.
template <int PIECES, int THREADS, int PER>
__global__ __launch_bounds__(THREADS) void evict_kernel(const EvictArgs a) {
  const int head = blockIdx.x % a.Hkv, rest = blockIdx.x / a.Hkv, r = rest % a.n_seqs, layer = rest / a.n_seqs;
  const Span s = span_of(a, r);
  keep_rows<THREADS, PER>(a, s, layer, r, head);
  unsigned char* const pool[2] = {a.pool.k, a.pool.v};
  close_up<PIECES, THREADS, kBothDeep, 2>(a, layer, r, head, pool, 0);
}

template <int PIECES>
static void launch_close_up(const EvictArgs& a, int64_t problems, int slices, hipStream_t stream) {
  const int pools = a.pool.k == a.pool.v ? 1 : 2;          // a cache whose values are its keys: rows move once
  close_up_kernel<PIECES, kMoveThreads><<<dim3((unsigned)(problems * pools * slices)), dim3(kMoveThreads), 0, stream>>>(a, slices, pools);
}

template <int PIECES>
static int launch_both(const EvictArgs& a, int64_t problems, hipStream_t stream) {
  if (a.max_kv <= kShortRows) evict_kernel<PIECES, kShortThreads, kShortRows / kShortThreads><<<dim3((unsigned)problems), dim3(kShortThreads), 0, stream>>>(a);
  else evict_kernel<PIECES, kBothThreads, 8><<<dim3((unsigned)problems), dim3(kBothThreads), 0, stream>>>(a);
  return (int)hipGetLastError();
}

int launch_evict(const EvictArgs& a, int d, hipStream_t stream) {
  const int64_t problems = (int64_t)a.n_layers * a.n_seqs * a.Hkv;
  const int pieces = d * (a.pool.fp8 ? 1 : 2) / 16;
  int slices = 1;
  while (problems * 2 * slices < kFewest && slices < pieces / 8) slices *= 2;
  while (problems * 2 * slices < kFewer && slices < pieces / 2 && a.max_budget > kManyRows) slices *= 2;
  if (problems * 2 * slices > kMostBlocks) return CODECOMP_EINVAL_SHAPE;
  if ((std::min(a.max_budget, a.max_kv) <= kFewKept && a.max_kv <= kHeldRows) || (problems >= kManyProblems && a.max_kv <= kBothRows)) {
    if (pieces == 16) return launch_both<16>(a, problems, stream);
    return pieces == 8 ? launch_both<8>(a, problems, stream) : launch_both<4>(a, problems, stream);
  }
  // As many threads and rows of each as the longest request needs: what registers do not hold is read again (4 heads, both kernels, us: 1088 rows with 256 threads of 8 | 1024 of
  // 32: 16.5 | 29; 8000 of which 50 stay, 256 of 16 | 512 of 16 | 1024 of 16: 27 | 13.5 | 16.6; 12000, 1024 of 16 | of 32: 16.5 | 23.9; 28 layers of 32768, 256 of 16 | 1024 of 32: 207 | 83).
  const dim3 grid((unsigned)problems);
  if (a.max_kv > 16384) keep_kernel<1024, 32><<<grid, dim3(1024), 0, stream>>>(a);
  else if (a.max_kv > 8192) keep_kernel<1024, 16><<<grid, dim3(1024), 0, stream>>>(a);
  else if (a.max_kv > 2048) keep_kernel<512, 16><<<grid, dim3(512), 0, stream>>>(a);
  else keep_kernel<256, 8><<<grid, dim3(256), 0, stream>>>(a);
  if (hipError_t e = hipGetLastError()) return (int)e;
  switch (pieces / slices) {
    case 16: launch_close_up<16>(a, problems, slices, stream); break;
    case 8: launch_close_up<8>(a, problems, slices, stream); break;
    case 4: launch_close_up<4>(a, problems, slices, stream); break;
    default: launch_close_up<2>(a, problems, slices, stream); break;
  }
  return (int)hipGetLastError();
}

}  // namespace codecomp
