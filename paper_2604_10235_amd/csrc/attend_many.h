// Internal header: attention of requests with many rows (new tokens x query heads per KV head; attend.hip says from how many on): prefill chunks and
// prompts.  Instantiated per head_dim and cache type in attend_many_*.hip, so that they compile side by side.
//
// The rows of a KV head, token by token and its query heads within, are cut into blocks of 256: eight waves of 32 rows,
// which share the keys and values that go through LDS in tiles of 64.  S^T = K Q^T leaves a row's logits in one lane of each half of the wave;
// O^T += V^T P^T takes them from there: the order of keys in a contraction is free, and chosen so that a lane's weights are its right operand as
// they stand.  V^T comes from LDS by the transposing read.  A row's reference (what is subtracted before exp2) moves only when a weight grows large, so
// that most steps neither look for a maximum nor touch the outputs.
//
// Bound by the matrix units and the vector instructions beside them, under the chip's power limit.  2048 tokens over 32768 keys, 28 query heads on 4 KV
// heads of 128: 760 to 810 us by the device, 1.15 to 1.23 PFLOP/s, where the library's product of two 8192 x 8192 matrices reaches 1.21 to 1.27 on the
// same devices; the matrix units are busy 69 % of the time at 1.5 to 1.9 GHz, 94 % of the reads meet L2, no LDS bank conflict.  head_dim 64 has as many
// vector instructions for half the products: 480 to 505 us, 0.93 to 0.97 PFLOP/s.  8-bit caches: 785 to 815 and 500 to 516 us, the codes are widened on the way to LDS.
// Weights are rounded to bf16 for the second product, which puts a bf16 output 1.3 to 1.45 times as far from the exact one as rounding alone; as two bf16, which
// requests of up to 64 rows have (they wait for memory), these chunks would take 1124 us instead of 783, and 712 instead of 494.
// The 50 to 75 scalar registers that do not fit are kept in lanes of vector registers and come back between parts: none in a step's instructions.
// Tried before: waves with 512 registers (the compiler keeps the accumulators in the half that vector instructions do not reach, and copies them); the page
// table looked up key by key (790 us; as one load per 1024 keys 760).
// Sending for a part's first tiles behind the last ones of the part before took as much time in the loop as it saved between parts; sending for them
// before the outputs are written, and writing these in whole rows by way of LDS, changed nothing or took registers that the loop needs.
#pragma once
#include <type_traits>

#include "attend.h"

namespace codecomp {

constexpr int kManyRows = 256, kManyKeys = 64, kManyWaves = 8, kManyThreads = 64 * kManyWaves;

// Blocks of rows are cut into equal parts by positions, kManyTile of them to a tile, and kManyLight to a tile of a block of up to 32 rows, one wave's, whose
// weights are two bf16 (512 tokens over 4096 keys and 64 steps over 500 .. 4096, us, with 5 | 6 | 7 | 8 | 9: 76 | 73 | 70 | 74 | 77 at head_dim 64,
// - | 102 | 102 | 107 | 109 at 128; 2048 over 8192 and 64 over 500 .. 16384: 279 | 255 | 247 | 244 | 255; - | 372 | 356 | 353 | 370).
constexpr int kManyTile = 8, kManyLight = 7;
// Tiles' worth of positions in front of a block's tiles: starting on a block (its queries, the first tiles) and
// ending it cost 11 us at head_dim 128 and 5 at 64, of 1.65 and 1.2 us a tile (a prompt of 4096 tokens, us, with 3 | 4 | 5 | 7 | 10 | 14: 185 |
// 170 | 155 | 141 | 146 | 149; head_dim 64 114 | 103 | 97 | 95).
constexpr int kManyLead = 7;
// Reference of a row before its first visible key: finite, so that hidden logits (minus infinity) less it still are minus infinity, and so low that a
// visible one's weight overflows, which makes it the reference.
constexpr float kNoReference = -3.402823466e38f;
constexpr int kManyLeast = 4;   // tiles' worth that a workgroup gets at least (with 8 a prompt of 100 tokens takes 32 us instead of 23)

struct ManyArgs {
  AttendArgs a;
  CutBlock* cuts;              // [workgroups]
  int workgroups, rows_from;   // requests of fewer rows are not this kernel's
  int whole;                   // 1: no block is shared (all are short): nothing to be joined
};

// Tiles of 64 keys that a block of rows of a request meets; at least one.
struct Blocks {
  int len, q0, nq, G, rows, count, causal;       // keys, first new token, new tokens, query heads per KV head, rows, blocks of them
  __device__ __forceinline__ int tiles(int block) const {
    int keys = len;
    if (causal) keys = min(len, len - nq + (min(block * kManyRows + kManyRows, rows) - 1) / G + 1);
    return max(1, (keys + kManyKeys - 1) / kManyKeys);
  }
};
__device__ __forceinline__ Blocks blocks_of(const ManyArgs& m, int len, int q0, int nq) {
  Blocks x;
  x.len = len; x.q0 = q0; x.nq = nq;
  x.G = m.a.b.G;
  x.rows = x.nq * x.G;
  x.count = x.rows >= m.rows_from ? (x.rows + kManyRows - 1) / kManyRows : 0;
  x.causal = m.a.b.causal;
  return x;
}
__device__ __forceinline__ Blocks blocks_of(const ManyArgs& m, int r) {
  return blocks_of(m, kv_len_of(m.a.b, r), m.a.b.cu_q[r], m.a.b.cu_q[r + 1] - m.a.b.cu_q[r]);
}

__device__ __forceinline__ Blocks uniform(Blocks x) {
  x.len = uniform(x.len); x.q0 = uniform(x.q0); x.nq = uniform(x.nq); x.rows = uniform(x.rows); x.count = uniform(x.count);
  return x;
}

// A tile in LDS: chunks of 1 KB, 16 rows of four 16-byte pieces, what a wave loads at a time.  Keys stand piece by piece in a chunk (16 rows of one,
// then of the next: a fragment's read meets every bank once), values row by row (four rows are the 256 bytes that the transposing read takes from
// half a wave).  Either way a fragment's number only adds a constant to a lane's address.
template <int D>
struct TileAt {
  static constexpr int GROUP = D / 32 * 1024;          // bytes of 16 rows
  static __device__ __forceinline__ int key(int row, int piece) { return (row >> 4) * GROUP + (piece >> 2) * 1024 + (piece & 3) * 256 + (row & 15) * 16; }
  static __device__ __forceinline__ int value(int row, int piece) { return (row >> 4) * GROUP + (piece >> 2) * 1024 + (row & 15) * 64 + (piece & 3) * 16; }
};

// ROWWISE: pages of less than 16 rows; else the 16 rows that a wave loads of a tile lie in one page, whose place is worked out in scalar registers.
template <int D, bool FP8, bool ROWWISE>
__global__ __launch_bounds__(kManyThreads, 2) void attend_many_kernel(const ManyArgs ma) {
  const AttendArgs& a = ma.a;
  constexpr int PIECES = D * (FP8 ? 1 : 2) / 16;               // 16-byte pieces of a stored row
  // 16-byte pieces of K and of V per thread and tile: of one row (8 bits), or of a wave's chunks, which lie side by side in 16 rows
  constexpr int LOADS = FP8 ? 1 : D / 64;
  // 8 bits at head_dim 64: half of the waves have the keys, the others the values
  constexpr bool HALVES = FP8 && D == 64;
  constexpr int SENT = HALVES ? 1 : 2 * LOADS;                    // loads of a wave for a tile
  using At = TileAt<D>;
  constexpr int KS = D / 16, DB = D / 32;
  constexpr int TILE = kManyKeys * 2 * D;                        // bytes of the keys of a tile in LDS; its values stand behind them
  static_assert(kManyRows == 32 * kManyWaves, "a block of 32 rows per wave");
  __shared__ __attribute__((aligned(1024))) unsigned char tiles_lds[4 * 2 * TILE];
  __shared__ int entries[ROWWISE ? 8 : 4][64];                    // of the page table: below
  auto k_tile = [&](int tile) __attribute__((always_inline)) { return tiles_lds + (tile & 3) * (2 * TILE); };
  __shared__ int not_finite;
  __shared__ int64_t wave_sum[kManyWaves];
  __shared__ int found[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), l32 = lane & 31, half = lane >> 5;

  // ---- this workgroup's share: the tiles of all blocks of all heads form one sequence, cut into equal parts.  Requests are shared out over the
  // threads to count their blocks, then blocks to count their tiles (one each, mostly: a prompt alone has many).
  const int n = a.b.n_seqs, per = (n + kManyThreads - 1) / kManyThreads;
  // positions of a tile and of a block
  auto per_tile = [&](const Blocks& x, int block) { return x.rows - block * kManyRows > 32 ? kManyTile : kManyLight; };
  auto weight = [&](const Blocks& x, int block) { return ma.whole ? 1 : kManyLead * kManyTile + x.tiles(block) * per_tile(x, block); };
  // Up to 2048 requests are kept in LDS: the loads of what follows are short then.
  __shared__ int requests[3][4 * kManyThreads];
  const bool kept = n <= 4 * kManyThreads;
  auto request = [&](int r) __attribute__((always_inline)) { return kept ? blocks_of(ma, requests[0][r], requests[1][r], requests[2][r]) : blocks_of(ma, r); };
  int my_blocks = 0;
  for (int r = min(tid * per, n); r < min(tid * per + per, n); ++r) {
    const Blocks x = blocks_of(ma, r);
    my_blocks += x.count;
    if (kept) { requests[0][r] = x.len; requests[1][r] = x.q0; requests[2][r] = x.nq; }
  }
  int blocks = my_blocks;                                        // up to here, inclusive
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int y = __shfl_up(blocks, off);
    if (lane >= off) blocks += y;
  }
  if (lane == 63) wave_sum[wave] = blocks;
  __syncthreads();
  int all_blocks = 0;
#pragma unroll
  for (int w = 0; w < kManyWaves; ++w) {
    if (w < wave) blocks += (int)wave_sum[w];
    all_blocks += (int)wave_sum[w];
  }
  int* first_block = reinterpret_cast<int*>(tiles_lds);           // of a thread's requests
  first_block[tid] = blocks - my_blocks;
  __syncthreads();
  const int block_per = (uniform(all_blocks) + kManyThreads - 1) / kManyThreads;
  const int b0 = min(tid * block_per, all_blocks), b1 = min(b0 + block_per, all_blocks);
  int my_r = 0, my_i = 0;                                         // request of block b0, and its number there
  int64_t mine = 0;                                               // positions of this thread's blocks
  if (b0 < b1) {
    int lo = 0;                                                  // last thread whose requests begin at b0 or before, and have blocks from there on
#pragma unroll
    for (int step = kManyThreads / 2; step > 0; step >>= 1)
      if (first_block[lo + step] <= b0) lo += step;
    my_r = lo * per;
    my_i = b0 - first_block[lo];
    Blocks x = request(my_r);
    while (my_i >= x.count) { my_i -= x.count; x = request(++my_r); }
    int r = my_r, i = my_i;
    for (int b = b0; b < b1; ++b, ++i) {
      while (i >= x.count) { i = 0; x = request(++r); }
      mine += weight(x, i);
    }
  }
  int64_t incl = mine;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int64_t y = __shfl_up(incl, off);
    if (lane >= off) incl += y;
  }
  __syncthreads();
  if (lane == 63) wave_sum[wave] = incl;
  __syncthreads();
  int64_t before = 0, per_head = 0;
#pragma unroll
  for (int w = 0; w < kManyWaves; ++w) {
    if (w < wave) before += wave_sum[w];
    per_head += wave_sum[w];
  }
  per_head = uniform(per_head);
  const int64_t total = per_head * a.b.Hkv;
  const int64_t workgroups = min((int64_t)ma.workgroups, ma.whole ? total : (total + kManyLeast * kManyTile - 1) / (kManyLeast * kManyTile));
  if (tid == 0 && blockIdx.x >= workgroups && !ma.whole) ma.cuts[blockIdx.x].r = -1;
  // neighbours in the sequence read the same keys: they run on the same die (workgroups go to the eight dies in turn)
  const int per_die = ((int)workgroups + 7) / 8, g = (int)(blockIdx.x & 7) * per_die + (int)(blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= per_die || g >= workgroups) return;
  const int64_t x0 = uniform(g * total / workgroups), x1 = uniform((g + 1) * total / workgroups);
  // From the end of the part back to its start: blocks are entered at their first keys, at about the same time by all workgroups, so
  // that the keys and values of a head are read by many at a time.
  int head = uniform((int)((x1 - 1) / per_head));
  {
    const int64_t at = x1 - 1 - head * per_head;
    int64_t start = before + incl - mine;
    if (at >= start && at < start + mine) {                      // one thread has it
      Blocks y = request(my_r);
      int r = my_r, i = my_i;
      for (;; ++i) {
        while (i >= y.count) { i = 0; y = request(++r); }
        const int positions = weight(y, i);
        if (at < start + positions) break;
        start += positions;
      }
      found[0] = r; found[1] = i; found[2] = (int)(at - start);
    }
  }
  __syncthreads();
  int r = uniform(found[0]), block = uniform(found[1]);
  int64_t start = uniform(x1 - 1 - found[2]);                     // position of the block
  Blocks of = uniform(request(r));
  CutBlock cut = {-1, 0, 0, 0};

  for (;;) {
    const int tiles = uniform(of.tiles(block));
    const int64_t first = start + kManyLead * kManyTile;          // position of its first tile
    const int each = uniform(per_tile(of, block));
    auto tiles_before = [&](int64_t x) { return uniform((int)min((max(x - first, (int64_t)0) + each - 1) / each, (int64_t)tiles)); };        // that begin before x
    const int tile0 = ma.whole ? 0 : tiles_before(x0), tile1 = ma.whole ? tiles : tiles_before(x1);
    if (tile1 > tile0) {
      const bool whole = tile0 == 0 && tile1 == tiles;
      const int slot = tile0 > 0 ? 2 * g : 2 * g + 1;
      if (tile0 == 0 && tile1 < tiles)                             // the rest of the block is the next workgroups'
        cut = {r, block, head, (int)(((first + (int64_t)(tiles - 1) * each + 1) * workgroups - 1) / total)};
      const int q0 = of.q0, row0 = block * kManyRows + wave * 32, row = row0 + l32;
      const bool active = row0 < of.rows;

      // query rows as right operands, and the keys that the lane's rows see
      u32x4 qf[KS];
      int limit;
      {
        const int rr = min(row, of.rows - 1), t = rr / of.G;
        const uint16_t* p = a.q + (q0 + t) * a.b.q_st + (head * of.G + rr - t * of.G) * a.b.q_sh + half * 8;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          qf[ks] = *reinterpret_cast<const u32x4*>(p + ks * 16);
          if (row >= of.rows) qf[ks] = u32x4{0, 0, 0, 0};
        }
        limit = of.causal ? min(of.len, of.len - of.nq + t + 1) : of.len;
      }
      const int seen_by_all = uniform(of.causal ? min(of.len, of.len - of.nq + block * kManyRows / of.G + 1) : of.len);

      const unsigned char* kb = a.pool.k + a.layer + head * a.pool.s_head;
      const unsigned char* vb = a.pool.v + a.layer + head * a.pool.s_head;
      const int32_t* table = a.b.table + (int64_t)r * a.b.table_width;
      const int in_page = (1 << a.pool.page_log2) - 1;

      // ---- the way of keys and values.  A tile goes into one of four LDS buffers three tiles ahead: 16-bit rows straight from memory, 8-bit rows by
      // way of registers, where they are widened.  Entries of the page table go ahead of them, 64 at a time: one for every 16 keys, the 16 tiles of a
      // stretch of 1024 keys at once (or, ROWWISE, one for every key of a tile, five tiles ahead).
      auto fetch_entries = [&](int stretch) __attribute__((always_inline)) {        // for the last key where there is none
        const int32_t* from = table + (max(min((stretch * 64 + lane) * (ROWWISE ? 1 : 16), of.len - 1), 0) >> a.pool.page_log2);
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds_address(entries[stretch & (ROWWISE ? 7 : 3)])), "v"(from) : "memory", "m0");
      };
      auto entry = [&](int tile, int row) __attribute__((always_inline)) { return ROWWISE ? entries[tile & 7][row] : entries[(tile >> 4) & 3][(tile & 15) * 4 + (row >> 4)]; };
      auto is_page = [&](int page) __attribute__((always_inline)) { return (unsigned)page < (unsigned)a.pool.n_pages; };
      // The rows of a tile that this thread loads pieces of.  16 bits: of the wave's 16 rows, the lane % 16th of K and the lane / 4th of V.  8 bits: of its
      // 8 or 16, in an order that makes the stores of eight lanes to LDS meet different banks: rows side by side in K, four rows and two pieces in V.
      constexpr int ROWS = FP8 ? 64 / PIECES : 16;
      const int wave_row = FP8 ? (wave * ROWS) & (kManyKeys - 1) : (wave >> 1) * 16;
      const int k_row = wave_row + (lane & (ROWS - 1)), v_row = wave_row + (FP8 ? (lane & 3) + ((lane >> 3) & (ROWS / 4 - 1)) * 4 : lane >> 2);
      const int k_piece = FP8 ? lane / ROWS : (wave & 1) * LOADS * 4 + (lane >> 4);
      const int v_piece = FP8 ? ((lane >> 2) & 1) + (lane >> 3) / (ROWS / 4) * 2 : (wave & 1) * LOADS * 4 + (lane & 3);
      const bool has_values = HALVES && wave >= kManyWaves / 2;
      // Where they are; rows that are not there: in page 0, taken out of the tile when it is used.  At `base` + `lane_off`.
      struct Place { int64_t base; uint32_t lane_off; };
      const uint32_t k_lane_off = (k_row - wave_row) * (uint32_t)a.pool.s_tok + k_piece * 16, v_lane_off = (v_row - wave_row) * (uint32_t)a.pool.s_tok + v_piece * 16;
      auto place = [&](int tile, int row, int piece, uint32_t lane_off) __attribute__((always_inline)) {
        const int page = ROWWISE ? entry(tile, row) : uniform(entry(tile, wave_row));
        const int64_t at = (uint64_t)(unsigned)(is_page(page) ? page : 0) * (uint64_t)a.pool.s_page;
        if constexpr (ROWWISE) return Place{at + (unsigned)((tile * kManyKeys + row) & in_page) * (unsigned)a.pool.s_tok, (uint32_t)piece * 16};
        return Place{at + (unsigned)((tile * kManyKeys + wave_row) & in_page) * (unsigned)a.pool.s_tok, lane_off};
      };
      auto k_place = [&](int tile) __attribute__((always_inline)) {
        return has_values ? place(tile, v_row, v_piece, v_lane_off) : place(tile, k_row, k_piece, k_lane_off);
      };
      auto v_place = [&](int tile, Place k) __attribute__((always_inline)) {
        if constexpr (HALVES) return k;
        if constexpr (!ROWWISE) return Place{k.base, v_lane_off};
        return place(tile, v_row, v_piece, v_lane_off);
      };
      u32x4 kr, vr;                                                // 8 bits: the tile after the next two, on its way
      auto fetch = [&](u32x4& into, uint32_t lds, const unsigned char* from, Place at) __attribute__((always_inline)) {
        if constexpr (FP8) {
          into = *reinterpret_cast<const u32x4*>(from + at.base + at.lane_off);
        } else {
#pragma unroll
          for (int i = 0; i < LOADS; ++i) {
            if constexpr (ROWWISE)
              asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds + (wave * LOADS + i) * 1024),
                           "v"(from + at.base + at.lane_off + i * 64) : "memory", "m0");
            else
              asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds + (wave * LOADS + i) * 1024),
                           "v"(at.lane_off), "s"(from + at.base + i * 64) : "memory", "m0");
          }
        }
      };
      auto fetch_keys = [&](int tile, Place at) __attribute__((always_inline)) { fetch(kr, lds_address(k_tile(tile)), has_values ? vb : kb, at); };
      auto fetch_values = [&](int tile, Place at) __attribute__((always_inline)) {
        if constexpr (!HALVES) fetch(vr, lds_address(k_tile(tile)) + TILE, vb, at);
      };
      const int park_at = has_values ? TILE + At::value(v_row, 2 * v_piece) : At::key(k_row, 2 * k_piece);
      const int park_at2 = has_values ? TILE + At::value(v_row, 2 * v_piece + 1) : At::key(k_row, 2 * k_piece + 1);
      auto park = [&](int tile, int quarter) __attribute__((always_inline)) {      // 8 bits: a half of the piece of K, or of that of V
        if constexpr (FP8) {
          unsigned char* at = k_tile(tile);
          if (quarter == 0) *reinterpret_cast<u32x4*>(at + park_at) = widen8(kr.x, kr.y);
          if (quarter == 1) *reinterpret_cast<u32x4*>(at + park_at2) = widen8(kr.z, kr.w);
          if constexpr (HALVES) return;
          if (quarter == 2) *reinterpret_cast<u32x4*>(at + TILE + At::value(v_row, 2 * v_piece)) = widen8(vr.x, vr.y);
          if (quarter == 3) *reinterpret_cast<u32x4*>(at + TILE + At::value(v_row, 2 * v_piece + 1)) = widen8(vr.z, vr.w);
        }
      };
      // The keys of a tile that there are; the tiles from `plain_end` on have keys that are not there, or that some rows do not see.
      auto is_there = [&](int tile, int page) __attribute__((always_inline)) { return __ballot(tile * kManyKeys + lane < of.len && is_page(page)); };
      const int plain_end = min(seen_by_all, of.len) >> 6;
      auto partly = [&](int tile) { return (tile + 1) * kManyKeys > seen_by_all && seen_by_all < of.len; };       // some rows do not see all of it
      // Values of a tile that has keys that are not there, or that some rows do not see: a weight of zero must not meet what stands in the one, nor an
      // infinite or NaN value in the other (added at the end, to the rows that see them).
      auto clean_values = [&](int tile, uint64_t valid) __attribute__((always_inline)) {
        unsigned any = 0;
        for (int i = tid; i < TILE / 16; i += kManyThreads) {
          u32x4* at = reinterpret_cast<u32x4*>(k_tile(tile) + TILE + i * 16);
          u32x4 v = *at;
          if (!((valid >> (i * 16 / At::GROUP * 16 + ((i >> 2) & 15))) & 1)) v = u32x4{0, 0, 0, 0};
          if (partly(tile)) v = finite_part<false>(v, any);
          *at = v;
        }
        if (any != 0) not_finite = 1;
      };

      f32x16 o[DB];
      float m = kNoReference, l = 0.0f;                            // a row's reference, this half's sum of weights
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[db][i] = 0.0f;
      f32x16 za, zb;                                               // logits of the first and of the second 32 keys of a tile
      // The tiles, with weights rounded to bf16, or (FINE) as two bf16, the rounded one and the rest: what requests of as many rows as the other kernel takes
      // have there, they have here as well, whatever is in the batch with them.
      auto walk = [&](auto two) __attribute__((always_inline)) {
        constexpr bool FINE = decltype(two)::value;
        struct Weights {                                             // of 16 keys each
          u32x4 p[2], rest[FINE ? 2 : 1];
        } pa, pb = {};
        auto pack = [&](Weights& to, int i, float x, float y) __attribute__((always_inline)) {      // of logits i and i + 1
          const unsigned p = pack2(x, y);
          to.p[i >> 3][(i & 7) >> 1] = p;
          if constexpr (FINE) to.rest[i >> 3][(i & 7) >> 1] = pack2(x - __uint_as_float(p << 16), y - __uint_as_float(p & 0xFFFF0000u));
        };

        // Key fragment f (16 of a row's elements of 32 keys), value fragment f (32 columns of 16 keys).
        const int k_lane = At::key(l32, half), v_lane = At::value(half * 4 + ((lane >> 2) & 3), 0) + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
        auto key_frag = [&](const unsigned char* kt, int f) __attribute__((always_inline)) { return *reinterpret_cast<const u32x4*>(kt + k_lane + f * 512); };
        auto value_frag = [&](const unsigned char* vt, int f) __attribute__((always_inline)) {
          const unsigned char* at = vt + v_lane + (f / DB) * At::GROUP + (f % DB) * 1024;
          const s16x4 v0 = read_columns(at), v1 = read_columns(at + 512);
          return __builtin_bit_cast(u32x4, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
        };
        constexpr int F = 2 * KS, RING = 4, PER = 16 / F, HALF = 2 * At::GROUP;      // fragments of a step, those held, logits per fragment; bytes of 32 rows
        u32x4 ring[RING];
        auto fill = [&](int f, const unsigned char* kt, const unsigned char* vt) __attribute__((always_inline)) {
          ring[f % RING] = f & 1 ? value_frag(vt, f / 2) : key_frag(kt, f / 2);
        };
        // One step: the weights p of the 32 keys from key0 on, whose logits are z (`masked`: not all rows see all of them; `valid`: which of them there are); beside them, on the matrix cores,
        // the logits zn of the next 32 keys (kt) and the outputs of the 32 before (vt), whose weights are pp.  The order is the source's: the LDS read that
        // the MFMA three further on needs (from the next step's tiles at the end), an MFMA, the vector work of a logit (two at head_dim 64), and
        // what `beside` has for this place.
        auto step = [&](f32x16& z, Weights& p, f32x16& zn, const unsigned char* kt, const Weights& pp, const unsigned char* vt, const unsigned char* kt_next,
                        const unsigned char* vt_next, int key0, bool masked, unsigned valid, auto&& beside) __attribute__((always_inline)) {
          if (__builtin_expect(masked, 0)) {
            int first = 4 * half;
            asm("" : "+v"(first));                                     // the places that follow from it are worked out here, not held in registers
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int j = 8 * (i >> 2) + first + (i & 3);
              if (!((valid >> j) & 1) || key0 + j >= limit) z[i] = -INFINITY;
            }
          }
          float sum = 0.0f, w[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) zn[i] = 0.0f;
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int f = 0; f < F; ++f) {
            beside(f);
            if (f + RING - 1 < F) fill(f + RING - 1, kt, vt);
            else fill(f + RING - 1 - F, kt_next, vt_next);
            const int i = f / 2;
            if (f & 1) {
              o[i % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag(ring[f % RING]), frag(pp.p[i / DB]), o[i % DB], 0, 0, 0);
              if constexpr (FINE) o[i % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag(ring[f % RING]), frag(pp.rest[i / DB]), o[i % DB], 0, 0, 0);
            } else zn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag(ring[f % RING]), frag(qf[i]), zn, 0, 0, 0);
#pragma unroll
            for (int e = f * PER; e < (f + 1) * PER; ++e) {
              w[e] = __builtin_amdgcn_exp2f(fmaf(z[e], a.c, -m));
              if (e > 0) sum += w[e - 1];
              if (e > 1 && (e & 1) == 0) pack(p, e - 2, w[e - 2], w[e - 1]);
            }
            __builtin_amdgcn_sched_barrier(0);
          }
          sum += w[15];
          pack(p, 14, w[14], w[15]);
          // here, beside the MFMAs, not behind the branch
          asm volatile("" ::"v"(sum), "v"(p.p[0]), "v"(p.p[1]));
          if constexpr (FINE) asm volatile("" ::"v"(p.rest[0]), "v"(p.rest[1]));
          // A logit far above its row's reference: move the references.  (Weights are positive: none is larger than their sum, and as
          // long as that is below 4096 nothing is lost in fp32 or bf16.)
          if (__builtin_expect(__ballot(sum > 4096.0f) != 0, 0)) {
            float t = -INFINITY;
#pragma unroll
            for (int i = 0; i < 16; ++i) t = fmaxf(t, z[i]);
            t *= a.c;
            t = fmaxf(t, __shfl_xor(t, 32));
            const float to = fmaxf(m, t), old = to == m ? 1.0f : __builtin_amdgcn_exp2f(m - to);
            m = to;
            l *= old;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
              for (int i = 0; i < 16; ++i) o[db][i] *= old;
            sum = 0.0f;
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
              const float x = __builtin_amdgcn_exp2f(fmaf(z[i], a.c, -m)), y = __builtin_amdgcn_exp2f(fmaf(z[i + 1], a.c, -m));
              sum += x + y;
              pack(p, i, x, y);
            }
          }
          l += sum;
        };

        // ---- before the first tile
        __syncthreads();                                             // the segment before is through with LDS
        if (tid == 0) not_finite = 0;
#pragma unroll
        for (int j = 0; j < (ROWWISE ? 5 : 3); ++j) fetch_entries((ROWWISE ? tile0 : tile0 >> 4) + j);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
        for (int j = 0; j < 3; ++j) {
          const Place from = k_place(tile0 + j);
          fetch_keys(tile0 + j, from);
          fetch_values(tile0 + j, v_place(tile0 + j, from));
          if (j < 2) { park(tile0 + j, 0); park(tile0 + j, 1); park(tile0 + j, 2); park(tile0 + j, 3); }
        }
        // in front of the first tile: values of zero
        for (int i = tid; i < HALF / 16; i += kManyThreads) *reinterpret_cast<u32x4*>(k_tile(tile0 + 3) + TILE + HALF + i * 16) = u32x4{0, 0, 0, 0};
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(SENT) : "memory");
        uint64_t valid = ROWWISE ? is_there(tile0, entry(tile0, lane)) : 0;
        uint64_t held = ROWWISE ? 0 : __ballot(is_page(entries[(tile0 >> 4) & 3][lane]));          // groups of 16 keys of the stretch whose pages there are
        if (active) {
#pragma unroll
          for (int i = 0; i < 16; ++i) za[i] = 0.0f;
#pragma unroll
          for (int f = 0; f < KS; ++f) za = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag(key_frag(k_tile(tile0), f)), frag(qf[f]), za, 0, 0, 0);
#pragma unroll
          for (int f = 0; f < RING - 1; ++f) fill(f, k_tile(tile0) + HALF, k_tile(tile0 + 3) + TILE + HALF);
        }
        for (int tile = tile0; tile < tile1; ++tile) {
          bool masked = tile >= plain_end;
          if constexpr (ROWWISE) {
            masked |= valid != ~0ull;
          } else {
            if ((tile & 15) == 13) fetch_entries((tile >> 4) + 2);   // three tiles ahead a new stretch begins: the one after it
            if ((tile & 15) == 0) held = __ballot(is_page(entries[(tile >> 4) & 3][lane]));
            masked |= (((unsigned)(held >> ((tile & 15) * 4)) & 15u) != 15u);
            if (masked) valid = is_there(tile, entry(tile, lane));
          }
          if (__builtin_expect(masked, 0)) clean_values(tile, valid);
          const unsigned char *t0 = k_tile(tile), *t1 = k_tile(tile + 1), *before = k_tile(tile + 3);
          // All of this step's LDS reads are on their way by the last places: from there on the tile before is nobody's, and the next one is everybody's.
          auto pass_on = [&](int f) __attribute__((always_inline)) {
            if (f == F - (RING - 1)) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(SENT + (ROWWISE ? 1 : 0)) : "memory");
          };
          Place k_from = {0, 0}, v_from = {0, 0};
          int next_entry = 0;
          auto send_for = [&](int f) __attribute__((always_inline)) {
            if (ROWWISE && f == 0) next_entry = entry(tile + 1, lane);
            if (f < 4) park(tile + 2, f);                            // before the next ones are sent for below
            if (f == 1) k_from = k_place(tile + 3);
            if (f == 2) v_from = v_place(tile + 3, k_from);
            if (f == 3) fetch_keys(tile + 3, k_from);
            if (f == 4) fetch_values(tile + 3, v_from);
            if (f == 5 && ROWWISE) fetch_entries(tile + 5);
          };
          if (active) {
            step(za, pa, zb, t0 + HALF, pb, before + TILE + HALF, t1, t0 + TILE, tile * kManyKeys, masked, (unsigned)valid, pass_on);
            step(zb, pb, za, t1, pa, t0 + TILE, t1 + HALF, t0 + TILE + HALF, tile * kManyKeys + 32, masked, (unsigned)(valid >> 32), send_for);
          } else {
            pass_on(F - (RING - 1));
#pragma unroll
            for (int f = 0; f < F; ++f) send_for(f);
          }
          if constexpr (ROWWISE) valid = is_there(tile + 1, next_entry);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");             // what was sent for beyond the last tile
        if (active) {
#pragma unroll
          for (int f = 0; f < KS; ++f) {
            const bf16x8 v = frag(value_frag(k_tile(tile1 + 3) + TILE + HALF, f));
            o[f % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, frag(pb.p[f / DB]), o[f % DB], 0, 0, 0);
            if constexpr (FINE) o[f % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, frag(pb.rest[f / DB]), o[f % DB], 0, 0, 0);
          }
        }
      };
      if (__builtin_expect(of.rows > kFewRowsMost, 1)) walk(std::false_type{});
      else walk(std::true_type{});
      if (active) {
        if (__builtin_expect(partly(tile1 - 1) && not_finite != 0, 0)) {
          // from the first tile that was cleaned on: the keys before seen_by_all in it were as well
          for (int key = max(seen_by_all & -kManyKeys, tile0 * kManyKeys); key < min(of.len, tile1 * kManyKeys); ++key) {
            const int at = table[key >> a.pool.page_log2];
            if (at < 0 || at >= a.pool.n_pages || key >= limit) continue;
            const unsigned char* from = a.pool.v + a.layer + head * a.pool.s_head + at * a.pool.s_page + (key & in_page) * a.pool.s_tok;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const f32x4 v = row4<FP8>(from + (db * 32 + i * 8 + half * 4) * (FP8 ? 1 : 2));
#pragma unroll
                for (int e = 0; e < 4; ++e) o[db][4 * i + e] = with_the_rest(o[db][4 * i + e], v[e]);
              }
          }
        }
        const float sum = l + __shfl_xor(l, 32);
        if (row < of.rows && whole) {
          const int t = row / of.G, h = head * of.G + row - t * of.G;
          const float inv = sum == 0.0f ? 0.0f : a.pool.v_scale / sum;
          uint16_t* out = a.out + (q0 + t) * a.b.o_st + h * a.b.o_sh + half * 4;
#pragma unroll
          for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              *reinterpret_cast<u32x2*>(out + db * 32 + i * 8) =
                  u32x2{pack2(o[db][4 * i] * inv, o[db][4 * i + 1] * inv), pack2(o[db][4 * i + 2] * inv, o[db][4 * i + 3] * inv)};
          if (a.lse && half == 0) a.lse[(int64_t)(q0 + t) * a.b.Hq + h] = sum == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(sum)) * kLn2;
        } else if (row < of.rows) {
          const int64_t part = (int64_t)slot * kManyRows + wave * 32 + l32;
#pragma unroll
          for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              *reinterpret_cast<f32x4*>(a.part_o + part * D + db * 32 + i * 8 + half * 4) = f32x4{o[db][4 * i], o[db][4 * i + 1], o[db][4 * i + 2], o[db][4 * i + 3]};
          if (half == 0) { a.part_ml[2 * part] = m; a.part_ml[2 * part + 1] = sum; }
        }
      }
    }
    if (start <= x0) break;
    if (--block < 0) {                                           // the request before that has blocks, or the last one of the head before: 64 at a time
      for (;;) {
        const int candidate = r - 1 - lane;
        const uint64_t some = __ballot(candidate >= 0 && request(max(candidate, 0)).count > 0);
        if (some != 0) { r -= 1 + __builtin_ctzll(some); break; }
        r -= 64;
        if (r <= 0) { r = n; --head; }
      }
      of = uniform(request(r));
      block = of.count - 1;
    }
    start -= uniform(weight(of, block));
  }
  if (tid == 0 && !ma.whole) ma.cuts[g] = cut;
}

template <int D, bool FP8>
int launch_many_of(const ManyArgs& m, hipStream_t stream) {
  if (m.a.pool.page_log2 < 4) attend_many_kernel<D, FP8, true><<<dim3(m.workgroups), dim3(kManyThreads), 0, stream>>>(m);
  else attend_many_kernel<D, FP8, false><<<dim3(m.workgroups), dim3(kManyThreads), 0, stream>>>(m);
  return (int)hipGetLastError();
}

}  // namespace codecomp
