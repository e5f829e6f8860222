// Attention weights summed up per cached row (codecomp_attend_mass): sums[j] = decay sums[j] + 1/G sum over rows (new tokens x query heads of the KV head) of
// exp(softmax_scale q.k_j - lse).
//
// The logits are formed again from queries and keys, with the log-sum-exp of every row known: half of attention's products, and no row has to wait for
// another.  A key's weights of all rows meet in one workgroup (or in a fixed number of parts, added in order): no atomics.
//
// Few rows (up to 64): every key is read once for a handful of products, bound by memory.  A workgroup of four waves has a chunk of the cache, each wave
// tiles of 32 or 64 keys of its own, the next one on its way into registers.  S = Q K^T, 16 rows x 16 keys per MFMA: lane = key, so that a key's weights are added
// in place, and by two exchanges between lanes at the end.
//
// Many rows: bound by the matrix units and the vector work beside them.  A workgroup keeps 256 keys in registers, 64 a wave, and takes the rows that see
// them 32 at a time through LDS, four tiles in turn, three of them on their way.  S^T = K Q^T: lane = row, whose log-sum-exp and limit are two
// registers; a lane adds up the weights of its rows for each of 32 keys, and the lanes are added up once, at the end.
#include <float.h>
#include <math.h>

#include <algorithm>

#include "serve.h"

namespace codecomp {

struct MassArgs {
  PagePool pool;
  PagedBatch b;
  const uint16_t* q;
  const float* lse;
  const int32_t* first;
  float* sums;                 // of the layer
  int64_t s_seq, s_head;
  float* part;                 // many rows: [split][request * head][row]
  int64_t layer;               // byte offset of the layer in the pool
  float c, decay, share;       // softmax_scale * k_scale * log2(e); 1 / G
  int chunk, splits, rows_each;
};

constexpr int kMassWaves = 4, kMassThreads = 64 * kMassWaves;
constexpr int kMassKeys = 64 * kMassWaves;      // many rows: keys of a workgroup
constexpr int kMassStage = 512;                 // rows whose log-sum-exp and limit stand in LDS at a time

__device__ __forceinline__ int first_of(const MassArgs& a, int r) { return a.first ? max(a.first[r], 0) : 0; }

// Keys that a row sees; none, if its log-sum-exp says that it saw nothing.
__device__ __forceinline__ int limit_of(const MassArgs& a, int len, int nq, int t, float lse) {
  return lse == -INFINITY ? 0 : a.b.causal ? min(len, len - nq + t + 1) : len;
}

// What stood there before, for rows that are not new.
__device__ __forceinline__ float old_sum(const MassArgs& a, const float* sums, int j, int len, int nq) {
  return a.decay != 0.0f && j < (a.b.causal ? len - nq : len) ? sums[j] : 0.0f;
}

template <int D, bool FP8>
__global__ __launch_bounds__(kMassThreads, FP8 && D == 128 ? 3 : 4) void mass_few_kernel(const MassArgs a) {
  constexpr int LOADS = D * (FP8 ? 1 : 2) / 64, KS = D / 32, CG = LOADS >= 4 ? 2 : 4, KEYS = 16 * CG, STRIP = kMassWaves * KEYS;
  __shared__ __attribute__((aligned(16))) float row_lse[kFewRowsMost];
  __shared__ __attribute__((aligned(16))) int row_limit[kFewRowsMost];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), l16 = lane & 15, quarter = lane >> 4;
  // chunk by chunk, all requests and heads of one: short requests lack the later ones
  const int items = a.b.n_seqs * a.b.Hkv, turn = blockIdx.x / items, item = blockIdx.x - turn * items;
  const int r = item / a.b.Hkv, head = item - r * a.b.Hkv;
  const int64_t chunk0 = (int64_t)turn * a.chunk;
  const int key0 = (int)chunk0;
  const int32_t* table = a.b.table + (int64_t)r * a.b.table_width;
  // Page entries for keys tile + 16 g + l16.  Those of the first two tiles are sent for before it is known how many keys there are: one wait less.
  int page[CG], next_page[CG];
  auto look_up = [&](int (&pg)[CG], int64_t tile, int end) __attribute__((always_inline)) {
#pragma unroll
    for (int g = 0; g < CG; ++g) pg[g] = table[max((int)min(tile + 16 * g + l16, (int64_t)end - 1), 0) >> a.pool.page_log2];
  };
  look_up(page, chunk0 + wave * KEYS, a.b.max_kv);
  look_up(next_page, chunk0 + (kMassWaves + wave) * KEYS, a.b.max_kv);
  const int q0 = a.b.cu_q[r], nq = a.b.cu_q[r + 1] - q0, rows = nq * a.b.G;
  if (nq <= 0 || nq > kFewRowsMost || rows > kFewRowsMost) return;
  const int len = uniform(kv_len_of(a.b, r)), from = uniform(first_of(a, r)), key1 = (int)min((int64_t)len, chunk0 + a.chunk);
  if (key0 >= key1 || key1 <= from) return;
  if (tid < kFewRowsMost) {
    const int t = min(tid, rows - 1) / a.b.G, g = min(tid, rows - 1) - t * a.b.G;
    const float x = a.lse[(int64_t)(q0 + t) * a.b.Hq + head * a.b.G + g];
    row_lse[tid] = x * kLog2e;
    row_limit[tid] = tid < rows ? limit_of(a, len, nq, t, x) : 0;
  }
  u32x4 qf[KS];
  auto queries = [&](int rb) __attribute__((always_inline)) {
    const int row = min(rb * 16 + l16, rows - 1), t = row / a.b.G, g = row - t * a.b.G;
    const uint16_t* p = a.q + (q0 + t) * a.b.q_st + (head * a.b.G + g) * a.b.q_sh;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)              // an 8-bit piece of a key is the fragments of two steps
      qf[ks] = *reinterpret_cast<const u32x4*>(p + (FP8 ? (ks >> 1) * 64 + quarter * 16 + (ks & 1) * 8 : ks * 32 + quarter * 8));
  };
  queries(0);
  __syncthreads();
  const int blocks = uniform((rows + 15) >> 4);

  const unsigned char* kb = a.pool.k + a.layer + head * a.pool.s_head + quarter * 16;
  float* sums = a.sums + r * a.s_seq + head * a.s_head;
  const int in_page = (1 << a.pool.page_log2) - 1;
  u32x4 kr[CG][LOADS];
  float old;
  auto send_for = [&](int tile, const int (&pg)[CG]) __attribute__((always_inline)) {
    const int j = tile + lane;
    old = lane < KEYS && j >= from && j < key1 ? old_sum(a, sums, j, len, nq) : 0.0f;
    int64_t off[CG];
#pragma unroll
    for (int g = 0; g < CG; ++g)                 // rows that are not there: page 0, without weight below
      off[g] = (pg[g] >= 0 && pg[g] < a.pool.n_pages ? pg[g] : 0) * a.pool.s_page + ((tile + 16 * g + l16) & in_page) * (int)a.pool.s_tok;
#pragma unroll
    for (int g = 0; g < CG; ++g)
#pragma unroll
      for (int i = 0; i < LOADS; ++i) kr[g][i] = *reinterpret_cast<const u32x4*>(kb + off[g] + i * 64);
  };
  int tile = key0 + wave * KEYS;
  while (tile + KEYS <= from && tile < key1) {   // protected rows: the first tile that is not of them alone
    tile += (from - tile) / STRIP * STRIP;
    if (tile + KEYS <= from) tile += STRIP;
    look_up(page, tile, key1);
    look_up(next_page, (int64_t)tile + STRIP, key1);
  }
  if (tile < key1) send_for(tile, page);
  while (tile < key1) {
    int limit_key[CG];                           // the key, or one that nothing sees
#pragma unroll
    for (int g = 0; g < CG; ++g) limit_key[g] = page[g] >= 0 && page[g] < a.pool.n_pages ? tile + 16 * g + l16 : INT32_MAX;
    u32x4 kf[CG][KS];
#pragma unroll
    for (int g = 0; g < CG; ++g)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        if constexpr (FP8) kf[g][ks] = ks & 1 ? widen8(kr[g][ks >> 1].z, kr[g][ks >> 1].w) : widen8(kr[g][ks >> 1].x, kr[g][ks >> 1].y);
        else kf[g][ks] = kr[g][ks];
      }
    const float before = old;
    const int next = tile + STRIP;
#pragma unroll
    for (int g = 0; g < CG; ++g) page[g] = next_page[g];
    if (next < key1) {
      send_for(next, page);
      look_up(next_page, (int64_t)next + STRIP, key1);
    }
    float sum[CG];
#pragma unroll
    for (int g = 0; g < CG; ++g) sum[g] = 0.0f;
    for (int rb = 0; rb < blocks; ++rb) {
      if (blocks > 1) queries(rb);
      f32x4 s[CG];
#pragma unroll
      for (int g = 0; g < CG; ++g) {
        s[g] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) s[g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(frag(qf[ks]), frag(kf[g][ks]), s[g], 0, 0, 0);
      }
      const f32x4 l = *reinterpret_cast<const f32x4*>(row_lse + rb * 16 + quarter * 4);
      const int4 limit = *reinterpret_cast<const int4*>(row_limit + rb * 16 + quarter * 4);
#pragma unroll
      for (int g = 0; g < CG; ++g) {
        float w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __builtin_amdgcn_exp2f(fmaf(s[g][i], a.c, -l[i]));
        sum[g] += (limit_key[g] < limit.x ? w[0] : 0.0f) + (limit_key[g] < limit.y ? w[1] : 0.0f);
        sum[g] += (limit_key[g] < limit.z ? w[2] : 0.0f) + (limit_key[g] < limit.w ? w[3] : 0.0f);
      }
    }
    float mine = 0.0f;
#pragma unroll
    for (int g = 0; g < CG; ++g) {
      float x = sum[g] + __shfl_xor(sum[g], 16);
      x += __shfl_xor(x, 32);
      if (quarter == g) mine = x;
    }
    const int j = tile + lane;
    if (lane < KEYS && j >= from && j < key1) sums[j] = fmaf(a.decay, before, a.share * mine);
    tile = next;
  }
}

// Rows that see the first key of a block of keys begin here.
__device__ __forceinline__ int first_row(const MassArgs& a, int len, int nq, int key) { return a.b.causal ? max(key - (len - nq), 0) * a.b.G : 0; }

template <int D, bool FP8>
__global__ __launch_bounds__(kMassThreads, 2) void mass_many_kernel(const MassArgs a) {
  constexpr int KS = D / 16, LOADS = D * (FP8 ? 1 : 2) / 32;       // fragments of a key; 16-byte pieces of it that a lane has
  constexpr int GROUP = D / 32 * 1024, TILE = 2 * GROUP;            // bytes of 16 rows and of 32 in LDS: chunks of 1 KB, 16 rows of four 16-byte pieces, piece by piece
  constexpr int SENT = TILE / 1024 / kMassWaves;                    // chunks of a tile that a wave sends for
  constexpr int RED = 33;                                           // floats between keys where lanes are added up
  constexpr int LDS = 4 * TILE > kMassKeys * RED * 4 ? 4 * TILE : kMassKeys * RED * 4;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[LDS];
  __shared__ float row_lse[2][kMassStage];
  __shared__ int row_limit[2][kMassStage];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), l32 = lane & 31, half = lane >> 5;
  // blocks of keys of one part of the rows side by side: they read the same queries
  const int blocks = (a.b.max_kv + kMassKeys - 1) / kMassKeys;
  const int block = blockIdx.x % blocks, rest = blockIdx.x / blocks, items = a.b.n_seqs * a.b.Hkv, split = rest / items, item = rest - split * items;
  const int r = item / a.b.Hkv, head = item - r * a.b.Hkv;
  const int q0 = a.b.cu_q[r], nq = a.b.cu_q[r + 1] - q0, rows = nq * a.b.G;
  if (rows <= kFewRowsMost) return;
  const int len = uniform(kv_len_of(a.b, r)), from = uniform(first_of(a, r)), key0 = block * kMassKeys;
  if (key0 >= len || key0 + kMassKeys <= from) return;
  const int row0 = uniform(max(first_row(a, len, nq, key0) & -32, split * a.rows_each)), row1 = uniform(min(rows, (split + 1) * a.rows_each));
  if (row0 >= row1) return;

  // keys as left operands
  const int wave_key = key0 + wave * 64;
  const int32_t* table = a.b.table + (int64_t)r * a.b.table_width;
  u32x4 kf[2][KS];
  unsigned there[2];
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const int key = wave_key + g * 32 + l32, at = table[min(key, len - 1) >> a.pool.page_log2];
    const bool held = at >= 0 && at < a.pool.n_pages;
    there[g] = (unsigned)__ballot(held && key < len);
    const unsigned char* p = a.pool.k + a.layer + head * a.pool.s_head + (held ? at : 0) * a.pool.s_page + (min(key, len - 1) & ((1 << a.pool.page_log2) - 1)) * a.pool.s_tok + half * 16;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(p + i * 32);
      if constexpr (FP8) {
        kf[g][2 * i] = widen8(x.x, x.y);
        kf[g][2 * i + 1] = widen8(x.z, x.w);
      } else {
        kf[g][i] = x;
      }
    }
  }
  const bool all_there = there[0] == 0xFFFFFFFFu && there[1] == 0xFFFFFFFFu;

  // ---- rows.  Step s has rows row0 + 32 s and on; the last row stands for those behind it, without weight.
  const int steps = (row1 - row0 + 31) >> 5, G = a.b.G;
  const int load_row = row0 + (wave >> 1) * 16 + (lane & 15), piece = (wave & 1) * SENT * 4 + (lane >> 4);
  int load_t = load_row / G, load_g = load_row - load_t * G;        // of the next tile that is sent for
  const int step_t = 32 / G, step_g = 32 - step_t * G, last_t = (rows - 1) / G, last_g = rows - 1 - last_t * G;
  const uint16_t* queries = a.q + q0 * a.b.q_st + head * G * a.b.q_sh + piece * 8;
  auto fetch = [&](int step) __attribute__((always_inline)) {
    const bool behind = load_t > last_t || (load_t == last_t && load_g > last_g);
    const uint16_t* p = queries + (behind ? last_t : load_t) * a.b.q_st + (behind ? last_g : load_g) * a.b.q_sh;
    const uint32_t to = lds_address(lds) + (step & 3) * TILE + wave * SENT * 1024;
#pragma unroll
    for (int i = 0; i < SENT; ++i)
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to + i * 1024), "v"(p + i * 32) : "memory", "m0");
    load_t += step_t;
    load_g += step_g;
    if (load_g >= G) { load_g -= G; ++load_t; }
  };
  auto stage = [&](int number) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kMassStage / kMassThreads; ++i) {
      const int at = i * kMassThreads + tid, row = row0 + number * kMassStage + at, rr = min(row, rows - 1), t = rr / G, g = rr - t * G;
      const float x = a.lse[(int64_t)(q0 + t) * a.b.Hq + head * G + g];
      row_lse[number & 1][at] = x * kLog2e;
      row_limit[number & 1][at] = row < row1 ? limit_of(a, len, nq, t, x) : 0;
    }
  };
  f32x16 sum[2];
#pragma unroll
  for (int g = 0; g < 2; ++g)
#pragma unroll
    for (int i = 0; i < 16; ++i) sum[g][i] = 0.0f;
  stage(0);
  fetch(0); fetch(1); fetch(2);
  const unsigned char* q_lane = lds + (l32 >> 4) * GROUP + (l32 & 15) * 16 + half * (FP8 ? 512 : 256);
  for (int s = 0; s < steps; ++s) {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(2 * SENT) : "memory");       // tile s has come, and tile s - 1 is nobody's
    fetch(s + 3);
    if ((s & 15) == 8) stage((s >> 4) + 1);
    const unsigned char* qt = q_lane + (s & 3) * TILE;
    f32x16 z[2];
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int i = 0; i < 16; ++i) z[g][i] = 0.0f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const int p = FP8 ? (ks >> 1) * 4 + (ks & 1) : 2 * ks;       // piece of the lower half of the lanes
      const bf16x8 qf = frag(*reinterpret_cast<const u32x4*>(qt + (p >> 2) * 1024 + (p & 3) * 256));
#pragma unroll
      for (int g = 0; g < 2; ++g) z[g] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag(kf[g][ks]), qf, z[g], 0, 0, 0);
    }
    const int at = (s & 15) * 32 + l32;
    const float l = row_lse[(s >> 4) & 1][at];
    const int limit = row_limit[(s >> 4) & 1][at];
    if (__builtin_expect(all_there && __ballot(limit < wave_key + 64) == 0, 1)) {
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int i = 0; i < 16; ++i) sum[g][i] += __builtin_amdgcn_exp2f(fmaf(z[g][i], a.c, -l));
    } else {
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int j = 8 * (i >> 2) + 4 * half + (i & 3);
          const float w = __builtin_amdgcn_exp2f(fmaf(z[g][i], a.c, -l));
          sum[g][i] += ((there[g] >> j) & 1) && wave_key + g * 32 + j < limit ? w : 0.0f;
        }
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");                  // what was sent for beyond the last row
  __syncthreads();
  // lanes added up: key by key, the 32 lanes of one side by side
  float* red = reinterpret_cast<float*>(lds) + wave * 64 * RED;
#pragma unroll
  for (int g = 0; g < 2; ++g)
#pragma unroll
    for (int i = 0; i < 16; ++i) red[(g * 32 + 8 * (i >> 2) + 4 * half + (i & 3)) * RED + l32] = sum[g][i];
  __syncthreads();
  float x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < 32; ++i) x[i & 3] += red[lane * RED + i];
  const float mine = (x[0] + x[1]) + (x[2] + x[3]);
  const int j = wave_key + lane;
  if (j < from || j >= len) return;
  if (a.splits > 1) {
    a.part[((int64_t)split * items + item) * a.b.max_kv + j] = mine;
    return;
  }
  float* sums = a.sums + r * a.s_seq + head * a.s_head;
  sums[j] = fmaf(a.decay, old_sum(a, sums, j, len, nq), a.share * mine);
}

// Parts of the rows added up, a thread for each key.
__global__ __launch_bounds__(kMassThreads) void mass_join_kernel(const MassArgs a) {
  const int items = a.b.n_seqs * a.b.Hkv, blocks = (a.b.max_kv + kMassKeys - 1) / kMassKeys, item = blockIdx.x / blocks, block = blockIdx.x - item * blocks;
  const int r = item / a.b.Hkv, head = item - r * a.b.Hkv, nq = a.b.cu_q[r + 1] - a.b.cu_q[r], rows = nq * a.b.G;
  if (rows <= kFewRowsMost) return;
  const int len = kv_len_of(a.b, r), j = block * kMassKeys + threadIdx.x;
  if (j < first_of(a, r) || j >= len) return;
  const int s0 = (first_row(a, len, nq, block * kMassKeys) & -32) / a.rows_each, s1 = (rows + a.rows_each - 1) / a.rows_each;
  float x = 0.0f;
#pragma unroll 8
  for (int s = s0; s < s1; ++s) x += a.part[((int64_t)s * items + item) * a.b.max_kv + j];
  float* sums = a.sums + r * a.s_seq + head * a.s_head;
  sums[j] = fmaf(a.decay, old_sum(a, sums, j, len, nq), a.share * x);
}

// Workgroups that a call of many rows is cut into where it can be.
constexpr int64_t kMassUnits = 2048;
constexpr int kMassLeastRows = 1024;             // of a part
constexpr int64_t kMostBlocks = (1 << 24) - 1;    // of 256 threads: an axis of a grid holds 2^32 threads

int make_mass_plan(const codecomp_batch* b, const codecomp_pages* p, const codecomp_mass* m, MassPlan* pl) {
  if (int rc = make_pool(p, &pl->pool)) return rc;
  if (int rc = make_batch(b, p, &pl->batch)) return rc;
  if (int rc = make_mass(m, &pl->mass)) return rc;
  const PagedBatch& x = pl->batch;
  if (m->n_layers != p->n_layers || m->n_seqs != b->n_seqs || m->n_kv_heads != p->n_kv_heads || m->width < b->max_kv_len) return CODECOMP_EINVAL_SHAPE;
  pl->d = p->head_dim;
  pl->scale = b->softmax_scale > 0.0f ? b->softmax_scale : 1.0f / sqrtf((float)p->head_dim);
  pl->few_rows = pl->many_rows = 0;
  int64_t most = 0;
  for (int r = 0; r < x.n_seqs; ++r) {
    const int64_t rows = (int64_t)(b->cu_q_host[r + 1] - b->cu_q_host[r]) * x.G;
    if (rows > kFewRowsMost) { ++pl->many_rows; most = std::max(most, rows); }
    else if (rows > 0) ++pl->few_rows;
  }
  const int64_t items = (int64_t)x.n_seqs * x.Hkv;
  int64_t chunk = (items * x.max_kv / 2048 + 255) / 256 * 256;
  chunk = std::min<int64_t>(std::max<int64_t>(chunk, 256), 2048);
  while (items * ((x.max_kv + chunk - 1) / chunk) > kMostBlocks && chunk < x.max_kv) chunk *= 2;
  pl->chunk = (int)std::min<int64_t>(chunk, 1 << 30);
  pl->chunks = (int)((x.max_kv + chunk - 1) / chunk);
  if (pl->few_rows > 0 && items * pl->chunks > kMostBlocks) return CODECOMP_EINVAL_SHAPE;
  pl->blocks = (x.max_kv + kMassKeys - 1) / kMassKeys;
  pl->splits = pl->rows_each = 0;
  pl->ws_bytes = 0;
  if (pl->many_rows > 0 && pl->blocks > 0) {
    if (items * pl->blocks > kMostBlocks) return CODECOMP_EINVAL_SHAPE;
    const int64_t units = (int64_t)pl->many_rows * x.Hkv * pl->blocks;
    int64_t splits = std::max<int64_t>(1, std::min(kMassUnits / units, most / kMassLeastRows));
    splits = std::min(splits, std::max<int64_t>(1, kMostBlocks / (items * pl->blocks)));
    pl->rows_each = (int)std::min<int64_t>(((most + splits - 1) / splits + 31) / 32 * 32, INT32_MAX & -32);
    pl->splits = (int)((most + pl->rows_each - 1) / pl->rows_each);
    if (pl->splits > 1) pl->ws_bytes = ((size_t)pl->splits * items * x.max_kv * sizeof(float) + 255) & ~(size_t)255;
  }
  return CODECOMP_OK;
}

template <int D, bool FP8>
static int launch_mass_of(const MassPlan& pl, const MassArgs& a, hipStream_t stream) {
  const int64_t items = (int64_t)pl.batch.n_seqs * pl.batch.Hkv;
  const dim3 block(kMassThreads);
  if (pl.few_rows > 0) {
    mass_few_kernel<D, FP8><<<dim3((unsigned)(items * pl.chunks)), block, 0, stream>>>(a);
    if (hipError_t e = hipGetLastError()) return (int)e;
  }
  if (pl.many_rows > 0) {
    mass_many_kernel<D, FP8><<<dim3((unsigned)(items * pl.blocks * pl.splits)), block, 0, stream>>>(a);
    if (hipError_t e = hipGetLastError()) return (int)e;
    if (pl.splits > 1) mass_join_kernel<<<dim3((unsigned)(items * pl.blocks)), block, 0, stream>>>(a);
  }
  return (int)hipGetLastError();
}

int launch_mass(const MassPlan& pl, const void* q, const float* lse, int layer, const int32_t* first, float decay, void* workspace, hipStream_t stream) {
  if (pl.batch.max_kv == 0) return 0;
  MassArgs a = {};
  a.pool = pl.pool; a.b = pl.batch; a.q = static_cast<const uint16_t*>(q); a.lse = lse; a.first = first;
  a.sums = pl.mass.sums + layer * pl.mass.s_layer; a.s_seq = pl.mass.s_seq; a.s_head = pl.mass.s_head;
  a.part = static_cast<float*>(workspace);
  a.layer = layer * pl.pool.s_layer;
  a.c = fminf(fmaxf(pl.scale * pl.pool.k_scale * kLog2e, FLT_MIN), FLT_MAX);
  a.decay = decay; a.share = 1.0f / pl.batch.G;
  a.chunk = pl.chunk; a.splits = pl.splits; a.rows_each = pl.rows_each;
  if (pl.d == 128) return pl.pool.fp8 ? launch_mass_of<128, true>(pl, a, stream) : launch_mass_of<128, false>(pl, a, stream);
  return pl.pool.fp8 ? launch_mass_of<64, true>(pl, a, stream) : launch_mass_of<64, false>(pl, a, stream);
}

}  // namespace codecomp
