// Attention weights summed up per cached row (codecomp_attend_mass): sums[j] = decay sums[j] + 1/G sum over rows (new tokens x query heads of the KV head) of
// exp(softmax_scale q.k_j - lse).
//
// The logits are formed again from queries and keys, with the log-sum-exp of every row known: half of attention's products, and no row has to wait for
// another.  A key's weights of all rows meet in one workgroup (or in a fixed number of parts, added in order): no atomics.  Logits, weights and sums are fp32.
//
// Few rows (up to 64; up to 16 beside requests of more): every key is read once for a handful of products, bound by memory.  A workgroup of four waves has a stretch of the cache, each wave
// tiles of 32 (head_dim 128) or 64 keys of its own, the next one on its way into registers.  S = Q K^T, 16 rows x 16 keys per MFMA: lane = key, so that a key's
// weights are added in place, and by two exchanges between lanes at the end.  64 requests of 500 to 16384 rows, 8 KV heads of 128, 8 bits: 118 us, 4.6 TB/s;
// 64 of 300 to 4100 behind 8192 protected ones, 4 KV heads, bf16: 38 us, 4.2 TB/s.  One token over 2113 rows: 7 us, which is what the launch takes.
// Tried before: two tiles on their way (no gain), tiles of 64 keys at head_dim 128 (202 us: registers spill), five waves (133).
//
// Many rows: bound by the matrix units and the vector work beside them (an exponential, a product and a sum a logit).  A workgroup of eight waves keeps 512 keys in
// registers, 64 a wave, and takes the rows that see them 32 at a time through LDS, eight tiles in turn, up to six of them on their way; waves meet at every
// second one (at each: 265 us instead of 263 below, 471 instead of 466 for 2048 tokens over 32768 8-bit rows).  S^T = K Q^T: lane = row, whose
// log-sum-exp and limit are two registers; a lane adds up the weights of its rows for each of 32 keys, and the lanes are added up once, at the end.
// The logits of a tile are formed while those of the tile before become weights, in an order that the source gives: MFMAs and vector work take turns.
// A prompt of 8191 tokens, 28 query heads of 128: 258 to 264 us, 0.91 to 0.93 PFLOP/s.  A step of 32 rows takes 0.97 us, 2040 cycles, of which the vector work of a SIMD's two
// waves takes 1670 (a logit is an exponential at a quarter of the rate, a product and a sum) and its MFMAs 1020.
// The work is cut into equal parts of rows over all blocks of keys, one for each compute unit, and the parts of a block that was cut are added by a second kernel: a
// workgroup for a block, or for two halves, took 293 us and more (blocks at the end of a causal prompt have few rows, and two workgroups on one
// compute unit do not share it evenly).  Tried before: four waves and two workgroups on a compute unit (278), three waves for a SIMD (273: registers spill),
// the keys waited for inside of the loop (496: the waits count what was sent for since).
#include <float.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "serve.h"

namespace codecomp {

// A block of keys whose rows several workgroups share: the first one has part 2 * share + 1, those after it 2 * share.
struct CutKeys {
  int32_t r, block, head;      // r < 0: none begins in this share
  int32_t last;                // share with the last rows
};

struct MassArgs {
  PagePool pool;
  PagedBatch b;
  const uint16_t* q;
  const float* lse;
  const int32_t* first;
  float* sums;                 // of the layer
  int64_t s_seq, s_head;
  float* part;                 // many rows: [2 * share][key of the block]
  CutKeys* cuts;               // [shares]
  int64_t layer;               // byte offset of the layer in the pool
  float c, decay, share;       // softmax_scale * k_scale * log2(e); 1 / G
  int chunk, shares, few_shares;
  int few_most;                // rows of a request up to which the kernel for few has it
};

constexpr int kMassWaves = 4, kMassThreads = 64 * kMassWaves;
constexpr int kManyMassWaves = 8, kManyMassThreads = 64 * kManyMassWaves, kMassKeys = 64 * kManyMassWaves;      // many rows: keys of a workgroup
constexpr int kMassStage = 512;                 // rows whose log-sum-exp and limit stand in LDS at a time
// Rows' worth of positions in front of a block's rows, for starting on its keys and ending it (a prompt of 8191 tokens, 16 of 20 to 400 over 400 to 3000 rows, four of 64
// over 500 to 4096, us: 256: 272, 76, 42; 384: 270, 81, 23; 512: 269, 81, 23; 768: 265, 80, 25; 1536: 273, 97, 29).
constexpr int kMassLead = 768;
// Rows' worth that a workgroup gets at least: more than the 32 of a tile, so that every workgroup between the first and the last of a block has some
// (100 tokens over 300 rows and 512 over 4096, us: 32: 16, 34; 64: 18, 34; 128: 19, 33; 256: 22, 33; 1024: 36, 48).
constexpr int kMassLeast = 64;

__device__ __forceinline__ int first_of(const MassArgs& a, int r) { return a.first ? max(a.first[r], 0) : 0; }

// Keys that a row sees; none, if its log-sum-exp says that it saw nothing.
__device__ __forceinline__ int limit_of(const MassArgs& a, int len, int nq, int t, float lse) {
  return lse == -INFINITY ? 0 : a.b.causal ? min(len, len - nq + t + 1) : len;
}

// What stood there before, for rows that are not new.
__device__ __forceinline__ float old_sum(const MassArgs& a, const float* sums, int j, int len, int nq) {
  return a.decay != 0.0f && j < (a.b.causal ? len - nq : len) ? sums[j] : 0.0f;
}

// Keys of a request that the kernel for few rows takes, in strips of what four waves read at a time: from the one with the first that counts on.
template <int STRIP>
__device__ __forceinline__ int mass_strips(const MassArgs& a, int r) {
  const int nq = a.b.cu_q[r + 1] - a.b.cu_q[r], len = kv_len_of(a.b, r), from = first_of(a, r);
  return nq <= 0 || nq > a.few_most || nq * a.b.G > a.few_most || from >= len ? 0 : (len + STRIP - 1) / STRIP - from / STRIP;
}

// EVEN: the strips of all requests and heads form one sequence, cut into equal parts; else a workgroup has one chunk of a request.
// ROWWISE: pages of less than 16 rows; else 16 rows of a tile lie in one page, whose place is worked out in scalar registers.
template <int D, bool FP8, bool EVEN, bool ROWWISE>
__global__ __launch_bounds__(kMassThreads, 4) void mass_few_kernel(const MassArgs a) {
  constexpr int LOADS = D * (FP8 ? 1 : 2) / 64, KS = D / 32, CG = D == 128 ? 2 : 4, KEYS = 16 * CG, STRIP = kMassWaves * KEYS;
  __shared__ __attribute__((aligned(16))) float row_lse[kFewRowsMost];
  __shared__ __attribute__((aligned(16))) int row_limit[kFewRowsMost];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  int l16 = lane & 15, quarter = lane >> 4;
  int r, head, key0, strip = 0;
  int64_t left = 0;                                              // EVEN: strips that are left
  const int32_t* table;
  // Page entries for keys tile + 16 g + l16.  Those of a chunk's first two tiles are sent for before it is known how many keys there are: one wait less.
  int page[CG], next_page[CG];
  auto look_up = [&](int (&pg)[CG], int64_t tile, int end) __attribute__((always_inline)) {
#pragma unroll
    for (int g = 0; g < CG; ++g) {
      const int at = max((int)min(tile + 16 * g + (ROWWISE ? l16 : 0), (int64_t)end - 1), 0) >> a.pool.page_log2;
      if constexpr (ROWWISE) pg[g] = table[at];
      else pg[g] = ((const __attribute__((address_space(4))) int32_t*)table)[at];
    }
  };
  if constexpr (EVEN) {
    __shared__ int64_t wave_sum[kMassWaves];
    __shared__ int found[2];
    const int n = a.b.n_seqs, per = (n + kMassThreads - 1) / kMassThreads, r0 = min(tid * per, n), r1 = min(r0 + per, n);
    int64_t mine = 0;
    for (int i = r0; i < r1; ++i) mine += mass_strips<STRIP>(a, i);
    int64_t incl = mine;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int64_t y = __shfl_up(incl, off);
      if (lane >= off) incl += y;
    }
    if (lane == 63) wave_sum[wave] = incl;
    __syncthreads();
    int64_t before = incl - mine, per_head = 0;
#pragma unroll
    for (int w = 0; w < kMassWaves; ++w) {
      if (w < wave) before += wave_sum[w];
      per_head += wave_sum[w];
    }
    per_head = uniform(per_head);
    const int64_t total = per_head * a.b.Hkv, shares = uniform(min((int64_t)a.few_shares, total)), share = blockIdx.x;
    if (share >= shares) return;
    const int64_t at_strip = uniform(share * total / shares);
    left = uniform((share + 1) * total / shares) - at_strip;
    head = uniform((int)(at_strip / per_head));
    int64_t at = at_strip - head * per_head - before;
    if (at >= 0 && at < mine) {                                  // one thread has it
      int i = r0;
      for (int w = mass_strips<STRIP>(a, i); at >= w; w = mass_strips<STRIP>(a, i)) { at -= w; ++i; }
      found[0] = i; found[1] = (int)at;
    }
    __syncthreads();
    r = uniform(found[0]); strip = uniform(found[1]);
  } else {
    // chunk by chunk, all requests and heads of one: short requests lack the later ones
    const int items = a.b.n_seqs * a.b.Hkv, turn = blockIdx.x / items, item = blockIdx.x - turn * items;
    r = item / a.b.Hkv; head = item - r * a.b.Hkv;
    key0 = (int)min((int64_t)turn * a.chunk, (int64_t)a.b.max_kv);
    table = a.b.table + (int64_t)r * a.b.table_width;
    look_up(page, key0 + wave * KEYS, a.b.max_kv);
    look_up(next_page, key0 + (kMassWaves + wave) * KEYS, a.b.max_kv);
  }
  for (;;) {
    if constexpr (EVEN) asm("" : "+v"(l16), "+v"(quarter));         // what follows from them is worked out per piece, not held in registers from piece to piece
    const int q0 = uniform(a.b.cu_q[r]), nq = uniform(a.b.cu_q[r + 1]) - q0, rows = nq * a.b.G;
    const int len = uniform(kv_len_of(a.b, r)), from = uniform(first_of(a, r));
    int key1;
    if constexpr (EVEN) {
      const int strips = uniform(mass_strips<STRIP>(a, r)), end = (int)min((int64_t)strips, strip + left), at = from / STRIP;
      key0 = (at + strip) * STRIP;
      key1 = (int)min((int64_t)len, (int64_t)(at + end) * STRIP);
      left -= end - strip;
      table = a.b.table + (int64_t)r * a.b.table_width;
      look_up(page, (int64_t)key0 + wave * KEYS, key1);
      look_up(next_page, (int64_t)key0 + (kMassWaves + wave) * KEYS, key1);
    } else {
      if (nq <= 0 || nq > a.few_most || rows > a.few_most) return;
      key1 = (int)min((int64_t)len, (int64_t)key0 + a.chunk);
      if (key0 >= key1 || key1 <= from) return;
    }
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
    const int blocks = uniform((rows + 15) >> 4);

    const unsigned char* kb = a.pool.k + a.layer + head * a.pool.s_head;
    float* sums = a.sums + r * a.s_seq + head * a.s_head;
    const int in_page = (1 << a.pool.page_log2) - 1;
    const uint32_t lane_off = quarter * 16 + (ROWWISE ? 0 : l16 * (uint32_t)a.pool.s_tok);
    u32x4 kr[CG][LOADS];
    float old;
    auto send_for = [&](int tile, const int (&pg)[CG]) __attribute__((always_inline)) {
      const int j = tile + lane;
      old = lane < KEYS && j >= from && j < key1 ? old_sum(a, sums, j, len, nq) : 0.0f;
      int64_t off[CG];
#pragma unroll
      for (int g = 0; g < CG; ++g)                 // rows that are not there: page 0, without weight below
        off[g] = (pg[g] >= 0 && pg[g] < a.pool.n_pages ? pg[g] : 0) * a.pool.s_page + ((tile + 16 * g + (ROWWISE ? l16 : 0)) & in_page) * (int)a.pool.s_tok;
#pragma unroll
      for (int g = 0; g < CG; ++g)
#pragma unroll
        for (int i = 0; i < LOADS; ++i) kr[g][i] = *reinterpret_cast<const u32x4*>(kb + off[g] + lane_off + i * 64);
    };
    int tile = key0 + wave * KEYS;
    while (tile + KEYS <= from && tile < key1) {   // protected rows: the first tile that is not of them alone
      tile += (from - tile) / STRIP * STRIP;
      if (tile + KEYS <= from) tile += STRIP;
      look_up(page, tile, key1);
      look_up(next_page, (int64_t)tile + STRIP, key1);
    }
    if (tile < key1) send_for(tile, page);
    __syncthreads();
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
      const int64_t next = (int64_t)tile + STRIP;
#pragma unroll
      for (int g = 0; g < CG; ++g) page[g] = next_page[g];
      if (next < key1) {
        send_for((int)next, page);
        look_up(next_page, next + STRIP, key1);
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
      tile = (int)min(next, (int64_t)key1);
    }
    if constexpr (!EVEN) return;
    if (left <= 0) break;
    strip = 0;
    for (++r;;) {                                                  // the next request with strips, or the first one of the next head: 64 at a time
      const uint64_t some = __ballot(r + lane < a.b.n_seqs && mass_strips<STRIP>(a, min(r + lane, a.b.n_seqs - 1)) > 0);
      if (some != 0) { r += __builtin_ctzll(some); break; }
      r += 64;
      if (r >= a.b.n_seqs) { r = 0; ++head; }
    }
    __syncthreads();                                               // through with LDS
  }
}

// Blocks of 512 keys of a request, and the rows that see them: of block b those from row_of(b) on, the first one's first key being seen by the most.
struct KeyBlocks {
  int len, nq, G, q0, rows, first, count, off;       // keys, tokens, ..., first block that is not of protected rows alone, blocks from there on, rows before the new ones
  __device__ __forceinline__ int row_of(int b) const { return off == INT32_MAX ? 0 : max(b * kMassKeys - off, 0) * G; }
  __device__ __forceinline__ int64_t weight(int b) const { return kMassLead + rows - row_of(b); }
  __device__ __forceinline__ int64_t before(int n) const {       // weight of the first n blocks
    int64_t rest = 0;
    if (off != INT32_MAX) {
      const int end = first + n, c = min(max(first, off < 0 ? 0 : off / kMassKeys + 1), end);       // blocks from c on are not seen by all rows
      rest = (int64_t)(end - 1 + c) * (end - c) / 2 * kMassKeys - (int64_t)off * (end - c);
    }
    return (int64_t)n * (kMassLead + rows) - rest * G;
  }
};
__device__ __forceinline__ KeyBlocks blocks_of(const MassArgs& a, int r) {
  KeyBlocks x;
  x.len = kv_len_of(a.b, r);
  x.q0 = a.b.cu_q[r];
  x.nq = a.b.cu_q[r + 1] - x.q0;
  x.G = a.b.G;
  x.rows = x.nq * x.G;
  x.off = a.b.causal ? x.len - x.nq : INT32_MAX;
  x.first = first_of(a, r) / kMassKeys;
  x.count = x.rows <= a.few_most || first_of(a, r) >= x.len ? 0 : (x.len + kMassKeys - 1) / kMassKeys - x.first;
  return x;
}

template <int D, bool FP8>
__global__ __launch_bounds__(kManyMassThreads, 2) void mass_many_kernel(const MassArgs a) {
  constexpr int KS = D / 16, LOADS = D * (FP8 ? 1 : 2) / 32;       // fragments of a key; 16-byte pieces of it that a lane has
  constexpr int GROUP = D / 32 * 1024, TILE = 2 * GROUP;            // bytes of 16 rows and of 32 in LDS: chunks of 1 KB, 16 rows of four 16-byte pieces, piece by piece
  constexpr int TILES = 8, AHEAD = TILES - 2;                       // in LDS, and on their way there
  constexpr int SENDERS = TILE / 1024;                              // waves that send for a chunk of a tile each
  constexpr int RED = 33;                                           // floats between keys where lanes are added up
  constexpr int LDS = TILES * TILE > kMassKeys * RED * 4 ? TILES * TILE : kMassKeys * RED * 4;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[LDS];
  __shared__ float row_lse[2][kMassStage];
  __shared__ int row_limit[2][kMassStage];
  __shared__ int64_t wave_sum[kManyMassWaves], found_at;
  __shared__ int found[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), l32 = lane & 31, half = lane >> 5;

  // ---- this workgroup's share: the rows of all blocks of keys of all requests and heads form one sequence, cut into equal parts
  const int n = a.b.n_seqs, per = (n + kManyMassThreads - 1) / kManyMassThreads, r0 = min(tid * per, n), r1 = min(r0 + per, n);
  auto weight_of = [&](int i) __attribute__((always_inline)) {
    const KeyBlocks x = blocks_of(a, i);
    return x.before(x.count);
  };
  int64_t mine = 0;
  for (int i = r0; i < r1; ++i) mine += weight_of(i);
  int64_t incl = mine;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int64_t y = __shfl_up(incl, off);
    if (lane >= off) incl += y;
  }
  if (lane == 63) wave_sum[wave] = incl;
  __syncthreads();
  int64_t before = incl - mine, per_head = 0;
#pragma unroll
  for (int w = 0; w < kManyMassWaves; ++w) {
    if (w < wave) before += wave_sum[w];
    per_head += wave_sum[w];
  }
  per_head = uniform(per_head);
  const int64_t total = per_head * a.b.Hkv, shares = uniform(min((int64_t)a.shares, (total + kMassLeast - 1) / kMassLeast));
  if (tid == 0 && blockIdx.x >= shares) a.cuts[blockIdx.x].r = -1;
  // neighbours in the sequence read the same queries: they run on the same die (workgroups go to the eight dies in turn)
  const int per_die = ((int)shares + 7) / 8, share = (int)(blockIdx.x & 7) * per_die + (int)(blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= per_die || share >= shares) return;
  const int64_t x0 = uniform(share * total / shares), x1 = uniform((share + 1) * total / shares);
  int head = uniform((int)(x0 / per_head));
  {
    int64_t at = x0 - head * per_head - before;
    if (at >= 0 && at < mine) {                                  // one thread has it
      int i = r0;
      for (int64_t w = weight_of(i); at >= w; w = weight_of(i)) { at -= w; ++i; }
      found[0] = i; found_at = at;
    }
  }
  __syncthreads();
  int r = uniform(found[0]);
  KeyBlocks of = blocks_of(a, r);
  {
    const int64_t at = found_at;
    for (int i = tid; i < of.count; i += kManyMassThreads) {
      const int64_t w = of.before(i);
      if (at >= w && at < w + of.weight(of.first + i)) { found[1] = of.first + i; wave_sum[0] = at - w; }
    }
  }
  __syncthreads();
  int block = uniform(found[1]);
  int64_t start = uniform(x0 - wave_sum[0]);                       // position of the block
  CutKeys cut = {-1, 0, 0, 0};

  for (;;) {
    const int len = uniform(of.len), nq = uniform(of.nq), q0 = uniform(of.q0), rows = uniform(of.rows), from = uniform(first_of(a, r)), G = a.b.G;
    const int key0 = block * kMassKeys, first_row = uniform(of.row_of(block)), all = rows - first_row;
    const int64_t front = start + kMassLead;                       // position of the block's first row
    const int row0 = uniform(first_row + (int)min((max(x0 - front, (int64_t)0) + 31) & -32, (int64_t)all));
    const int row1 = uniform(x1 >= front + all ? rows : first_row + (int)min((max(x1 - front, (int64_t)0) + 31) & -32, (int64_t)all));
    const int64_t next_block = front + all;
    if (row0 < row1) {
      const bool whole = row0 == first_row && row1 == rows;
      const int slot = row0 > first_row ? 2 * share : 2 * share + 1;
      if (row0 == first_row && row1 < rows)                        // the rest of the rows is the next workgroups'
        cut = {r, block, head, uniform((int)(((front + (all - 1) / 32 * 32 + 1) * shares - 1) / total))};
      __syncthreads();                                             // through with LDS
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

      // They have come before the loop, whose own waits count what it sends for.
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) asm volatile("" ::"v"(kf[g][ks]));

      // ---- rows.  Step s has rows row0 + 32 s and on; the last row stands for those behind it, without weight.
      const int steps = (row1 - row0 + 31) >> 5;
      const int piece = wave % (D / 32) * 4 + (lane >> 4);
      int load_row = row0 + wave / (D / 32) * 16 + (lane & 15), load_g = load_row % G;        // of the next tile that is sent for
      const int64_t step_row = (32 / G) * a.b.q_st + (32 % G) * a.b.q_sh, wrap = a.b.q_st - G * a.b.q_sh;
      const uint16_t* queries = a.q + q0 * a.b.q_st + head * G * a.b.q_sh + piece * 8;
      const uint16_t* load_at = queries + (load_row / G) * a.b.q_st + load_g * a.b.q_sh;
      const uint16_t* last_at = queries + (nq - 1) * a.b.q_st + (G - 1) * a.b.q_sh;
      auto fetch = [&](int step) __attribute__((always_inline)) {
        const uint16_t* p = load_row < rows ? load_at : last_at;
        if (wave < SENDERS)
          asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds_address(lds) + (step & (TILES - 1)) * TILE + wave * 1024), "v"(p) : "memory", "m0");
        load_row += 32;
        load_g += 32 % G;
        load_at += step_row;
        if (load_g >= G) { load_g -= G; load_at += wrap; }
      };
      auto stage = [&](int number) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kMassStage / kManyMassThreads; ++i) {
          const int at = i * kManyMassThreads + tid, row = row0 + number * kMassStage + at, rr = min(row, rows - 1), t = rr / G, g = rr - t * G;
          const float x = a.lse[(int64_t)(q0 + t) * a.b.Hq + head * G + g];
          row_lse[number & 1][at] = x == -INFINITY ? 0.0f : x * kLog2e;
          row_limit[number & 1][at] = row < row1 ? limit_of(a, len, nq, t, x) : 0;
        }
      };
      f32x16 sum[2], za[2], zb[2];
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int i = 0; i < 16; ++i) sum[g][i] = zb[g][i] = 0.0f;
      stage(0);
#pragma unroll
      for (int f = 0; f < AHEAD; ++f) fetch(f);
      const unsigned char* q_lane = lds + (l32 >> 4) * GROUP + (l32 & 15) * 16 + half * (FP8 ? 512 : 256);
      auto query_frag = [&](const unsigned char* qt, int ks) __attribute__((always_inline)) {
        const int p = FP8 ? (ks >> 1) * 4 + (ks & 1) : 2 * ks;         // piece of the lower half of the lanes
        return *reinterpret_cast<const u32x4*>(qt + (p >> 2) * 1024 + (p & 3) * 256);
      };
      // One step: the logits z of its rows on the matrix cores, beside them the weights of the rows before, whose logits are zp and log-sum-exp lp.  The order is the
      // source's: an LDS read for some fragments further on (from the next tile at the end), two MFMAs, the vector work of some logits.
      float lp = INFINITY;                                             // before the first step: no weight
      int limit_p = INT32_MAX;
      constexpr int RING = D == 128 ? 6 : 4, PER = 16 / KS;                           // fragments held; logits of each 32 keys beside a fragment
      u32x4 ring[RING];
      auto weigh = [&](f32x16 (&zp)[2], int f) __attribute__((always_inline)) {
#pragma unroll
        for (int i = f * PER; i < (f + 1) * PER; ++i)
#pragma unroll
          for (int g = 0; g < 2; ++g) sum[g][i] += __builtin_amdgcn_exp2f(fmaf(zp[g][i], a.c, -lp));
      };
      // Logits of keys that a row does not see.
      auto mask = [&](f32x16 (&zp)[2]) __attribute__((always_inline)) {
        if (__builtin_expect(all_there && __ballot(limit_p < wave_key + 64) == 0, 1)) return;
        const bool odd = lp != lp;                                     // a row whose log-sum-exp is NaN: what it sees is, what it does not see is not
        if (__builtin_expect(__ballot(odd) != 0, 0)) {
#pragma unroll
          for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int i = 0; i < 16; ++i) zp[g][i] = odd ? lp : zp[g][i];
          if (odd) lp = 0.0f;
        }
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          const int n = min(max(limit_p - (wave_key + g * 32), 0), 32);
          const unsigned seen = (there[g] & (unsigned)(((uint64_t)1 << n) - 1)) >> (4 * half);
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int m = (int)(seen << (31 - 8 * (i >> 2) - (i & 3))) >> 31;       // all ones or zeros
            zp[g][i] = __int_as_float((m & __float_as_int(zp[g][i])) | (~m & 0xFF800000));
          }
        }
      };
      auto step = [&](int s, f32x16 (&z)[2], f32x16 (&zp)[2], auto even) __attribute__((always_inline)) {
        const unsigned char *qt = q_lane + (s & (TILES - 1)) * TILE, *next = q_lane + ((s + 1) & (TILES - 1)) * TILE;
        if constexpr (decltype(even)::value) asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(AHEAD - 3) : "memory");       // tiles s + 1 and s + 2 have come, and tiles s - 2 and s - 1 are nobody's
        mask(zp);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int f = 0; f < KS; ++f) {
          ring[(f + RING - 1) % RING] = f + RING - 1 < KS ? query_frag(qt, f + RING - 1) : query_frag(next, f + RING - 1 - KS);
#pragma unroll
          for (int g = 0; g < 2; ++g) z[g] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag(kf[g][f]), frag(ring[f % RING]), f == 0 ? f32x16{} : z[g], 0, 0, 0);      // zero as an operand: no registers to clear
          weigh(zp, f);
          if (f == 0) fetch(s + AHEAD);
          __builtin_amdgcn_sched_barrier(0);
        }
        asm volatile("" ::"v"(sum[0]), "v"(sum[1]));                   // here, beside the MFMAs, not behind the next step's branch
        // fragment f of the next step is in place f
        if constexpr (KS % RING != 0) {
          u32x4 turned[RING - 1];
#pragma unroll
          for (int f = 0; f < RING - 1; ++f) turned[f] = ring[(KS + f) % RING];
#pragma unroll
          for (int f = 0; f < RING - 1; ++f) ring[f] = turned[f];
        }
        if ((s & 15) == 8) stage((s >> 4) + 1);
        const int at = (s & 15) * 32 + l32;
        lp = row_lse[(s >> 4) & 1][at];
        limit_p = row_limit[(s >> 4) & 1][at];
      };
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(AHEAD - 1) : "memory");
#pragma unroll
      for (int f = 0; f < RING - 1; ++f) ring[f] = query_frag(q_lane, f);
      int s = 0;
      for (; s + 1 < steps; s += 2) {
        step(s, za, zb, std::true_type{});
        step(s + 1, zb, za, std::false_type{});
      }
      if (s < steps) {
        step(s, za, zb, std::true_type{});
        mask(za);
#pragma unroll
        for (int f = 0; f < KS; ++f) weigh(za, f);
      } else {
        mask(zb);
#pragma unroll
        for (int f = 0; f < KS; ++f) weigh(zb, f);
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
      if (!whole) {
        a.part[(int64_t)slot * kMassKeys + wave * 64 + lane] = mine;
      } else if (j >= from && j < len) {
        float* sums = a.sums + r * a.s_seq + head * a.s_head;
        sums[j] = fmaf(a.decay, old_sum(a, sums, j, len, nq), a.share * mine);
      }
    }
    if (next_block >= x1) break;
    start = next_block;
    if (++block >= of.first + of.count) {                          // the next request with blocks, or the first one of the next head: 64 at a time
      for (++r;;) {
        const uint64_t some = __ballot(r + lane < n && blocks_of(a, min(r + lane, n - 1)).count > 0);
        if (some != 0) { r += __builtin_ctzll(some); break; }
        r += 64;
        if (r >= n) { r = 0; ++head; }
      }
      of = blocks_of(a, r);
      block = of.first;
    }
    block = uniform(block);
  }
  if (tid == 0) a.cuts[share] = cut;
}

// Parts of a block of keys added up, in the order of the rows: two threads a key, each some of the parts.
__global__ __launch_bounds__(2 * kMassKeys) void mass_join_kernel(const MassArgs a) {
  __shared__ float sum_of[2][kMassKeys];
  const int first = blockIdx.x;
  const CutKeys cut = a.cuts[first];
  if (cut.r < 0) return;
  const int key = threadIdx.x & (kMassKeys - 1), q = threadIdx.x / kMassKeys, parts = cut.last - first + 1;
  float x = 0.0f;
#pragma unroll 8
  for (int p = q * parts / 2; p < (q + 1) * parts / 2; ++p) x += a.part[(int64_t)(p == 0 ? 2 * first + 1 : 2 * (first + p)) * kMassKeys + key];
  sum_of[q][key] = x;
  __syncthreads();
  const KeyBlocks of = blocks_of(a, cut.r);
  const int j = cut.block * kMassKeys + key;
  if (q != 0 || j < first_of(a, cut.r) || j >= of.len) return;
  float* sums = a.sums + cut.r * a.s_seq + cut.head * a.s_head;
  sums[j] = fmaf(a.decay, old_sum(a, sums, j, of.len, of.nq), a.share * (sum_of[0][key] + sum_of[1][key]));
}

// Few rows: chunks, a workgroup each, up to so many bytes of keys that there may be, else equal shares of all that there are, which take a look at all requests first
// (us, chunks | shares: 64 requests of 300 rows 7.7 | 8.9, 16 of 500 to 4000 12.2 | 16.0, one of 100000 21 | 25, 32 of 4000, 131 MB, 25 | 27;
// 48 of 1000 to 4000 30 | 28, 64 of 300 to 4100 39 | 33, 8 of 4000 to 32000 38 | 28).
constexpr int64_t kMassEvenBytes = 1 << 27;
// Four for each compute unit (512, 1024, 2048: 136, 118, 123 us for the 8-bit steps above).
constexpr int kMassFewShares = 1024;
// Where some request has more than 64 rows, and the kernel for many runs, it has all of more than 16, and what is left as well if that is no more than 64 blocks of keys: a
// launch less (us, split at 64 | so: 9 requests of 5 to 15 tokens of 7 query heads over 526 to 3688 rows 31 | 19, 16 of up to 20 over 100 to 2000 31 | 20, two over 13 to 15
// rows 19 | 14, 40 of up to 20 over 100 to 2000 41 | 32, 64 of up to 12 over 500 to 8000 128 | 129; 30 steps beside a prompt, 240 blocks, 25 | 25, with all together 34).
constexpr int kMassSteps = 16;
constexpr int64_t kMassTogether = 64;
constexpr int kMassShares = 256;                 // many rows: a workgroup for each compute unit
constexpr int64_t kMostBlocks = (1 << 24) - 1;    // of 256 threads: an axis of a grid holds 2^32 threads

int make_mass_plan(const codecomp_batch* b, const codecomp_pages* p, const codecomp_mass* m, MassPlan* pl) {
  if (int rc = make_pool(p, &pl->pool)) return rc;
  if (int rc = make_batch(b, p, &pl->batch)) return rc;
  if (int rc = make_mass(m, &pl->mass)) return rc;
  const PagedBatch& x = pl->batch;
  if (m->n_layers != p->n_layers || m->n_seqs != b->n_seqs || m->n_kv_heads != p->n_kv_heads || m->width < b->max_kv_len) return CODECOMP_EINVAL_SHAPE;
  pl->d = p->head_dim;
  pl->scale = b->softmax_scale > 0.0f ? b->softmax_scale : 1.0f / sqrtf((float)p->head_dim);
  auto count = [&](int few_most) {
    pl->few_most = few_most;
    pl->few_rows = pl->many_rows = 0;
    for (int r = 0; r < x.n_seqs; ++r) {
      const int64_t rows = (int64_t)(b->cu_q_host[r + 1] - b->cu_q_host[r]) * x.G;
      if (rows > few_most) ++pl->many_rows;
      else if (rows > 0) ++pl->few_rows;
    }
  };
  count(kFewRowsMost);
  if (pl->many_rows > 0) count(kMassSteps);
  if (pl->many_rows > 0 && pl->few_rows > 0 && (int64_t)pl->few_rows * x.Hkv * ((x.max_kv + kMassKeys - 1) / kMassKeys) <= kMassTogether) count(0);
  const int64_t items = (int64_t)x.n_seqs * x.Hkv;
  const int64_t chunk = items * x.max_kv > 256 * 2048 ? 512 : 256;        // two tiles of every wave (one at head_dim 64), or four where there are enough workgroups all the same (128 to 1024: within 0.4 us)
  pl->chunk = (int)chunk;
  pl->chunks = (int)((x.max_kv + chunk - 1) / chunk);
  const int64_t keys = (int64_t)pl->few_rows * x.Hkv * x.max_kv;
  pl->shares = keys > kMassEvenBytes / (p->head_dim * (pl->pool.fp8 ? 1 : 2)) || items * pl->chunks > kMostBlocks ? kMassFewShares : 0;
  pl->ws_bytes = pl->many_rows > 0 && x.max_kv > 0 ? kMassShares * (2 * kMassKeys * sizeof(float) + sizeof(CutKeys)) : 0;
  return CODECOMP_OK;
}

template <int D, bool FP8>
static int launch_mass_of(const MassPlan& pl, const MassArgs& a, hipStream_t stream) {
  const int64_t items = (int64_t)pl.batch.n_seqs * pl.batch.Hkv;
  const dim3 block(kMassThreads);
  if (pl.few_rows > 0) {
    const dim3 even((unsigned)pl.shares), chunks((unsigned)(items * pl.chunks));
    if (pl.pool.page_log2 < 4) {
      if (pl.shares > 0) mass_few_kernel<D, FP8, true, true><<<even, block, 0, stream>>>(a);
      else mass_few_kernel<D, FP8, false, true><<<chunks, block, 0, stream>>>(a);
    } else {
      if (pl.shares > 0) mass_few_kernel<D, FP8, true, false><<<even, block, 0, stream>>>(a);
      else mass_few_kernel<D, FP8, false, false><<<chunks, block, 0, stream>>>(a);
    }
    if (hipError_t e = hipGetLastError()) return (int)e;
  }
  if (pl.many_rows > 0) {
    mass_many_kernel<D, FP8><<<dim3(kMassShares), dim3(kManyMassThreads), 0, stream>>>(a);
    if (hipError_t e = hipGetLastError()) return (int)e;
    mass_join_kernel<<<dim3(kMassShares), dim3(2 * kMassKeys), 0, stream>>>(a);
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
  a.cuts = reinterpret_cast<CutKeys*>(a.part + 2 * kMassShares * kMassKeys);
  a.few_most = pl.few_most;
  a.chunk = pl.chunk; a.shares = kMassShares; a.few_shares = pl.shares;
  if (pl.d == 128) return pl.pool.fp8 ? launch_mass_of<128, true>(pl, a, stream) : launch_mass_of<128, false>(pl, a, stream);
  return pl.pool.fp8 ? launch_mass_of<64, true>(pl, a, stream) : launch_mass_of<64, false>(pl, a, stream);
}

}  // namespace codecomp
