// Attention of requests with few rows (new tokens x query heads per KV head, up to 32, or 64 of them by two workgroups): the step of one token, and
// short chunks.
//
// Every key and value is read once for a handful of products: bound by memory.  So the cache is cut into chunks of keys, one workgroup of four
// waves per (request, KV head, chunk), each wave with tiles of 32 keys of its own: a tile is on its way into registers while the one
// before it is multiplied, and no wave waits for another until the chunk is done.  Large batches are cut into equal parts instead, one for each
// workgroup that the chip holds, whatever the lengths.  Chunks and parts are joined by a second kernel (a row's reference, sum of weights and unscaled
// output each), in order.
//
// Per tile, S^T = K Q^T (lane = row; 16 keys x 16 rows per MFMA), weights exp2(c s - reference) in place, O^T += V^T P^T.  The
// order of keys inside an MFMA's contraction is free, and chosen so that a lane's weights are the right operand as they stand (keys 4 q + i
// and 16 + 4 q + i of lane group q); V^T is read from LDS by the transposing read.  A weight enters the product as two bf16, its
// rounded value and the rest: 16 bits of it, for MFMA time that memory hides.
//
// Measured (a kernel that only reads reaches 6.4 TB/s): 64 steps over 500 .. 16384 keys, 4 KV heads of 128 elements, bf16: 187 us, 5.3 TB/s; with 8 KV heads, 8
// bits: 184 us, 5.5 TB/s; one step over 131072 keys: 56 us, 4.8 TB/s (51 the kernel, 6 the join); one over 2113: 10 us (7 and 4), a chain of small loads
// (lengths, table, rows, parts) that nothing hides.
#include <type_traits>

#include "attend.h"

namespace codecomp {

constexpr int kFewWaves = 4, kFewKeys = 32, kFewStrip = kFewWaves * kFewKeys;

// A lane loads 16-byte pieces of two keys of a tile, l16 and 16 + l16: those that its K fragments are made of, in registers as they come (the
// order of a row's elements in the contraction is free as well: an 8-bit piece is the fragments of two steps), and the same ones of V, which go
// through LDS.
template <int D, bool FP8>
struct FewTile {
  static constexpr int LOADS = D * (FP8 ? 1 : 2) / 64;        // pieces of a row per lane
  static constexpr int V_ROW = 2 * D + 32;                     // bytes between rows in LDS: two groups of four V rows hit all banks once
  static constexpr int BYTES = kFewKeys * V_ROW;
  static __device__ __forceinline__ int q_element(int ks, int quarter) {        // that goes with the K fragment of step ks
    return FP8 ? (ks >> 1) * 64 + quarter * 16 + (ks & 1) * 8 : ks * 32 + quarter * 8;
  }
  static __device__ __forceinline__ u32x4 k_frag(const u32x4* piece, int ks) {
    if constexpr (!FP8) return piece[ks];
    const u32x4 x = piece[ks >> 1];
    return ks & 1 ? widen8(x.z, x.w) : widen8(x.x, x.y);
  }
};

// Keys of a request that this kernel takes, in strips of what the four waves read at a time; at least one.
__device__ __forceinline__ int strips_of(const AttendArgs& a, int r) {
  const int rows = (a.b.cu_q[r + 1] - a.b.cu_q[r]) * a.b.G;
  return rows <= 0 || rows > a.row_slots ? 0 : max(1, (kv_len_of(a.b, r) + kFewStrip - 1) / kFewStrip);
}

// 16 rows of a request's own keys, from row0 on, joined to the parts of the shared ones: D / 4 threads a row.  Parts come from memory (other dies wrote them):
// as many as registers hold are sent for at a time, and the reference moves on from one lot to the next.
template <int D>
__device__ __forceinline__ void join_rows(const SharedArgs& a, const float (&own_o)[16][D], const float (&own_ml)[16][2], int q0, int head, int row0, int rows) {
  constexpr int THREADS = D / 4, LOT = 16;
  const int e = threadIdx.x % THREADS * 4;
  const GroupParts parts = parts_of_group(a.sh, q0);
  for (int n = threadIdx.x / THREADS; n < 16; n += 64 * kFewWaves / THREADS) {
    const int row = row0 + n, t = row / a.b.G, h = head * a.b.G + row - t * a.b.G;
    if (row >= rows) return;
    const int64_t at = row_part(a, parts.first, q0 + t, h), step = parts.step * a.b.Hq;
    float top = own_ml[n][0], all = own_ml[n][1];
    f32x4 x = *reinterpret_cast<const f32x4*>(&own_o[n][e]);
    for (int p0 = 0; p0 < parts.count; p0 += LOT) {
      f32x4 v[LOT];
      float m[LOT], l[LOT], to = top;
#pragma unroll
      for (int i = 0; i < LOT; ++i) {
        const int64_t part = at + min(p0 + i, parts.count - 1) * step;
        m[i] = a.part_ml[2 * part];
        l[i] = p0 + i < parts.count ? a.part_ml[2 * part + 1] : kNoPart;
        v[i] = *reinterpret_cast<const f32x4*>(a.part_o + part * D + e);
      }
#pragma unroll
      for (int i = 0; i < LOT; ++i) to = fmaxf(to, l[i] == kNoPart ? -INFINITY : m[i]);
      const float old = to == top ? 1.0f : __builtin_amdgcn_exp2f(top - to);
      top = to;
      x *= old;
      all *= old;
#pragma unroll
      for (int i = 0; i < LOT; ++i) {
        const float f = m[i] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m[i] - to);       // times zeros, or an infinity or NaN that it saw
        const bool some = l[i] != kNoPart;
        all += some ? f * l[i] : 0.0f;
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] += some ? f * v[i][k] : 0.0f;
      }
    }
    const float inv = all == 0.0f ? 0.0f : a.pool.v_scale / all;
    *reinterpret_cast<u32x2*>(a.out + (q0 + t) * a.b.o_st + h * a.b.o_sh + e) = u32x2{pack2(x.x * inv, x.y * inv), pack2(x.z * inv, x.w * inv)};
    if (a.lse && e == 0) a.lse[(int64_t)(q0 + t) * a.b.Hq + h] = all == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(all)) * kLn2;
  }
}

// EVEN: the strips of all requests and heads form one sequence, cut into equal parts; else a workgroup has one chunk of a request, or (SHARED 1) of the rows that
// a group shares, or of a request's rows behind them, and leaves parts of all rows, or (2) all rows of a request, the shared ones among them.
template <int D, bool FP8, int RB, bool EVEN, int SHARED = 0>
__global__ __launch_bounds__(64 * kFewWaves, RB == 2 || EVEN ? 2 : 3) void attend_few_kernel(const std::conditional_t<SHARED != 0, SharedArgs, AttendArgs> a) {
  using T = FewTile<D, FP8>;
  constexpr int KS = D / 32, DB = D / 16;
  __shared__ __attribute__((aligned(16))) unsigned char lds[kFewWaves * T::BYTES];
  __shared__ float row_m[kFewWaves][16], row_l[kFewWaves][16];
  __shared__ __attribute__((aligned(16))) float own_o[SHARED == 1 ? 16 : 1][D], own_ml[SHARED == 1 ? 16 : 1][2];       // what the workgroup joins the shared rows' parts to
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  int l16 = lane & 15, quarter = lane >> 4;
  int r, head, row0, key0, share = 0, strip = 0;                 // request, head, first of this workgroup's rows, first of its keys
  int64_t left = 0, part0 = 0;                                   // EVEN: strips that are left; else the chunk's part
  const int32_t* table;
  // Entries of the page table for keys tile + l16 and 16 + tile + l16, not looked at before they are needed.  Those of the first two tiles are sent for
  // before it is known how many keys there are: one wait less.
  int page[2], next_page[2];
  const int32_t* lead_table = nullptr;                           // SHARED 2: of the group's first request, for the shared rows
  int lead_keys = 0;
  auto table_of = [&](int key) __attribute__((always_inline)) {
    if constexpr (SHARED == 2) return key < lead_keys ? lead_table : table;
    return table;
  };
  auto look_up = [&](int (&pg)[2], int tile, int end) __attribute__((always_inline)) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int key = max(min(tile + 16 * b + l16, end - 1), 0);
      pg[b] = table_of(key)[key >> a.pool.page_log2];
    }
  };
  int64_t total = 0, shares = 0, at_strip = 0;
  CutBlock cut = {-1, 0, 0, 0};
  int shared_q0 = 0, shared_nq = 0, shared_len = 0, key_end = 0;        // SHARED: tokens of the group or request, keys up to which there are some
  int shared_part = 0;                                           // SHARED 1: number of its part
  bool shared_own = false;                                       // SHARED 1: of rows behind the shared ones
  auto part_base = [&]() __attribute__((always_inline)) {
    if constexpr (SHARED == 1) {
      if (shared_own) return a.sh.own_base + (int64_t)shared_part * a.b.T;
      const GroupParts parts = parts_of_group(a.sh, shared_q0);
      return parts.first + shared_part * parts.step;
    }
    return (int64_t)0;
  };
  int causal = SHARED ? 0 : a.b.causal;
  bool shared_join = false;                                       // these are a request's own rows, and the parts of the shared ones are joined to them
  if constexpr (EVEN) {
    share = blockIdx.x;
    row0 = 0;
    __shared__ int64_t wave_sum[kFewWaves];
    __shared__ int found[2];
    const int n = a.b.n_seqs, per = (n + 64 * kFewWaves - 1) / (64 * kFewWaves), r0 = min(tid * per, n), r1 = min(r0 + per, n);
    int64_t mine = 0;
    for (int i = r0; i < r1; ++i) mine += strips_of(a, i);
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
    for (int w = 0; w < kFewWaves; ++w) {
      if (w < wave) before += wave_sum[w];
      per_head += wave_sum[w];
    }
    per_head = uniform(per_head);
    total = per_head * a.b.Hkv;
    shares = uniform(min((int64_t)a.shares, total));
    if (share >= shares) {
      if (tid == 0) a.cuts[share].r = -1;
      return;
    }
    at_strip = uniform(share * total / shares);
    left = uniform((share + 1) * total / shares) - at_strip;
    head = uniform((int)(at_strip / per_head));
    int64_t at = at_strip - head * per_head - before;
    if (at >= 0 && at < mine) {                                  // one thread has it
      int i = r0;
      for (int s = strips_of(a, i); at >= s; s = strips_of(a, i)) { at -= s; ++i; }
      found[0] = i; found[1] = (int)at;
    }
    __syncthreads();
    r = uniform(found[0]); strip = uniform(found[1]);
  } else if constexpr (SHARED == 2) {
    const int item = blockIdx.x / a.row_parts;
    row0 = ((int)blockIdx.x - item * a.row_parts) * (16 * RB);
    r = item / a.b.Hkv; head = item - r * a.b.Hkv;
    shared_q0 = a.b.cu_q[r];
    shared_nq = a.b.cu_q[r + 1] - shared_q0;
    if (shared_nq * a.b.G <= row0) return;
    const int g = uniform(request_of(a.sh.cu_groups, a.sh.n_groups, r));
    lead_keys = uniform(prefix_of(a.sh, g));
    shared_len = uniform((int)min((int64_t)kv_len_of(a.b, r), (int64_t)lead_keys + a.sh.max_own));
    lead_table = a.b.table + (int64_t)a.sh.cu_groups[g] * a.b.table_width;
    table = a.b.table + (int64_t)r * a.b.table_width;
    key0 = 0;
    key_end = shared_len;
    causal = a.b.causal;
    look_up(page, wave * kFewKeys, key_end);
    look_up(next_page, (kFewWaves + wave) * kFewKeys, key_end);
  } else if constexpr (SHARED) {
    const bool group = (int)blockIdx.x < a.sh.few_units;
    const int unit = group ? blockIdx.x : blockIdx.x - a.sh.few_units, parts = group ? a.sh.few_parts : a.row_parts;
    const int items = (group ? a.sh.n_groups : a.b.n_seqs) * a.b.Hkv, turn = unit / items, item = unit - turn * items, split = turn / parts;
    row0 = (turn - split * parts) * (16 * RB);
    r = item / a.b.Hkv; head = item - r * a.b.Hkv;
    if (group) {
      const int g = r, end = a.sh.cu_groups[g + 1];
      r = a.sh.cu_groups[g];
      if (r >= end) return;
      shared_q0 = a.b.cu_q[r];
      shared_nq = a.b.cu_q[end] - shared_q0;
      if (shared_nq * a.b.G > a.sh.few_rows || shared_nq * a.b.G <= row0) return;
      shared_len = uniform(prefix_of(a.sh, g));
      key0 = split * a.sh.few_chunk;
      key_end = key0 + a.sh.few_chunk;
      shared_part = split;
    } else {
      shared_q0 = a.b.cu_q[r];
      shared_nq = a.b.cu_q[r + 1] - shared_q0;
      if (shared_nq * a.b.G <= row0) return;
      const int before = uniform(prefix_of(a.sh, request_of(a.sh.cu_groups, a.sh.n_groups, r)));
      shared_len = uniform((int)min((int64_t)kv_len_of(a.b, r), (int64_t)before + a.sh.max_own));
      key0 = (int)min(before + (int64_t)split * a.chunk, (int64_t)INT32_MAX);
      key_end = (int)min((int64_t)key0 + a.chunk, (int64_t)INT32_MAX);
      shared_part = split;
      shared_own = true;
      causal = a.b.causal;
      shared_join = a.sh.join != 0;
    }
    if (key0 >= shared_len && (group || !a.sh.join)) {
      no_part<64 * kFewWaves>(a, part_base(), shared_q0, head, row0, min(shared_nq * a.b.G, row0 + 16 * RB));
      return;
    }
    table = a.b.table + (int64_t)r * a.b.table_width;
    key_end = min(key_end, shared_len);
    look_up(page, key0 + wave * kFewKeys, key_end);
    look_up(next_page, key0 + (kFewWaves + wave) * kFewKeys, key_end);
  } else {
    // Chunk by chunk, all requests and heads of one: neighbouring workgroups run on different dies, and must not be the same chunks of all
    // requests there (short requests lack the later ones).
    const int items = a.b.n_seqs * a.b.Hkv, turn = blockIdx.x / items, item = blockIdx.x - turn * items, split = turn / a.row_parts;
    row0 = (turn - split * a.row_parts) * (16 * RB);
    r = item / a.b.Hkv; head = item - r * a.b.Hkv;
    key0 = split * a.chunk;
    part0 = ((int64_t)item * a.splits + split) * a.row_slots;
    table = a.b.table + (int64_t)r * a.b.table_width;
    look_up(page, key0 + wave * kFewKeys, a.b.max_kv);
    look_up(next_page, key0 + (kFewWaves + wave) * kFewKeys, a.b.max_kv);
  }
  for (;;) {
    if constexpr (EVEN) asm("" : "+v"(l16), "+v"(quarter));         // what follows from them is worked out per piece, not held in registers from piece to piece
    const int q0 = SHARED ? shared_q0 : a.b.cu_q[r], nq = SHARED ? shared_nq : a.b.cu_q[r + 1] - q0, rows = nq * a.b.G;
    const int len = SHARED ? shared_len : uniform(kv_len_of(a.b, r));
    int key1;
    bool whole;                                                    // no other workgroup has keys of these rows
    if constexpr (EVEN) {
      const int strips = uniform(strips_of(a, r)), end = (int)min((int64_t)strips, strip + left);
      table = a.b.table + (int64_t)r * a.b.table_width;
      key0 = strip * kFewStrip;
      key1 = min(len, end * kFewStrip);
      whole = strip == 0 && end == strips;
      part0 = (int64_t)(strip > 0 ? 2 * share : 2 * share + 1) * a.row_slots;
      if (strip == 0 && end < strips) cut = {r, 0, head, uniform((int)(((at_strip + strips) * shares - 1) / total))};
      left -= end - strip;
      at_strip += end - strip;
      look_up(page, key0 + wave * kFewKeys, key1);
      look_up(next_page, key0 + (kFewWaves + wave) * kFewKeys, key1);
    } else if constexpr (SHARED) {
      key1 = causal ? min(key_end, len - nq + (min(row0 + 16 * RB, rows) - 1) / a.b.G + 1) : key_end;       // nothing behind what the last row sees
      whole = SHARED == 2 || shared_join;
    } else {
      if (rows <= row0 || rows > a.row_slots) return;
      key1 = min(len, key0 + a.chunk);
      if (key0 > 0 && key0 >= len) return;
      whole = len <= a.chunk;
    }

    // query rows as right operands
    u32x4 qf[RB][KS];
    int limit[RB];                                                // keys that the lane's row sees
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int row = row0 + rb * 16 + l16, t = min(row, rows - 1) / a.b.G, g = min(row, rows - 1) - t * a.b.G;
      const uint16_t* p = a.q + (q0 + t) * a.b.q_st + (head * a.b.G + g) * a.b.q_sh;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        qf[rb][ks] = *reinterpret_cast<const u32x4*>(p + T::q_element(ks, quarter));
        if (!SHARED && row >= rows) qf[rb][ks] = u32x4{0, 0, 0, 0};
      }
      limit[rb] = causal ? min(len, len - nq + t + 1) : len;
    }
    const int seen_by_all = causal ? len - nq + 1 : len;

    const unsigned char* kb = a.pool.k + a.layer + head * a.pool.s_head + quarter * 16;
    const unsigned char* vb = a.pool.v + a.layer + head * a.pool.s_head + quarter * 16;
    const int in_page = (1 << a.pool.page_log2) - 1;
    unsigned char* vs_lds = lds + wave * T::BYTES;

    u32x4 kr[2][T::LOADS], vr[2][T::LOADS];
    auto send_for = [&](int tile, const int (&pg)[2]) __attribute__((always_inline)) {
      int64_t off[2];
#pragma unroll
      for (int b = 0; b < 2; ++b)                                  // rows that are not there: page 0, masked or zeroed below
        off[b] = (pg[b] >= 0 && pg[b] < a.pool.n_pages ? pg[b] : 0) * a.pool.s_page + ((tile + 16 * b + l16) & in_page) * (int)a.pool.s_tok;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < T::LOADS; ++i) kr[b][i] = *reinterpret_cast<const u32x4*>(kb + off[b] + i * 64);
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < T::LOADS; ++i) vr[b][i] = *reinterpret_cast<const u32x4*>(vb + off[b] + i * 64);
    };

    f32x4 o[RB][DB];
    float m[RB], l[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      m[rb] = -INFINITY; l[rb] = 0.0f;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[rb][db] = f32x4{0, 0, 0, 0};
    }

    unsigned left_out = 0;
    int tile = key0 + wave * kFewKeys;
    if (tile < key1) send_for(tile, page);
    if constexpr (SHARED != 0) {                                   // rows that are not there; the queries are waited for behind the keys
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
          if (row0 + rb * 16 + l16 >= rows) qf[rb][ks] = u32x4{0, 0, 0, 0};
    }
    for (; tile < key1; tile += kFewWaves * kFewKeys) {
      bool there[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) there[b] = tile + 16 * b + l16 < key1 && page[b] >= 0 && page[b] < a.pool.n_pages;
      const unsigned valid = ((unsigned)__ballot(there[0]) & 0xFFFFu) | (unsigned)__ballot(there[1]) << 16;
      const bool plain = valid == 0xFFFFFFFFu && tile + kFewKeys <= seen_by_all;
      f32x4 s[RB][2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) s[rb][b] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const bf16x8 kf = frag(T::k_frag(kr[b], ks));
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) s[rb][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, frag(qf[rb][ks]), s[rb][b], 0, 0, 0);
        }
      }
      if (__builtin_expect(!plain, 0)) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < T::LOADS; ++i)
            if (!there[b]) vr[b][i] = u32x4{0, 0, 0, 0};
        // a weight of zero must not meet an infinite or NaN value: such values are added at the end, to the rows that see them
        if (tile + kFewKeys > seen_by_all && seen_by_all < len) {
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < T::LOADS; ++i) vr[b][i] = finite_part<FP8>(vr[b][i], left_out);
        }
      }
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < T::LOADS; ++i) {
          unsigned char* at = vs_lds + (16 * b + l16) * T::V_ROW + (i * 64 + quarter * 16) * (FP8 ? 2 : 1);
          if constexpr (FP8) {
            *reinterpret_cast<u32x4*>(at) = widen8(vr[b][i].x, vr[b][i].y);
            *reinterpret_cast<u32x4*>(at + 16) = widen8(vr[b][i].z, vr[b][i].w);
          } else {
            *reinterpret_cast<u32x4*>(at) = vr[b][i];
          }
        }
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int b = 0; b < 2; ++b) page[b] = next_page[b];
      if (tile + kFewWaves * kFewKeys < key1) {
        send_for(tile + kFewWaves * kFewKeys, page);
        look_up(next_page, tile + 2 * kFewWaves * kFewKeys, key1);
      }

      float p[RB][8];
      bool grows = false;
      float top[RB];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[rb][i] = s[rb][i >> 2][i & 3] * a.c;
        if (__builtin_expect(!plain, 0)) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int j = (i >> 2) * 16 + quarter * 4 + (i & 3);
            if (!((valid >> j) & 1) || tile + j >= limit[rb]) p[rb][i] = -INFINITY;
          }
        }
        float x = fmaxf(fmaxf(fmaxf(p[rb][0], p[rb][1]), fmaxf(p[rb][2], p[rb][3])), fmaxf(fmaxf(p[rb][4], p[rb][5]), fmaxf(p[rb][6], p[rb][7])));
        x = fmaxf(x, __shfl_xor(x, 16));
        x = fmaxf(x, __shfl_xor(x, 32));
        top[rb] = x;
        grows |= x > m[rb] + kSlack;
      }
      if (__builtin_expect(__ballot(grows) != 0, 0)) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          const float to = fmaxf(m[rb], top[rb]);
          const float old = to == m[rb] ? 1.0f : __builtin_amdgcn_exp2f(m[rb] - to);
          m[rb] = to;
          l[rb] *= old;
#pragma unroll
          for (int db = 0; db < DB; ++db) o[rb][db] *= old;
        }
      }
      bf16x8 hi[RB], lo[RB];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const float ref = m[rb] == -INFINITY ? 0.0f : m[rb];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          p[rb][i] = __builtin_amdgcn_exp2f(p[rb][i] - ref);
          l[rb] += p[rb][i];
        }
        u32x4 h, w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          h[i] = pack2(p[rb][2 * i], p[rb][2 * i + 1]);
          w[i] = pack2(p[rb][2 * i] - __uint_as_float(h[i] << 16), p[rb][2 * i + 1] - __uint_as_float(h[i] & 0xFFFF0000u));
        }
        hi[rb] = frag(h); lo[rb] = frag(w);
      }
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const unsigned char* at = vs_lds + (quarter * 4 + (l16 >> 2)) * T::V_ROW + db * 32 + (l16 & 3) * 8;
        const s16x4 v0 = read_columns(at), v1 = read_columns(at + 16 * T::V_ROW);
        const bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          o[rb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, hi[rb], o[rb][db], 0, 0, 0);
          o[rb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, lo[rb], o[rb][db], 0, 0, 0);
        }
      }
      __builtin_amdgcn_wave_barrier();
    }

    if (__builtin_expect(__ballot(left_out != 0) != 0, 0)) {
      // from the first tile that was cleaned on: the keys before seen_by_all in it were as well
      for (int key = SHARED ? key0 + (max(seen_by_all - key0, 0) & -kFewKeys) : max(seen_by_all & -kFewKeys, key0); key < key1; ++key) {
        const int at = table_of(key)[key >> a.pool.page_log2];
        if ((key - key0) / kFewKeys % kFewWaves != wave || at < 0 || at >= a.pool.n_pages) continue;          // another wave's
        const unsigned char* row = a.pool.v + a.layer + head * a.pool.s_head + at * a.pool.s_page + (key & in_page) * a.pool.s_tok;
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const f32x4 v = row4<FP8>(row + (db * 16 + quarter * 4) * (FP8 ? 1 : 2));
#pragma unroll
          for (int rb = 0; rb < RB; ++rb)
            if (key < limit[rb]) {
#pragma unroll
              for (int i = 0; i < 4; ++i) o[rb][db][i] = with_the_rest(o[rb][db][i], v[i]);
            }
        }
      }
    }

    // the four waves' shares of every row, 16 rows at a time
    constexpr int O_ROW = D + 4;
    float* o_lds = reinterpret_cast<float*>(lds);
    static_assert(16 * O_ROW * 4 <= T::BYTES, "rows of a block fit the tiles");
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      if (row0 + rb * 16 >= rows) break;
      float sum = l[rb];
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      __syncthreads();
      if (quarter == 0) { row_m[wave][l16] = m[rb]; row_l[wave][l16] = sum; }
#pragma unroll
      for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4*>(o_lds + (wave * 16 + l16) * O_ROW + db * 16 + quarter * 4) = o[rb][db];
      __syncthreads();
      constexpr int E = D / 16;                                   // elements of a row per thread
      const int n = tid >> 4, row = row0 + rb * 16 + n, e = (tid & 15) * E;
      if (row < rows) {
        float to = -INFINITY;
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) to = fmaxf(to, row_m[w][n]);
        float all = 0.0f, x[E];
#pragma unroll
        for (int i = 0; i < E; ++i) x[i] = 0.0f;
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) {
          const float f = row_m[w][n] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(row_m[w][n] - to);       // times zeros, or an infinity or NaN that it saw
          all += f * row_l[w][n];
#pragma unroll
          for (int i = 0; i < E; ++i) x[i] += f * o_lds[(w * 16 + n) * O_ROW + e + i];
        }
        if (SHARED == 1 && whole) {                                     // joined below
#pragma unroll
          for (int i = 0; i < E; ++i) own_o[n][e + i] = x[i];
          if ((tid & 15) == 0) { own_ml[n][0] = to; own_ml[n][1] = all; }
        } else if (whole) {
          const int t = row / a.b.G, h = head * a.b.G + row - t * a.b.G;
          const float inv = all == 0.0f ? 0.0f : a.pool.v_scale / all;
          uint16_t* out = a.out + (q0 + t) * a.b.o_st + h * a.b.o_sh + e;
#pragma unroll
          for (int i = 0; i < E; i += 2) *reinterpret_cast<unsigned*>(out + i) = pack2(x[i] * inv, x[i + 1] * inv);
          if (a.lse && (tid & 15) == 0) a.lse[(int64_t)(q0 + t) * a.b.Hq + h] = all == 0.0f ? -INFINITY : (to + __builtin_amdgcn_logf(all)) * kLn2;
        } else {
          int64_t part;
          if constexpr (SHARED) part = row_part(a, part_base(), q0 + row / a.b.G, head * a.b.G + row % a.b.G);
          else part = part0 + row;
#pragma unroll
          for (int i = 0; i < E; i += 4) *reinterpret_cast<f32x4*>(a.part_o + part * D + e + i) = f32x4{x[i], x[i + 1], x[i + 2], x[i + 3]};
          if ((tid & 15) == 0) { a.part_ml[2 * part] = to; a.part_ml[2 * part + 1] = all; }
        }
      }
      if constexpr (SHARED == 1) {
        if (shared_join) {
          __syncthreads();
          join_rows<D>(a, own_o, own_ml, q0, head, row0 + rb * 16, rows);
        }
      }
    }
    if constexpr (!EVEN) return;
    if (left <= 0) break;
    strip = 0;
    for (++r;;) {                                                  // the next request with strips, or the first one of the next head: 64 at a time
      const uint64_t some = __ballot(r + lane < a.b.n_seqs && strips_of(a, min(r + lane, a.b.n_seqs - 1)) > 0);
      if (some != 0) { r += __builtin_ctzll(some); break; }
      r += 64;
      if (r >= a.b.n_seqs) { r = 0; ++head; }
    }
    __syncthreads();                                               // through with LDS
  }
  if (tid == 0) a.cuts[share] = cut;
}

// Parts joined: a workgroup per row of a request and head that several workgroups had keys of.  Weights of all parts first, then the outputs, four
// elements a thread, the parts shared out over the workgroup's groups of D / 4 threads and these added up in order.
template <int D, bool EVEN>
__global__ __launch_bounds__(256) void join_few_kernel(const AttendArgs a) {
  constexpr int GROUPS = 256 / (D / 4);
  __shared__ float weight[kFewMostSplits];
  __shared__ float red[4];
  __shared__ f32x4 sums[GROUPS][D / 4];
  constexpr int AHEAD = 4;
  const int row_slots = a.row_slots, row = blockIdx.x % row_slots, item = blockIdx.x / row_slots, tid = threadIdx.x;       // EVEN: the workgroup with the first part
  const int group = tid / (D / 4), e = tid % (D / 4);
  int r = item / a.b.Hkv, head = item - r * a.b.Hkv, most = a.splits;
  if constexpr (EVEN) {
    const CutBlock cut = a.cuts[item];
    if (cut.r < 0) return;
    r = cut.r; head = cut.head; most = cut.last - item + 1;
  }
  auto part = [&](int s) { return (EVEN ? (int64_t)(s == 0 ? 2 * item + 1 : 2 * (item + s)) : (int64_t)item * a.splits + s) * row_slots + row; };
  // What a thread needs first is sent for before it is known how many chunks there are (workspace, whatever stands there).
  float m0 = 0.0f, l0 = 0.0f;
  f32x4 ahead[AHEAD];
  if (tid < most) {
    m0 = a.part_ml[2 * part(tid)];
    l0 = a.part_ml[2 * part(tid) + 1];
  }
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) ahead[i] = *reinterpret_cast<const f32x4*>(a.part_o + part(min(group + i * GROUPS, most - 1)) * D + e * 4);
  const int q0 = a.b.cu_q[r], rows = (a.b.cu_q[r + 1] - q0) * a.b.G;
  if (rows > row_slots || row >= rows) return;
  int n = most;
  if constexpr (!EVEN) {
    const int len = kv_len_of(a.b, r);
    if (len <= a.chunk) return;                                  // written by its only chunk
    n = (len + a.chunk - 1) / a.chunk;
  }
  float top = -INFINITY;
  for (int s = tid; s < n; s += 256) {
    const float m = s < 256 ? m0 : a.part_ml[2 * part(s)];
    weight[s] = m;
    top = fmaxf(top, m);
  }
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) top = fmaxf(top, __shfl_xor(top, off));
  if ((tid & 63) == 0) red[tid >> 6] = top;
  __syncthreads();
  top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  __syncthreads();
  float all = 0.0f;
  for (int s = tid; s < n; s += 256) {
    const float f = weight[s] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(weight[s] - top);
    const float l = s < 256 ? l0 : a.part_ml[2 * part(s) + 1];
    weight[s] = f;
    all += l != l ? l : f * l;
  }
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) all += __shfl_xor(all, off);
  if ((tid & 63) == 0) red[tid >> 6] = all;
  __syncthreads();
  all = red[0] + red[1] + red[2] + red[3];
  f32x4 x = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < AHEAD; ++i)
    if (group + i * GROUPS < n) x += ahead[i] * weight[group + i * GROUPS];
#pragma unroll 8
  for (int s = group + AHEAD * GROUPS; s < n; s += GROUPS) {
    const f32x4 v = *reinterpret_cast<const f32x4*>(a.part_o + part(s) * D + e * 4);
    x += v * weight[s];
  }
  sums[group][e] = x;
  __syncthreads();
  if (group == 0) {
#pragma unroll
    for (int g = 1; g < GROUPS; ++g) x += sums[g][e];
    const float inv = all == 0.0f ? 0.0f : a.pool.v_scale / all;
    const int t = row / a.b.G, h = head * a.b.G + row - t * a.b.G;
    *reinterpret_cast<u32x2*>(a.out + (q0 + t) * a.b.o_st + h * a.b.o_sh + e * 4) = u32x2{pack2(x.x * inv, x.y * inv), pack2(x.z * inv, x.w * inv)};
    if (a.lse && e == 0) a.lse[(int64_t)(q0 + t) * a.b.Hq + h] = all == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(all)) * kLn2;
  }
}

template <int D, bool FP8, int RB>
static int launch_few_of(const AttendArgs& a, hipStream_t stream) {
  const int64_t items = (int64_t)a.b.n_seqs * a.b.Hkv;
  const dim3 block(64 * kFewWaves), join_block(256);
  if (a.shares > 0) {
    attend_few_kernel<D, FP8, RB, true><<<dim3((unsigned)a.shares), block, 0, stream>>>(a);
    if (hipError_t e = hipGetLastError()) return (int)e;
    join_few_kernel<D, true><<<dim3((unsigned)(a.shares * a.row_slots)), join_block, 0, stream>>>(a);
    return (int)hipGetLastError();
  }
  attend_few_kernel<D, FP8, RB, false><<<dim3((unsigned)(items * a.splits * a.row_parts)), block, 0, stream>>>(a);
  if (hipError_t e = hipGetLastError()) return (int)e;
  if (a.splits > 1) join_few_kernel<D, false><<<dim3((unsigned)(items * a.row_slots)), join_block, 0, stream>>>(a);
  return (int)hipGetLastError();
}
template <int D, bool FP8>
static int launch_few_rows(const AttendArgs& a, hipStream_t stream) {
  return a.row_slots <= 16 ? launch_few_of<D, FP8, 1>(a, stream) : launch_few_of<D, FP8, 2>(a, stream);
}

int launch_few(const AttendPlan& pl, const AttendArgs& a, hipStream_t stream) {
  if (pl.d == 128) return pl.pool.fp8 ? launch_few_rows<128, true>(a, stream) : launch_few_rows<128, false>(a, stream);
  return pl.pool.fp8 ? launch_few_rows<64, true>(a, stream) : launch_few_rows<64, false>(a, stream);
}

template <int D, bool FP8>
static int launch_few_shared_of(bool two_blocks, int64_t units, const SharedArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)units), block(64 * kFewWaves);
  if (a.sh.alone) {
    if (two_blocks) attend_few_kernel<D, FP8, 2, false, 2><<<grid, block, 0, stream>>>(a);
    else attend_few_kernel<D, FP8, 1, false, 2><<<grid, block, 0, stream>>>(a);
  } else {
    if (two_blocks) attend_few_kernel<D, FP8, 2, false, 1><<<grid, block, 0, stream>>>(a);
    else attend_few_kernel<D, FP8, 1, false, 1><<<grid, block, 0, stream>>>(a);
  }
  return (int)hipGetLastError();
}

int launch_few_shared(int d, bool fp8, bool two_blocks, int64_t units, const SharedArgs& a, hipStream_t stream) {
  if (d == 128) return fp8 ? launch_few_shared_of<128, true>(two_blocks, units, a, stream) : launch_few_shared_of<128, false>(two_blocks, units, a, stream);
  return fp8 ? launch_few_shared_of<64, true>(two_blocks, units, a, stream) : launch_few_shared_of<64, false>(two_blocks, units, a, stream);
}

}  // namespace codecomp
