// Internal header: attention of requests with many rows (new tokens x query heads per KV head, more than 64): prefill chunks and prompts.
// Instantiated per head_dim and cache type in attend_many_*.hip, so that they compile side by side.
//
// The rows of a KV head, token by token and its query heads within, are cut into blocks of 256: four waves of 64 rows, two MFMA tiles of 32
// each, which share the keys and values that go through LDS in tiles of 64.  S^T = K Q^T leaves a row's logits in one lane of each half of the wave;
// O^T += V^T P^T takes them from there: the order of keys in a contraction is free, and chosen so that a lane's weights are its right operand as
// they stand.  V^T comes from LDS by the transposing read.
#pragma once
#include "attend.h"

namespace codecomp {

constexpr int kManyRows = 256, kManyKeys = 64;

// What a workgroup leaves for the kernel that joins blocks of rows whose keys several workgroups share.
struct CutBlock {
  int32_t r, block, head;      // r < 0: none
  int32_t first_slot, last;    // slot of this workgroup's part; last workgroup with a part (slot 2 * workgroup)
};

struct ManyArgs {
  AttendArgs a;
  CutBlock* cuts;              // [workgroups]
  int workgroups, few_rows_most;
};

// Tiles of 64 keys that a block of rows of a request meets; at least one.
struct Blocks {
  int len, nq, G, rows, count, causal;
  __device__ __forceinline__ int tiles(int block) const {
    int keys = len;
    if (causal) keys = min(len, len - nq + (min(block * kManyRows + kManyRows, rows) - 1) / G + 1);
    return max(1, (keys + kManyKeys - 1) / kManyKeys);
  }
};
__device__ __forceinline__ Blocks blocks_of(const ManyArgs& m, int r) {
  Blocks x;
  x.len = kv_len_of(m.a.b, r);
  x.nq = m.a.b.cu_q[r + 1] - m.a.b.cu_q[r];
  x.G = m.a.b.G;
  x.rows = x.nq * x.G;
  x.count = x.rows > m.few_rows_most ? (x.rows + kManyRows - 1) / kManyRows : 0;
  x.causal = m.a.b.causal;
  return x;
}

template <int D, bool FP8>
__global__ __launch_bounds__(256, D == 128 ? 1 : 2) void attend_many_kernel(const ManyArgs ma) {
  const AttendArgs& a = ma.a;
  constexpr int PIECES = D * (FP8 ? 1 : 2) / 16;               // 16-byte pieces of a stored row
  constexpr int ROWS = 256 / PIECES, LOADS = kManyKeys / ROWS;  // rows per load of the workgroup, loads per tile
  constexpr int K_ROW = 2 * D + 16, V_ROW = 2 * D + 64;          // bytes between rows in LDS: no bank conflicts in either read
  constexpr int KS = D / 16, DB = D / 32;
  __shared__ __attribute__((aligned(16))) unsigned char k_lds[2][kManyKeys * K_ROW];
  __shared__ __attribute__((aligned(16))) unsigned char v_lds[2][kManyKeys * V_ROW];
  __shared__ uint64_t apart_lds[2][4];
  __shared__ int64_t wave_sum[4];
  __shared__ int found[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l32 = lane & 31, half = lane >> 5;

  // ---- this workgroup's share: the tiles of all blocks of all heads form one sequence, cut into equal parts
  const int n = a.b.n_seqs, per = (n + 255) / 256;
  int64_t mine = 0;
  for (int r = min(tid * per, n); r < min(tid * per + per, n); ++r) {
    const Blocks x = blocks_of(ma, r);
    for (int i = 0; i < x.count; ++i) mine += x.tiles(i);
  }
  int64_t incl = mine;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int64_t y = __shfl_up(incl, off);
    if (lane >= off) incl += y;
  }
  if (lane == 63) wave_sum[wave] = incl;
  __syncthreads();
  int64_t before = 0, per_head = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if (w < wave) before += wave_sum[w];
    per_head += wave_sum[w];
  }
  const int64_t total = per_head * a.b.Hkv;
  const int64_t workgroups = min((int64_t)ma.workgroups, total);
  const int g = blockIdx.x;
  if (g >= workgroups) {
    if (tid == 0) ma.cuts[g].r = -1;
    return;
  }
  int64_t x = g * total / workgroups;
  const int64_t x_end = (g + 1) * total / workgroups;
  int head = (int)(x / per_head);
  {
    const int64_t at = x - head * per_head;
    int64_t start = before + incl - mine;
    if (at >= start && at < start + mine) {                      // one thread has it
      for (int r = tid * per;; ++r) {
        const Blocks y = blocks_of(ma, r);
        int64_t t = 0;
        int i = 0;
        for (; i < y.count; ++i) {
          const int tiles = y.tiles(i);
          if (at < start + t + tiles) break;
          t += tiles;
        }
        start += t;
        if (i < y.count) { found[0] = r; found[1] = i; found[2] = (int)(at - start); break; }
      }
    }
  }
  __syncthreads();
  int r = __builtin_amdgcn_readfirstlane(found[0]), block = __builtin_amdgcn_readfirstlane(found[1]), tile0 = __builtin_amdgcn_readfirstlane(found[2]);
  Blocks of = blocks_of(ma, r);
  bool first_segment = true;
  CutBlock cut = {-1, 0, 0, 0, 0};

  for (; x < x_end;) {
    if (block >= of.count) {                                     // the next request that has blocks, or the next head
      do {
        if (++r == n) { r = 0; ++head; }
        of = blocks_of(ma, r);
      } while (of.count == 0);
      block = 0;
    }
    const int tiles = of.tiles(block);
    const int tile1 = (int)min((int64_t)tiles, tile0 + (x_end - x));
    const bool whole = tile0 == 0 && tile1 == tiles;
    const int slot = first_segment ? 2 * g : 2 * g + 1;
    if (tile0 == 0 && tile1 < tiles) {
      const int64_t end = x + tiles;                             // position behind the block
      cut = {r, block, head, slot, (int)((end * workgroups - 1) / total)};
    }
    const int q0 = a.b.cu_q[r], row0 = block * kManyRows + wave * 64;
    const bool active = row0 < of.rows;

    // query rows as right operands, and the keys that the lane's rows see
    u32x4 qf[2][KS];
    int limit[2];
#pragma unroll
    for (int rb = 0; rb < 2; ++rb) {
      const int row = row0 + rb * 32 + l32, rr = min(row, of.rows - 1), t = rr / of.G;
      const uint16_t* p = a.q + (q0 + t) * a.b.q_st + (head * of.G + rr - t * of.G) * a.b.q_sh + half * 8;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        qf[rb][ks] = *reinterpret_cast<const u32x4*>(p + ks * 16);
        if (row >= of.rows) qf[rb][ks] = u32x4{0, 0, 0, 0};
      }
      limit[rb] = of.causal ? min(of.len, of.len - of.nq + t + 1) : of.len;
    }
    const int seen_by_all = of.causal ? min(of.len, of.len - of.nq + block * kManyRows / of.G + 1) : of.len;

    const unsigned char* kb = a.pool.k + a.layer + head * a.pool.s_head + (tid % PIECES) * 16;
    const unsigned char* vb = a.pool.v + a.layer + head * a.pool.s_head + (tid % PIECES) * 16;
    const int32_t* table = a.b.table + (int64_t)r * a.b.table_width;
    const int in_page = (1 << a.pool.page_log2) - 1;
    auto look_up = [&](int tile) {                               // page of key 64 tile + lane; -1: no such key
      const int key = tile * kManyKeys + lane;
      int page = -1;
      if (tile < tile1 && key < of.len) {
        page = table[key >> a.pool.page_log2];
        if (page >= a.pool.n_pages) page = -1;
      }
      return page;
    };
    auto send_for = [&](const unsigned char* base, u32x4* into, int tile, int page) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int row = i * ROWS + tid / PIECES;
        const int at = max(__shfl(page, row), 0);                // rows that are not there: page 0, zeroed below
        into[i] = *reinterpret_cast<const u32x4*>(base + at * a.pool.s_page + ((tile * kManyKeys + row) & in_page) * a.pool.s_tok);
      }
    };
    auto park = [&](unsigned char* lds, int row_bytes, const u32x4* from) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        unsigned char* at = lds + (i * ROWS + tid / PIECES) * row_bytes + (tid % PIECES) * (FP8 ? 32 : 16);
        if constexpr (FP8) {
          *reinterpret_cast<u32x4*>(at) = widen8(from[i].x, from[i].y);
          *reinterpret_cast<u32x4*>(at + 16) = widen8(from[i].z, from[i].w);
        } else {
          *reinterpret_cast<u32x4*>(at) = from[i];
        }
      }
    };
    u32x4 kr[LOADS], vr[LOADS];

    f32x16 o[2][DB];
    float m[2] = {-1.0e30f, -1.0e30f}, l[2] = {0.0f, 0.0f};
#pragma unroll
    for (int rb = 0; rb < 2; ++rb)
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[rb][db][i] = 0.0f;

    f32x16 s[2], s_next[2];
    bf16x8 p_prev[2][2];                                         // weights of the 32 keys before, [rows][16 keys]
#pragma unroll
    for (int rb = 0; rb < 2; ++rb)
#pragma unroll
      for (int k2 = 0; k2 < 2; ++k2) p_prev[rb][k2] = frag(u32x4{0, 0, 0, 0});

    auto logits = [&](f32x16 (&z)[2], const unsigned char* kt) {
#pragma unroll
      for (int rb = 0; rb < 2; ++rb)
#pragma unroll
        for (int i = 0; i < 16; ++i) z[rb][i] = 0.0f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const u32x4 kf = *reinterpret_cast<const u32x4*>(kt + l32 * K_ROW + ks * 32 + half * 16);
#pragma unroll
        for (int rb = 0; rb < 2; ++rb) z[rb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag(kf), frag(qf[rb][ks]), z[rb], 0, 0, 0);
      }
    };
    auto weigh_values = [&](const unsigned char* vt) {
#pragma unroll
      for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const unsigned char* at = vt + (k2 * 16 + half * 4 + ((lane >> 2) & 3)) * V_ROW + db * 64 + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
          const s16x4 v0 = read_columns(at), v1 = read_columns(at + 8 * V_ROW);
          const bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
          for (int rb = 0; rb < 2; ++rb) o[rb][db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, p_prev[rb][k2], o[rb][db], 0, 0, 0);
        }
    };
    // Values that some rows of the block do not see and that are infinite or NaN: zeros in LDS, added here to the rows that see them.
    auto add_apart = [&](unsigned bits, int key0, int page) {
      while (bits) {
        const int j = __ffs(bits) - 1;
        bits &= bits - 1;
        const int key = key0 + j;
        const unsigned char* row = a.pool.v + a.layer + head * a.pool.s_head + __shfl(page, key & 63) * a.pool.s_page + (key & in_page) * a.pool.s_tok;
#pragma unroll
        for (int rb = 0; rb < 2; ++rb) {
          unsigned w = 0;
#pragma unroll
          for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (k2 == (j >> 4) && i == ((j & 3) >> 1) + 2 * ((j & 15) >> 3)) w = __builtin_bit_cast(u32x4, p_prev[rb][k2])[i];
          w = __shfl(w, ((j >> 2) & 1) * 32 + l32);
          const float f = __uint_as_float((j & 1) ? w & 0xFFFF0000u : w << 16);
          const bool sees = key < limit[rb];
#pragma unroll
          for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const f32x4 v = row4<FP8>(row + (db * 32 + i * 8 + half * 4) * (FP8 ? 1 : 2));
#pragma unroll
              for (int e = 0; e < 4; ++e) o[rb][db][4 * i + e] = sees ? fmaf(f, v[e], o[rb][db][4 * i + e]) : o[rb][db][4 * i + e];
            }
        }
      }
    };
    // Weights of the 32 keys from key0 on; `valid`: which of them there are.
    auto weights = [&](f32x16 (&z)[2], int key0, unsigned valid) {
      if (__builtin_expect(valid != 0xFFFFFFFFu || key0 + 32 > seen_by_all, 0)) {
#pragma unroll
        for (int rb = 0; rb < 2; ++rb)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int j = 8 * (i >> 2) + 4 * half + (i & 3);
            if (!((valid >> j) & 1) || key0 + j >= limit[rb]) z[rb][i] = -INFINITY;
          }
      }
      float p[2][16], sum[2];
      float top = 0.0f;
      auto form = [&]() {
        top = 0.0f;
#pragma unroll
        for (int rb = 0; rb < 2; ++rb) {
          sum[rb] = 0.0f;
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            p[rb][i] = __builtin_amdgcn_exp2f(fmaf(z[rb][i], a.c, -m[rb]));
            sum[rb] += p[rb][i];
            top = fmaxf(top, p[rb][i]);
          }
        }
      };
      form();
      if (__builtin_expect(__ballot(top > 256.0f) != 0, 0)) {    // a logit far above its row's reference: move the references
#pragma unroll
        for (int rb = 0; rb < 2; ++rb) {
          float t = -INFINITY;
#pragma unroll
          for (int i = 0; i < 16; ++i) t = fmaxf(t, z[rb][i]);
          t *= a.c;
          t = fmaxf(t, __shfl_xor(t, 32));
          const float to = fmaxf(m[rb], t), old = to == m[rb] ? 1.0f : __builtin_amdgcn_exp2f(m[rb] - to);
          m[rb] = to;
          l[rb] *= old;
#pragma unroll
          for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[rb][db][i] *= old;
        }
        form();
      }
#pragma unroll
      for (int rb = 0; rb < 2; ++rb) {
        l[rb] += sum[rb];
#pragma unroll
        for (int k2 = 0; k2 < 2; ++k2) {
          u32x4 w;
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = pack2(p[rb][8 * k2 + 2 * i], p[rb][8 * k2 + 2 * i + 1]);
          p_prev[rb][k2] = frag(w);
        }
      }
    };

    // ---- tiles.  A tile's keys are in LDS a step before its values: while the weights of 32 keys are formed, the matrix cores form the
    // logits of the next 32 and take in the values of the 32 before.
    __syncthreads();                                             // the segment before is through with LDS
    int page = look_up(tile0), page_next = look_up(tile0 + 1), page_prev = -1;
    send_for(kb, kr, tile0, page);
    send_for(vb, vr, tile0, page);
    auto park_keys = [&](int tile, int pg) {
      const uint64_t valid = __ballot(pg >= 0);
      if (__builtin_expect(valid != ~0ull, 0)) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
          if (!((valid >> (i * ROWS + tid / PIECES)) & 1)) kr[i] = u32x4{0, 0, 0, 0};
      }
      park(k_lds[tile & 1], K_ROW, kr);
    };
    auto park_values = [&](int tile, int pg) {
      const uint64_t valid = __ballot(pg >= 0);
      const bool partly = (tile + 1) * kManyKeys > seen_by_all && seen_by_all < of.len;
      if (__builtin_expect(valid != ~0ull || partly, 0)) {
        uint64_t apart = 0;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
          const int row = i * ROWS + tid / PIECES;
          if (!((valid >> row) & 1)) vr[i] = u32x4{0, 0, 0, 0};
          const uint64_t bad = partly ? __ballot(not_finite<FP8>(vr[i])) : 0;
#pragma unroll
          for (int j = 0; j < 64 / PIECES; ++j)
            if ((bad >> (j * PIECES)) & ((1ull << PIECES) - 1)) apart |= 1ull << (i * ROWS + wave * (64 / PIECES) + j);
          if ((apart >> row) & 1) vr[i] = u32x4{0, 0, 0, 0};
        }
        if (lane == 0) apart_lds[tile & 1][wave] = apart;
      }
      park(v_lds[tile & 1], V_ROW, vr);
    };
    park_keys(tile0, page);
    if (tile0 + 1 < tile1) send_for(kb, kr, tile0 + 1, page_next);
    __syncthreads();
    if (active) logits(s, k_lds[tile0 & 1]);
    for (int tile = tile0; tile < tile1; ++tile) {
      const uint64_t valid = __ballot(page >= 0);
      const bool partly = (tile + 1) * kManyKeys > seen_by_all && seen_by_all < of.len;
      const bool partly_before = tile > tile0 && tile * kManyKeys > seen_by_all && seen_by_all < of.len;
      if (active) {
        logits(s_next, k_lds[tile & 1] + 32 * K_ROW);
        if (tile > tile0) weigh_values(v_lds[(tile + 1) & 1] + 32 * V_ROW);        // of the tile before
        if (__builtin_expect(partly_before, 0)) {
          const uint64_t* w = apart_lds[(tile + 1) & 1];
          add_apart((unsigned)((w[0] | w[1] | w[2] | w[3]) >> 32), (tile - 1) * kManyKeys + 32, page_prev);
        }
        weights(s, tile * kManyKeys, (unsigned)valid);
      }
      // the next tile's keys and this one's values
      if (tile + 1 < tile1) park_keys(tile + 1, page_next);
      park_values(tile, page);
      const int page_after = look_up(tile + 2);
      if (tile + 2 < tile1) send_for(kb, kr, tile + 2, page_after);
      if (tile + 1 < tile1) send_for(vb, vr, tile + 1, page_next);
      __syncthreads();
      if (active) {
        if (tile + 1 < tile1) logits(s, k_lds[(tile + 1) & 1]);
        weigh_values(v_lds[tile & 1]);
        if (__builtin_expect(partly, 0)) {
          const uint64_t* w = apart_lds[tile & 1];
          add_apart((unsigned)(w[0] | w[1] | w[2] | w[3]), tile * kManyKeys, page);
        }
        weights(s_next, tile * kManyKeys + 32, (unsigned)(valid >> 32));
      }
      page_prev = page; page = page_next; page_next = page_after;
    }
    if (active) {
      weigh_values(v_lds[(tile1 + 1) & 1] + 32 * V_ROW);
      if (__builtin_expect(tile1 * kManyKeys > seen_by_all && seen_by_all < of.len, 0)) {
        const uint64_t* w = apart_lds[(tile1 + 1) & 1];
        add_apart((unsigned)((w[0] | w[1] | w[2] | w[3]) >> 32), (tile1 - 1) * kManyKeys + 32, page_prev);
      }
#pragma unroll
      for (int rb = 0; rb < 2; ++rb) {
        const float sum = l[rb] + __shfl_xor(l[rb], 32);
        const int row = row0 + rb * 32 + l32;
        if (row >= of.rows) continue;
        if (whole) {
          const int t = row / of.G, h = head * of.G + row - t * of.G;
          const float inv = sum == 0.0f ? 0.0f : a.pool.v_scale / sum;
          uint16_t* out = a.out + (q0 + t) * a.b.o_st + h * a.b.o_sh + half * 4;
#pragma unroll
          for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              *reinterpret_cast<u32x2*>(out + db * 32 + i * 8) = u32x2{pack2(o[rb][db][4 * i] * inv, o[rb][db][4 * i + 1] * inv),
                                                                     pack2(o[rb][db][4 * i + 2] * inv, o[rb][db][4 * i + 3] * inv)};
          if (a.lse && half == 0) a.lse[(int64_t)(q0 + t) * a.b.Hq + h] = sum == 0.0f ? -INFINITY : (m[rb] + __builtin_amdgcn_logf(sum)) * kLn2;
        } else {
          const int64_t part = (int64_t)slot * kManyRows + wave * 64 + rb * 32 + l32;
#pragma unroll
          for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              *reinterpret_cast<f32x4*>(a.part_o + part * D + db * 32 + i * 8 + half * 4) =
                  f32x4{o[rb][db][4 * i], o[rb][db][4 * i + 1], o[rb][db][4 * i + 2], o[rb][db][4 * i + 3]};
          if (half == 0) { a.part_ml[2 * part] = m[rb]; a.part_ml[2 * part + 1] = sum; }
        }
      }
    }
    x += tile1 - tile0;
    tile0 = 0;
    ++block;
    first_segment = false;
  }
  if (tid == 0) ma.cuts[g] = cut;
}

template <int D, bool FP8>
int launch_many_of(const ManyArgs& m, hipStream_t stream) {
  attend_many_kernel<D, FP8><<<dim3(m.workgroups), dim3(256), 0, stream>>>(m);
  return (int)hipGetLastError();
}

}  // namespace codecomp
