// Rotary positions, by themselves and on the way into the pages.
//
// A pair (x0, x1) at position p becomes magnitude * (x0 cos a - x1 sin a, x0 sin a + x1 cos a), a = p * freq.  Both kernels only
// move memory: 4 bytes per element against a few operations, and what the angles cost is shared by the heads that a thread takes.
// Measured: 32768 tokens of 40 heads of 128 elements 115 us, 5.8 TB/s (as much as any copy here); four chunks of together 10500 tokens into an FP8
// cache 58 us, 4.5 TB/s; 16 tokens 3.3 us, of which the launch and one chain of loads are all.
// The angle of a far position loses all its digits in fp32 (p * freq at 10^6 has steps of 0.06 rad): it is formed in turns as a 64-bit
// fraction (rounded once, on the host), whose product with a whole position wraps around where the angle does.  What is left of it after taking out the nearest
// quarter turn is at most pi / 4, known to 2^-27 of a turn, where the Taylor series of sine and cosine to the 9th and 10th power are good to 2e-9 and 1.2e-10
// (pi/4^11 / 11!, pi/4^12 / 12!).
#include "cache.h"

namespace codecomp {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kRotaryThreads = 256;
// Units of 16 elements up to which every thread takes one head, beyond it four, which share their angles (40 heads of 128, us, one | four: 256 tokens
// 3.8 | 4.8, 1024 6.5 | 5.8; append of 500 tokens 6.0 | 7.0, of 2000 12.8 | 11.6).
constexpr int kRotaryFew = 3 << 16;

struct Vectors {               // bf16 [tokens][heads][d]
  const uint16_t* p;
  int64_t st, sh;
};
struct RotateArgs {
  RotaryArgs rot;
  const int32_t* positions;
  Vectors x, k, v;             // x: what is rotated into `out`; k, v: append only
  uint16_t* out;
  int64_t o_st, o_sh;
  int T, heads, groups;        // heads that threads walk through (append: q, k and v heads), thread groups they are cut into
  int q_heads;                 // append: heads of x among them (0: none given)
  PagedBatch b;
  PagePool pool;
  int64_t layer;               // byte offset of the layer
};

__device__ __forceinline__ void sine_cosine(uint64_t turns, float magnitude, float& s, float& c) {
  const uint64_t quarter = (turns + (1ull << 61)) >> 62;                       // nearest, modulo 4
  const int32_t rest = (int32_t)((int64_t)(turns - (quarter << 62)) >> 30);     // what is left, in 2^-34 of a turn
  const float a = (float)rest * (float)(6.283185307179586477 / 17179869184.0), z = a * a;
  float sn = fmaf(z, 2.7557319e-6f, -1.9841270e-4f), cs = fmaf(z, -2.7557319e-7f, 2.4801587e-5f);
  sn = fmaf(z, sn, 8.3333333e-3f); cs = fmaf(z, cs, -1.3888889e-3f);
  sn = fmaf(z, sn, -1.6666667e-1f); cs = fmaf(z, cs, 4.1666667e-2f);
  sn = fmaf(a * z, sn, a); cs = fmaf(z, cs, -0.5f);
  cs = fmaf(z, cs, 1.0f);
  const bool odd = quarter & 1;
  const float s0 = odd ? cs : sn, c0 = odd ? sn : cs;
  s = ((quarter & 2) ? -s0 : s0) * magnitude;
  c = (((quarter + 1) & 2) ? -c0 : c0) * magnitude;
}

__device__ __forceinline__ void widen(u32x4 a, float* f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(a[i] << 16);
    f[2 * i + 1] = __uint_as_float(a[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ u32x4 narrow(const float* f) {          // to the nearest bf16, ties to even
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = __builtin_bit_cast(unsigned, bf16x2{(__bf16)f[2 * i], (__bf16)f[2 * i + 1]});
  return r;
}
__device__ __forceinline__ float to_e4m3_range(float x) { return x != x ? x : fminf(fmaxf(x, -448.0f), 448.0f); }
__device__ __forceinline__ u32x2 narrow8(const float* f) {         // to the nearest E4M3 code, ties to even, beyond 448 to 448
  float g[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) g[i] = to_e4m3_range(f[i]);
  int lo = __builtin_amdgcn_cvt_pk_fp8_f32(g[0], g[1], 0, false), hi = __builtin_amdgcn_cvt_pk_fp8_f32(g[4], g[5], 0, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(g[2], g[3], lo, true);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(g[6], g[7], hi, true);
  return u32x2{(unsigned)lo, (unsigned)hi};
}

// A thread takes unit u of a token, 16 elements of a head, for HPT heads in turn: elements 8 u .. and dim / 2 + 8 u .. (pairs of halves), or
// 16 u .. (neighbours, and what is not rotated).  Consecutive threads take consecutive units: whole lines of a head.
template <int HPT, bool INTERLEAVED, bool APPEND>
__global__ __launch_bounds__(kRotaryThreads) void rotary_kernel(const RotateArgs a, int units_log2) {
  // Long calls write past the caches what these could not hold until it is read (bf16 append of 8800 tokens 64 -> 53 us), and read past them what they
  // rotate (32768 tokens 125 -> 120 -> 115 us; loads of append 53 -> 55: not there).
  auto put = [](auto* at, auto v) __attribute__((always_inline)) {
    auto* p = reinterpret_cast<decltype(v)*>(at);
    if constexpr (HPT > 1) __builtin_nontemporal_store(v, p);
    else *p = v;
  };
  auto get = [](const uint16_t* at) __attribute__((always_inline)) {
    const u32x4* p = reinterpret_cast<const u32x4*>(at);
    if constexpr (HPT > 1 && !APPEND) return __builtin_nontemporal_load(p);
    return *p;
  };
  const unsigned id = blockIdx.x * kRotaryThreads + threadIdx.x;
  const int u = id & ((1 << units_log2) - 1);
  const unsigned rest = id >> units_log2;
  int t = (int)(rest / (unsigned)a.groups);
  const int group = (int)rest - t * a.groups;
  const bool there = t < a.T;
  t = min(t, a.T - 1);
  const bool turned = u * 16 < a.rot.dim;
  const int e0 = turned && !INTERLEAVED ? u * 8 : u * 16, e1 = turned && !INTERLEAVED ? a.rot.dim / 2 + u * 8 : u * 16 + 8;
  // The vectors are sent for first: what follows up to their use is a chain of small loads, and the angles.
  const int kv = APPEND ? a.b.Hkv : 0;
  u32x4 lo[HPT], hi[HPT];
#pragma unroll
  for (int j = 0; j < HPT; ++j) {
    const int h = group * HPT + j;
    if (h >= a.heads || !there) continue;
    const uint16_t* p;
    if (!APPEND || h < a.q_heads) p = a.x.p + t * a.x.st + h * a.x.sh;
    else if (h < a.q_heads + kv) p = a.k.p + t * a.k.st + (h - a.q_heads) * a.k.sh;
    else p = a.v.p + t * a.v.st + (h - a.q_heads - kv) * a.v.sh;
    lo[j] = get(p + e0);
    hi[j] = get(p + e1);
  }
  int64_t row = -1;            // where the token's K and V go
  if constexpr (APPEND) {
    int r = request_of(a.b.cu_q, a.b.n_seqs, __builtin_amdgcn_readfirstlane(t));
    while (r + 1 < a.b.n_seqs && a.b.cu_q[r + 1] <= t) ++r;
    const int slot = kv_len_of(a.b, r) - a.b.cu_q[r + 1] + t;
    if (slot >= 0) {
      const int page = a.b.table[(int64_t)r * a.b.table_width + (slot >> a.pool.page_log2)];
      if (page >= 0 && page < a.pool.n_pages) row = a.layer + page * a.pool.s_page + (slot & ((1 << a.pool.page_log2) - 1)) * a.pool.s_tok;
    }
  }
  if (!there) return;
  float s[8], c[8];
  if (turned) {
    const uint64_t p = (uint64_t)(int64_t)a.positions[t];
#pragma unroll
    for (int i = 0; i < 8; ++i) sine_cosine(p * a.rot.turns[u * 8 + i], a.rot.magnitude, s[i], c[i]);
  }
#pragma unroll
  for (int j = 0; j < HPT; ++j) {
    const int h = group * HPT + j;
    if (h >= a.heads) continue;
    const bool value = APPEND && h >= a.q_heads + kv, key = APPEND && !value && h >= a.q_heads;
    float f[16];
    if ((turned && !value) || key || value) { widen(lo[j], f); widen(hi[j], f + 8); }
    if (turned && !value) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int i0 = INTERLEAVED ? 2 * i : i, i1 = INTERLEAVED ? 2 * i + 1 : 8 + i;
        const float x0 = f[i0], x1 = f[i1];
        f[i0] = x0 * c[i] - x1 * s[i];
        f[i1] = x0 * s[i] + x1 * c[i];
      }
    }
    if (!key && !value) {
      uint16_t* o = a.out + t * a.o_st + h * a.o_sh;
      put(o + e0, turned ? narrow(f) : lo[j]);
      put(o + e1, turned ? narrow(f + 8) : hi[j]);
      continue;
    }
    if (row < 0) continue;
    const float scale = value ? a.pool.v_scale : a.pool.k_scale;
    if (scale != 1.0f) {
#pragma unroll
      for (int i = 0; i < 16; ++i) f[i] = f[i] / scale;
    }
    unsigned char* o = (value ? a.pool.v : a.pool.k) + row + (h - a.q_heads - (value ? kv : 0)) * a.pool.s_head;
    // a value head's unit has the same elements as a key head's: e0 and e1
    if (a.pool.fp8) {
      const u32x2 x = narrow8(f), y = narrow8(f + 8);
      if (e1 == e0 + 8) {
        put(o + e0, u32x4{x.x, x.y, y.x, y.y});
      } else {
        put(o + e0, x);
        put(o + e1, y);
      }
    } else {
      put(o + 2 * e0, narrow(f));
      put(o + 2 * e1, narrow(f + 8));
    }
  }
}

template <int HPT, bool APPEND>
static int launch_rotary_of(RotateArgs& a, int units_log2, hipStream_t stream) {
  a.groups = (a.heads + HPT - 1) / HPT;
  const int64_t threads = ((int64_t)a.T * a.groups) << units_log2;
  const dim3 grid((unsigned)((threads + kRotaryThreads - 1) / kRotaryThreads)), block(kRotaryThreads);
  if (a.rot.interleaved) rotary_kernel<HPT, true, APPEND><<<grid, block, 0, stream>>>(a, units_log2);
  else rotary_kernel<HPT, false, APPEND><<<grid, block, 0, stream>>>(a, units_log2);
  return (int)hipGetLastError();
}

template <bool APPEND>
static int launch_rotary(RotateArgs& a, int d, hipStream_t stream) {
  const int units_log2 = d == 128 ? 3 : 2;
  if (((int64_t)a.T * a.heads << units_log2) <= kRotaryFew) return launch_rotary_of<1, APPEND>(a, units_log2, stream);
  return launch_rotary_of<4, APPEND>(a, units_log2, stream);
}

int launch_rotate(const RotaryArgs& rot, const void* x, const int32_t* positions, int T, int H, int d, int64_t x_st, int64_t x_sh, void* out, int64_t o_st,
                  int64_t o_sh, hipStream_t stream) {
  RotateArgs a = {};
  a.rot = rot; a.positions = positions;
  a.x = {static_cast<const uint16_t*>(x), x_st, x_sh};
  a.out = static_cast<uint16_t*>(out); a.o_st = o_st; a.o_sh = o_sh;
  a.T = T; a.heads = H;
  return launch_rotary<false>(a, d, stream);
}

int launch_append(const RotaryArgs& rot, const PagedBatch& b, const PagePool& pool, int layer, int d, const void* q, const void* k, const void* v,
                  const int32_t* positions, void* q_out, hipStream_t stream) {
  RotateArgs a = {};
  a.rot = rot; a.positions = positions;
  a.x = {static_cast<const uint16_t*>(q), b.q_st, b.q_sh};
  a.k = {static_cast<const uint16_t*>(k), b.n_st, b.n_sh};
  a.v = {static_cast<const uint16_t*>(v), b.n_st, b.n_sh};
  a.out = static_cast<uint16_t*>(q_out); a.o_st = b.o_st; a.o_sh = b.o_sh;
  a.T = b.T; a.q_heads = q ? b.Hq : 0; a.heads = a.q_heads + 2 * b.Hkv;
  a.b = b; a.pool = pool; a.layer = layer * pool.s_layer;
  return launch_rotary<true>(a, d, stream);
}

}  // namespace codecomp
