// Internal header: what the kernels of codecomp_attend share.
#pragma once
#include "cache.h"

namespace codecomp {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// A row's reference (what is subtracted from its logits before exp2) only moves when a logit is this far above it: weights up to 2^8
// lose nothing in fp32 or in bf16, and most tiles then leave the sums and the outputs as they are.
constexpr float kSlack = 8.0f;

constexpr int kFewRowsMost = 64;          // rows of a request up to which weights are two bf16, in either kernel, and most rows that the one for few takes

// What a workgroup leaves for the kernel that joins rows whose keys several workgroups had.
struct CutBlock {
  int32_t r, block, head;      // of the block of rows whose first part is this workgroup's (slot 2 * workgroup + 1); r < 0: none
  int32_t last;                // last workgroup with a part of it (those after the first in slot 2 * workgroup)
};

// Groups of requests that share the rows at the start of their caches (attend_shared.hip).
struct SharedRows {
  const int32_t* cu_groups;
  const int32_t* prefix_lens;
  int n_groups, max_prefix, max_own;
  int few_rows;                // rows of a group up to which the kernel for few rows has its shared rows
  int few_units, few_parts, few_chunk, few_splits;       // shared rows of groups of few rows: workgroups, parts of the rows, keys of a chunk, chunks
  int many_units, many_tiles, many_splits;               // of many: workgroups, tiles of a chunk, chunks
  int fine;                    // of many, weights of the shared rows as two bf16: 0 never, 1 always, 2 in waves with rows of a request of up to kFewRowsMost
  int many_tokens, few_tokens; // tokens of groups of each kind; a row has a part for each chunk of its kind's
  int32_t* place;              // where there are both: of a token among those of its kind, few: ~place (written by the kernel for many rows, which does not need them)
  int64_t own_base;            // tokens' parts of shared rows, all together; behind them those of the rows behind, chunk by chunk of all tokens
  int own_units, own_tiles, own_splits;                  // of many, behind the shared rows: the same, and their parts; 0: the kernel for few rows has those
  int alone;                   // 1: everything is short, and a request's shared rows are attended to with its own ones, by the kernel for few rows: no parts
  int join;                    // 1: whoever has a request's own rows joins the parts of the shared ones to them, and writes the outputs
};
// What a row's parts say that had no keys: not to be read any further.
constexpr float kNoPart = -1.0f;

struct AttendArgs {
  PagePool pool;
  PagedBatch b;
  const uint16_t* q;
  uint16_t* out;
  float* lse;
  float* part_o;               // [part][rows of a part][D], not yet divided by the sum of weights
  float* part_ml;              // [part][rows of a part][2]: reference, sum of weights
  int64_t layer;               // byte offset of the layer in the pool
  float c;                     // softmax_scale * k_scale * log2(e): logits in powers of two
  int chunk, splits, row_slots, row_parts;       // few rows: keys of a chunk, most chunks, most rows, workgroups that they are shared out to
  int shares;                  // few rows: equal parts that all keys are cut into; 0: chunks
  CutBlock* cuts;              // [shares]
};
struct SharedArgs : AttendArgs {
  SharedRows sh;
};

__device__ __forceinline__ int prefix_of(const SharedRows& sh, int g) { return min(max(sh.prefix_lens[g], 0), sh.max_prefix); }
// Parts lie chunk by chunk, all rows of a kind of groups, [chunk][token][head]: part p of a group's token and a head is row_part(first + p * step, token, head).
struct GroupParts { int64_t first, step; int count; };
__device__ __forceinline__ GroupParts parts_of_group(const SharedRows& sh, int token) {
  if (!sh.place) return {0, sh.many_tokens + sh.few_tokens, max(sh.many_splits, sh.few_splits)};
  const int at = sh.place[token];
  if (at >= 0) return {at - token, sh.many_tokens, sh.many_splits};
  return {(int64_t)sh.many_splits * sh.many_tokens + ~at - token, sh.few_tokens, sh.few_splits};
}
__device__ __forceinline__ int64_t row_part(const AttendArgs& a, int64_t base, int token, int head) { return (base + token) * a.b.Hq + head; }
// A part of rows row0 .. row1 - 1 of a KV head, which has tokens from q0 on: nothing in it.
template <int THREADS>
__device__ __forceinline__ void no_part(const AttendArgs& a, int64_t base, int q0, int head, int row0, int row1) {
  for (int row = row0 + threadIdx.x; row < row1; row += THREADS) {
    const int t = row / a.b.G, h = head * a.b.G + row - t * a.b.G;
    const int64_t part = row_part(a, base, q0 + t, h);
    a.part_ml[2 * part] = -INFINITY; a.part_ml[2 * part + 1] = kNoPart;
  }
}

// The same in all lanes, and known to be: in scalar registers.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform(int64_t x) {
  return (int64_t)((uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 | (unsigned)__builtin_amdgcn_readfirstlane((int)x));
}

__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p; }

__device__ __forceinline__ bf16x8 frag(u32x4 v) { return __builtin_bit_cast(bf16x8, v); }
__device__ __forceinline__ unsigned pack2(float a, float b) { return __builtin_bit_cast(unsigned, bf16x2{(__bf16)a, (__bf16)b}); }

// 8 E4M3 codes as 8 bf16: every E4M3 number is a bf16 number.
__device__ __forceinline__ u32x4 widen8(unsigned a, unsigned b) {
  u32x4 r;
  r.x = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false));
  r.y = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true));
  r.z = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false));
  r.w = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true));
  return r;
}

// A 16-byte piece with zeros for its infinities and NaN (E4M3 has no infinity); `any`: not 0 where there were some.  Their exponents are all ones
// (E4M3: all bits but the sign), to which one at the bottom makes a carry into the sign's place.
template <bool FP8>
__device__ __forceinline__ u32x4 finite_part(u32x4 v, unsigned& any) {
  constexpr unsigned ONES = FP8 ? 0x7F7F7F7Fu : 0x7F807F80u, ONE = FP8 ? 0x01010101u : 0x00800080u, SIGNS = FP8 ? 0x80808080u : 0x80008000u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const unsigned found = ((v[i] & ONES) + ONE) & SIGNS;
    any |= found;
    v[i] &= ~((found >> (FP8 ? 7 : 15)) * (FP8 ? 0xFFu : 0xFFFFu));
  }
  return v;
}

// 4 elements of a stored row as floats.
template <bool FP8>
__device__ __forceinline__ f32x4 row4(const unsigned char* p) {
  f32x4 r;
  if constexpr (FP8) {
    const unsigned x = *reinterpret_cast<const unsigned*>(p);
    const unsigned lo = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.0f, false));
    const unsigned hi = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.0f, true));
    r = f32x4{__uint_as_float(lo << 16), __uint_as_float(lo & 0xFFFF0000u), __uint_as_float(hi << 16), __uint_as_float(hi & 0xFFFF0000u)};
  } else {
    const u32x2 x = *reinterpret_cast<const u32x2*>(p);
    r = f32x4{__uint_as_float(x.x << 16), __uint_as_float(x.x & 0xFFFF0000u), __uint_as_float(x.y << 16), __uint_as_float(x.y & 0xFFFF0000u)};
  }
  return r;
}

// What finite_part left out, for a row that sees the value: weights are positive, so an infinity or NaN is what the sum becomes, whatever
// the weight.
__device__ __forceinline__ float with_the_rest(float sum, float v) { return __builtin_isfinite(v) ? sum : sum + v; }

// The transposing read: a group of 16 lanes addresses four rows of 16 elements in LDS, four lanes a row, and lane i gets column i.
__device__ __forceinline__ s16x4 read_columns(const unsigned char* lds) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)lds);
}

int launch_few(const AttendPlan& pl, const AttendArgs& a, hipStream_t stream);
int launch_few_shared(int d, bool fp8, bool two_blocks, int64_t units, const SharedArgs& a, hipStream_t stream);

}  // namespace codecomp
