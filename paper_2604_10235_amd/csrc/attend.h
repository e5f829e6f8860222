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

}  // namespace codecomp
