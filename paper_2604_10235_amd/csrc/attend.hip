// Attention of new tokens over a paged cache.
#include <math.h>

#include "cache.h"

namespace codecomp {

struct AttendArgs {
  PagePool pool;
  PagedBatch b;
  const uint16_t* q;
  uint16_t* out;
  float* lse;
  int64_t layer;
  float scale;
  int d;
};

__device__ __forceinline__ float element(const unsigned char* p, int i, bool fp8) {
  if (!fp8) return __uint_as_float((unsigned)reinterpret_cast<const uint16_t*>(p)[i] << 16);
  return __builtin_amdgcn_cvt_f32_fp8((int)p[i], 0);
}

// One wave per (token, query head): logits of 64 keys, a lane each, then the weighted rows, two elements a lane.
__global__ __launch_bounds__(64) void attend_plain_kernel(const AttendArgs a) {
  const int t = blockIdx.x, h = blockIdx.y, lane = threadIdx.x, kvh = h / a.b.G;
  const int r = request_of(a.b.cu_q, a.b.n_seqs, t);
  const int len = kv_len_of(a.b, r), at = len - a.b.cu_q[r + 1] + t;
  const int seen = a.b.causal ? max(min(len, at + 1), 0) : len;
  __shared__ float q[128];
  for (int i = lane; i < a.d; i += 64) q[i] = element(reinterpret_cast<const unsigned char*>(a.q + t * a.b.q_st + h * a.b.q_sh), i, false);
  __syncthreads();
  float top = -INFINITY, sum = 0.0f, o0 = 0.0f, o1 = 0.0f;
  for (int key0 = 0; key0 < seen; key0 += 64) {
    const int key = key0 + lane;
    int64_t row = -1;
    float x = -INFINITY;
    if (key < seen) {
      const int page = a.b.table[(int64_t)r * a.b.table_width + (key >> a.pool.page_log2)];
      if (page >= 0 && page < a.pool.n_pages)
        row = a.layer + page * a.pool.s_page + kvh * a.pool.s_head + (key & ((1 << a.pool.page_log2) - 1)) * a.pool.s_tok;
    }
    if (row >= 0) {
      x = 0.0f;
      for (int i = 0; i < a.d; ++i) x = fmaf(q[i], element(a.pool.k + row, i, a.pool.fp8), x);
      x *= a.scale * a.pool.k_scale;
    }
    float m = x;
    for (int off = 1; off < 64; off <<= 1) m = fmaxf(m, __shfl_xor(m, off));
    if (m == -INFINITY) continue;
    const float to = fmaxf(top, m), old = expf(top - to);
    const float p = row >= 0 ? expf(x - to) : 0.0f;
    top = to; sum = sum * old + p; o0 *= old; o1 *= old;
    for (int j = 0; j < min(64, seen - key0); ++j) {
      const int64_t vrow = __shfl(row, j);
      const float w = __shfl(p, j);
      if (vrow < 0) continue;
      const int e = lane * (a.d / 64);
      o0 = fmaf(w, element(a.pool.v + vrow, e, a.pool.fp8), o0);
      if (a.d == 128) o1 = fmaf(w, element(a.pool.v + vrow, e + 1, a.pool.fp8), o1);
    }
  }
  for (int off = 1; off < 64; off <<= 1) sum += __shfl_xor(sum, off);
  const float inv = sum > 0.0f ? a.pool.v_scale / sum : sum;
  __bf16* o = reinterpret_cast<__bf16*>(a.out + t * a.b.o_st + h * a.b.o_sh) + lane * (a.d / 64);
  o[0] = (__bf16)(o0 * inv);
  if (a.d == 128) o[1] = (__bf16)(o1 * inv);
  if (a.lse && lane == 0) a.lse[(int64_t)t * a.b.Hq + h] = top == -INFINITY ? -INFINITY : top + logf(sum);
}

int make_attend_plan(const codecomp_batch* b, const codecomp_pages* p, AttendPlan* pl) {
  if (int rc = make_pool(p, &pl->pool)) return rc;
  if (int rc = make_batch(b, p, &pl->batch)) return rc;
  if (pl->batch.Hq > 65535) return CODECOMP_EINVAL_HEADS;
  pl->d = p->head_dim;
  pl->scale = b->softmax_scale > 0.0f ? b->softmax_scale : 1.0f / sqrtf((float)p->head_dim);
  pl->ws_bytes = 0;
  return CODECOMP_OK;
}

int launch_attend(const AttendPlan& pl, const void* q, int layer, void* out, float* lse, void* workspace, hipStream_t stream) {
  AttendArgs a;
  a.pool = pl.pool; a.b = pl.batch; a.q = static_cast<const uint16_t*>(q); a.out = static_cast<uint16_t*>(out); a.lse = lse;
  a.layer = layer * pl.pool.s_layer; a.scale = pl.scale; a.d = pl.d;
  attend_plain_kernel<<<dim3(pl.batch.T, pl.batch.Hq), dim3(64), 0, stream>>>(a);
  return (int)hipGetLastError();
}

}  // namespace codecomp
