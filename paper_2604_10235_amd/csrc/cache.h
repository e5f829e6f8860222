// Internal header: what the operators on a paged cache (codecomp_cache.h) share.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "codecomp_cache.h"

namespace codecomp {

// A pool of pages with its strides in bytes.
struct PagePool {
  unsigned char* k;
  unsigned char* v;
  int n_pages, page_log2, fp8;
  int64_t s_layer, s_page, s_head, s_tok;
  float k_scale, v_scale;
};

// Requests over a pool; strides in elements.
struct PagedBatch {
  const int32_t* cu_q;
  const int32_t* kv_lens;
  const int32_t* table;
  int n_seqs, table_width, max_kv, causal, Hq, Hkv, G, T;
  int64_t q_st, q_sh, n_st, n_sh, o_st, o_sh;
};

// Validate and translate (0 or a CODECOMP_E* code).  Host only.
int make_pool(const codecomp_pages* p, PagePool* pool);
int make_batch(const codecomp_batch* b, const codecomp_pages* p, PagedBatch* batch);

// Rows of the cache that a request has: what is on the device, cut to what the host said.
__device__ __forceinline__ int kv_len_of(const PagedBatch& b, int r) { return min(max(b.kv_lens[r], 0), b.max_kv); }

// The request of packed token `t`, the same for all lanes of the wave: the last r with cu[r] <= t (a request without tokens shares
// its start with the next one, so it is never the last).  64 candidates a round; all lanes of the wave take part.
__device__ __forceinline__ int request_of(const int32_t* cu, int n_seqs, int t) {
  int lo = 0;                                    // cu[lo] <= t, and the answer is in [lo, lo + span)
  for (int span = n_seqs; span > 1;) {
    const int step = (span + 63) >> 6, at = lo + (int)(threadIdx.x & 63) * step;
    const int hits = __popcll(__ballot(at < lo + span && cu[at] <= t));          // a prefix of the candidates, lo among them
    const int next = lo + max(hits - 1, 0) * step;
    span = min(step, lo + span - next);
    lo = next;
  }
  return lo;
}

struct RotaryArgs {
  uint64_t turns[64];          // of a pair per position, in 2^-64 of a turn, modulo 1
  int dim, interleaved;
  float magnitude;
};
int make_rotary(const codecomp_rotary* r, int head_dim, RotaryArgs* a);

constexpr int kFewMostSplits = 2048;      // most chunks that a request's keys are cut into

// codecomp_attend as laid out on the host.
struct AttendPlan {
  PagePool pool;
  PagedBatch batch;
  int d;
  float scale;
  int few_rows, many_rows;     // requests of each kind (attend.hip)
  int row_slots, row_parts;    // few rows: rows of the largest, workgroups that they are shared out to
  int chunk, splits;           // few rows: keys of a workgroup, and workgroups per request and head,
  int shares;                  // or (not 0) equal parts of the keys of all requests and heads, one for each workgroup
  int workgroups, many_from, many_blocks;        // many rows: workgroups, rows from which a request is of this kind, blocks of rows,
  int many_whole;              // none of them shared
  size_t off_few, off_many, ws_bytes;
};
int make_attend_plan(const codecomp_batch* b, const codecomp_pages* p, AttendPlan* plan);
int launch_attend(const AttendPlan& pl, const void* q, int layer, void* out, float* lse, void* workspace, hipStream_t stream);

int launch_rotate(const RotaryArgs& rot, const void* x, const int32_t* positions, int T, int H, int d, int64_t x_st, int64_t x_sh, void* out, int64_t o_st,
                  int64_t o_sh, hipStream_t stream);
int launch_append(const RotaryArgs& rot, const PagedBatch& b, const PagePool& pool, int layer, int d, const void* q, const void* k, const void* v,
                  const int32_t* positions, void* q_out, hipStream_t stream);

// One side of a move of rows: dense rows packed by request (table NULL), or pages.  Strides in bytes.
struct RowSide {
  unsigned char* k;
  unsigned char* v;
  const int32_t* table;
  const int32_t* first;        // pages: row of the cache that is the request's row 0; NULL = 0
  const int32_t* cu;           // dense: where a request's rows begin
  int table_width, n_pages, page_log2;
  int64_t s_layer, s_page, s_head, s_tok;
};
struct MoveArgs {
  RowSide from, to;
  const int32_t* idx;          // [L * Hkv][rows] request-local source rows, or NULL: row i is source row i
  const int32_t* cu_rows;      // requests of the moved rows
  const int32_t* cu_source;    // lengths of the requests that idx points into
  int n_seqs, Hkv, rows, pieces_log2;
};
int launch_move(const MoveArgs& a, int problems, hipStream_t stream);
int launch_pages_copy(const PagePool& pool, int L, int Hkv, int d, const int32_t* pairs, int n_pairs, hipStream_t stream);

}  // namespace codecomp
