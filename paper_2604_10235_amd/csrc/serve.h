// Internal header: what the operators of codecomp_serve.h share.
#pragma once
#include "attend.h"
#include "codecomp_serve.h"

namespace codecomp {

// Sums of attention weights; strides in elements.
struct MassSums {
  float* sums;
  int64_t s_layer, s_seq, s_head;
};
int make_mass(const codecomp_mass* m, MassSums* out);

// codecomp_attend_shared as laid out on the host.
struct SharedPlan {
  PagePool pool;
  PagedBatch batch;
  SharedRows sh;
  int d;
  float scale;
  int few_groups, many_groups; // groups of each kind (attend_shared.hip)
  bool prompts;                // the kernel for many rows has what requests have behind the shared rows
  int few_two, own_two;        // kernel for few rows, shared and own: 32 rows a workgroup, not 16
  int row_parts, chunk, own_splits;    // rows behind the shared ones: parts of a request's rows, keys of a chunk, chunks
  int64_t own_units;
  int own_parts;               // parts of a row behind the shared ones
  int64_t parts;               // of all rows
  bool both;                   // groups of either kind
  size_t ws_bytes;
};
int make_shared_plan(const codecomp_batch* b, const codecomp_groups* g, const codecomp_pages* p, SharedPlan* plan);
int launch_shared(const SharedPlan& pl, const void* q, int layer, void* out, float* lse, void* workspace, hipStream_t stream);

// codecomp_attend_mass as laid out on the host.
struct MassPlan {
  PagePool pool;
  PagedBatch batch;
  MassSums mass;
  int d;
  float scale;
  int few_rows, many_rows;     // requests of each kind (mass.hip)
  int few_most;                // rows of a request up to which it is of the first kind
  int chunk, chunks;           // few rows: keys of a workgroup, and workgroups for a request and head,
  int shares;                  // or (not 0) equal parts of the keys of all requests and heads
  size_t ws_bytes;
};
int make_mass_plan(const codecomp_batch* b, const codecomp_pages* p, const codecomp_mass* m, MassPlan* plan);
int launch_mass(const MassPlan& pl, const void* q, const float* lse, int layer, const int32_t* first, float decay, void* workspace, hipStream_t stream);

struct EvictArgs {
  PagePool pool;
  MassSums from, to;           // sums as they are, and those of the kept rows (the same, or elsewhere)
  const int32_t* kv_lens;
  const int32_t* table;
  const int32_t* budgets;
  const int32_t* first;
  int32_t* kept;
  int32_t* new_lens;
  int n_layers, n_seqs, Hkv, table_width, max_kv, max_budget, recent;
};
int launch_evict(const EvictArgs& a, int d, hipStream_t stream);

}  // namespace codecomp
