// C ABI of the operators for shared and evicted caches (codecomp_serve.h): validation, and what is launched.  Validation happens before the first HIP
// call, as in api.hip.
#include <math.h>

#include "serve.h"

namespace codecomp {

static bool misaligned16(const void* p) { return ((uintptr_t)p & 15) != 0; }
static bool misaligned4(const void* p) { return ((uintptr_t)p & 3) != 0; }

int make_mass(const codecomp_mass* m, MassSums* out) {
  if (!m || !m->sums) return CODECOMP_EINVAL_NULL;
  if (m->n_layers < 1 || m->n_seqs < 1 || m->n_kv_heads < 1 || m->width < 0 || misaligned4(m->sums)) return CODECOMP_EINVAL_SHAPE;
  if (m->n_layers > (1 << 20) || m->n_seqs > 65535 || m->n_kv_heads > 65535) return CODECOMP_EINVAL_SHAPE;       // with which sizes can be multiplied in 64 bits
  if (m->stride_layer < 0 || m->stride_seq < 0 || m->stride_head < 0) return CODECOMP_EINVAL_SHAPE;
  out->sums = m->sums;
  out->s_head = m->stride_head ? m->stride_head : m->width;
  out->s_seq = m->stride_seq ? m->stride_seq : m->n_kv_heads * (int64_t)m->width;
  out->s_layer = m->stride_layer ? m->stride_layer : (int64_t)m->n_seqs * m->n_kv_heads * m->width;
  return CODECOMP_OK;
}

static int bad_workspace(const void* workspace, size_t have, size_t need) {
  return need > 0 && (!workspace || ((uintptr_t)workspace & 255) != 0 || have < need) ? CODECOMP_EINVAL_WORKSPACE : CODECOMP_OK;
}

}  // namespace codecomp

using namespace codecomp;

extern "C" {

int codecomp_attend_shared_validate(const codecomp_batch* batch, const codecomp_groups* groups, const codecomp_pages* pages) {
  SharedPlan pl;
  return make_shared_plan(batch, groups, pages, &pl);
}

size_t codecomp_attend_shared_workspace_bytes(const codecomp_batch* batch, const codecomp_groups* groups, const codecomp_pages* pages) {
  SharedPlan pl;
  return make_shared_plan(batch, groups, pages, &pl) ? 0 : pl.ws_bytes;
}

int codecomp_attend_shared(const void* q, const codecomp_batch* batch, const codecomp_groups* groups, const codecomp_pages* pages, int32_t layer, void* out,
                           float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
  SharedPlan pl;
  if (int rc = make_shared_plan(batch, groups, pages, &pl)) return rc;
  if (pl.batch.T > 0 && (!q || !out)) return CODECOMP_EINVAL_NULL;
  if (layer < 0 || layer >= pages->n_layers) return CODECOMP_EINVAL_PAGES;
  if (misaligned16(q) || misaligned16(out) || misaligned4(lse)) return CODECOMP_EINVAL_SHAPE;
  if (int rc = bad_workspace(workspace, workspace_bytes, pl.ws_bytes)) return rc;
  if (pl.batch.T == 0) return CODECOMP_OK;
  return launch_shared(pl, q, layer, out, lse, workspace, (hipStream_t)hip_stream);
}

int codecomp_attend_mass_validate(const codecomp_batch* batch, const codecomp_pages* pages, const codecomp_mass* mass) {
  MassPlan pl;
  return make_mass_plan(batch, pages, mass, &pl);
}

size_t codecomp_attend_mass_workspace_bytes(const codecomp_batch* batch, const codecomp_pages* pages, const codecomp_mass* mass) {
  MassPlan pl;
  return make_mass_plan(batch, pages, mass, &pl) ? 0 : pl.ws_bytes;
}

int codecomp_attend_mass(const void* q, const float* lse, const codecomp_batch* batch, const codecomp_pages* pages, int32_t layer, const int32_t* first,
                         float decay, const codecomp_mass* mass, void* workspace, size_t workspace_bytes, void* hip_stream) {
  MassPlan pl;
  if (int rc = make_mass_plan(batch, pages, mass, &pl)) return rc;
  if (pl.batch.T > 0 && (!q || !lse)) return CODECOMP_EINVAL_NULL;
  if (layer < 0 || layer >= pages->n_layers) return CODECOMP_EINVAL_PAGES;
  if (!(decay >= 0.0f && decay <= 1.0f)) return CODECOMP_EINVAL_PRIOR;
  if (misaligned16(q) || misaligned4(lse) || misaligned4(first)) return CODECOMP_EINVAL_SHAPE;
  if (int rc = bad_workspace(workspace, workspace_bytes, pl.ws_bytes)) return rc;
  if (pl.batch.T == 0) return CODECOMP_OK;
  return launch_mass(pl, q, lse, layer, first, decay, workspace, (hipStream_t)hip_stream);
}

int codecomp_evict(const codecomp_mass* mass, const codecomp_eviction* e, const codecomp_pages* pages, int32_t* kept, int32_t* new_lens,
                   const codecomp_mass* kept_mass, void* hip_stream) {
  EvictArgs a = {};
  if (int rc = make_mass(mass, &a.from)) return rc;
  if (int rc = make_pool(pages, &a.pool)) return rc;
  if (!e || !e->kv_lens_dev || !e->table_dev || !e->budgets_dev || !kept || !new_lens) return CODECOMP_EINVAL_NULL;
  if (kept_mass) {
    if (int rc = make_mass(kept_mass, &a.to)) return rc;
    if (kept_mass->n_layers != mass->n_layers || kept_mass->n_seqs != mass->n_seqs || kept_mass->n_kv_heads != mass->n_kv_heads || kept_mass->width != mass->width)
      return CODECOMP_EINVAL_SHAPE;
  } else {
    a.to = a.from;
  }
  // in place means with the same strides: sums that are written where others are still to be read would be lost
  if (a.to.sums == a.from.sums && (a.to.s_layer != a.from.s_layer || a.to.s_seq != a.from.s_seq || a.to.s_head != a.from.s_head)) return CODECOMP_EINVAL_SHAPE;
  if (e->n_seqs < 1 || e->n_seqs > 65535 || e->n_seqs != mass->n_seqs || mass->n_layers != pages->n_layers || mass->n_kv_heads != pages->n_kv_heads) return CODECOMP_EINVAL_SHAPE;
  if (e->table_width < 1 || e->max_kv_len < 0 || e->max_kv_len > (int64_t)e->table_width * pages->page_size || e->max_kv_len > (1 << 30)) return CODECOMP_EINVAL_PAGES;
  if (e->max_kv_len > mass->width) return CODECOMP_EINVAL_SHAPE;
  if (e->max_budget < 1 || e->max_budget > (1 << 30) || e->recent < 0 || e->recent > e->max_budget) return CODECOMP_EINVAL_BUDGET;
  if (misaligned4(kept) || misaligned4(new_lens)) return CODECOMP_EINVAL_SHAPE;
  if (new_lens == e->kv_lens_dev || new_lens == e->budgets_dev || new_lens == e->first_dev) return CODECOMP_EINVAL_SHAPE;       // read when it is written
  a.kv_lens = e->kv_lens_dev; a.table = e->table_dev; a.budgets = e->budgets_dev; a.first = e->first_dev;
  a.kept = kept; a.new_lens = new_lens;
  a.n_layers = pages->n_layers; a.n_seqs = e->n_seqs; a.Hkv = pages->n_kv_heads;
  a.table_width = e->table_width; a.max_kv = e->max_kv_len; a.max_budget = e->max_budget; a.recent = e->recent;
  return launch_evict(a, pages->head_dim, (hipStream_t)hip_stream);
}

}  // extern "C"
