// C ABI of the operators on a paged cache (codecomp_cache.h): validation, rotary frequencies, and what is launched.  Validation
// happens before the first HIP call, as in api.hip.
#include <math.h>

#include "cache.h"
#include "plan.h"

namespace codecomp {

constexpr int kMostHeads = 65535;      // with which sizes can be multiplied in 64 bits

static bool misaligned16(const void* p) { return ((uintptr_t)p & 15) != 0; }
static bool bad_strides(std::initializer_list<int64_t> strides, int multiple) {
  for (int64_t s : strides)
    if (s < 0 || s % multiple != 0) return true;
  return false;
}

int make_pool(const codecomp_pages* p, PagePool* pool) {
  if (!p || !p->k || !p->v) return CODECOMP_EINVAL_NULL;
  if (p->head_dim != 64 && p->head_dim != 128) return CODECOMP_EINVAL_HEADDIM;
  if (p->kv_dtype != CODECOMP_KV_BF16 && p->kv_dtype != CODECOMP_KV_FP8_E4M3) return CODECOMP_EINVAL_MODE;
  if (p->n_kv_heads < 1) return CODECOMP_EINVAL_HEADS;
  if (p->n_layers < 1 || (int64_t)p->n_layers * p->n_kv_heads > 65535) return CODECOMP_EINVAL_SHAPE;       // one grid axis
  if (p->n_pages < 1 || p->page_size < 1 || p->page_size > 65536 || (p->page_size & (p->page_size - 1)) != 0) return CODECOMP_EINVAL_PAGES;
  const int esz = p->kv_dtype == CODECOMP_KV_FP8_E4M3 ? 1 : 2;
  if (misaligned16(p->k) || misaligned16(p->v)) return CODECOMP_EINVAL_SHAPE;
  if (bad_strides({p->stride_layer, p->stride_page, p->stride_head, p->stride_tok}, 16 / esz)) return CODECOMP_EINVAL_SHAPE;
  if (!(p->k_scale >= 0.0f) || !(p->v_scale >= 0.0f) || !isfinite(p->k_scale) || !isfinite(p->v_scale)) return CODECOMP_EINVAL_PRIOR;
  const int64_t d = p->head_dim;
  const int64_t st = p->stride_tok ? p->stride_tok : d, sh = p->stride_head ? p->stride_head : p->page_size * d;
  const int64_t sp = p->stride_page ? p->stride_page : p->n_kv_heads * (p->page_size * d);
  const int64_t sl = p->stride_layer ? p->stride_layer : p->n_pages * (p->n_kv_heads * (p->page_size * d));
  if (st < d || st > INT32_MAX / (p->page_size * esz)) return CODECOMP_EINVAL_SHAPE;       // places inside a page are counted in 32 bits
  pool->k = static_cast<unsigned char*>(p->k); pool->v = static_cast<unsigned char*>(p->v);
  pool->n_pages = p->n_pages; pool->page_log2 = __builtin_ctz((unsigned)p->page_size); pool->fp8 = esz == 1;
  pool->s_layer = sl * esz; pool->s_page = sp * esz; pool->s_head = sh * esz; pool->s_tok = st * esz;
  pool->k_scale = p->k_scale > 0.0f ? p->k_scale : 1.0f;
  pool->v_scale = p->v_scale > 0.0f ? p->v_scale : 1.0f;
  return CODECOMP_OK;
}

int make_batch(const codecomp_batch* b, const codecomp_pages* p, PagedBatch* out) {
  if (!b || !b->cu_q_host || !b->cu_q_dev || !b->kv_lens_dev || !b->table_dev) return CODECOMP_EINVAL_NULL;
  if (b->n_seqs < 1 || b->n_seqs > 65535) return CODECOMP_EINVAL_SHAPE;
  if (b->n_q_heads < 1 || b->n_q_heads > kMostHeads || b->n_q_heads % p->n_kv_heads != 0) return CODECOMP_EINVAL_HEADS;
  if (b->causal != 0 && b->causal != 1) return CODECOMP_EINVAL_MODE;
  if (!(b->softmax_scale >= 0.0f) || !isfinite(b->softmax_scale)) return CODECOMP_EINVAL_PRIOR;
  if (b->table_width < 1 || b->max_kv_len < 0 || b->max_kv_len > (int64_t)b->table_width * p->page_size) return CODECOMP_EINVAL_PAGES;
  if (b->max_kv_len > (1 << 30)) return CODECOMP_EINVAL_PAGES;
  if (b->cu_q_host[0] != 0) return CODECOMP_EINVAL_SEQLENS;
  for (int r = 0; r < b->n_seqs; ++r)
    if (b->cu_q_host[r + 1] < b->cu_q_host[r]) return CODECOMP_EINVAL_SEQLENS;
  if (bad_strides({b->q_stride_tok, b->q_stride_head, b->new_stride_tok, b->new_stride_head, b->out_stride_tok, b->out_stride_head}, 8))
    return CODECOMP_EINVAL_SHAPE;
  const int64_t d = p->head_dim;
  out->cu_q = b->cu_q_dev; out->kv_lens = b->kv_lens_dev; out->table = b->table_dev;
  out->n_seqs = b->n_seqs; out->table_width = b->table_width; out->max_kv = b->max_kv_len; out->causal = b->causal;
  out->Hq = b->n_q_heads; out->Hkv = p->n_kv_heads; out->G = b->n_q_heads / p->n_kv_heads;
  out->T = b->cu_q_host[b->n_seqs];
  // rows and units of work are counted in 32 bits
  if ((int64_t)out->T * (out->Hq + 2 * (int64_t)out->Hkv) * (d / 16) > INT32_MAX) return CODECOMP_EINVAL_SHAPE;
  out->q_sh = b->q_stride_head ? b->q_stride_head : d;
  out->q_st = b->q_stride_tok ? b->q_stride_tok : out->Hq * d;
  out->n_sh = b->new_stride_head ? b->new_stride_head : d;
  out->n_st = b->new_stride_tok ? b->new_stride_tok : out->Hkv * d;
  out->o_sh = b->out_stride_head ? b->out_stride_head : d;
  out->o_st = b->out_stride_tok ? b->out_stride_tok : out->Hq * d;
  if (out->q_sh < d || out->n_sh < d || out->o_sh < d) return CODECOMP_EINVAL_SHAPE;
  return CODECOMP_OK;
}

// Turns per position of a frequency, modulo 1, in 2^-64 of a turn, rounded to the nearest: a position of 2^31 is off by 2^-34 of a turn.  After Payne and
// Hanek: freq = m 2^e with a whole m < 2^53; of the places of 1 / (2 pi) only those from e + 1 on make less than whole turns, and the first 128 of
// them are enough, modulo whole turns, for any double.  (A product in doubles is off by 2^-53 of the turns: 0.2 radians at position 2^31 for a
// frequency of 10^6.)
static uint64_t turns_of(double freq) {
  static constexpr uint64_t kPerRadian[18] = {          // 1 / (2 pi), 64 places a word from the point on
      0x28BE60DB9391054Au, 0x7F09D5F47D4D3770u, 0x36D8A5664F10E410u, 0x7F9458EAF7AEF158u, 0x6DC91B8E909374B8u, 0x01924BBA82746487u,
      0x3F877AC72C4A69CFu, 0xBA208D7D4BAED121u, 0x3A671C09AD17DF90u, 0x4E64758E60D4CE7Du, 0x272117E2EF7E4A0Eu, 0xC7FE25FFF7816603u,
      0xFBCBC462D6829B47u, 0xDB4D9FB3C9F2C26Du, 0xD3D18FD9A797FA8Bu, 0x5D49EEB1FAF97C5Eu, 0xCF41CE7DE294A4BAu, 0x9AFED7EC47E35742u};
  int e;
  const uint64_t m = (uint64_t)ldexp(frexp(fabs(freq), &e), 53);
  e -= 53;                                                  // at most 1024 - 53: 971 + 128 places are in the table
  unsigned __int128 places = 0;                             // e + 1 .. e + 128, those before the point zeros
  if (e > -128) {
    const int skip = e > 0 ? e : 0, word = skip >> 6, shift = skip & 63;
    places = (unsigned __int128)kPerRadian[word] << 64 | kPerRadian[word + 1];
    if (shift > 0) places = places << shift | kPerRadian[word + 2] >> (64 - shift);
    if (e < 0) places >>= -e;
  }
  return (uint64_t)((m * places + ((uint64_t)1 << 63)) >> 64);
}

int make_rotary(const codecomp_rotary* r, int head_dim, RotaryArgs* a) {
  if (r->dim < 0 || r->dim > head_dim || r->dim % 16 != 0) return CODECOMP_EINVAL_MODE;
  if (r->interleaved != 0 && r->interleaved != 1) return CODECOMP_EINVAL_MODE;
  if (r->inverse != 0 && r->inverse != 1) return CODECOMP_EINVAL_MODE;
  if (!isfinite(r->magnitude)) return CODECOMP_EINVAL_MODE;
  a->dim = r->dim; a->interleaved = r->interleaved;
  a->magnitude = r->magnitude == 0.0f ? 1.0f : r->magnitude;
  for (int i = 0; i < r->dim / 2; ++i) {
    if (!isfinite(r->freq[i])) return CODECOMP_EINVAL_MODE;
    // positions are whole numbers, so whole turns per position do not count, and the inverse is exactly the rotation at minus the position
    const uint64_t turns = turns_of(r->freq[i]);
    a->turns[i] = (r->freq[i] < 0.0) != (r->inverse != 0) ? 0 - turns : turns;
  }
  return CODECOMP_OK;
}

// Rows of `params` against a pool: the shapes that have to agree.
static int check_rows(const Plan& pl, const codecomp_params* params, const codecomp_pages* pages, PagePool* pool) {
  if (int rc = make_pool(pages, pool)) return rc;
  if (pages->n_layers != pl.L || pages->n_kv_heads != pl.Hkv) return CODECOMP_EINVAL_SHAPE;
  if (pages->head_dim != pl.d) return CODECOMP_EINVAL_HEADDIM;
  if (pages->kv_dtype != params->kv_dtype) return CODECOMP_EINVAL_MODE;
  return CODECOMP_OK;
}

static RowSide paged_side(const PagePool& pool, const int32_t* table, int table_width, const int32_t* first) {
  RowSide s = {};
  s.k = pool.k; s.v = pool.v; s.table = table; s.first = first; s.table_width = table_width;
  s.n_pages = pool.n_pages; s.page_log2 = pool.page_log2;
  s.s_layer = pool.s_layer; s.s_page = pool.s_page; s.s_head = pool.s_head; s.s_tok = pool.s_tok;
  return s;
}

// compact: the layout of k_out, v_out; else that of k, v.
static RowSide dense_side(const Plan& pl, bool compact, const void* k, const void* v) {
  RowSide s = {};
  const int esz = pl.kv_fp8 ? 1 : 2;
  s.k = static_cast<unsigned char*>(const_cast<void*>(k)); s.v = static_cast<unsigned char*>(const_cast<void*>(v));
  s.cu = compact ? pl.cu_budgets_dev : pl.cu_seqlens_dev;
  s.s_layer = (compact ? pl.o_sl : pl.kv_sl) * esz; s.s_head = (compact ? pl.o_sh : pl.kv_sh) * esz; s.s_tok = (compact ? pl.o_st : pl.kv_st) * esz;
  return s;
}

static MoveArgs move_args(const Plan& pl, const int32_t* idx, bool budgets) {
  MoveArgs a = {};
  a.idx = idx;
  a.cu_rows = budgets ? pl.cu_budgets_dev : pl.cu_seqlens_dev;
  a.cu_source = pl.cu_seqlens_dev;
  a.n_seqs = pl.n_seqs; a.Hkv = pl.Hkv; a.rows = budgets ? pl.TB : pl.T;
  a.pieces_log2 = (pl.d == 128 ? 4 : 3) - (pl.kv_fp8 ? 1 : 0);
  return a;
}

static int check_table(const int32_t* table, int32_t table_width) {
  if (!table) return CODECOMP_EINVAL_NULL;
  return table_width < 1 ? CODECOMP_EINVAL_PAGES : CODECOMP_OK;
}

}  // namespace codecomp

using namespace codecomp;

extern "C" {

int codecomp_rotary_init(codecomp_rotary* r, int32_t dim, int32_t interleaved, double base, int32_t scaling, double factor, double context,
                         double low, double high) {
  if (!r) return CODECOMP_EINVAL_NULL;
  if (dim < 16 || dim > 128 || dim % 16 != 0 || (interleaved != 0 && interleaved != 1)) return CODECOMP_EINVAL_MODE;
  if (!(base > 1.0) || !isfinite(base)) return CODECOMP_EINVAL_MODE;
  if (scaling < CODECOMP_ROTARY_PLAIN || scaling > CODECOMP_ROTARY_RAMP) return CODECOMP_EINVAL_MODE;
  if (scaling != CODECOMP_ROTARY_PLAIN && (!(factor >= 1.0) || !isfinite(factor))) return CODECOMP_EINVAL_MODE;
  const bool blend = scaling == CODECOMP_ROTARY_WAVELENGTH || scaling == CODECOMP_ROTARY_RAMP;
  if (blend && (!(context > 0.0) || !isfinite(context) || !(low > 0.0) || !(low < high) || !isfinite(high))) return CODECOMP_EINVAL_MODE;
  const double two_pi = 6.283185307179586477, n = dim;
  if (scaling == CODECOMP_ROTARY_BASE) base *= pow(factor, n / (n - 2.0));
  r->dim = dim; r->interleaved = interleaved; r->inverse = 0; r->magnitude = 1.0f;
  for (int i = 0; i < 64; ++i) r->freq[i] = 0.0;
  double from = 0.0, to = 0.0;
  if (scaling == CODECOMP_ROTARY_RAMP) {
    from = fmax(floor(n * log(context / (two_pi * high)) / (2.0 * log(base))), 0.0);
    to = fmin(ceil(n * log(context / (two_pi * low)) / (2.0 * log(base))), n - 1.0);
  }
  for (int i = 0; i < dim / 2; ++i) {
    double f = pow(base, -2.0 * i / n), keep = 1.0;             // share of the unscaled frequency
    if (scaling == CODECOMP_ROTARY_LINEAR) keep = 0.0;
    if (scaling == CODECOMP_ROTARY_WAVELENGTH) keep = (context * f / two_pi - low) / (high - low);
    if (scaling == CODECOMP_ROTARY_RAMP) keep = 1.0 - (i - from) / fmax(to - from, 0.001);
    keep = fmin(fmax(keep, 0.0), 1.0);
    r->freq[i] = keep < 1.0 ? (1.0 - keep) * (f / factor) + keep * f : f;
  }
  return CODECOMP_OK;
}

int codecomp_rotate(const void* x, const int32_t* positions, const codecomp_rotary* rotary, int32_t n_tokens, int32_t n_heads, int32_t head_dim,
                    int64_t x_stride_tok, int64_t x_stride_head, void* out, int64_t out_stride_tok, int64_t out_stride_head, void* hip_stream) {
  if (!rotary || (n_tokens > 0 && (!x || !positions || !out))) return CODECOMP_EINVAL_NULL;
  if (head_dim != 64 && head_dim != 128) return CODECOMP_EINVAL_HEADDIM;
  if (n_heads < 1 || n_heads > kMostHeads) return CODECOMP_EINVAL_HEADS;
  if (n_tokens < 0 || (int64_t)n_tokens * n_heads * (head_dim / 16) > INT32_MAX) return CODECOMP_EINVAL_SHAPE;
  if (bad_strides({x_stride_tok, x_stride_head, out_stride_tok, out_stride_head}, 8) || misaligned16(x) || misaligned16(out)) return CODECOMP_EINVAL_SHAPE;
  const int64_t x_sh = x_stride_head ? x_stride_head : head_dim, o_sh = out_stride_head ? out_stride_head : head_dim;
  if (x_sh < head_dim || o_sh < head_dim) return CODECOMP_EINVAL_SHAPE;
  RotaryArgs rot;
  if (int rc = make_rotary(rotary, head_dim, &rot)) return rc;
  if (n_tokens == 0) return CODECOMP_OK;
  return launch_rotate(rot, x, positions, n_tokens, n_heads, head_dim, x_stride_tok ? x_stride_tok : (int64_t)n_heads * head_dim, x_sh, out,
                       out_stride_tok ? out_stride_tok : (int64_t)n_heads * head_dim, o_sh, (hipStream_t)hip_stream);
}

int codecomp_append(const void* q, const void* k, const void* v, const int32_t* positions, const codecomp_rotary* rotary, const codecomp_batch* batch,
                    const codecomp_pages* pages, int32_t layer, void* q_out, void* hip_stream) {
  PagePool pool;
  PagedBatch b;
  if (int rc = make_pool(pages, &pool)) return rc;
  if (int rc = make_batch(batch, pages, &b)) return rc;
  if (b.T > 0 && (!k || !v || (!q) != (!q_out) || (rotary && !positions))) return CODECOMP_EINVAL_NULL;
  if (layer < 0 || layer >= pages->n_layers) return CODECOMP_EINVAL_PAGES;
  if (misaligned16(q) || misaligned16(k) || misaligned16(v) || misaligned16(q_out)) return CODECOMP_EINVAL_SHAPE;
  RotaryArgs rot = {};
  rot.magnitude = 1.0f;
  if (rotary)
    if (int rc = make_rotary(rotary, pages->head_dim, &rot)) return rc;
  if (b.T == 0) return CODECOMP_OK;
  return launch_append(rot, b, pool, layer, pages->head_dim, q, k, v, positions, q_out, (hipStream_t)hip_stream);
}

int codecomp_pages_store(const void* k, const void* v, const int32_t* idx, const codecomp_params* params, const codecomp_pages* pages,
                         const int32_t* table, int32_t table_width, const int32_t* first, void* hip_stream) {
  if (!k || !v) return CODECOMP_EINVAL_NULL;
  Plan pl;
  PagePool pool;
  if (int rc = make_plan(params, &pl)) return rc;
  if (int rc = check_rows(pl, params, pages, &pool)) return rc;
  if (int rc = check_table(table, table_width)) return rc;
  if (misaligned16(k) || misaligned16(v)) return CODECOMP_EINVAL_SHAPE;
  MoveArgs a = move_args(pl, idx, true);
  a.from = dense_side(pl, idx == nullptr, k, v);
  a.to = paged_side(pool, table, table_width, first);
  return launch_move(a, pl.L * pl.Hkv, (hipStream_t)hip_stream);
}

int codecomp_pages_load(const codecomp_pages* pages, const int32_t* table, int32_t table_width, const int32_t* first, const int32_t* idx,
                        const codecomp_params* params, void* k, void* v, void* hip_stream) {
  if (!k || !v) return CODECOMP_EINVAL_NULL;
  Plan pl;
  PagePool pool;
  if (int rc = make_plan(params, &pl)) return rc;
  if (int rc = check_rows(pl, params, pages, &pool)) return rc;
  if (int rc = check_table(table, table_width)) return rc;
  if (misaligned16(k) || misaligned16(v)) return CODECOMP_EINVAL_SHAPE;
  MoveArgs a = move_args(pl, idx, idx != nullptr);
  a.from = paged_side(pool, table, table_width, first);
  a.to = dense_side(pl, idx != nullptr, k, v);
  return launch_move(a, pl.L * pl.Hkv, (hipStream_t)hip_stream);
}

int codecomp_pages_compact(const codecomp_pages* pages, const int32_t* table, int32_t table_width, const int32_t* first, const int32_t* idx,
                           const codecomp_params* params, const codecomp_pages* to, const int32_t* to_table, int32_t to_table_width,
                           const int32_t* to_first, void* hip_stream) {
  if (!idx) return CODECOMP_EINVAL_NULL;
  Plan pl;
  PagePool pool, to_pool;
  if (int rc = make_plan(params, &pl)) return rc;
  if (int rc = check_rows(pl, params, pages, &pool)) return rc;
  if (int rc = check_rows(pl, params, to, &to_pool)) return rc;
  if (int rc = check_table(table, table_width)) return rc;
  if (int rc = check_table(to_table, to_table_width)) return rc;
  // rows are moved as they are stored: the values only stay the same where the scales are
  if (pool.k_scale != to_pool.k_scale || pool.v_scale != to_pool.v_scale) return CODECOMP_EINVAL_MODE;
  MoveArgs a = move_args(pl, idx, true);
  a.from = paged_side(pool, table, table_width, first);
  a.to = paged_side(to_pool, to_table, to_table_width, to_first);
  return launch_move(a, pl.L * pl.Hkv, (hipStream_t)hip_stream);
}

int codecomp_pages_copy(const codecomp_pages* pages, const int32_t* pairs, int32_t n_pairs, void* hip_stream) {
  PagePool pool;
  if (int rc = make_pool(pages, &pool)) return rc;
  if (n_pairs < 0) return CODECOMP_EINVAL_SHAPE;
  if (n_pairs == 0) return CODECOMP_OK;
  if (!pairs) return CODECOMP_EINVAL_NULL;
  return launch_pages_copy(pool, pages->n_layers, pages->n_kv_heads, pages->head_dim, pairs, n_pairs, (hipStream_t)hip_stream);
}

int codecomp_attend_validate(const codecomp_batch* batch, const codecomp_pages* pages) {
  AttendPlan pl;
  return make_attend_plan(batch, pages, &pl);
}

size_t codecomp_attend_workspace_bytes(const codecomp_batch* batch, const codecomp_pages* pages) {
  AttendPlan pl;
  return make_attend_plan(batch, pages, &pl) ? 0 : pl.ws_bytes;
}

int codecomp_attend(const void* q, const codecomp_batch* batch, const codecomp_pages* pages, int32_t layer, void* out, float* lse, void* workspace,
                    size_t workspace_bytes, void* hip_stream) {
  AttendPlan pl;
  if (int rc = make_attend_plan(batch, pages, &pl)) return rc;
  if (pl.batch.T > 0 && (!q || !out)) return CODECOMP_EINVAL_NULL;
  if (layer < 0 || layer >= pages->n_layers) return CODECOMP_EINVAL_PAGES;
  if (misaligned16(q) || misaligned16(out) || ((uintptr_t)lse & 3) != 0) return CODECOMP_EINVAL_SHAPE;
  if (pl.ws_bytes > 0 && (!workspace || ((uintptr_t)workspace & 255) != 0 || workspace_bytes < pl.ws_bytes)) return CODECOMP_EINVAL_WORKSPACE;
  if (pl.batch.T == 0) return CODECOMP_OK;
  return launch_attend(pl, q, layer, out, lse, workspace, (hipStream_t)hip_stream);
}

}  // extern "C"
