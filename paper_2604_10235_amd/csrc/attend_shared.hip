// codecomp_attend_shared: attention of requests whose caches begin with the same rows.
//
// The shared rows are attended to once for a group, by the rows (new tokens x query heads of a KV head) of all of its requests together: they lie side by
// side in the packed batch, and all of them see all of the shared rows.  What a request has behind them is its own.  Both leave parts of every row (reference, sum
// of weights, unscaled output, fp32), which are joined in order: o = sum of 2^(m_p - m) o_p, l the same, m the largest m_p; output o / l, log-sum-exp m + log2 l.
//
// Groups of many rows: the kernel of attend_many.h, whose blocks of 256 rows share keys and values through LDS.  Groups of few: that of
// attend_few.hip, which reads keys and values once for up to 32 rows.  Rows behind the shared ones: the kernel for few rows, in which whoever has the rows joins the
// parts of the shared ones to them, or, for prompts, the kernel for many, in the same launch as the shared rows.  Where all is short nothing is shared: the kernel for few rows
// takes a request's shared and own rows together.
//
// Single tokens wait for memory, and shared rows are read once for all: 64 steps of 28 query heads on 4 KV heads of 128 over 32768 shared rows and up to 700 of their own, 73 us
// where codecomp_attend over the same caches takes 470 (the shared rows 54, by 448 rows in blocks of 256, whose weights are two bf16: half as many products again; their own 20, of which
// a compute unit reads 32 bytes a ns).  96 steps in eight groups of twelve behind 2001 to 9001 rows, 8 KV heads, 8 bits: 99 us instead of 219.
// Prompts wait for the matrix units, which sharing takes no work off: 24 of up to 401 tokens in two groups behind 16000 rows, head_dim 64, 215 to 223 us, codecomp_attend 220.
// Four steps behind 2049 rows: 12 us, two launches of dependent waits, as in codecomp_attend.
// Tried before, kernel for few rows: eight waves a workgroup (four steps 9.5 us instead of 8.7), three blocks of 16 rows (shared rows of 48 rows 52 us instead of 57, but their
// own ones 69 instead of 62); kernel for many: a loop over units (206 -> 214 us).
#include <float.h>
#include <math.h>

#include <algorithm>

#include "attend_many.h"
#include "serve.h"

namespace codecomp {

extern template int launch_many_shared_of<64, false>(const ManyArgs&, hipStream_t);
extern template int launch_many_shared_of<64, true>(const ManyArgs&, hipStream_t);
extern template int launch_many_shared_of<128, false>(const ManyArgs&, hipStream_t);
extern template int launch_many_shared_of<128, true>(const ManyArgs&, hipStream_t);

constexpr int kChip = 256;                       // compute units: workgroups of the kernel for many rows that run at once
constexpr int64_t kMostBlocks = (1 << 23) - 1;    // of up to 512 threads: an axis of a grid holds 2^32 threads
constexpr int64_t kMostSplits = 1024, kMostParts = 1 << 21;       // chunks of a request's keys; of all rows together, where there are more than eight chunks: workspace
// Up to so many keys in all nothing is cut, shared rows are read once for every 16 or 32 rows, and there is nothing to join: one launch (us, with parts | without: 64 steps behind 16
// rows 12.0 | 7.3, 1024 in groups of 8 behind 300, 8 bits, 128 | 116, 226 tokens behind 47 23 | 12, 1000 requests of up to 20 tokens behind 400, head_dim 64, 195 | 129; beyond: 8
// steps behind 700 12.8 | 14.6, 256 behind 500 and up to 300 of their own 41 | 51, two prompts of 600 tokens behind 600 50 | 79).  Not where that is much work, and at least twice as
// much as the kernel for many rows would have (1024 steps in groups of 128 behind 300 82 | 96).
constexpr int kAloneKeys = 512;
constexpr int64_t kAloneStrips = 8192;
// Empty workgroups that are let pass, beside four for each that is not (a prompt of 400 tokens among steps over 50 rows, 30 of them shared, us, with the kernel for many rows | mostly
// empty: 50 steps 33 | 40, 200 46 | 121, 700 127 | 390).
constexpr int64_t kEmptyBlocks = 4096;
// Little work, in strips of 128 keys by 32 rows: all of it in one launch of the kernel for few rows, and one that joins (us, one | the kernel for many as well: 64 steps of 7 query
// heads on 4 KV heads behind 2048 rows, 896 strips, 29 | 33, 4096 34.6 | 37.1, 8192 46 | 41; 16 steps behind 16000, 2000 strips, 34.3 | 35.5, 32000 46 | 42; 64 steps behind 4096, 8 KV
// heads, 8 bits, 2048 strips, 31 | 38; behind 16000, head_dim 64, 2000 strips, 23 | 29).  Less where a request has more than 64 rows, whose weights the kernel for many rounds.
constexpr int64_t kFewStrips = 2048, kFewStripsRounded = 1024;
// Groups of 33 to 64 rows: the kernel for few rows reads the shared rows twice, the one for many has most of a block empty, but a tile's keys for all of it at once (us,
// few | many: one group of 56 rows behind 2000 rows 13 | 23, 8192 21 | 28, 32768 33 | 39; eight behind 2000 to 9000 51 | 45, of 64 rows at head_dim 64 31 | 36; 8 bits, 48 rows, 99 |
// 118: never there).  By keys of all such groups and heads.
constexpr int kFewRows = 32;
constexpr int64_t kFewKeys8 = INT64_MAX, kFewKeys16 = 1 << 17;
// Most keys of a chunk in the kernel for few rows, shared and own (us, eight groups of 48 rows behind 9001: 512 77, 1024 65, 2048 57, 4096 57; 96 requests' own 2000: 512 96, 1024 85,
// 2048 88; of 20 to 2000: 66, 61, 62).
constexpr int kFewChunk = 2048, kOwnChunk = 1024;
// Requests of more rows: what they have behind the shared ones is the kernel for many rows' too, once that runs (us, few | many: 8 tokens of 7 query heads over 100 to 1000 rows
// behind 2000, 32 requests, 59 | 47, 14: 71 | 42, 18: 73 | 43; 16 prompts of up to 512 over up to 2500: 856 | 281; 4 tokens 51 | 45, but at head_dim 64, 6 tokens of 4 over up to 2000,
// 38 | 56).
constexpr int kOwnRows = 32;
// Otherwise one workgroup has a request's own rows, and joins, where they are short or where there are enough of these, else chunks do and a kernel that joins (us, chunks |
// one: 16 requests of 4 heads, up to 300 rows, 25 | 26, up to 2000 39 | 58; 64 of up to 4000 94 | 100, of 8000 227 | 215, of up to 16000 230 | 276; 128 of up to 1000 88 | 85;
// 200 of up to 9000 432 | 446).
constexpr int kJoinKeys = 512, kJoinMost = 8192;
constexpr int64_t kJoinItems = 192;
// The kernel that joins: several groups of threads a row, for many parts and few rows (us, one | eight: four steps of 18 parts 14.3 | 12.3, one behind 32768 rows 39 | 23, eight 41 |
// 33, 64 of 10 parts 23 | 23, 96 of 7 parts 99 | 101; 32 requests of 16 tokens, 14336 rows of 4 parts, 51 | 58).
constexpr int kJoinParts = 8;
constexpr int64_t kJoinRows = 16384;
// Chunks of shared rows for the kernel for many: the time of a tile is the unit.  A chunk starts and ends in 5 of them (8.6 us of 1.6 each at head_dim 128), and what it leaves
// goes through memory twice: 600000 elements in a tile's time.
constexpr double kLead = 5.0, kPartElements = 600000.0;
// Of the own rows of prompts: a third of what a compute unit has to do in all, and 2048 keys at least (with the tile that the shared ones end in; us, whole | in chunks: 512 tokens over
// 60000 own rows 1097 | 455, 8 requests of up to 300 over 300 to 30000 592 | 562; with halves of the work 427, 725, before they went to the dies in turn; 100 tokens over 4000
// with chunks of 24 | 33 | 40 tiles 46 | 57 | 64, but 48 requests of 14 over up to 2000, 8 bits, head_dim 64, with 24 | 40 62 | 51).
constexpr double kOwnTiles = 33.0;

int make_shared_plan(const codecomp_batch* b, const codecomp_groups* g, const codecomp_pages* p, SharedPlan* pl) {
  if (int rc = make_pool(p, &pl->pool)) return rc;
  if (int rc = make_batch(b, p, &pl->batch)) return rc;
  const PagedBatch& x = pl->batch;
  if (!g || !g->cu_groups_host || !g->cu_groups_dev || !g->prefix_lens_dev) return CODECOMP_EINVAL_NULL;
  if (g->n_groups < 1 || g->n_groups > 65535) return CODECOMP_EINVAL_SHAPE;
  if (g->max_prefix_len < 0 || g->max_prefix_len > b->max_kv_len || g->max_own_len < 0 || g->max_own_len > b->max_kv_len) return CODECOMP_EINVAL_PAGES;
  if (g->cu_groups_host[0] != 0 || g->cu_groups_host[g->n_groups] != b->n_seqs) return CODECOMP_EINVAL_SEQLENS;
  for (int i = 0; i < g->n_groups; ++i)
    if (g->cu_groups_host[i + 1] < g->cu_groups_host[i]) return CODECOMP_EINVAL_SEQLENS;
  pl->d = p->head_dim;
  pl->scale = b->softmax_scale > 0.0f ? b->softmax_scale : 1.0f / sqrtf((float)p->head_dim);
  SharedRows& s = pl->sh;
  s = SharedRows{};
  s.cu_groups = g->cu_groups_dev; s.prefix_lens = g->prefix_lens_dev;
  s.n_groups = g->n_groups; s.max_prefix = g->max_prefix_len; s.max_own = g->max_own_len;
  int64_t few_most = 0, blocks = 0, own_most = 0;
  const int64_t items = (int64_t)x.n_seqs * x.Hkv;
  int64_t own_parts = 0, group_parts = 0, group_most = 0;      // parts of 32 rows of all requests, of all groups; rows of the largest one
  for (int r = 0; r < x.n_seqs; ++r) {
    const int64_t rows = (int64_t)(b->cu_q_host[r + 1] - b->cu_q_host[r]) * x.G;
    own_most = std::max(own_most, rows);
    own_parts += (rows + 31) / 32;
  }
  int64_t middle = 0;                              // groups of more than 32 rows that either kernel can take
  for (int i = 0; i < g->n_groups; ++i) {
    const int64_t rows = (int64_t)(b->cu_q_host[g->cu_groups_host[i + 1]] - b->cu_q_host[g->cu_groups_host[i]]) * x.G;
    middle += rows > kFewRows && rows <= kFewRowsMost;
    group_most = std::max(group_most, rows);
    group_parts += (rows + 31) / 32;
  }
  // The kernel for few rows has workgroups for as many parts of every request, or group, as the largest one has: not where most of them would find nothing.
  auto alike = [&](int64_t count, int64_t most, int64_t parts) { return count * ((most + 31) / 32) * x.Hkv <= 4 * parts * x.Hkv + kEmptyBlocks; };
  // Work in strips of 128 keys by 32 rows, with the shared rows read for every request, and once for a group.
  auto strips_of = [&](int64_t keys) { return (keys + 127) / 128; };
  const int64_t apart = own_parts * strips_of(s.max_prefix + (int64_t)s.max_own) * x.Hkv;
  const int64_t together = (group_parts * strips_of(s.max_prefix) + own_parts * strips_of(s.max_own)) * x.Hkv;
  const bool pays = group_most > kFewRowsMost && apart > kAloneStrips && apart > 2 * together;
  if (s.max_prefix + (int64_t)s.max_own <= kAloneKeys && !pays && alike(x.n_seqs, own_most, own_parts)) {
    pl->own_two = own_most > 16;
    pl->row_parts = std::max<int>(1, (int)((own_most + (pl->own_two ? 31 : 15)) / (pl->own_two ? 32 : 16)));
    pl->own_units = items * pl->row_parts;
    if (pl->own_units > kMostBlocks) return CODECOMP_EINVAL_SHAPE;
    pl->few_groups = pl->many_groups = pl->few_two = pl->chunk = pl->own_splits = 0;
    pl->prompts = false;
    s.alone = 1;
    pl->ws_bytes = 0;
    return CODECOMP_OK;
  }
  pl->few_groups = pl->many_groups = 0;
  s.many_tokens = s.few_tokens = 0;
  int64_t strips = group_parts * strips_of(s.max_prefix);        // of the shared rows, and of the own ones of requests that the kernel for many rows would take
  for (int r = 0; r < x.n_seqs; ++r) {
    const int64_t rows = (int64_t)(b->cu_q_host[r + 1] - b->cu_q_host[r]) * x.G;
    if (rows > kOwnRows) strips += (rows + 31) / 32 * strips_of(s.max_own);
  }
  if (strips * x.Hkv <= (own_most > kFewRowsMost ? kFewStripsRounded : kFewStrips) && alike(x.n_seqs, own_most, own_parts) && alike(s.n_groups, group_most, group_parts)) s.few_rows = INT32_MAX;
  else s.few_rows = middle * x.Hkv * s.max_prefix > (pl->pool.fp8 ? kFewKeys8 : kFewKeys16) ? kFewRows : kFewRowsMost;
  bool fine = false, rounded = false;              // in groups of many rows: requests of up to 64 rows, of more
  for (int i = 0; i < g->n_groups; ++i) {
    const int64_t rows = (int64_t)(b->cu_q_host[g->cu_groups_host[i + 1]] - b->cu_q_host[g->cu_groups_host[i]]) * x.G;
    if (rows > s.few_rows) {
      ++pl->many_groups;
      s.many_tokens += (int)(rows / x.G);
      blocks += (rows + kManyRows - 1) / kManyRows;
      for (int r = g->cu_groups_host[i]; r < g->cu_groups_host[i + 1]; ++r) {
        const int64_t own = (int64_t)(b->cu_q_host[r + 1] - b->cu_q_host[r]) * x.G;
        if (own > kFewRowsMost) rounded = true;
        else if (own > 0) fine = true;
      }
    } else if (rows > 0) {
      ++pl->few_groups;
      s.few_tokens += (int)(rows / x.G);
      few_most = std::max(few_most, rows);
    }
  }
  s.fine = !fine ? 0 : rounded ? 2 : 1;
  int64_t own_blocks = 0;                          // of rows, if the kernel for many rows has the own ones too
  for (int r = 0; r < x.n_seqs; ++r) {
    const int64_t rows = (int64_t)(b->cu_q_host[r + 1] - b->cu_q_host[r]) * x.G;
    own_blocks += (rows + kManyRows - 1) / kManyRows;
  }
  pl->prompts = pl->many_groups > 0 && own_most > kOwnRows;
  if (!pl->prompts || s.max_own == 0) own_blocks = 0;
  own_blocks *= x.Hkv;
  blocks *= x.Hkv;
  auto most_of = [&](int64_t tokens) { return std::min(kMostSplits, std::max<int64_t>(8, kMostParts / std::max<int64_t>(1, tokens * x.Hq))); };
  const int64_t most_splits = most_of(x.T);
  double own = 0.0;                                // tiles' worth of time of a chunk of them
  if (own_blocks > 0) {
    // long ones in chunks of a third of what there is to do for a compute unit, at most
    const int tiles = std::max(1, (s.max_prefix + kManyKeys - 1) / kManyKeys), own_tiles = (s.max_own + kManyKeys - 1) / kManyKeys + 1;
    const double work = (blocks * (tiles + kLead) + own_blocks * (0.75 * own_tiles + kLead)) / kChip;
    const int64_t chunk = std::max<int64_t>((int64_t)std::max(work / 3, kOwnTiles), (own_tiles + most_splits - 1) / most_splits);
    s.own_tiles = (int)std::min<int64_t>(chunk, own_tiles);
    s.own_splits = (own_tiles + s.own_tiles - 1) / s.own_tiles;
    own_blocks *= s.own_splits;
    own = 0.75 * s.own_tiles + kLead;
  }
  const int64_t most_units = kMostBlocks - (pl->few_groups > 0 ? kPlacers : 0);
  if (blocks + own_blocks > most_units) return CODECOMP_EINVAL_SHAPE;
  s.own_units = (int)own_blocks;
  s.join = pl->many_groups > 0 && !pl->prompts && (s.max_own <= kJoinKeys || (s.max_own <= kJoinMost && items * ((own_most + 31) / 32) >= kJoinItems));
  pl->few_two = s.join || pl->prompts ? few_most > 16 : std::max(few_most, own_most) > 16;
  pl->own_two = s.join ? own_most > 16 : pl->few_two;
  const int few_each = pl->few_two ? 32 : 16, own_each = pl->own_two ? 32 : 16;

  // Shared rows, many: chunks for which the last workgroup ends early (rounds of as many as there are compute units, then the requests' own blocks, which fill what the last
  // round leaves free) and not much is done in all (the chip's clock goes by it).  1, 2, 3, 4, 5 and 8 chunks, us: the 24 questions 307, 273, 223, 228, 228, 245; four prompts of
  // 200 to 500 tokens behind 8000 rows 217, 234, 253, 256, 268, 304; 32 of 16 tokens behind 4000 92, 58, 53, 65, 65, 79; 24, 32 and 43: 64 steps behind 32768 rows 77, 74, 97.  Own rows count as three quarters of their bound.
  s.many_splits = s.few_splits = 0;
  if (pl->many_groups > 0) {
    const int tiles = std::max(1, (s.max_prefix + kManyKeys - 1) / kManyKeys);
    const double part = (double)s.many_tokens * x.Hq * p->head_dim / kPartElements;
    int best = 1;
    double least = 0.0;
    for (int n = 1; n <= std::min(tiles, kChip) && blocks * n + own_blocks <= most_units; ++n) {
      const double each = (tiles + n - 1) / n + kLead;
      const int64_t rounds = ((blocks * n + 7) / 8 + kChip / 8 - 1) / (kChip / 8);       // of a die's compute units
      const int64_t left = own_blocks > 0 ? own_blocks - (rounds * kChip - blocks * n) * (int64_t)(each / own) : 0;
      const double end = rounds * each + (left > 0 ? (left + kChip - 1) / kChip * own : 0.0), work = (blocks * n * each + own_blocks * own) / kChip;
      const double time = end + work + n * (0.04 + part);
      if (n == 1 || time < least) { best = n; least = time; }
    }
    s.many_tiles = (tiles + best - 1) / best;
    s.many_splits = (tiles + s.many_tiles - 1) / s.many_tiles;
    s.many_units = (int)(blocks * s.many_splits);
  }
  // Chunks of keys for `items` that have some, of `all` that there is a workgroup for.
  auto cut = [&](int64_t items, int64_t all, int most, int64_t largest, int64_t most_splits, int* chunk, int* splits) {
    int64_t keys = (items * most / 512 + 127) / 128 * 128;
    keys = std::min<int64_t>(std::max<int64_t>(keys, 128), largest);
    while ((most + keys - 1) / keys > most_splits || (all * ((most + keys - 1) / keys) > kMostBlocks / 2 && keys < most)) keys *= 2;
    *chunk = (int)std::min<int64_t>(keys, 1 << 30);
    *splits = (int)((most + keys - 1) / keys);
  };
  // shared rows, few
  s.few_parts = std::max<int>(1, (int)((few_most + few_each - 1) / few_each));
  int64_t few_units = 0;
  if (pl->few_groups > 0) {
    const int64_t units = (int64_t)s.n_groups * x.Hkv * s.few_parts;
    cut((int64_t)pl->few_groups * x.Hkv * s.few_parts, units, s.max_prefix, kFewChunk, most_of(s.few_tokens), &s.few_chunk, &s.few_splits);
    s.few_splits = std::max(s.few_splits, 1);
    few_units = units * s.few_splits;
    if (few_units > kMostBlocks) return CODECOMP_EINVAL_SHAPE;
  }
  s.few_units = (int)few_units;
  // rows behind them
  pl->row_parts = std::max<int>(1, (int)std::min<int64_t>((own_most + own_each - 1) / own_each, INT32_MAX));
  pl->own_units = pl->chunk = pl->own_splits = 0;
  if (!pl->prompts) {
    if (items * pl->row_parts > kMostBlocks) return CODECOMP_EINVAL_SHAPE;
    if (s.join) {
      pl->chunk = s.max_own;
      pl->own_splits = 1;
    } else {
      cut(items * pl->row_parts, items * pl->row_parts, s.max_own, kOwnChunk, most_splits, &pl->chunk, &pl->own_splits);
    }
    pl->own_units = items * pl->row_parts * pl->own_splits;
  }
  if (pl->own_units + few_units > kMostBlocks) return CODECOMP_EINVAL_SHAPE;
  // parts, and where there are groups of both kinds, places of tokens
  pl->own_parts = s.own_units > 0 ? s.own_splits : s.join ? 0 : pl->own_splits;
  s.own_base = (int64_t)s.many_splits * s.many_tokens + (int64_t)s.few_splits * s.few_tokens;
  pl->parts = (s.own_base + (int64_t)pl->own_parts * x.T) * x.Hq;
  pl->both = s.many_tokens > 0 && s.few_tokens > 0;
  pl->ws_bytes = x.T == 0 ? 0 : ((size_t)pl->parts * (p->head_dim + 2) * sizeof(float) + (pl->both ? x.T * sizeof(int32_t) : 0) + 255) & ~(size_t)255;
  return CODECOMP_OK;
}

// A row's parts, those of the shared rows first: GROUPS times D / 4 threads a row, the parts shared out over the groups and these added up in order.
// BOTH: there are groups of few rows and of many; else all rows have as many parts, one behind the other.
template <int D, int GROUPS, bool BOTH>
__global__ __launch_bounds__(256) void join_shared_kernel(const SharedArgs a, int own_parts) {
  constexpr int THREADS = D / 4, ROWS = 256 / THREADS / GROUPS;
  __shared__ f32x4 sums[GROUPS][ROWS][THREADS];
  __shared__ float tops[GROUPS][ROWS], alls[GROUPS][ROWS];
  const int in = threadIdx.x / THREADS, group = in % GROUPS, slot = in / GROUPS, th = threadIdx.x % THREADS, e = th * 4;
  const int64_t rows = (int64_t)a.b.T * a.b.Hq, row = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * ROWS + slot;
  const bool there = row < rows;
  GroupParts shared = {0, 0, max(a.sh.many_splits, a.sh.few_splits)};
  if (BOTH && there) shared = parts_of_group(a.sh, (int)(row / a.b.Hq));
  const int parts = shared.count + own_parts;
  auto place = [&](int p) __attribute__((always_inline)) {
    if constexpr (BOTH) return (p < shared.count ? shared.first + p * shared.step : a.sh.own_base + (int64_t)(p - shared.count) * a.b.T) * a.b.Hq + row;
    return p * rows + row;
  };
  // Parts come from memory (other dies wrote them): a lot is sent for before one of it is looked at, and the reference moves on from lot to lot.
  constexpr int LOT = 4;
  float top = -INFINITY, all = 0.0f;
  f32x4 x = {0, 0, 0, 0};
  if (there) {
    for (int p0 = group; p0 < parts; p0 += LOT * GROUPS) {
      float2 ml[LOT];
      f32x4 v[LOT];
      float to = top;
#pragma unroll
      for (int i = 0; i < LOT; ++i) {
        const int64_t part = place(min(p0 + i * GROUPS, parts - 1));
        ml[i] = *reinterpret_cast<const float2*>(a.part_ml + 2 * part);
        v[i] = *reinterpret_cast<const f32x4*>(a.part_o + part * D + e);
      }
#pragma unroll
      for (int i = 0; i < LOT; ++i) {
        if (p0 + i * GROUPS >= parts) ml[i] = float2{-INFINITY, kNoPart};
        to = fmaxf(to, ml[i].x);
      }
      const float old = to == top ? 1.0f : __builtin_amdgcn_exp2f(top - to);
      top = to;
      x *= old;
      all *= old;
#pragma unroll
      for (int i = 0; i < LOT; ++i) {
        const float f = ml[i].x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ml[i].x - to);       // times zeros, or an infinity or NaN that it saw
        const bool some = ml[i].y != kNoPart;
        all += some ? f * ml[i].y : 0.0f;
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] += some ? f * v[i][k] : 0.0f;
      }
    }
  }
  if constexpr (GROUPS > 1) {
    if (th == 0) tops[group][slot] = top;
    __syncthreads();
    float to = top;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) to = fmaxf(to, tops[g][slot]);
    const float f = to == top ? 1.0f : __builtin_amdgcn_exp2f(top - to);
    top = to;
    sums[group][slot][th] = x * f;
    if (th == 0) alls[group][slot] = all * f;
    __syncthreads();
    if (group > 0) return;
    x = sums[0][slot][th]; all = alls[0][slot];
#pragma unroll
    for (int g = 1; g < GROUPS; ++g) { x += sums[g][slot][th]; all += alls[g][slot]; }
  }
  if (!there) return;
  const int64_t t = row / a.b.Hq, h = row - t * a.b.Hq;
  const float inv = all == 0.0f ? 0.0f : a.pool.v_scale / all;
  *reinterpret_cast<u32x2*>(a.out + t * a.b.o_st + h * a.b.o_sh + e) = u32x2{pack2(x.x * inv, x.y * inv), pack2(x.z * inv, x.w * inv)};
  if (a.lse && e == 0) a.lse[row] = all == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(all)) * kLn2;
}

template <int D, int GROUPS>
static int launch_join(const SharedArgs& a, int own_parts, hipStream_t stream) {
  constexpr int ROWS = 256 / (D / 4) / GROUPS;
  const int64_t blocks = ((int64_t)a.b.T * a.b.Hq + ROWS - 1) / ROWS, width = std::min<int64_t>(blocks, 1 << 20);       // an axis of a grid holds 2^32 threads
  const dim3 grid((unsigned)width, (unsigned)((blocks + width - 1) / width));
  if (a.sh.place) join_shared_kernel<D, GROUPS, true><<<grid, dim3(256), 0, stream>>>(a, own_parts);
  else join_shared_kernel<D, GROUPS, false><<<grid, dim3(256), 0, stream>>>(a, own_parts);
  return (int)hipGetLastError();
}

int launch_shared(const SharedPlan& pl, const void* q, int layer, void* out, float* lse, void* workspace, hipStream_t stream) {
  SharedArgs a = {};
  a.pool = pl.pool; a.b = pl.batch; a.q = static_cast<const uint16_t*>(q); a.out = static_cast<uint16_t*>(out); a.lse = lse;
  a.layer = layer * pl.pool.s_layer;
  a.c = fminf(fmaxf(pl.scale * pl.pool.k_scale * kLog2e, FLT_MIN), FLT_MAX);       // a hidden logit of minus infinity times it stays one
  a.chunk = pl.chunk; a.row_parts = pl.row_parts;
  a.sh = pl.sh;
  if (pl.sh.alone) return launch_few_shared(pl.d, pl.pool.fp8, pl.own_two, pl.own_units, a, stream);
  const int64_t rows = (int64_t)pl.batch.T * pl.batch.Hq;
  a.part_o = static_cast<float*>(workspace);
  a.part_ml = a.part_o + pl.parts * pl.d;
  if (pl.both) a.sh.place = reinterpret_cast<int32_t*>(a.part_ml + 2 * pl.parts);
  if (pl.many_groups > 0) {
    ManyArgs m = {};
    m.a = a;
    m.sh = a.sh;
    m.rows_from = a.sh.few_rows + 1;
    int rc;
    if (pl.d == 128) rc = pl.pool.fp8 ? launch_many_shared_of<128, true>(m, stream) : launch_many_shared_of<128, false>(m, stream);
    else rc = pl.pool.fp8 ? launch_many_shared_of<64, true>(m, stream) : launch_many_shared_of<64, false>(m, stream);
    if (rc) return rc;
  }
  if (pl.sh.join) {
    if (pl.sh.few_units > 0)
      if (int rc = launch_few_shared(pl.d, pl.pool.fp8, pl.few_two, pl.sh.few_units, a, stream)) return rc;
    a.sh.few_units = 0;
    return launch_few_shared(pl.d, pl.pool.fp8, pl.own_two, pl.own_units, a, stream);
  }
  if (pl.sh.few_units + pl.own_units > 0)
    if (int rc = launch_few_shared(pl.d, pl.pool.fp8, pl.few_two, pl.sh.few_units + pl.own_units, a, stream)) return rc;
  const bool many = std::max(pl.sh.many_splits, pl.sh.few_splits) + pl.own_parts >= kJoinParts && rows <= kJoinRows;
  if (pl.d == 128) return many ? launch_join<128, 8>(a, pl.own_parts, stream) : launch_join<128, 1>(a, pl.own_parts, stream);
  return many ? launch_join<64, 16>(a, pl.own_parts, stream) : launch_join<64, 1>(a, pl.own_parts, stream);
}

}  // namespace codecomp
