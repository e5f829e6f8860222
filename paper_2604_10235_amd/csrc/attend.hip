// codecomp_attend: which kernels a batch takes, and the workspace they share.
#include <float.h>
#include <math.h>

#include <algorithm>

#include "attend_many.h"

namespace codecomp {

extern template int launch_many_of<64, false>(const ManyArgs&, hipStream_t);
extern template int launch_many_of<64, true>(const ManyArgs&, hipStream_t);
extern template int launch_many_of<128, false>(const ManyArgs&, hipStream_t);
extern template int launch_many_of<128, true>(const ManyArgs&, hipStream_t);

// Which kernel a request takes goes by its rows (new tokens x query heads per KV head; figures in us for 28 query heads on 4 KV heads of 128
// elements, few | many rows' kernel).  Up to kFewRows it is attend_few_kernel's, which gives a chunk of keys to a workgroup: 4 tokens over 8192 keys 15 |
// 23, over 131072 60 | 72; only from a few GB on the other is ahead (64 requests over 8192 keys 212 | 190).  Up to kFewRowsMost two workgroups share the
// rows and both read the keys, which pays while these are few: 9 tokens over 8192 keys 19 | 24, over 32768 38 | 41, over 131072 92 | 76; 64 requests
// over 8192 keys 353 | 204; and always from an 8-bit cache: 17 | 24, 31 | 39, 59 | 69, 205 | 205.  Beyond, a third and a fourth workgroup do not pay
// from 8192 keys on (18 tokens over 32768 keys 57 | 44; over 2000 15 | 21).  Up to kFewRowsMost, weights enter the product as two bf16 in either kernel,
// by a request's own rows alone (the many-row one with rounded ones: 64 requests 191).
constexpr int kFewRows = 32;
constexpr int64_t kFewKeysMost = 1 << 17;        // keys of all requests and KV heads, at their largest, up to which kFewRowsMost holds for bf16
// In a batch with longer chunks, short requests go along with them while they are few: fewer launches, and the bandwidth that long ones have.  Beyond, what
// starting on a block costs, and one wave's work for its tiles, take longer than a kernel and a join of their own.  Most of them, as blocks of rows (requests times KV
// heads) and as tiles of keys (at the largest length); us, 4 KV heads, apart | along.
// head_dim 128: beside 512 tokens over 4096 keys 64 steps over 500 .. 4000 125 | 95, 256 of them 277 | 242; beside 2048 over 8192 64 over 8000 .. 16384
// 502 | 436; beside a prompt of 20 64 over 300 .. 1000 41 | 37, 256 97 | 101; 256 over 50 .. 300 beside 512 tokens 88 | 91, 1000 158 | 229.
// head_dim 64 has half the bytes for as much of a wave's work: 64 over 500 .. 4000 73 | 66, 128 94 | 104; 64 over 300 .. 1000 beside a prompt of 20 29 | 29, 128 37 | 45;
// 16 over 8000 .. 16384 beside 512 tokens 86 | 78, 64 196 | 214; (lost: 128 over 300 .. 1000 beside 2048 over 8192 158 | 145).
// 8 bits, every tile of which is widened for a whole block's rows: beside 512 tokens over 4096 keys 4 over 4000 67 | 57 (head_dim 64 49 | 44), 16 72 | 69 (50 | 50), 64
// 102 | 135 (64 | 97); beside a prompt of 20 33 | 27 (27 | 22), 39 | 41 (31 | 33), 69 | 107 (45 | 81).
struct Along { int64_t blocks, tiles; };
constexpr Along kAlong128 = {1024, INT64_MAX}, kAlong64 = {256, 1 << 15}, kAlongFp8 = {INT64_MAX, 1 << 10};

// Cache bytes (at the largest lengths) from which the keys of several requests of few rows are cut into equal parts instead of chunks: all workgroups
// run at once and end together, for 5 us more before the first key and for the parts (64 steps over 500 .. 16384 keys, 4 KV heads of 128: 210 us in
// chunks, 190 in parts; 8 bits 118, 103; 16 over 300 .. 9000 45, 37, 8 bits 25.7, 25.9; 64 over 8192 192, 196; one over 131072 57, 64).  Not where a
// request is one chunk: no join to begin with (1000 steps over 100 .. 1000 keys 223, 235; 8 bits, head_dim 64 52, 87).  Two workgroups
// per compute unit: with three or four 195 and 198.
constexpr int64_t kEvenBytes = 1 << 28;
constexpr int kShares = 512;
constexpr int64_t kMostFewBlocks = (1 << 24) - 1;
// Tiles of the longest block of rows up to which blocks are not shared by workgroups: no parts to be joined (a prompt of 500 tokens 27 us, 32 with
// sharing; of 100 19, 23).
constexpr int kWholeTiles = 8;

static size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

int make_attend_plan(const codecomp_batch* b, const codecomp_pages* p, AttendPlan* pl) {
  if (int rc = make_pool(p, &pl->pool)) return rc;
  if (int rc = make_batch(b, p, &pl->batch)) return rc;
  const PagedBatch& x = pl->batch;
  pl->d = p->head_dim;
  pl->scale = b->softmax_scale > 0.0f ? b->softmax_scale : 1.0f / sqrtf((float)p->head_dim);
  int few_most, few_limit = kFewRowsMost;
  for (;;) {
    few_most = pl->few_rows = pl->many_rows = 0;
    for (int r = 0; r < x.n_seqs; ++r) {
      const int64_t rows = (int64_t)(b->cu_q_host[r + 1] - b->cu_q_host[r]) * x.G;
      if (rows == 0) continue;
      if (rows > few_limit) { ++pl->many_rows; continue; }
      ++pl->few_rows;
      if (rows > few_most) few_most = (int)rows;
    }
    if (few_most <= kFewRows || pl->pool.fp8 || (int64_t)pl->few_rows * x.Hkv * x.max_kv <= kFewKeysMost) break;
    few_limit = kFewRows;
  }
  const Along along = pl->pool.fp8 ? kAlongFp8 : pl->d == 64 ? kAlong64 : kAlong128;
  const int64_t few_blocks = (int64_t)pl->few_rows * x.Hkv, few_tiles = few_blocks * ((x.max_kv + kManyKeys - 1) / kManyKeys);
  if (pl->many_rows > 0 && few_blocks <= along.blocks && few_tiles <= along.tiles) {
    pl->many_rows += pl->few_rows;
    pl->few_rows = few_most = 0;
  }
  pl->many_from = pl->few_rows > 0 ? few_limit + 1 : 1;
  int64_t blocks = 0;
  for (int r = 0; r < x.n_seqs; ++r) {
    const int64_t rows = (int64_t)(b->cu_q_host[r + 1] - b->cu_q_host[r]) * x.G;
    if (rows >= pl->many_from) blocks += (rows + kManyRows - 1) / kManyRows;
  }
  pl->many_blocks = blocks * x.Hkv < INT32_MAX ? (int)(blocks * x.Hkv) : INT32_MAX;
  pl->row_parts = (few_most + 31) / 32;
  pl->row_slots = few_most;
  const int64_t items = (int64_t)x.n_seqs * x.Hkv;
  // chunks of keys: about two workgroups per compute unit if all requests are of the largest length, of at least 128 keys each (one tile for each wave; 256: 1 us more for one request)
  // and at most 2048 (one token over 131072 keys, 4 KV heads: chunks of 512 58 us, of 1024 55, of 4096 68; 64 requests of 500 .. 16384 keys, 8 bits: 512
  // 215, 1024 200, 2048 199, 4096 209)
  int64_t chunk = (items * x.max_kv / 512 + 127) / 128 * 128;
  if (chunk < 128) chunk = 128;
  if (chunk > 2048) chunk = 2048;
  // One chunk of short caches: no join, which costs 4 us and more with many requests (one step, us, one chunk | several: 200 keys, 1 request 8.3 | 11.9;
  // 400 keys 11 | 11, 64 requests 13.9 | 19; 800 keys 15 | 11.7, 21 | 27; 8 bits 400 keys 8.4 | 10, 10.5 | 15; 800 keys 10.8 | 10.2, 13.4 | 18; 4 tokens
  // over 400 keys, 64 requests 16 | 30).
  const int once = (p->head_dim * (pl->pool.fp8 ? 1 : 2) <= 128 ? 512 : 256) << (items >= 256 ? 2 : items >= 64 ? 1 : 0);
  if (x.max_kv <= std::min(once, 1024)) chunk = 1024;
  // so many at most: the list of a row's chunks stands in LDS, and an axis of a grid holds 2^32 threads
  while ((x.max_kv + chunk - 1) / chunk > kFewMostSplits || (x.max_kv > chunk && items * pl->row_parts * ((x.max_kv + chunk - 1) / chunk) > kMostFewBlocks)) chunk *= 2;
  pl->chunk = (int)chunk;
  pl->splits = x.max_kv > chunk ? (int)((x.max_kv + chunk - 1) / chunk) : 1;
  if (pl->few_rows > 0 && (items * pl->row_parts > kMostFewBlocks || items * pl->row_slots > kMostFewBlocks)) return CODECOMP_EINVAL_SHAPE;
  const int64_t bytes = (int64_t)pl->few_rows * x.Hkv * x.max_kv * p->head_dim * (pl->pool.fp8 ? 2 : 4);
  pl->shares = pl->few_rows > 1 && pl->row_parts == 1 && pl->splits > 1 && bytes > kEvenBytes ? kShares : 0;
  size_t off = 0;
  pl->off_few = off;
  if (pl->shares > 0) off = align256(off + (size_t)pl->shares * (2 * (size_t)pl->row_slots * (p->head_dim + 2) * sizeof(float) + sizeof(CutBlock)));
  else if (pl->few_rows > 0 && pl->splits > 1) off = align256(off + (size_t)(items * pl->splits * pl->row_slots) * (p->head_dim + 2) * sizeof(float));
  pl->off_many = off;
  pl->workgroups = 256;
  pl->many_whole = x.max_kv <= kWholeTiles * kManyKeys;
  if (pl->many_rows > 0 && !pl->many_whole)
    off = align256(off + (size_t)pl->workgroups * 2 * kManyRows * (p->head_dim + 2) * sizeof(float) + pl->workgroups * sizeof(CutBlock));
  pl->ws_bytes = off;
  return CODECOMP_OK;
}

// Blocks of rows whose keys several workgroups shared: blockIdx.y the workgroup that has a block's first part, blockIdx.x some of its rows, one
// after the other by D / 4 threads each.  (In that order: the first parts may be a multiple of eight workgroups apart, which would put all the work on one die.)
template <int D>
__global__ __launch_bounds__(256) void join_many_kernel(const ManyArgs ma, int rows_each) {
  const AttendArgs& a = ma.a;
  const CutBlock cut = ma.cuts[blockIdx.y];
  if (cut.r < 0) return;
  constexpr int THREADS = D / 4;
  const int first = blockIdx.y, e = (threadIdx.x % THREADS) * 4;
  const int q0 = a.b.cu_q[cut.r], rows = (a.b.cu_q[cut.r + 1] - q0) * a.b.G;
  for (int i = threadIdx.x / THREADS; i < rows_each; i += 256 / THREADS) {
    const int in_block = blockIdx.x * rows_each + i, row = cut.block * kManyRows + in_block;
    if (row >= rows) return;
    auto part_of = [&](int g) { return (int64_t)(g == first ? 2 * g + 1 : 2 * g) * kManyRows + in_block; };
    float top = kNoReference, all = 0.0f;
#pragma unroll 8
    for (int g = first; g <= cut.last; ++g) top = fmaxf(top, a.part_ml[2 * part_of(g)]);
    f32x4 x = {0, 0, 0, 0};
#pragma unroll 8
    for (int g = first; g <= cut.last; ++g) {
      const int64_t part = part_of(g);
      const float m = a.part_ml[2 * part], f = m == top ? 1.0f : __builtin_amdgcn_exp2f(m - top);
      all += a.part_ml[2 * part + 1] * f;
      x += *reinterpret_cast<const f32x4*>(a.part_o + part * D + e) * f;
    }
    const int t = row / a.b.G, h = cut.head * a.b.G + row - t * a.b.G;
    const float inv = all == 0.0f ? 0.0f : a.pool.v_scale / all;
    *reinterpret_cast<u32x2*>(a.out + (q0 + t) * a.b.o_st + h * a.b.o_sh + e) = u32x2{pack2(x.x * inv, x.y * inv), pack2(x.z * inv, x.w * inv)};
    if (a.lse && e == 0) a.lse[(int64_t)(q0 + t) * a.b.Hq + h] = all == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(all)) * kLn2;
  }
}

static int launch_many(const AttendPlan& pl, const AttendArgs& a, char* workspace, hipStream_t stream) {
  ManyArgs m;
  m.a = a;
  m.workgroups = pl.workgroups;
  m.rows_from = pl.many_from;
  m.whole = pl.many_whole;
  m.a.part_o = reinterpret_cast<float*>(workspace);
  m.a.part_ml = m.a.part_o + (size_t)pl.workgroups * 2 * kManyRows * pl.d;
  m.cuts = reinterpret_cast<CutBlock*>(m.a.part_ml + (size_t)pl.workgroups * 2 * kManyRows * 2);
  int rc;
  if (pl.d == 128) rc = pl.pool.fp8 ? launch_many_of<128, true>(m, stream) : launch_many_of<128, false>(m, stream);
  else rc = pl.pool.fp8 ? launch_many_of<64, true>(m, stream) : launch_many_of<64, false>(m, stream);
  if (rc || pl.many_whole) return rc;
  // A few blocks of many parts: their rows over more workgroups (20 tokens over 131072 keys 83 us, 16 rows each 96, 64 rows each 213); many blocks of
  // a part or two: fewer workgroups (12 x 1024 tokens over 4096 keys, head_dim 64: 8 rows each 125, 16 124).
  const int rows_each = pl.many_blocks <= 32 ? 256 / (pl.d / 4) : 16;
  const dim3 grid(kManyRows / rows_each, pl.workgroups), block(256);
  if (pl.d == 128) join_many_kernel<128><<<grid, block, 0, stream>>>(m, rows_each);
  else join_many_kernel<64><<<grid, block, 0, stream>>>(m, rows_each);
  return (int)hipGetLastError();
}

int launch_attend(const AttendPlan& pl, const void* q, int layer, void* out, float* lse, void* workspace, hipStream_t stream) {
  AttendArgs a = {};
  a.pool = pl.pool; a.b = pl.batch; a.q = static_cast<const uint16_t*>(q); a.out = static_cast<uint16_t*>(out); a.lse = lse;
  a.layer = layer * pl.pool.s_layer;
  a.c = fminf(fmaxf(pl.scale * pl.pool.k_scale * kLog2e, FLT_MIN), FLT_MAX);       // a hidden logit of minus infinity times it stays one
  a.chunk = pl.chunk; a.splits = pl.splits; a.row_slots = pl.row_slots; a.row_parts = pl.row_parts; a.shares = pl.shares;
  if (pl.few_rows > 0) {
    a.part_o = reinterpret_cast<float*>(static_cast<char*>(workspace) + pl.off_few);
    const size_t parts = (pl.shares > 0 ? 2 * (size_t)pl.shares : (size_t)pl.batch.n_seqs * pl.batch.Hkv * pl.splits) * pl.row_slots;
    a.part_ml = a.part_o + parts * pl.d;
    a.cuts = reinterpret_cast<CutBlock*>(a.part_ml + parts * 2);
    if (int rc = launch_few(pl, a, stream)) return rc;
  }
  if (pl.many_rows > 0)
    if (int rc = launch_many(pl, a, static_cast<char*>(workspace) + pl.off_many, stream)) return rc;
  return 0;
}

}  // namespace codecomp
