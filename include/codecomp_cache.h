/*
 * codecomp_cache.h - C ABI for serving from a compressed cache on MI355X (gfx950): the compact rows of codecomp.h in
 *                    pages, the new tokens behind them, and the attention that reads both.
 *
 * What follows the compression in the paper's pipeline (section "Position Encoding"): the compressed chunks stand one
 * behind the other in the cache with their original positions, the query's tokens take positions of their own, and
 * attention runs over what was kept.  The paper gives no kernels for it; pages, 8-bit storage and splits are this library's.
 *
 *   codecomp_rotate          rotary positions on query or key vectors, or the gradient of that
 *   codecomp_append          new tokens: queries rotated, keys rotated and values stored in the pages
 *   codecomp_pages_store     dense rows (a compact cache, or kept rows of a dense one) into pages
 *   codecomp_pages_load      rows of pages into the dense layout that codecomp_score and codecomp_gather read
 *   codecomp_pages_compact   kept rows of a paged cache into other pages
 *   codecomp_pages_copy      whole pages (requests that fork)
 *   codecomp_attend          attention of new tokens over the pages
 *
 * Everything said at the head of codecomp.h holds here as well: device pointers unless the name ends in _host, nothing is
 * allocated, nothing synchronises, work goes to `hip_stream`, calls are re-entrant and deterministic, a rejected call has
 * enqueued nothing, device data is not validated.  What a corrupt table or length can do is bounded: a page number outside
 * the pool is a page that is not held (its keys take no part in attention, rows read from it are zeros, rows written to
 * it are dropped), a length is cut to [0, max_kv_len].  Calls may be captured into a graph; the lengths, tables and
 * tokens may then change between replays (cu_q may not: it sizes the launches).
 */
#ifndef CODECOMP_CACHE_H
#define CODECOMP_CACHE_H

#include "codecomp.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { CODECOMP_EINVAL_PAGES = -12 };     /* page pool, page table, layer, cu_q or max_kv_len out of order */

/* A pool of pages: for every layer n_pages pages, each of page_size rows of every KV head.  All layers of a request use
 * the same page numbers; a row's K and V lie at the same place of their pools.
 *   element of (layer, page, head, row, i) at layer * stride_layer + page * stride_page + head * stride_head + row * stride_tok + i
 * The value of an element is what is stored there times k_scale (v_scale). */
typedef struct codecomp_pages {
  void* k;                     /* DEVICE, 16-byte aligned                                                        */
  void* v;
  int32_t n_layers, n_pages;
  int32_t page_size;           /* rows of a page: a power of two, at most 65536                                  */
  int32_t n_kv_heads;
  int32_t head_dim;            /* 64 or 128                                                                      */
  int32_t kv_dtype;            /* CODECOMP_KV_BF16 or CODECOMP_KV_FP8_E4M3                                       */
  int64_t stride_layer, stride_page, stride_head, stride_tok; /* elements, multiples of 16 bytes; a page's rows within 2^31 bytes; 0 = dense
                                  [n_layers][n_pages][n_kv_heads][page_size][head_dim]                           */
  float k_scale, v_scale;      /* finite, > 0; 0 = 1                                                             */
} codecomp_pages;

/* The new tokens of a batch of requests, and where the requests' caches are.  New token t of the packed batch belongs to the
 * request r with cu_q[r] <= t < cu_q[r + 1]; requests without a new token are allowed.  kv_lens[r] counts the rows of
 * the request in the cache, its new tokens among them: they are the last ones, so token t has row
 * kv_lens[r] - cu_q[r + 1] + t.  Row j lies in page table[r][j / page_size]. */
typedef struct codecomp_batch {
  int32_t n_seqs;              /* 1 .. 65535                                                                     */
  int32_t n_q_heads;           /* a multiple of the pool's n_kv_heads, at most 65535                              */
  int32_t table_width;         /* entries of a request's row of the table                                        */
  int32_t max_kv_len;          /* HOST bound of kv_lens, <= table_width * page_size: sizes launches and workspace */
  int32_t causal;              /* 1: a new token sees the rows up to its own; 0: all rows of its request (attention
                                  to an encoder's states, for one)                                               */
  float softmax_scale;         /* 0 selects 1/sqrt(head_dim)                                                     */
  const int32_t* cu_q_host;    /* [n_seqs + 1] HOST                                                              */
  const int32_t* cu_q_dev;     /* [n_seqs + 1] DEVICE copy of the same values                                    */
  const int32_t* kv_lens_dev;  /* [n_seqs]                                                                       */
  const int32_t* table_dev;    /* [n_seqs][table_width]                                                          */
  /* strides in elements, multiples of 8; 0 = dense [T][heads][head_dim] */
  int64_t q_stride_tok, q_stride_head;        /* q                                                               */
  int64_t new_stride_tok, new_stride_head;    /* new k and v                                                     */
  int64_t out_stride_tok, out_stride_head;    /* q_out of codecomp_append, out of codecomp_attend                */
} codecomp_batch;

/* Rotary positions: the first `dim` elements of a head are dim / 2 pairs, pair i of a vector at position p is turned by the
 * angle p * freq[i] and multiplied by `magnitude`; the other elements are copied.
 *   (x0, x1) -> magnitude * (x0 cos a - x1 sin a, x0 sin a + x1 cos a)
 * Pairs are elements (i, i + dim / 2), or (2 i, 2 i + 1) when interleaved.  inverse: by -a, which with the same
 * magnitude is the gradient at the input from the gradient at the output (the transpose).
 * Angles are reduced in turns of 64 bits, to which any frequency is rounded once: at position 2^31 they are off by 2^-34 of a turn, less than fp32 can
 * tell.  The inverse at a position is bit for bit the rotation at minus the position. */
typedef struct codecomp_rotary {
  int32_t dim;                 /* a multiple of 16, 0 .. head_dim                                                */
  int32_t interleaved;
  int32_t inverse;
  float magnitude;             /* finite; 0 = 1                                                                  */
  double freq[64];             /* radians per position, finite, of each of the dim / 2 pairs                     */
} codecomp_rotary;

/* Host-only: fills freq (and dim, interleaved; inverse = 0, magnitude = 1) with base^(-2 i / dim), scaled for contexts longer than the trained one:
 *   PLAIN       as it is;
 *   LINEAR      divided by `factor`;
 *   BASE        from base * factor^(dim / (dim - 2));
 *   WAVELENGTH  by the turns f * context / (2 pi) that a pair makes in the trained context: at most `low` divided by factor,
 *               at least `high` as it is, between them a blend, linear in the turns;
 *   RAMP        the same, linear in the pair's number between floor(n(high)) and ceil(n(low)), cut to [0, dim - 1], with n(turns) =
 *               dim ln(context / (2 pi turns)) / (2 ln base).  (The usual magnitude with it is 0.1 ln(factor) + 1: set it.)
 * CODECOMP_EINVAL_MODE for an unknown scaling, dim not a multiple of 16 in 16 .. 128, base <= 1, factor < 1, context <= 0 or not low < high. */
enum { CODECOMP_ROTARY_PLAIN = 0, CODECOMP_ROTARY_LINEAR = 1, CODECOMP_ROTARY_BASE = 2, CODECOMP_ROTARY_WAVELENGTH = 3, CODECOMP_ROTARY_RAMP = 4 };
int codecomp_rotary_init(codecomp_rotary* rotary, int32_t dim, int32_t interleaved, double base, int32_t scaling, double factor,
                         double context, double low, double high);

/* out[t][h][:] = rotary(x[t][h][:], positions[t]) for n_tokens tokens of n_heads heads; x and out bf16, rotated in fp32 and
 * rounded once; n_heads at most 65535.  positions: DEVICE int32 [n_tokens], any value.  Strides in elements, multiples of 8; 0 = dense.
 * out may be x with the same strides.  n_tokens = 0 is a call that does nothing (as is a batch without new tokens below): vectors may be NULL then. */
int codecomp_rotate(const void* x, const int32_t* positions, const codecomp_rotary* rotary, int32_t n_tokens, int32_t n_heads,
                    int32_t head_dim, int64_t x_stride_tok, int64_t x_stride_head, void* out, int64_t out_stride_tok,
                    int64_t out_stride_head, void* hip_stream);

/* The new tokens of a batch in one launch: q_out = rotary(q); the rows of the new tokens in layer `layer` of the pool =
 * rotary(k) / k_scale and v / v_scale, rounded to the pool's type (FP8: to the nearest code, beyond 448 to 448; infinities
 * count as beyond, NaN stays NaN).  q, k, v, q_out bf16 [T][heads][head_dim]; rotary may be NULL (positions then, too): no rotation.  q and q_out
 * may both be NULL (only the cache is written); q_out may be q with the same strides.  A token whose row would be negative is dropped from the cache.  Two tokens must
 * not have the same place in the pool.  Rounding: the rotated fp32 value is rounded once. */
int codecomp_append(const void* q, const void* k, const void* v, const int32_t* positions, const codecomp_rotary* rotary,
                    const codecomp_batch* batch, const codecomp_pages* pages, int32_t layer, void* q_out, void* hip_stream);

/* Rows between the dense layouts of codecomp.h and pages, all layers and heads in one launch, bit for bit.  `params` is what
 * the compression was called with: n_layers, n_kv_heads, head_dim, kv_dtype (equal to the pool's), cu_seqlens, cu_budgets and
 * strides are used.  table: DEVICE int32 [n_seqs][table_width], a row per request of `params`; first: DEVICE int32 [n_seqs], the row of the
 * cache that a request's row 0 goes to or comes from, NULL = 0.  (The paper's chunks, compressed as requests of one call, go one
 * behind the other into the pages of the request that they belong to: the same table row for all of them, and `first`
 * the budgets summed up.)  Rows that lie outside [0, table_width * page_size) are treated as those of pages that are not held.
 *
 * store: row first[r] + i of the pages, i < B_r = k[cu_budgets[r] + i] of the compact layout (out strides) when idx is NULL,
 *        else k[cu_seqlens[r] + idx[l][h][cu_budgets[r] + i]] of the cache's layout (kv strides): codecomp_gather into pages. */
int codecomp_pages_store(const void* k, const void* v, const int32_t* idx, const codecomp_params* params,
                         const codecomp_pages* pages, const int32_t* table, int32_t table_width, const int32_t* first,
                         void* hip_stream);
/* load: with idx NULL k[cu_seqlens[r] + j] (kv strides) = row first[r] + j of the pages, j < N_r; else k[cu_budgets[r] + i] (out
 *       strides) = row first[r] + idx[l][h][cu_budgets[r] + i]: codecomp_gather from pages. */
int codecomp_pages_load(const codecomp_pages* pages, const int32_t* table, int32_t table_width, const int32_t* first,
                        const int32_t* idx, const codecomp_params* params, void* k, void* v, void* hip_stream);
/* compact: row to_first[r] + i of `to` = row first[r] + idx[l][h][cu_budgets[r] + i] of `pages`, i < B_r.  `to` may be the same pool; the pages
 *          written must not be pages read.  (idx values are cut into [0, N_r) in all three calls.) */
int codecomp_pages_compact(const codecomp_pages* pages, const int32_t* table, int32_t table_width, const int32_t* first,
                           const int32_t* idx, const codecomp_params* params, const codecomp_pages* to, const int32_t* to_table,
                           int32_t to_table_width, const int32_t* to_first, void* hip_stream);

/* Page pairs[i][1] = page pairs[i][0], all layers and heads, K and V; pairs: DEVICE int32 [n_pairs][2].  A pair with a page outside the pool, or
 * of a page with itself, is left out.  No page may be written twice, or be read and written. */
int codecomp_pages_copy(const codecomp_pages* pages, const int32_t* pairs, int32_t n_pairs, void* hip_stream);

/* Host-only: 0 or the code with which codecomp_attend refuses this batch on this pool. */
int codecomp_attend_validate(const codecomp_batch* batch, const codecomp_pages* pages);

/* Host-only: bytes of workspace that codecomp_attend needs (0 when the arguments are invalid, or when it needs none). */
size_t codecomp_attend_workspace_bytes(const codecomp_batch* batch, const codecomp_pages* pages);

/* out[t][h][:] = sum_j p_j v_j,  p = softmax_j(softmax_scale * q[t][h] . k_j),  over the rows j that token t of request r sees:
 * j < kv_lens[r], and j <= kv_lens[r] - cu_q[r + 1] + t when causal; K and V of KV head h / (n_q_heads / n_kv_heads) of layer `layer`.
 * lse[t][h] = ln sum_j exp(softmax_scale * q . k_j) (f32, dense [T][n_q_heads]; may be NULL): two caches attended to apart are joined with it.
 * A token that sees no row (or rows of pages that are not held alone) gets out = 0, lse = -inf.  What stands in rows that a token
 * does not see, NaN and infinities too, has no part in its result.  An infinity or NaN in a value that it does see makes that element of its result infinite or NaN, whatever the
 * weight; one in its query or in a key that it sees may make all of it so.  Logits, sums and outputs are fp32; the weights enter the second
 * product rounded to bf16, or as two bf16, 16 bits together, for requests of up to 64 rows (new tokens * query heads per KV head).
 * workspace: >= codecomp_attend_workspace_bytes(), 256-byte aligned, contents on entry do not matter; NULL when that is 0.
 * Calls that may run at the same time need workspaces of their own. */
int codecomp_attend(const void* q, const codecomp_batch* batch, const codecomp_pages* pages, int32_t layer, void* out, float* lse,
                    void* workspace, size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* CODECOMP_CACHE_H */
