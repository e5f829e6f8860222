/*
 * codecomp_serve.h - C ABI for long and branching service from a compressed cache on MI355X (gfx950): requests that share the start of
 *                    their caches, attention weights summed up per cached row, eviction by these sums.
 *
 * The paper compresses a prompt once, by the attention of its last tokens (section "Attention-based KV Cache Compression").
 * What comes behind - answers, the steps of an agent, several of them on one compressed prompt - grows the cache again, and
 * is ranked by nothing.  The paper gives no kernels for that; these operators are this library's, on the pages of codecomp_cache.h.
 *
 *   codecomp_attend_shared   codecomp_attend for groups of requests whose caches begin with the same rows: these are read once for a group
 *   codecomp_attend_mass     the attention weights that a call's new tokens give to every cached row, added to sums per request, head and row
 *   codecomp_evict           rows behind a protected start: the last few and those of the largest sums stay, all layers and heads in one call
 *
 * Used together: requests fork from one prompt (codecomp_pages_copy for the page that the shared rows end in), codecomp_append and
 * codecomp_attend_shared per layer and step, codecomp_attend_mass with its log-sum-exp, and from time to time codecomp_evict; `first` of the latter
 * two is the number of shared rows, which are everybody's and stay.
 *
 * Everything said at the heads of codecomp.h and codecomp_cache.h holds here as well: device pointers unless the name ends in _host, nothing is
 * allocated, nothing synchronises, work goes to `hip_stream`, calls are re-entrant and deterministic, a rejected call has enqueued nothing, device data is
 * not validated, what a corrupt table, length or budget can do is bounded.  Calls may be captured into a graph; lengths, budgets,
 * tables and tokens may then change between replays (what has a copy on the host may not).
 */
#ifndef CODECOMP_SERVE_H
#define CODECOMP_SERVE_H

#include "codecomp_cache.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Requests cu_groups[g] .. cu_groups[g + 1] - 1 of a batch share their rows 0 .. prefix_lens[g] - 1: the same pages hold them (the page in which they end
 * may differ: a copy).  They are read by way of the table of the group's first request, be it one without new tokens.  A group of one
 * request, and a length of 0, are allowed; a group may be empty. */
typedef struct codecomp_groups {
  int32_t n_groups;                /* 1 .. 65535                                                                  */
  int32_t max_prefix_len;          /* HOST bound of prefix_lens, 0 .. the batch's max_kv_len: sizes launches and workspace, as does */
  int32_t max_own_len;             /* HOST bound of the rows behind the shared ones, 0 .. the batch's max_kv_len: kv_lens[r] is cut to prefix_lens[g] + max_own_len */
  const int32_t* cu_groups_host;   /* [n_groups + 1] HOST, from 0 to n_seqs, not decreasing                        */
  const int32_t* cu_groups_dev;    /* [n_groups + 1] DEVICE copy of the same values                                */
  const int32_t* prefix_lens_dev;  /* [n_groups], cut to [0, max_prefix_len]                                       */
} codecomp_groups;

/* Host-only: 0 or the code with which codecomp_attend_shared refuses these arguments. */
int codecomp_attend_shared_validate(const codecomp_batch* batch, const codecomp_groups* groups, const codecomp_pages* pages);

/* Host-only: bytes of workspace that codecomp_attend_shared needs (0 when the arguments are invalid or there is no new token). */
size_t codecomp_attend_shared_workspace_bytes(const codecomp_batch* batch, const codecomp_groups* groups, const codecomp_pages* pages);

/* out and lse as of codecomp_attend over the same batch: a token of request r in group g sees rows j < prefix_lens[g], and the rows from there on that
 * codecomp_attend would let it see (j < kv_lens[r]; causal: j <= kv_lens[r] - cu_q[r + 1] + t).  The shared rows are to lie before the new
 * tokens of every request, prefix_lens[g] <= kv_lens[r] - (cu_q[r + 1] - cu_q[r]), and then the result is that of codecomp_attend but for roundings.
 * What stands in rows that a token does not see has no part in its result; an infinity or NaN in what it sees counts as for codecomp_attend.
 * Logits, sums and outputs are fp32.  Weights enter the second product rounded to bf16, or as two bf16, 16 bits together, for requests of up to 64 rows (new
 * tokens * query heads per KV head), as in codecomp_attend, whatever is in the group and the batch with them.
 * What it is for: single tokens and short chunks, which wait for memory, behind long shared rows (64 steps behind 32768 rows 73 us, codecomp_attend 471).  Prompts wait for
 * the matrix units, which sharing takes no work off: behind long shared rows either call takes as long, but from 8-bit caches, or with long rows of their own, codecomp_attend over
 * the same batch (with the shared pages in every request's table) is faster, by up to a fifth, and it needs less workspace.
 * workspace: >= codecomp_attend_shared_workspace_bytes(), 256-byte aligned, contents on entry do not matter; calls that may run at the same
 * time need workspaces of their own.  It grows with the tokens: head_dim + 2 floats for every token, query head and chunk that the keys are cut into (64 steps behind 32768 rows
 * 30 MB, 16 prompts of 4096 tokens behind 8192, 28 heads of 128, 1.9 GB). */
int codecomp_attend_shared(const void* q, const codecomp_batch* batch, const codecomp_groups* groups, const codecomp_pages* pages, int32_t layer, void* out,
                           float* lse, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Sums of attention weights, f32: element of (layer, request, KV head, row) at layer * stride_layer + request * stride_seq + head * stride_head + row.
 * Two elements must not lie at one place. */
typedef struct codecomp_mass {
  float* sums;                                     /* DEVICE                                                          */
  int32_t n_layers, n_seqs, n_kv_heads;
  int32_t width;                                   /* rows that there is room for                                     */
  int64_t stride_layer, stride_seq, stride_head;   /* elements; 0 = dense [n_layers][n_seqs][n_kv_heads][width]        */
} codecomp_mass;

/* Host-only: 0 or the code with which codecomp_attend_mass refuses these arguments; bytes of workspace that it needs (0 when they are invalid, or when
 * it needs none). */
int codecomp_attend_mass_validate(const codecomp_batch* batch, const codecomp_pages* pages, const codecomp_mass* mass);
size_t codecomp_attend_mass_workspace_bytes(const codecomp_batch* batch, const codecomp_pages* pages, const codecomp_mass* mass);

/* For every request with new tokens, KV head and row first[r] <= j < kv_lens[r]:
 *   sums[j] = (j is old ? decay * sums[j] : 0) + 1/G * sum_{t, h} exp(softmax_scale * q[t][h] . k_j - lse[t][h])
 * over its new tokens t that see row j (as in codecomp_attend) and the G query heads h of the KV head: the attention mass u(j) of
 * codecomp_score, mean over the heads.  lse is what codecomp_attend or codecomp_attend_shared has left for the same batch (or any other f32 [T][n_q_heads], dense, e.g. one
 * joined over several caches); a token and head whose lse is -inf gives no weight.  Old rows are those before the new tokens
 * (j < kv_lens[r] - (cu_q[r + 1] - cu_q[r])) when causal, and all rows otherwise; sums of rows that are not old are not read: they need no clearing when causal.  Without
 * the mask no row is known to be new: the caller clears the sums of rows that it appends, also where evicted ones stood.  decay in [0, 1]; 0 reads no sums.
 * Rows of pages that are not held get no weight; rows outside of first[r] .. kv_lens[r] - 1, and all of a request without new tokens, stay as they are.
 * first: DEVICE int32 [n_seqs] (below 0 counts as 0), NULL = 0.
 * The batch's max_kv_len is at most the width, its n_seqs that of the sums.  Weights and sums are fp32; every sum has a fixed order.
 * What an infinity or NaN in a key, a query or lse makes of a weight - NaN, infinite, or zero where z - lse is minus infinity - the sum of that row becomes; no other
 * sum changes.
 * workspace: >= codecomp_attend_mass_workspace_bytes(), 256-byte aligned, contents on entry do not matter; NULL when that is 0. */
int codecomp_attend_mass(const void* q, const float* lse, const codecomp_batch* batch, const codecomp_pages* pages, int32_t layer, const int32_t* first,
                         float decay, const codecomp_mass* mass, void* workspace, size_t workspace_bytes, void* hip_stream);

/* What is evicted from: request r has n = kv_lens[r] rows (cut to [0, max_kv_len]), row j in page table[r][j / page_size]; its first f = first[r] rows (cut to [0, n]) stay
 * as they are, and of the rows behind them at most budgets[r] (cut to [recent, max_budget]) are kept.  Two requests, or two entries of one request, must
 * not have a page in common in which rows behind their first ones lie. */
typedef struct codecomp_eviction {
  int32_t n_seqs;                  /* 1 .. 65535                                                                  */
  int32_t table_width;
  int32_t max_kv_len;              /* HOST bound of kv_lens, <= table_width * page_size                           */
  int32_t max_budget;              /* HOST bound of budgets, >= 1; the width of `kept`                            */
  int32_t recent;                  /* the last so many rows always stay: 0 .. max_budget                          */
  const int32_t* kv_lens_dev;      /* [n_seqs]                                                                    */
  const int32_t* table_dev;        /* [n_seqs][table_width]                                                       */
  const int32_t* budgets_dev;      /* [n_seqs]                                                                    */
  const int32_t* first_dev;        /* [n_seqs]; NULL = 0                                                          */
} codecomp_eviction;

/* For every layer, request and KV head: m = min(n - f, B_r) rows of [f, n) are kept - all of them, or the last `recent` and, of the others, the B_r - recent
 * of the largest sums (equal ones: the lower row; ordered as IEEE floats, -0 == +0, NaN below everything else) - and move together:
 *   row f + i = row kept[l][r][h][i], K and V bit for bit, and kept_mass[l][r][h][f + i] = mass[l][r][h][kept[l][r][h][i]],  i < m,
 * with kept ascending, -1 from m on (DEVICE int32 [n_layers][n_seqs][n_kv_heads][max_budget], dense), and new_lens[r] = f + m (DEVICE int32 [n_seqs]).  Rows of K and V, and
 * sums, from f + m on stay as they are (of causal batches codecomp_attend_mass does not read them; before others, clear the sums of the rows that come there).  kept_mass NULL: `mass` itself; else sums of the same shape
 * elsewhere, and `mass` stays as it is.  new_lens must not be kv_lens, budgets or first.  A row that moves from a page that is not held becomes zeros, one that moves to such a
 * page is dropped.  mass->n_layers and n_kv_heads are the pool's, n_seqs the eviction's, width at least max_kv_len. */
int codecomp_evict(const codecomp_mass* mass, const codecomp_eviction* eviction, const codecomp_pages* pages, int32_t* kept, int32_t* new_lens,
                   const codecomp_mass* kept_mass, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* CODECOMP_SERVE_H */
