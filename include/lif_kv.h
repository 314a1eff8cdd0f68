/*
 * lif_kv.h — the attention side of a decoded token: a paged key-value cache in device memory, what
 * writes it (norm of queries and keys per head, rotation of positions, one pass) and what reads it
 * (attention of the new tokens over the cached ones).
 *
 * The paper keeps attention resident and leaves it to the host framework (Section 3.1, "Selective
 * Persistence Strategy"; the key-value cache appears in Appendix C's memory accounting only).  A
 * program that steps the FFN layers of lif.h one by one has this between them:
 *
 *   once per token:      lif_kv_reserve                       room for the step's tokens
 *   layer by layer:      (projections) lif_kv_append          q, k normed and rotated; k, v cached
 *                        lif_kv_attention (projection)
 *                        lif_decode_step                      the layer's FFN (lif.h)
 *   when drafts fail,
 *   beams reorder,
 *   sequences end:       lif_kv_fork                          cut back, copy, reorder, free
 *
 * Conventions are those of lif.h: "dev" pointers are device addresses, "host" pointers host
 * addresses, streams are `cudaStream_t` as `void*`, the caller owns all memory, calls with a stream
 * only enqueue (so all of them can be captured into a graph; every size they need is read from
 * device memory when they run).  Argument errors are returned at once; what only the device can see
 * goes to the cache's sticky status word (LIF_KV_CNT_STATUS, lif_kv_get_stats): such a call is
 * refused as a whole and changes nothing but what its description says.
 * All calls of one cache use its workspace: they are to be ordered one behind the other (one stream,
 * or events between streams).  Different caches are independent.  The device that was current at
 * lif_kv_create has to be current in every later call with a stream and in lif_kv_get_stats
 * (LIF_ERR_STATE otherwise, and nothing is done).
 *
 * Sequences have places 0 .. max_seqs-1.  Place b holds `lens[b]` tokens, of which the last
 * `n_new[b]` are the tokens of the step under way; a free place has length 0.  Token p of it is row
 * p % page_tokens of page table[b][p / page_tokens]; a page id is the same in every layer.  Pages
 * can be shared: refs[page] counts the table entries that name it.
 */
#ifndef LIF_KV_H
#define LIF_KV_H

#include "lif.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element type of queries, keys, values, norm weights and outputs.  Sums, softmax statistics, norms
 * and rotations are fp32 (angles: 64-bit fractions of a turn). */
enum { LIF_TYPE_F16 = 0, LIF_TYPE_BF16 = 1 };

/* Norm of every query and key head over its head_dim elements, ahead of the rotation:
 * RMS    x / sqrt(mean(x^2) + eps) * weight
 * LAYER  (x - mean(x)) / sqrt(var(x) + eps) * weight + bias */
enum { LIF_NORM_NONE = 0, LIF_NORM_RMS = 1, LIF_NORM_LAYER = 2 };

/* Rotation of the first rope_dims elements of every query and key head by position: pairs
 * (i, i + rope_dims/2) or (2i, 2i+1), pair i at position p by the angle p * host_rope_freq[i]:
 *   (u, v) -> rope_scale * (u cos - v sin, u sin + v cos). */
enum { LIF_ROPE_NONE = 0, LIF_ROPE_HALF = 1, LIF_ROPE_INTERLEAVED = 2 };

#define LIF_KV_MAX_SEQS 1024
#define LIF_KV_MAX_NEW 64

typedef struct lif_kv lif_kv;

typedef struct {
  int32_t n_layers;        /* 1 .. 1024 */
  int32_t n_heads;         /* query heads: a multiple of n_kv_heads, <= 1024 */
  int32_t n_kv_heads;      /* query head i reads key-value head i / (n_heads / n_kv_heads) */
  int32_t head_dim;        /* 64, 80, 96, 128 or 256 */
  int32_t dtype;           /* LIF_TYPE_* */
  int32_t page_tokens;     /* power of two, 8 .. 256 */
  int32_t n_pages;         /* pages of the pool, 1 .. 2^24 */
  int32_t max_seqs;        /* places, 1 .. LIF_KV_MAX_SEQS */
  int32_t max_pages;       /* pages a sequence may have; max_pages * page_tokens <= 2^30, and over all places, key-value
                              heads and blocks of rows at most 2^31 - 2^26 tiles of 64 tokens */
  int32_t max_new;         /* tokens of one sequence in one step, 1 .. LIF_KV_MAX_NEW */
  int32_t window;          /* 0: a token sees itself and everything before it; w > 0: itself and the
                              w - 1 tokens before it */
  float scale;             /* factor on <q, k> ahead of the softmax, > 0; 0: 1 / sqrt(head_dim) */
  int32_t norm;            /* LIF_NORM_* */
  float norm_eps;          /* >= 0 */
  int32_t rope;            /* LIF_ROPE_* */
  int32_t rope_dims;       /* even, 2 .. head_dim (0 without rotation) */
  float rope_scale;        /* factor on the rotated elements (1: none), finite */
  const double* host_rope_freq; /* [rope_dims/2] radians per position, |f| <= 2 pi; read by
                              lif_kv_create only.  Scaling for long contexts is a matter of these. */
  void* dev_pages;         /* [n_layers][n_pages][2][n_kv_heads][page_tokens][head_dim], keys then
                              values, 16-byte aligned */
  void* dev_workspace;     /* 256-byte aligned, lif_kv_workspace_bytes() bytes: tables and scratch */
  size_t workspace_bytes;
} lif_kv_desc;

/* The rows of one operand of lif_kv_append: head h of token t of place b is the head_dim
 * consecutive elements at dev + (b * max_new + t) * token_stride + h * head_stride (in elements;
 * both multiples of 8, >= 0; dev 16-byte aligned), so a fused projection's output is taken as it is. */
typedef struct {
  const void* dev;
  int64_t token_stride;
  int64_t head_stride;
} lif_kv_rows;

/* Norm weights of one layer, [head_dim] of the cache's type, 16-byte aligned, shared by its heads.
 * Biases: LIF_NORM_LAYER only, may be NULL. */
typedef struct {
  const void* dev_q_weight;
  const void* dev_q_bias;
  const void* dev_k_weight;
  const void* dev_k_bias;
} lif_kv_norms;

/* Indices into the counts block (int32[LIF_KV_CNT_LEN] on the device). */
enum {
  LIF_KV_CNT_STATUS = 0,    /* sticky lif_status */
  LIF_KV_CNT_FREE = 1,      /* pages that no table entry names */
  LIF_KV_CNT_COPIES = 2,    /* pages copied (per layer) by the last reserve or compact */
  LIF_KV_CNT_REFUSED = 3,   /* calls refused so far */
  LIF_KV_CNT_LEN = 32
};

/* Device addresses inside the workspace, valid for the cache's lifetime: counts, lens[max_seqs],
 * n_new[max_seqs], table[max_seqs][max_pages] (-1 past a sequence's pages), refs[n_pages]. */
typedef struct {
  int32_t* counts;
  int32_t* lens;
  int32_t* n_new;
  int32_t* table;
  int32_t* refs;
} lif_kv_state;

/* Bytes of workspace for this description (pointer fields ignored). */
lif_status lif_kv_workspace_bytes(const lif_kv_desc* desc, size_t* out_bytes);

/* Check `desc`, create the handle and empty the cache.  Allocates no device memory; copies the
 * frequencies into the workspace and synchronises the device. */
lif_status lif_kv_create(const lif_kv_desc* desc, lif_kv** out);
lif_status lif_kv_destroy(lif_kv* kv);
lif_status lif_kv_get_state(lif_kv* kv, lif_kv_state* host_out);

/* All places free, all pages free, status cleared. */
lif_status lif_kv_reset(lif_kv* kv, void* stream);

/* Room for the next tokens: place b grows by dev_n_new[b] tokens (int32[max_seqs] on the device, 0 ..
 * max_new; 0: the place takes no part in the step).  Pages are given out lowest id first, in order of
 * the places.  A partly filled last page that another table entry names too is copied first (its
 * filled rows, every layer) and the copy takes its place in the table, unless all who hold the page
 * grow out of it in this call: then the lowest place keeps it and the others get copies.
 * Refused: LIF_ERR_INVALID_ARG (a count out of range), LIF_ERR_CAPACITY (too few free pages, or a
 * sequence past max_pages): nothing grows and n_new becomes 0 for every place, so that the step's
 * append and attention calls do nothing. */
lif_status lif_kv_reserve(lif_kv* kv, const int32_t* dev_n_new, void* stream);

/* The new tokens' queries, keys and values of one layer: q and k through norm and rotation (positions
 * are places in the sequence: lens[b] - n_new[b] + t), k and v into the pages, q to dev_q_out
 * [max_seqs][max_new][n_heads][head_dim] (16-byte aligned; may be q->dev itself where q is laid out
 * so; otherwise no row of q, k or v may lie in it: LIF_ERR_INVALID_ARG).  Rows t >= n_new[b] are neither used nor written.
 * norms: required (its weights too) with a norm, ignored without. */
lif_status lif_kv_append(lif_kv* kv, int32_t layer, const lif_kv_rows* q, const lif_kv_rows* k,
                         const lif_kv_rows* v, const lif_kv_norms* norms, void* dev_q_out, void* stream);

/* Attention of the new tokens of one layer over their sequences (the new tokens included, each sees
 * those up to itself):
 *   out[b][t][i] = sum_j w_j v_j / sum_j w_j,  w_j = exp(scale <q[b][t][i], k_j> - max_j ...),
 * j over the tokens that the position of token t sees.  dev_q and dev_out: [max_seqs][max_new]
 * [n_heads][head_dim], 16-byte aligned; rows t >= n_new[b] are neither read nor written.  dev_out may
 * not overlap dev_q (LIF_ERR_INVALID_ARG).  What a token does not see never enters its result, infinities and NaN included
 * (rows of a sequence's pages that no token sees may be read all the same).
 * The w_j are rounded to the cache's type: by half a unit in the last place, and with LIF_TYPE_F16 by up to 2^-32 of
 * the row's largest where they are below 2^-21 of it.  Scores scale <q, k> may be up to 10^8 in magnitude (beyond,
 * fp32 is too coarse for a softmax in any case).
 * The same cache, tables and inputs give the same bits.  Waits inside the kernels are bounded: one that ran
 * out sets LIF_ERR_TIMEOUT, over any other status, and that call's output is not to be used. */
lif_status lif_kv_attention(lif_kv* kv, int32_t layer, const void* dev_q, void* dev_out, void* stream);

/* Rearranges the places, all at once: afterwards place b holds the first dev_len[b] tokens of what
 * place dev_src[b] held before (sharing its pages), or is free where dev_src[b] is -1.  dev_src
 * (int32[max_seqs], NULL: b itself) may name a place any number of times; dev_len (int32[max_seqs],
 * NULL: all) is 0 .. the source's length, or -1 for all of it.  Pages that nobody names any more are
 * free.  n_new becomes 0.  Refused: LIF_ERR_INVALID_ARG for a source or length out of range. */
lif_status lif_kv_fork(lif_kv* kv, const int32_t* dev_src, const int32_t* dev_len, void* stream);

/* Takes over tables from elsewhere: lengths (int32[max_seqs]), page ids (int32[max_seqs][max_pages],
 * entries past a sequence's pages are not looked at) and the tokens of the step under way (NULL: none;
 * 0 .. min(max_new, length)).  Pages may be shared, but not those that hold tokens of the step.  The
 * pages' contents are the caller's.  Refused: LIF_ERR_INVALID_ARG. */
lif_status lif_kv_load(lif_kv* kv, const int32_t* dev_lens, const int32_t* dev_table,
                       const int32_t* dev_n_new, void* stream);

/* Moves the pages in use to ids 0 .. used-1, in every layer: the lowest free one takes the highest
 * used one's contents, and so on, as deleted cache rows are filled in Section 3.3.  Tables and counts
 * follow; sequences, and a step under way, stay as they are. */
lif_status lif_kv_compact(lif_kv* kv, void* stream);

/* Synchronises the device and copies the counts block (int32[LIF_KV_CNT_LEN]). */
lif_status lif_kv_get_stats(lif_kv* kv, int32_t* host_counts);
lif_status lif_kv_clear_status(lif_kv* kv, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* LIF_KV_H */
