/*
 * mar_kernels.h - per-kernel entry points of the cached MAR step.
 *
 * The same kernels mar_step runs, exposed one at a time so that each step of
 * the path can be checked on its own.  Conventions as in mar_cache.h:
 * device pointers, row-major dense layouts, `dtype` is mar_dtype (storage
 * type; products accumulate in fp32), asynchronous on `stream`, arguments
 * checked on the host before any launch (an error launches nothing).
 * Buffers read or written in 16-byte vectors must be 16-byte aligned.
 *
 * Row mapping used below: with `idx` given, row m of a compact matrix belongs
 * to slot m / per_slot and token idx[m] of that slot; without it, row m is
 * token m % per_slot of slot m / per_slot (and per_slot must equal seq).
 * The key and value caches [slots, H, seq, d_head] hold one slot's keys (or
 * values) of head h as a contiguous seq x d_head block.
 */
#ifndef MAR_KERNELS_H
#define MAR_KERNELS_H

#include <stddef.h>
#include <stdint.h>

#include "mar_cache.h"

#ifdef __cplusplus
extern "C" {
#endif

/* LayerNorm of the pre-LN block (LN1 / LN2), optionally gathering the rows
 * first (Eq. 9: only the computed rows enter blocks P..L-1).
 *   out[m]      = (r - mean(r)) / sqrt(var(r) + eps) * w + b   in dtype
 *   copy_f32[m] = r (nullable)
 * with r the source row of m: src is [slots, seq, d] (fp32 if src_f32 else
 * dtype), m < `m`.  Statistics in fp32, biased variance.  d % 8 == 0,
 * d <= 2048; src, w, b, out and copy_f32 16-byte aligned (MAR_E_ARG
 * otherwise). */
mar_status mar_k_layernorm(int32_t dtype, const void* src, int32_t src_f32, const int32_t* idx,
                           int32_t per_slot, int32_t seq, int32_t m, int32_t d, const float* w,
                           const float* b, float eps, float* copy_f32, void* out, void* stream);

/* out[m, n] = act(a w^T + bias) in dtype; a [m, k], w [n, k] (nn.Linear
 * layout), bias [n] fp32; act = exact-erf GELU when `act` != 0 (the block's
 * first MLP product), identity otherwise.  k % 64 == 0, n % 8 == 0; a, w
 * and out 16-byte aligned (MAR_E_ARG otherwise). */
mar_status mar_k_linear(int32_t dtype, int32_t act, const void* a, const void* w, const float* bias,
                        int32_t m, int32_t n, int32_t k, void* out, void* stream);

/* Residual product (output projection, second MLP product):
 *   x[m, n] = resid[m, n] + (a w^T)[m, n] + bias[n]      fp32
 * written to out[m, n] (out may equal resid), or, when out_idx is given, to
 * out[(m / per_slot) * seq + out_idx[m], n] (the scatter of the fresh rows
 * into the output cache, Eq. 9) with resid_copy[m, n] = x (nullable).
 * k % 64 == 0, n % 8 == 0; a, w, resid, out and resid_copy 16-byte
 * aligned (MAR_E_ARG otherwise). */
mar_status mar_k_linear_residual(int32_t dtype, const void* a, const void* w, const float* bias,
                                 int32_t m, int32_t n, int32_t k, const float* resid, float* out,
                                 const int32_t* out_idx, int32_t per_slot, int32_t seq,
                                 float* resid_copy, void* stream);

/* Query/key/value projection with the key/value cache update (Eq. 9: the
 * computed rows replace their cached keys and values).  Columns
 * [n_offset, n_offset + n_cols) of the stacked [3D, D] projection, with w
 * and bias pointing at column n_offset:
 *   query columns  -> q_out[m, c]                  ([m, D], dtype)
 *   key columns    -> k_cache[slot, head, tok, :]  ([slots, H, seq, dh])
 *   value columns  -> v_cache[slot, head, tok, :]  ([slots, H, seq, dh];
 *                     nullable) and v_copy, a second buffer of the same
 *                     layout (nullable); one of them required
 * slot/tok from the row mapping.  d_model % 64 == 0, d_head % 16 == 0,
 * n_offset % 32 == 0, n_cols % 8 == 0; every matrix argument 16-byte
 * aligned (MAR_E_ARG otherwise). */
mar_status mar_k_qkv(int32_t dtype, const void* a, const void* w, const float* bias, int32_t m,
                     int32_t n_cols, int32_t n_offset, int32_t d_model, int32_t n_heads, int32_t seq,
                     int32_t per_slot, const int32_t* idx, void* q_out, void* k_cache, void* v_cache,
                     void* v_copy, void* stream);

/* Eq. (3) without mask for per_slot query rows per slot against all seq
 * keys of the slot: q, out [n_slots * per_slot, H * d_head] (head h at
 * columns h * d_head ...), k and v [n_slots, H, seq, d_head] (the cache
 * layout).  Scale
 * 1/sqrt(d_head); softmax statistics in fp32.  d_head in {16, 32, ..., 128}.
 * per_slot == seq is the dense block; per_slot = N the cached one.  q, k,
 * v and out 16-byte aligned (MAR_E_ARG otherwise). */
mar_status mar_k_attention(int32_t dtype, const void* q, const void* k, const void* v, void* out,
                           int32_t n_slots, int32_t n_heads, int32_t seq, int32_t d_head,
                           int32_t per_slot, void* stream);

/* Eq. (8) similarity of every token: scores[slot, t] (fp64) = cosine of
 * v_cur and v_ref rows (layout [n_slots, H, seq, d_head]; a token's row is
 * its d_head slices over all heads), products and sums in fp64; 1 if both
 * rows are zero, 0 if one is.  With update_ref != 0, v_ref receives v_cur
 * afterwards.  d_head % 8 == 0; v_cur and v_ref 16-byte aligned
 * (MAR_E_ARG otherwise). */
mar_status mar_k_scores(int32_t dtype, const void* v_cur, void* v_ref, int32_t n_slots, int32_t n_heads,
                        int32_t seq, int32_t d_head, double* scores, int32_t update_ref, void* stream);

/* Eq. (8) selection: idx[slot, 0..n) = the n tokens of the slot with the
 * smallest score (NaN ranks as +inf, ties to the lower index), ascending.
 * seq <= 4096. */
mar_status mar_k_select(const double* scores, int32_t n_slots, int32_t seq, int32_t n, int32_t* idx,
                        void* stream);

/* The opposite ranking (Table 3, the strategy that caches the
 * minimum-similarity tokens): idx[slot, 0..n) = the n tokens of the slot
 * with the largest score (NaN ranks last, ties to the lower index),
 * ascending.  seq <= 4096. */
mar_status mar_k_select_most_similar(const double* scores, int32_t n_slots, int32_t seq, int32_t n,
                                     int32_t* idx, void* stream);

/* Tuning hook: force tile configuration `variant` (0 .. MAR_GEMM_VARIANTS-1)
 * for every later matrix product of the process, or -1 to restore the
 * choice by shape (which also knows the tiles for few rows, not named here).
 * Every configuration sums the k of an output in the same order, so results
 * do not change by a single bit.
 * Not thread-safe with concurrent launches. */
#define MAR_GEMM_VARIANTS 16
mar_status mar_k_gemm_variant(int32_t variant);

/* ---------------------------------------------------------------------------
 * Positions, the paged key/value cache and its attention: next to the slots of
 * one fixed length above, a cache whose sequences grow page by page (several
 * images or frames after each other, prompts of any length), share key/value
 * heads between query heads, and may be causal.
 *
 * Rows of a batch are ragged: sequence s owns rows q_start[s] ..
 * q_start[s + 1] - 1 of every row matrix, its n new tokens, and holds
 * kv_len[s] tokens with them: its row i is token kv_len[s] - n + i.  Row
 * matrices have a row stride of their own (`ld`, elements), so that the column
 * blocks of one product's output can be passed in place.
 *
 * What a kernel reads from the device it bounds itself: an entry of `table`
 * outside [0, n_pages) names no page (its keys are not visible, what is stored
 * there is dropped), tokens below 0 or at max_kv and above are not stored and
 * not visible, rows of no sequence (behind the last one) are left as they were,
 * a sequence's rows at m and above are not there.  q_start must ascend;
 * otherwise which sequence a row belongs to is undefined, but nothing outside the
 * buffers is touched. */

/* Which elements of a head make pair i of its n_pairs pairs: */
typedef enum {
  MAR_ROTARY_HALVES = 0,    /* (i, i + n_pairs) */
  MAR_ROTARY_NEIGHBOURS = 1 /* (2 i, 2 i + 1) */
} mar_rotary_layout;

/* Rotary positions: pair i of every head of a row turns by the angle
 *   pos[row, axis[i]] * freq[i]   (radians, reduced in fp64),
 * (a, b) -> (a cos - b sin, b cos + a sin); elements from 2 n_pairs on stay.
 * The axes are the caller's (time, height, width, ...): pairs may be divided
 * among them in any way.  An axis outside [0, n_axes) leaves its pairs as they
 * are; negated frequencies turn back. */
typedef struct {
  const double* freq;  /* device [n_pairs] */
  const int32_t* axis; /* device [n_pairs] */
  int32_t n_pairs;     /* multiple of 8, 8 <= n_pairs <= d_head / 2 */
  int32_t n_axes;      /* 1 .. 4 */
  int32_t layout;      /* mar_rotary_layout */
} mar_rotary;

/* The pages of a cache and a batch of sequences that live in them.  Token t of
 * sequence s is row t % page of page table[s, t / page].  Pages of one
 * sequence need no order, and sequences may share pages that none of them
 * stores to.  k, v: 16-byte aligned.  page: a power of two, 16 .. 4096.
 * d_head: a multiple of 16, 16 .. 128.  max_kv bounds every kv_len
 * (1 <= max_kv <= max_pages * page <= 2^30): work is divided for that many
 * keys, so a bound far above the lengths leaves few workgroups to each of them.
 * n_heads <= 4096, n_seqs <= 65536. */
typedef struct {
  void *k, *v;            /* device [n_pages, n_heads, page, d_head] in dtype */
  const int32_t* table;   /* device [n_seqs, max_pages] */
  const int32_t* q_start; /* device [n_seqs + 1] */
  const int32_t* kv_len;  /* device [n_seqs], the new tokens included */
  int32_t n_pages, n_heads, page, d_head, n_seqs, max_pages, max_kv;
} mar_paged_batch;

/* out[m, n_heads * d_head] = rotary positions of the rows of x (head h at
 * columns h * d_head ...), pos [m, n_axes] int32.  fp32 arithmetic, one
 * rounding.  ld_x, ld_out: multiples of 8, at least n_heads * d_head; x and
 * out 16-byte aligned; out may be x itself (same pointer and stride), else
 * they must not overlap.  m * n_heads < 2^30. */
mar_status mar_k_rotary(int32_t dtype, const mar_rotary* rotary, const void* x, int64_t ld_x,
                        const int32_t* pos, int32_t m, int32_t n_heads, int32_t d_head, void* out,
                        int64_t ld_out, void* stream);

/* New tokens into the cache: keys k (rotated) and values v, [m, batch->n_heads
 * * d_head] each, go to their pages; with q given, its n_heads_q heads are
 * rotated into q_out (which may be q itself).  rotary NULL (pos is then
 * ignored): no rotation, keys are stored and queries copied as they are.
 * Strides, alignment and overlaps as in mar_k_rotary; k, v, q and q_out must not
 * overlap the pages.  Two rows must not name the same place in the cache. */
mar_status mar_k_paged_store(int32_t dtype, const mar_paged_batch* batch, const mar_rotary* rotary,
                             const int32_t* pos, int32_t m, const void* k, int64_t ld_k, const void* v,
                             int64_t ld_v, int32_t n_heads_q, const void* q, int64_t ld_q, void* q_out,
                             int64_t ld_q_out, void* stream);

/* Attention of every row of the batch over its sequence's tokens in the cache:
 * q, out [m, n_heads_q * d_head], n_heads_q a multiple of batch->n_heads (query
 * head h reads key/value head h / (n_heads_q / batch->n_heads)), scale
 * 1/sqrt(d_head), softmax statistics and sums in fp32.  In bf16 the weights, up to
 * 2^13 before they are divided by their sum, are rounded to bf16 for the product
 * with the values, and the rounded ones are summed.  Finite values stay finite as
 * long as |v| * (kv_len + 32) < 2^118.  The row at token p sees token j of its
 * sequence if
 *   j < kv_len,  (not causal, or j <= p),
 *   (window == 0, or j > p - window, or j < sinks):
 * with a window the last `window` tokens up to its own, and the first `sinks`
 * ones; without `causal` every token after it too.  A row that sees no token
 * becomes zeros, one whose scores are all -infinity NaN (0 / 0); what unseen
 * tokens hold (infinities, NaN) does not matter.
 * out must not overlap q or the pages.
 *
 * workspace: device, 16-byte aligned, of mar_k_paged_attention_workspace_bytes
 * (or NULL with 0 bytes): where few rows read long sequences, their keys are
 * divided among workgroups that leave their parts there.  A smaller one will
 * do, with fewer parts and in less haste.  Calls that may overlap (on two
 * streams, in two graphs) need a workspace each.  Sums are taken in an order
 * that depends on the host's arguments and the lengths alone: equal calls give
 * equal bits. */
mar_status mar_k_paged_attention(int32_t dtype, const mar_paged_batch* batch, int32_t m, int32_t n_heads_q,
                                 const void* q, int64_t ld_q, int32_t causal, int32_t window, int32_t sinks,
                                 void* workspace, size_t workspace_bytes, void* out, int64_t ld_out,
                                 void* stream);

/* Bytes of workspace that mar_k_paged_attention makes use of (0 if none, or if
 * an argument is refused; mar_last_error() then says why). */
size_t mar_k_paged_attention_workspace_bytes(int32_t dtype, const mar_paged_batch* batch, int32_t m,
                                             int32_t n_heads_q, int32_t window, int32_t sinks);

#ifdef __cplusplus
}
#endif

#endif /* MAR_KERNELS_H */
