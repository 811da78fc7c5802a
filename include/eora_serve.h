/*
 * eora_serve.h -- what a serving step needs around and beside the compensated layers of eora_linear.h (same library,
 * same conventions): low-rank adapters of many requests, head norms with the position rotation, a paged key-value
 * cache, and the attention of one new token over it.  A decoder block of a served model is then
 *
 *     q|k|v  eora_linear_forward_fused, with eora_adapters_forward where requests have adapters of their own
 *            eora_qk_norm_rope: norms, rotation, the new keys and values into the cache
 *            eora_attention_forward over the cache
 *     o      eora_linear_forward (+ adapters);  gate|up, down likewise
 *
 * (The paper's method ends at the projections, Eq. 4; Section 3 has the low-rank modules of several tasks switched on and
 * off beside one compressed model, which eora_adapters_forward does for a batch.)
 *
 * All pointers are DEVICE pointers, caller-owned; nothing here is a torch type.  Every function returns an int status
 * (codes of eora_linear.h); nothing throws, aborts or traps; nothing synchronises or allocates; work is enqueued on
 * `stream` (a cudaStream_t; NULL: the default stream) of the current device, whose memory the pointers must be.  All calls can be captured into a CUDA graph: what changes from step to step (ids, positions, slots,
 * lengths, page tables) is read from device memory by the kernels.  16-bit types: EORA_X_F16 or EORA_X_BF16.  Pointers are
 * 16-byte aligned (those to int32, to scales and to lse: 4-byte), strides are in elements and multiples of 8 (EORA_ERR_MISALIGNED);
 * that of a page table is any.  Arithmetic is fp32 (sums, norms,
 * softmax statistics) with the inputs as 16-bit operands of the matrix products; what is computed on the way into one (t, softmax weights) goes into
 * it as two 16-bit parts.  Results are rounded once.
 * Integers in device memory are not trusted: an id, position, slot, length or page outside its range has the effect stated
 * with the call, never an access out of bounds.
 */
#ifndef EORA_SERVE_H
#define EORA_SERVE_H

#include <stddef.h>

#include "eora_linear.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- low-rank adapters of many requests ------------------------------------------------------------------------------
 *
 *     y[i] = base[i] + scales[j] * (x[i] . A_j[:, :r]) . B_j[:r, :],   j = ids[i],  r = ranks[j]
 *     y[i] = base[i]                                                   where ids[i] is not in [0, n_adapters)
 *
 * beside a projection that all tokens share: base is its output (of eora_linear_forward or any other), y may be base (rows
 * without an adapter are then left as they are).  base == NULL stands for zeros.  Unlike eora_linear_forward_multi, the
 * bank belongs to the caller, who may load another adapter into a slot between calls (stream order is enough); it holds any
 * number of adapters up to 4096; only those that ids name are read; ids are in device memory; and m is up to 2^20.
 *
 *   a  [n_adapters][d_in][max_rank],  b [n_adapters][max_rank][d_out]   row-major, of x's type
 *   ranks  int32 [n_adapters], NULL: all max_rank; clamped to [0, max_rank] (0: no adapter).  Columns of A and rows of B
 *          from an adapter's rank on are not used, whatever they hold.
 *   scales fp32 [n_adapters], NULL: 1
 *   ids    int32 [m]
 * x [m][d_in] and y, base [m][d_out] with row strides.  y and base are of y_dtype (EORA_Y_*); except for base == y,
 * outputs must not overlap inputs.  The sum base + s t B is rounded to y_dtype once; t = x . A is kept as a high and a low
 * 16-bit part, scaled by a power of two per token.  Infinities and NaN in x, A and base give what the formula gives, those of a token in its row
 * only; an infinity in B may come out as NaN.  The order of the sums goes by the config and m alone: a token's result does
 * not depend on what the other tokens of its call are, and the same call gives the same bits.  Keeps no state: calls may overlap.
 * Errors: NULL_ARG, BAD_SHAPE (d_in not a positive multiple of 128, d_out of 32, max_rank not a multiple of 8 in [8, 256],
 * n_adapters not in [1, 4096], m < 0 or above 2^20, a row stride shorter than a row), UNSUPPORTED (types), MISALIGNED, CUDA.
 */
typedef struct {
  int32_t d_in, d_out, max_rank, n_adapters;
  int32_t x_dtype;     /* of x, a and b */
  int32_t y_dtype;     /* of base and y */
} eora_adapters_config;
typedef struct {
  const void* a;
  const void* b;
  const int32_t* ranks;
  const float* scales;
} eora_adapters_weights;
int eora_adapters_forward(const eora_adapters_config* cfg, const eora_adapters_weights* w, const void* x, int64_t x_stride,
                          int32_t m, const int32_t* ids, const void* base, int64_t base_stride, void* y, int64_t y_stride,
                          void* stream);

/* ---- a paged key-value cache -------------------------------------------------------------------------------------------
 *
 * Keys and values of n_pages pages of page_size tokens each.  Channel d of key head h of the token in row `row` of page p is
 *     k[p * page_stride + h * head_stride + row * token_stride + d]
 * (v with the same strides), so both orders of heads and tokens, and K and V interleaved in one buffer, are expressed by
 * strides; [page][head][token][channel] is the one that the attention reads in the longest runs.  A slot is
 * page * page_size + row.  page_size is a power of two; n_pages * page_size <= 2^31 - 1.
 */
typedef struct {
  void* k;
  void* v;
  int64_t page_stride, head_stride, token_stride;
  int32_t n_pages, page_size, n_kv_heads, head_dim;
  int32_t dtype;
} eora_kv_cache;

/* ---- norms of queries and keys, rotation, cache write ------------------------------------------------------------------
 *
 * For each of m tokens and each head of q [m][n_heads * head_dim] and k [m][n_kv_heads * head_dim]:
 *     u = x * rsqrt(mean(x^2) + eps) * w        (w: q_weight / k_weight [head_dim] of the inputs' type; NULL: u = x)
 *     (u_a, u_b) -> (u_a c - u_b s, u_b c + u_a s)   for the rot_dim / 2 pairs of the first rot_dim channels
 * where pair i is (i, i + rot_dim/2) (EORA_ROPE_HALF) or (2i, 2i + 1) (EORA_ROPE_ADJACENT) and
 * c = cos_sin[pos][i], s = cos_sin[pos][rot_dim/2 + i], cos_sin fp32 [n_positions][rot_dim], pos = positions[i].
 * q goes to q_out, k to k_out (NULL: not written) and, with a cache, k and v [m][n_kv_heads * head_dim] to the cache's row
 * slots[i]; a slot outside the cache (-1) keeps the token out of it.  A token whose position is not in [0, n_positions) is
 * skipped: nothing of it is written anywhere.  Several tokens with one slot: which of them the cache holds is not defined.
 * q_out may be q and k_out may be k (with the same stride); outputs must not overlap inputs otherwise.
 * Row strides (q_stride ...) let q, k and v be columns of one product.  m == 0 is a no-op.  Keeps no state.
 * Errors: NULL_ARG (q, k, q_out, cos_sin or positions missing; a cache without v and slots, v or slots without a cache),
 * BAD_SHAPE (head_dim not a multiple of 16 in [16, 256], rot_dim not a multiple of 16 in [0, head_dim] (0: no rotation,
 * cos_sin may be NULL), heads < 1 or above 1024, n_heads no multiple of n_kv_heads, eps not in [0, inf), m < 0 or above 2^20,
 * strides below a row, a cache of another shape), UNSUPPORTED (types, pairing), MISALIGNED, CUDA.
 */
enum { EORA_ROPE_HALF = 0, EORA_ROPE_ADJACENT = 1 };
typedef struct {
  int32_t n_heads, n_kv_heads, head_dim, rot_dim;
  int32_t pairs;         /* EORA_ROPE_HALF or EORA_ROPE_ADJACENT */
  int32_t dtype;         /* of q, k, v, the weights, the outputs and the cache */
  int32_t n_positions;   /* rows of cos_sin */
  float eps;
  const void* q_weight;
  const void* k_weight;
  const float* cos_sin;
} eora_qk_config;
int eora_qk_norm_rope(const eora_qk_config* cfg, const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                      int64_t v_stride, const int32_t* positions, int32_t m, void* q_out, int64_t q_out_stride, void* k_out,
                      int64_t k_out_stride, const int32_t* slots, const eora_kv_cache* cache, void* stream);

/* ---- attention of one new token per sequence over the cache ------------------------------------------------------------
 *
 * For each of `batch` sequences and each of n_heads query heads (head h reads key head h / (n_heads / n_kv_heads)):
 *     out = sum_t softmax_t(scale q . k_t) v_t,    lse = log sum_t exp(scale q . k_t)   (natural logarithm, fp32)
 * over the tokens t in [max(0, n - window), n), n = lengths[i] (window 0: all), the new token among them (its key and value
 * are in the cache already).  Token t is row t % page_size of page page_table[i * table_stride + t / page_size].
 *   q, out [batch][n_heads * head_dim] with row strides, of the cache's type; out may be q (with the same stride), outputs must not overlap inputs
 *              otherwise; lse fp32 [batch][n_heads], may be NULL
 *   page_table int32 [batch][max_pages] with a row stride; entries behind the last token's page are not read
 *   lengths    int32 [batch]; below 1: no token, out = 0 and lse = -inf; clamped to max_pages * page_size
 * Tokens on a page that is not in [0, n_pages) are left out of the sums.  What the cache holds in rows that no sequence
 * sees (NaN included) has no effect.  Infinities and NaN in what one sees give what the formula gives, in the heads and channels that they reach:
 * out is NaN where a score is +inf or NaN or all scores are -inf (lse then inf, NaN or -inf); where only some scores are -inf, those tokens count nothing;
 * an infinity in v is one in out (NaN where the token's weight is below 2^-29 of the largest).  Rows of out behind `batch` are not touched.
 * The sums are split over the cache's length and joined in a fixed order: the same call gives the same bits.
 *
 * workspace: eora_attention_workspace_bytes(cfg) bytes (0 for a config that is refused), zeroed by the caller before its first
 * use; a call leaves it as the next one expects it.  Calls that may overlap on the GPU need workspaces of their own (in stream
 * order one serves all, graphs that were captured with it too, as long as they are replayed one after the other).
 * batch == 0 is a no-op.
 * Errors: NULL_ARG, BAD_SHAPE (head_dim not 64, 96, 128 or 256; heads < 1 or above 1024, n_heads no multiple of n_kv_heads;
 * max_batch not in [1, 65536]; max_pages < 1; max_pages * page_size above 2^30; window < 0; scale not finite and
 * positive; a cache of another shape than the config's; strides below a row; a workspace that is too small),
 * M_TOO_LARGE (batch > max_batch), UNSUPPORTED (types), MISALIGNED, CUDA.
 */
typedef struct {
  int32_t n_heads, n_kv_heads, head_dim, dtype;
  int32_t page_size, max_pages;      /* of a sequence */
  int32_t max_batch;
  int32_t window;
  float scale;
} eora_attention_config;
size_t eora_attention_workspace_bytes(const eora_attention_config* cfg);
int eora_attention_forward(const eora_attention_config* cfg, const void* q, int64_t q_stride, const eora_kv_cache* cache,
                           const int32_t* page_table, int64_t table_stride, const int32_t* lengths, int32_t batch, void* out,
                           int64_t out_stride, float* lse, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* EORA_SERVE_H */
