/*
 * smetric_kv.h -- C ABI of libsmetric.so, the instance's side of a routed request: the paged
 * KV cache behind the blocks that the router matches, on one MI355X (gfx950).
 *
 * The router sends a request to the instance that holds c blocks of its prompt (Sec. 4.1);
 * the instance computes the L - B c tokens that are left and caches them (Sec. 2), which is
 * what Eq. (1) prices: work per new token, and the attention of the new tokens over
 * everything before them.  This header holds the operators of that step which touch the
 * cache, for a ragged batch of requests with one new token each (decoding), a few (drafts
 * to be checked) or thousands (a prompt's chunk), mixed as they come:
 *   smetric_qk_rotate     queries and keys normed per head and rotated to their positions
 *   smetric_kv_append     the same with the keys and the values entered into the pages
 *   smetric_kv_read       cached tokens read back as activations
 *   smetric_attend_plan   how a step's attention is split over the GPU (once per step)
 *   smetric_attend        the attention of the new tokens over the pages (once per layer)
 *   smetric_attend_scores the same with capped scores, or a bias by distance
 *
 * Conventions are those of smetric.h: device pointers unless marked (host), no allocation,
 * work enqueued on `stream`, host-visible errors returned with nothing enqueued, and errors
 * in device-resident inputs found by the kernels, which never read or write out of bounds
 * for them and set `status` (device int32, optional: NULL) to SMETRIC_EINVAL if it is 0.
 */
#ifndef SMETRIC_KV_H
#define SMETRIC_KV_H

#include "smetric.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types.  Activations are BF16 or F16; a cache has the activations' type or
 *   E4M3  the 8-bit float without infinities, largest value 448, with one scale per head
 *   E2M1  the 4-bit float +-{0, 0.5, 1, 1.5, 2, 3, 4, 6} (codes 0 .. 7, 8 for the sign), two in a
 *         byte, the even component in the lower half, and for every 32 neighbouring components of a
 *         head's token an exponent byte e: a stored x stands for x 2^(e - 127), for NaN where e
 *         is 255.  4.25 bits a component. */
enum { SMETRIC_BF16 = 0, SMETRIC_F16 = 1, SMETRIC_E4M3 = 2, SMETRIC_E2M1 = 3 };

/* An activation of shape [n_tokens, heads, head_dim]: components are contiguous, tokens and
 * heads any number of elements apart that keeps every head 16-byte aligned (a slice of a
 * fused product of queries, keys and values is one). */
typedef struct smetric_heads {
  void *data;
  int64_t token_stride, head_stride; /* elements, multiples of 8 */
} smetric_heads;

/* The exponent bytes of E2M1 pages: that of components 32 g .. 32 g + 31 of (page, head, token) is
 * k[page * k_stride[0] + head * k_stride[1] + token * k_stride[2] + g].  A page's keys' and values'
 * exponents of a head beside each other fill whole lines of memory ([page][head][k, v][token][g]). */
typedef struct smetric_kv_exps {
  uint8_t *k, *v;                    /* aligned to head_dim / 32 bytes */
  int64_t k_stride[3], v_stride[3];  /* bytes, >= 0; multiples of head_dim / 32 */
} smetric_kv_exps;

/* A paged cache: keys and values of n_pages pages of page_size tokens.  Element (page, head,
 * token, component) of the keys is k[page * k_stride[0] + head * k_stride[1] + token *
 * k_stride[2] + component]; [page][head][token] order keeps what one head reads of a page in
 * one piece and is what the kernels are timed with, any other order works. */
typedef struct smetric_kv_cache {
  void *k, *v;                       /* 16-byte aligned */
  int64_t n_pages;                   /* in [1, 2^31) */
  int64_t k_stride[3], v_stride[3];  /* elements, >= 0; multiples of 8 (E4M3: 16, E2M1: 32) */
  int32_t page_size;                 /* tokens, in [1, 65536] */
  int32_t n_kv_heads;
  int32_t head_dim;                  /* 64, 128 or 256 */
  int32_t dtype;
  const float *k_scale, *v_scale;    /* float32[n_kv_heads], E4M3: a stored x stands for x * scale, any number */
  const smetric_kv_exps *exps;       /* (host) E2M1; not read for other types */
} smetric_kv_cache;

/* A ragged batch: request r's new tokens are q_off[r] .. q_off[r+1] of the activations and
 * the last ones of its kv_len[r] tokens in the cache, so new token i is at place
 * kv_len[r] - (q_off[r+1] - q_off[r]) + i of the request; a token with a negative place is
 * padding.  Place p lives in page table[r * table_stride + p / page_size]; entries that no
 * place needs are not read.  Domain: q_off non-decreasing from 0 to n_tokens, kv_len in
 * [0, min(max_pages * page_size, 2^24)], needed pages in [0, n_pages). */
typedef struct smetric_batch {
  const int32_t *table;
  int64_t table_stride; /* >= max_pages */
  int32_t max_pages;    /* entries in a request's row */
  int32_t n_req;
  const int64_t *q_off;  /* int64[n_req + 1] */
  const int32_t *kv_len; /* int32[n_req] */
  int64_t n_tokens;      /* new tokens of the batch, < 2^31 / (query heads per key-value head) */
} smetric_batch;

/* ---------------------------------------------------------------------------------
 * Norm and rotation of one head's components x[0 .. head_dim):
 *   y_j = x_j * w_j / sqrt(mean(x^2) + eps)    with a weight w; y = x without one
 *   pairs (a, b) = (y_i, y_{i + rot_dim/2}), or (y_{2i}, y_{2i+1}) when interleaved, for
 *   i < rot_dim/2:  a' = a cos - b sin,  b' = b cos + a sin,  components from rot_dim on kept
 * computed in float32 and rounded once.
 *   q_weight, k_weight  activation type[head_dim], 16-byte aligned, or NULL: no norm
 *   table               float32[n_pos * rot_dim], row p: the cosines of position p's
 *                       rot_dim/2 angles, then their sines; 16-byte aligned; may be NULL
 *                       with rot_dim = 0 (no rotation)
 *   rot_dim             a multiple of 16 in [0, head_dim]
 * --------------------------------------------------------------------------------- */
typedef struct smetric_rotary {
  const void *q_weight, *k_weight;
  const float *table;
  int64_t n_pos;
  int32_t rot_dim;
  int32_t interleaved;
  float eps; /* >= 0 */
} smetric_rotary;

/* Queries and keys normed and rotated in one pass.
 *   positions  int32[n_tokens]; one outside [0, n_pos) sets status, its token's outputs are
 *              zeros (not read when rot_dim = 0; may then be NULL)
 *   q -> q_out, k -> k_out  may be the same memory with the same strides; a head count of 0
 *              leaves that side out
 * Host errors: EINVAL (bad types, sizes, strides or alignment, null pointers). */
int smetric_qk_rotate(int32_t dtype, int32_t head_dim, int64_t n_tokens, const smetric_rotary *rotary /* host */,
                      const int32_t *positions, int32_t n_q_heads, const smetric_heads *q /* host */,
                      const smetric_heads *q_out /* host */, int32_t n_kv_heads, const smetric_heads *k /* host */,
                      const smetric_heads *k_out /* host */, int32_t *status, hipStream_t stream);

/* The new tokens' keys (normed and rotated) and values (as they are) written to their
 * places in the pages, and, when n_q_heads > 0, their queries normed and rotated into q_out.
 *   rotary     NULL: neither norm nor rotation
 *   positions  int32[n_tokens] or NULL: a token's place in its request is its position
 * A padding token writes nothing to the cache and zeros to q_out; so does one with a bad
 * input (an inconsistent request, page or position), which also sets status.  E4M3 pages
 * hold x / scale rounded to nearest even, saturated at 448 (NaN, also that of 0 / 0, stays NaN).
 * E2M1 pages: 32 components whose largest magnitude is a get e = 127 + k for the smallest k with
 * a <= 7 2^k, in [-125, 125] (F16: [-23, 13]), where the activations' type holds what the codes stand
 * for exactly; x / 2^k is rounded to the nearest code, of two equally near ones to the even one, and
 * saturated at 6, so that no component is further from what it becomes than half of the largest step
 * (bar what F16 keeps in range); a NaN among the 32 makes e 255, all 32 NaN.  Tokens that
 * share a place race; pages shared by requests may be read but not appended to.
 * Host errors: EINVAL. */
int smetric_kv_append(int32_t dtype, const smetric_kv_cache *cache /* host */, const smetric_batch *batch /* host */,
                      const smetric_rotary *rotary /* host */, const int32_t *positions, int32_t n_q_heads,
                      const smetric_heads *q /* host */, const smetric_heads *q_out /* host */,
                      const smetric_heads *k /* host */, const smetric_heads *v /* host */, int32_t *status,
                      hipStream_t stream);

/* Cached tokens read back: row i of request r of k_out and v_out ([n_tokens, n_kv_heads,
 * head_dim] of type `dtype`) is place kv_len[r] - (q_off[r+1] - q_off[r]) + i of the request, as
 * of the new tokens of a step; a whole session's tokens are q_off[r+1] - q_off[r] = kv_len[r].
 * 16-bit pages are copied bit for bit, 8- and 4-bit values times their scale or power of two in
 * float32, rounded once.  Rows of padding are zeros; so are those of a bad input (an inconsistent
 * request or page), which also sets status.  NULL for k_out or v_out leaves that side out.
 * Host errors: EINVAL. */
int smetric_kv_read(int32_t dtype, const smetric_kv_cache *cache /* host */, const smetric_batch *batch /* host */,
                    const smetric_heads *k_out /* host */, const smetric_heads *v_out /* host */, int32_t *status,
                    hipStream_t stream);

/* ---------------------------------------------------------------------------------
 * Attention of the new tokens over the cache.  Query head h reads key-value head
 * h / (n_q_heads / n_kv_heads).  A token at place p sees the request's cached tokens
 * j <= p and, with window > 0, j > p - window:
 *   s_j = scale (q . k_j),  out = sum_j exp(s_j - lse) v_j,  lse = log(sum_j exp(s_j))
 * and out = 0, lse = -inf when it sees nothing.  Scores, maxima, sums and the output are
 * held in float32; exp(s_j - m), with m the largest score so far or at most log(2^8) below it, is
 * rounded to the activations' type for the product with the values and for the sum that this is divided
 * by (F16 loses bits of those below 2^-21 of the largest, BF16 holds 8 of any), not for lse's.  What
 * E2M1 pages hold is rounded to the activations' type first: exact for what smetric_kv_append enters.
 * Tokens that a row does not see change not a bit of it, whatever they hold; nor does what a page holds
 * past kv_len.  Splits are joined in a fixed order, so the same call gives the same bits.
 *
 * The plan holds how the batch's rows and cached tokens are split into pieces of work.  It
 * depends on the lengths alone: one smetric_attend_plan per step serves every layer's
 * smetric_attend with the same scalars, as long as q_off, kv_len and the plan's buffer stay.
 *   max_new  (host) the most new tokens of a request, at least 1: decides the shape of the
 *            pieces; a larger request is computed all the same, less efficiently
 *   plan, workspace  >= the bytes smetric_attend_plan_bytes reports, 256-byte aligned; the
 *            workspace is scratch that calls ordered on one stream may share
 *   lse      float32[n_tokens * n_q_heads] or NULL
 * A batch outside its domain marks the plan invalid (and sets status); smetric_attend then
 * writes zeros, lse -inf, and sets status, as it does for a plan made with other scalars and
 * for a request longer than its table's row.  A page outside [0, n_pages) sets status and
 * leaves its request's rows unspecified.
 * Host errors: EINVAL (bad types, sizes, strides or alignment, null pointers, scale not a
 * positive finite number), EWORKSPACE (short plan or workspace).
 * --------------------------------------------------------------------------------- */
int smetric_attend_plan_bytes(int32_t n_req, int64_t n_tokens, int32_t n_q_heads, int32_t n_kv_heads,
                              int32_t head_dim, int32_t max_new, uint64_t *plan_bytes /* host */,
                              uint64_t *ws_bytes /* host */);
int smetric_attend_plan(const int64_t *q_off, const int32_t *kv_len, int32_t n_req, int64_t n_tokens,
                        int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_new, int32_t window,
                        void *plan, uint64_t plan_bytes, int32_t *status, hipStream_t stream);
int smetric_attend(int32_t dtype, const smetric_kv_cache *cache /* host */, const smetric_batch *batch /* host */,
                   int32_t n_q_heads, const smetric_heads *q /* host */, const smetric_heads *out /* host */,
                   float *lse, float scale, int32_t max_new, int32_t window, const void *plan, uint64_t plan_bytes,
                   void *workspace, uint64_t ws_bytes, int32_t *status, hipStream_t stream);

/* The same attention with other scores: for query head h and a token at place p
 *   s_j = cap tanh(scale (q . k_j) / cap) + slopes[h] (j - p)
 * The plan is smetric_attend_plan's.
 *   cap     0: scores as they are; else a number in [2^-20, 2^20]
 *   slopes  float32[n_q_heads], of either sign, magnitudes up to 2^20, or NULL: no bias
 * Scores are float32's: capped ones are off by some 2^-23 cap of caps up to 64, of larger ones by some
 * 2^-21 of themselves, a bias by (head_dim / 16 + 8) 2^-24 of how far it is below the largest that the
 * row sees.
 * Values' range: BF16 chunks with a cap up to 50.5 and no slopes have a fixed maximum in place of the
 * running one, which values whose magnitude is 0 or in [2^-x, 2^x], x = 115 - 1.443 cap, bear: 2^42
 * either way at 50, 2^71 at 30.  Smaller ones may become zeros there, larger ones infinite.
 * Host errors: smetric_attend's, and EINVAL for another cap. */
typedef struct smetric_scores {
  float cap;
  const float *slopes;
} smetric_scores;
int smetric_attend_scores(int32_t dtype, const smetric_kv_cache *cache /* host */, const smetric_batch *batch /* host */,
                          int32_t n_q_heads, const smetric_heads *q /* host */, const smetric_heads *out /* host */,
                          float *lse, float scale, const smetric_scores *scores /* host */, int32_t max_new, int32_t window,
                          const void *plan, uint64_t plan_bytes, void *workspace, uint64_t ws_bytes, int32_t *status,
                          hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* SMETRIC_KV_H */
