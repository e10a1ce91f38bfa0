/*
 * mohge_block.h — what stands around the MoHGE layer in a decoder block, for MI355X (gfx950): the
 * root-mean-square norm in front of it with the residual's addition (forward and backward), and for
 * decoding a paged cache of keys and values, attention of one new token per sequence over it, and the
 * product with 4-bit weights of the projections.  Part of libmohge.so.
 *
 * Conventions (return codes, DEVICE pointers and their alignment, streams, mohge_last_error) are those of
 * mohge.h: calls only enqueue kernels, allocate nothing and keep nothing.  Sums, statistics and softmax
 * weights are fp32.  E4M3 codes (one byte each) and their conversion are those of mohge_expert_ffn_w8:
 * the value is scale * value(code), where a row of n values x has
 *   scale = max(max|x| * (1/448), 2^-126), or 1 for a row of zeros, and code = x * (1/scale) rounded to nearest even,
 * reciprocals and products in fp32, each rounded to nearest.  (For bf16 x the codes are those of x / scale too.)
 */
#ifndef MOHGE_BLOCK_H
#define MOHGE_BLOCK_H

#include "mohge.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { MOHGE_E4M3 = 2 };    /* next to MOHGE_F32 and MOHGE_BF16, where a call says so */

/* ---- Norm -------------------------------------------------------------------------------------- */

typedef struct mohge_norm_config {
  int32_t T;         /* rows (tokens), 0..2^21                                                     */
  int32_t d;         /* columns: a multiple of 8, 8..32768                                         */
  int32_t dtype;     /* MOHGE_F32 or MOHGE_BF16: x, residual, sum_out, dy, h, dsum, dx             */
  int32_t y_dtype;   /* dtype, or MOHGE_E4M3: y as codes with one scale per row                    */
  float eps;         /* added to the mean of the squares, >= 0                                     */
} mohge_norm_config;

/*
 * h = x + residual (h = x without one), rstd_t = 1 / sqrt(mean_j h_tj^2 + eps), y_tj = h_tj rstd_t weight_j.
 * In:  x DEVICE [T,d]; residual DEVICE [T,d] or NULL; weight DEVICE [d] f32.
 * Out: sum_out DEVICE [T,d] = h or NULL (may be x or residual itself); y DEVICE [T,d]; y_scale DEVICE [T] f32,
 *      required for MOHGE_E4M3 and NULL otherwise; rstd DEVICE [T] f32 or NULL (the backward pass reads it).
 * The statistic and y are those of the fp32 sum, before it is rounded for sum_out.  (A row whose sum of squares passes the largest fp32
 * number has rstd = 0 and y = 0.)
 */
int mohge_rmsnorm(const mohge_norm_config* cfg, const void* x, const void* residual, const float* weight,
                  void* sum_out, void* y, float* y_scale, float* rstd, void* stream);

/*
 * Backward: with n_tj = h_tj rstd_t and g_tj = weight_j dy_tj,
 *   dx_tj = dsum_tj + rstd_t (g_tj - n_tj mean_k(g_tk n_tk)),   dweight_j = sum_t dy_tj n_tj.
 * dx is the gradient of x and of residual alike.
 * In:  dy DEVICE [T,d]; h DEVICE [T,d] = sum_out (x where there was no residual); weight; rstd as written by
 *      mohge_rmsnorm; dsum DEVICE [T,d], the gradient that reaches h past the norm, or NULL.
 * Out: dx DEVICE [T,d] (may be dy or dsum itself); dweight DEVICE [d] f32, overwritten (zero for T = 0).
 * workspace DEVICE, mohge_norm_workspace_size(cfg) bytes (it depends on d alone).  y_dtype is not looked at.
 * The sums over tokens have a fixed order (deterministic).
 */
int mohge_rmsnorm_bwd(const mohge_norm_config* cfg, const void* dy, const void* h, const float* weight,
                      const float* rstd, const void* dsum, void* dx, float* dweight, void* workspace,
                      size_t workspace_bytes, void* stream);
size_t mohge_norm_workspace_size(const mohge_norm_config* cfg);

/* ---- Paged cache of keys and values, and attention over it --------------------------------------- */

/*
 * k_pages and v_pages are DEVICE [n_pages, n_kv_heads, page_size, head_size] (cache_dtype); with MOHGE_E4M3,
 * k_scale and v_scale are DEVICE [n_pages, n_kv_heads, page_size] f32, one scale per position and head.
 * Position p of sequence b is row p % page_size of page block_table[b, p / page_size].
 * block_table DEVICE [n_seqs, max_pages]: entries past the page of a sequence's last position are not read.
 * seq_lens DEVICE [n_seqs]: positions of every sequence, the new ones of the step among them.
 */
typedef struct mohge_cache_config {
  int32_t n_seqs;
  int32_t n_heads;      /* query heads, a multiple of n_kv_heads; query head h reads kv head h / (n_heads / n_kv_heads) */
  int32_t n_kv_heads;
  int32_t head_size;    /* 64, 128 or 256                                                          */
  int32_t page_size;    /* 16, 32, 64, 128 or 256                                                  */
  int32_t n_pages;
  int32_t max_pages;    /* columns of block_table; max_pages * page_size <= 2^30                   */
  int32_t dtype;        /* MOHGE_F32 or MOHGE_BF16: q, k, v, out                                   */
  int32_t cache_dtype;  /* dtype, or MOHGE_E4M3 with MOHGE_BF16                                    */
} mohge_cache_config;

/*
 * Writes new keys and values into their pages.  Sequence b has the rows tok_offsets[b] .. tok_offsets[b+1] - 1 of
 * k and v as its last positions: row i is position seq_lens[b] - (tok_offsets[b+1] - i).
 * In:  n_tokens rows in all; k, v DEVICE [n_tokens, n_kv_heads, head_size] (dtype) with k_stride and v_stride elements
 *      from row to row (multiples of 8, at least n_kv_heads * head_size): slices of the projection's output
 *      need no copy; tok_offsets DEVICE [n_seqs+1] ascending from 0 to n_tokens, or NULL for one row per sequence
 *      (n_tokens = n_seqs).
 * A row whose position is outside the block table, or whose page number is outside 0..n_pages-1, is not written
 * (a sequence that is to sit a step out has seq_lens[b] = 0, or no rows).
 */
int mohge_cache_append(const mohge_cache_config* cfg, int32_t n_tokens, const void* k, int64_t k_stride,
                       const void* v, int64_t v_stride, const int32_t* tok_offsets, const int32_t* block_table,
                       const int32_t* seq_lens, void* k_pages, void* v_pages, float* k_scale, float* v_scale,
                       void* stream);

/*
 * Attention of one query row per sequence over all its positions, n = seq_lens[b]:
 *   s_j = scale q . k_j,   out = sum_{j<n} softmax(s)_j v_j,   lse = log sum_{j<n} exp s_j.
 * A sequence of length 0, or whose scores are all -infinity, gives out = 0 and lse = -infinity.  An infinite value in a position that counts
 * gives an infinite element or NaN.
 * In:  q DEVICE [n_seqs, n_heads, head_size] (dtype), q_stride elements from sequence to sequence (a multiple of 8, at
 *      least n_heads * head_size).
 * Out: out DEVICE [n_seqs, n_heads, head_size] (dtype); lse DEVICE [n_seqs, n_heads] f32 or NULL.
 * A sequence that is longer than its block table, or that has a page number outside 0..n_pages-1 among the pages
 * it reads, gets NaN (out and lse): a wrong number can never pass for a result.
 * workspace DEVICE, mohge_cache_workspace_size(cfg) bytes (a few MB, whatever the lengths; never less for more sequences).  It
 * holds counters that MUST BE ZERO when the call starts and that the call leaves zero: clear it once (hipMemset) and keep
 * it for calls of one cfg, issued in stream order; calls that overlap on one workspace race.  Were the counters not zero, results that
 * are joined from parts are NaN, in this call and in later ones, until the workspace is cleared.
 * The positions of all sequences are divided evenly over the workgroups, by the lengths found on the device; parts are
 * joined in a fixed order (deterministic).
 */
int mohge_cache_attention(const mohge_cache_config* cfg, const void* q, int64_t q_stride, const int32_t* block_table,
                          const int32_t* seq_lens, const void* k_pages, const void* v_pages, const float* k_scale,
                          const float* v_scale, float scale, void* out, float* lse, void* workspace,
                          size_t workspace_bytes, void* stream);
size_t mohge_cache_workspace_size(const mohge_cache_config* cfg);

/* ---- Product with 4-bit weights ------------------------------------------------------------------- */

typedef struct mohge_proj_config {
  int32_t T;         /* rows of x, 0..32                                                           */
  int32_t n_in;      /* a multiple of group                                                        */
  int32_t n_out;     /* >= 1                                                                       */
  int32_t group;     /* weights of a row that share a scale: 32, 64 or 128                         */
  int32_t x_dtype;   /* MOHGE_BF16, or MOHGE_E4M3 with one scale per row (as mohge_rmsnorm writes it) */
  int32_t y_dtype;   /* MOHGE_BF16 or MOHGE_F32                                                    */
} mohge_proj_config;

/*
 * y[t,n] = sum_k x[t,k] w[n,k],   w[n,k] = scales[n, k / group] * (code[n,k] - zeros[n, k / group]).
 * In:  x DEVICE [T, n_in]; x_scale DEVICE [T] f32, required for MOHGE_E4M3 and NULL otherwise;
 *      codes DEVICE [n_out, n_in/2] bytes: two 4-bit codes 0..15 per byte, the element with the even index in the
 *      low four bits; scales DEVICE [n_out, n_in/group] bf16; zeros DEVICE [n_out, n_in/group] bytes 0..15, or NULL: 8.
 * Out: y DEVICE [T, n_out].
 * Codes and x are exact in the matrix cores' bf16 operands; sums are fp32, a group's sum is multiplied by its scale.
 * Infinite x give what the definition gives (infinities, NaN where a code is its zero point or both signs meet); such rows take longer.
 */
int mohge_proj_w4(const mohge_proj_config* cfg, const void* x, const float* x_scale, const void* codes,
                  const void* scales, const void* zeros, void* y, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* MOHGE_BLOCK_H */
