/*
 * jq_block.h -- C ABI of the operators of libjq that stand around a decoder
 * block's W4A4 linears (jq.h) when a model is served: the RMS norm that feeds
 * a quantised linear, an 8-bit linear for the layers that do not take 4 bits,
 * the rotation of new queries and keys with their append to a paged cache, and
 * the attention of the new tokens over that cache.
 *
 * The conventions are those of jq.h: device pointers owned by the caller,
 * asynchronous on `stream`, nothing allocated, synchronised or printed,
 * arguments checked before anything is launched (on any error nothing is
 * written), no global state.  What the host cannot see (positions, slots, page
 * numbers, lengths) is checked on the device, as stated at each call; no value
 * of them makes a call read or write outside the arrays that it is given.
 *
 * e4m3 is the 8-bit float without infinities (largest 448), one byte a code.
 * A scale of a set of values v is
 *     s = max(fl32(max|v| * fl32(1 / 448)), 2^-126),  or 0 where every v is 0,
 * and its codes are rne_e4m3(fl32(v / s)), 0 where s = 0.  An
 * infinity or NaN among the values makes the scale an infinity or NaN, so it
 * shows in whatever is computed from the codes.
 */
#ifndef JQ_BLOCK_H
#define JQ_BLOCK_H

#include <stddef.h>
#include <stdint.h>

#include "jq.h"

#ifdef __cplusplus
extern "C" {
#endif

/* What jq_rmsnorm writes. */
typedef enum {
  JQ_NORM_BF16 = 0, /* y [M,D] bf16 */
  JQ_NORM_FP8 = 1,  /* y [M,D] e4m3, scale [M, ceil(D/128)]: the operand of jq_fp8_gemm */
  JQ_NORM_INT4 = 2  /* y [M,D/2] packed int4, scale [M]: the operand of jq_w4a4_gemm */
} jq_norm_out;

/*
 * RMS norm with the residual's addition, per row, in fp32 with one rounding at
 * the end:
 *     h = x + residual        (h = x where residual is NULL)
 *     residual_out = bf16(h)  (only with a residual)
 *     y = (h * r) * weight,   r = 1 / sqrt(mean(h^2) + eps)
 * JQ_NORM_BF16 rounds y to bf16.  JQ_NORM_FP8 quantises each 128 columns of y
 * as above.  JQ_NORM_INT4 takes s = fl32(max|y| / 7) of the row and
 * clamp(rne(fl32(y / s)), -8, 7), the rule of jq_quantize_act, on the fp32 y.
 * Where the sum of squares passes fp32's range (|h| near 2^64), r is 0.
 *   x            in   [M,D] bf16, rows x_stride elements apart
 *   residual     in   [M,D] bf16, rows residual_stride apart, or NULL
 *   weight       in   [D] bf16
 *   y            out  contiguous, by `out`
 *   scale        out  fp32, by `out`; NULL for JQ_NORM_BF16
 *   residual_out out  [M,D] bf16, rows residual_out_stride apart; it may be
 *                     `residual` itself (or x) with the same stride; NULL if
 *                     and only if residual is NULL
 * D % 8 == 0 (for JQ_NORM_INT4, D % 64 == 0, which jq_w4a4_gemm asks for too),
 * D <= 65536, M <= 2^30; strides >= D and % 8 == 0; matrix pointers and weight
 * 16-byte aligned.
 * Errors: JQ_ERR_INVALID_ARG, JQ_ERR_UNSUPPORTED_SHAPE, JQ_ERR_MISALIGNED, JQ_ERR_HIP.
 */
jq_status jq_rmsnorm(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride,
                     const void* weight, int64_t M, int64_t D, float eps, jq_norm_out out, void* y, float* scale,
                     void* residual_out, int64_t residual_out_stride, void* stream);

/*
 * Activations of the 8-bit linear: x [M,K] bf16 (rows x_stride apart) to e4m3
 * codes q [M,K] with a scale for each row and 128 columns, scale
 * [M, ceil(K/128)] (the last block of a row may be short).
 * K % 16 == 0, 16 <= K <= 65536, M <= 2^30 and M * ceil(K/512) < 2^31;
 * x_stride >= K and % 8 == 0; x and q 16-byte aligned.
 */
jq_status jq_quantize_act_fp8(const void* x_bf16, int64_t x_stride, int64_t M, int64_t K, void* q, float* scale,
                              void* stream);

/*
 * Weights of the 8-bit linear, once when a model is loaded: w [N,K] bf16 to
 * e4m3 codes wq [N,K] with a scale for each 128 rows x 128 columns, w_scale
 * [ceil(N/128), ceil(K/128)].  Sizes as above.
 */
jq_status jq_pack_weight_fp8(const void* w_bf16, int64_t N, int64_t K, void* wq, float* w_scale, void* stream);

/* Bytes of workspace of jq_fp8_linear for an [M,K] input: its codes and their
 * scales, each rounded up to 256 bytes.  0 for invalid sizes. */
size_t jq_fp8_workspace_bytes(int64_t M, int64_t K);

/*
 * The product of the 8-bit linear on quantised activations:
 *     y[m,n] = bf16( sum_b (scale[m,b] * w_scale[n/128,b]) * sum_{k in b} q[m,k] * wq[n,k]  + bias[n] )
 * with blocks b of 128 k.  A block's sum is taken by the matrix cores in fp32,
 * which cut the products of eight neighbouring k at 2^-14 of the largest of them;
 * the sum over blocks and the bias are fp32, rounded once to bf16.  Products
 * with few output tiles add their blocks in several interleaved runs, in an
 * order that depends on the shape alone.
 *   q, scale     in   [M,K] e4m3, [M, ceil(K/128)] fp32
 *   wq, w_scale  in   [N,K] e4m3, [ceil(N/128), ceil(K/128)] fp32
 *   bias_bf16    in   [N] bf16, or NULL
 *   y_bf16       out  [M,N] bf16
 * K % 16 == 0, 16 <= K <= 65536; M <= 2^30, N <= 2^22, M * N < 2^38; q, wq and
 * y 16-byte aligned.
 */
jq_status jq_fp8_gemm(const void* q, const float* scale, int64_t M, int64_t K, const void* wq, const float* w_scale,
                      int64_t N, const void* bias_bf16, void* y_bf16, void* stream);

/* The whole 8-bit linear: jq_quantize_act_fp8 into the workspace (256-byte
 * aligned, at least jq_fp8_workspace_bytes(M,K)), then jq_fp8_gemm. */
jq_status jq_fp8_linear(const void* x_bf16, int64_t x_stride, int64_t M, int64_t K, const void* wq,
                        const float* w_scale, int64_t N, const void* bias_bf16, void* y_bf16, void* workspace,
                        size_t workspace_bytes, void* stream);

/* What a paged cache holds. */
typedef enum {
  JQ_CACHE_BF16 = 0,
  JQ_CACHE_FP8 = 1 /* e4m3 codes with an fp32 scale for each token and head */
} jq_cache_type;

/*
 * Rotation and append.  Queries and keys of T new tokens are rotated by their
 * positions, on the first R elements of each head:
 *     (a, b) -> (a c - b s, a s + b c),  c, s = cos, sin[position, i], i < R/2,
 * of the pairs (i, i + R/2), or (2i, 2i + 1) if `interleaved`; queries go to
 * q_out, keys and the (unrotated) values into the cache.
 *   q            in   [T,Hq,D] bf16, tokens q_stride elements apart (NULL with Hq = 0: append only)
 *   k, v         in   [T,Hk,D] bf16, tokens k_stride, v_stride apart
 *   positions    in   [T] int32, rows of the tables
 *   cos, sin     in   [P, R/2] fp32
 *   slots        in   [T] int64: page * page_size + place in the page
 *   q_out        out  [T,Hq,D] bf16, tokens q_out_stride apart; it may be q itself
 *   k_cache, v_cache   [num_pages, Hk, page_size, D], bf16 or e4m3
 *   k_scale, v_scale   [num_pages, Hk, page_size] fp32 for JQ_CACHE_FP8, else NULL
 * A token whose slot lies outside [0, num_pages * page_size), as -1 does, is
 * not appended.  A position outside [0, P) gives NaN in the rotated elements
 * (and, by its scale, in the whole key of an 8-bit cache).  What a slot holds
 * that two tokens of one call share is unspecified: a token and head is written
 * by several stores, so it may be parts of both, an 8-bit cache's codes of one
 * beside the scale of the other.  No other slot is affected.
 * D % 16 == 0, 16 <= D <= 256 (jq_paged_attention reads caches of D = 64, 128 and
 * 256); R % 16 == 0, 0 <= R <= D (cos and sin may be
 * NULL with R = 0); page_size a power of two, 16 .. 65536; strides % 8 == 0 and
 * at least a token's elements; T * (Hq + 2 Hk) < 2^31; pointers 16-byte
 * aligned (positions, scales 4, slots 8).
 */
jq_status jq_rope_append(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                         int64_t v_stride, int64_t T, int64_t Hq, int64_t Hk, int64_t D, const int32_t* positions,
                         const float* cos, const float* sin, int64_t P, int64_t R, int interleaved,
                         const int64_t* slots, void* q_out, int64_t q_out_stride, void* k_cache, void* v_cache,
                         float* k_scale, float* v_scale, int64_t num_pages, int64_t page_size, jq_cache_type type,
                         void* stream);

/* Bytes of workspace of jq_paged_attention (0 where none is needed, and for
 * invalid sizes). */
size_t jq_paged_attention_workspace_bytes(int64_t B, int64_t Tq, int64_t Hq, int64_t Hk, int64_t D, int64_t max_len);

/*
 * Attention of each sequence's Tq newest tokens over its cached tokens, the
 * new ones (already appended) among them:
 *     out = sum_t p_t v_t,  p = softmax over visible t of sm_scale * (q . k_t)
 * A token t is visible if t < lens[b] and, for causal calls, t <= lens[b] - Tq + i
 * for new token i.  A query that sees no token gives zeros, and lse = -inf.
 * Query head h reads key head h / (Hq / Hk).
 *   q            in   [B,Tq,Hq,D] bf16
 *   k_cache, v_cache, k_scale, v_scale, num_pages, page_size, type: as jq_rope_append
 *   page_table   in   [B,table_cols] int32: the pages of a sequence in order
 *   lens         in   [B] int32; a length above max_len counts as max_len, one
 *                     below 0 as 0
 *   out          out  [B,Tq,Hq,D] bf16
 *   lse          out  [B,Tq,Hq] fp32 log of the softmax's denominator (natural
 *                     logarithm, with the maximum in it), or NULL
 *   workspace    at least jq_paged_attention_workspace_bytes, 256-byte aligned
 *                     (NULL where that is 0)
 * A page number outside [0, num_pages) among those that a sequence's length
 * reaches makes its outputs NaN; entries past those are not read.  Of a
 * sequence's last page, places past its end may be read (up to the end of a group
 * of 16 tokens), whatever they hold, and count for nothing.
 * An infinity or NaN among a token's cached values reaches the queries that see
 * the token, and no other; a score of -infinity is a weight of 0, and a query with
 * no other scores is as one that sees nothing.
 * D = 64, 128 or 256; Hq % Hk == 0; page_size as above;
 * max_len <= table_cols * page_size, max_len <= 2^30; B * Tq * Hq < 2^24, and so
 * the parts that the key axis is cut into, over all sequences and heads.
 */
jq_status jq_paged_attention(const void* q, const void* k_cache, const void* v_cache, const float* k_scale,
                             const float* v_scale, const int32_t* page_table, int64_t table_cols,
                             const int32_t* lens, int64_t B, int64_t Tq, int64_t Hq, int64_t Hk, int64_t D,
                             int64_t num_pages, int64_t page_size, int64_t max_len, float sm_scale, int causal,
                             jq_cache_type type, void* out, float* lse, void* workspace, size_t workspace_bytes,
                             void* stream);

#ifdef __cplusplus
}
#endif

#endif /* JQ_BLOCK_H */
