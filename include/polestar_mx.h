/*
 * polestar_mx.h -- a layer's forward in the OCP microscaling formats: rows and
 * weights quantized, products of them, a norm that writes quantized rows, and
 * attention over K/V caches held in 4 bits.  Conventions (device pointers,
 * dense row-major arrays, validation before anything is enqueued, errors,
 * workspaces, streams) are those of polestar.h.
 *
 * Formats (polestar_codec of polestar.h): 32 consecutive channels of a row
 * share a scale 2^e, stored as the byte e + 127 (E8M0).  With amax the block's
 * largest magnitude, e = max(floor(log2 amax) - emax, -127), and -127 for a
 * block of zeros; a channel is v / 2^e rounded to nearest, ties to even, and
 * saturated, without negative zeros:
 *   POLESTAR_MXFP4: E2M1 (emax 2, at most 6), two codes per byte, the lower
 *                   channel in the low nibble, sign in bit 3;
 *   POLESTAR_MXFP8: E4M3 (emax 8, at most 448), one byte per code.
 * A block that holds a NaN or an infinity gets the byte 255 and zero codes; a
 * block with that byte reads as NaN, whatever its codes.  A row of n channels is
 * polestar_codec_row_bytes(fmt, n) bytes of codes and n / 32 bytes of scales,
 * and n % 32 must be 0 (UNSUPPORTED otherwise).  Codes must be 16-byte aligned,
 * scales may start at any byte.
 */
#ifndef POLESTAR_MX_H
#define POLESTAR_MX_H

#include "polestar.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * polestar_mx_quantize -- codes and scales of the rows [row_start, row_start +
 * n_rows) of every sequence.
 *   x : [batch][seq][n] dtype
 *   codes : out [batch][n_rows][row bytes];  scales : out [batch][n_rows][n / 32]
 * Weights are laid out by one call with batch 1, seq = n_rows = n_out.
 * UNSUPPORTED above 65535 sequences or 2^35 channels of one sequence's rows.
 */
polestar_status polestar_mx_quantize(int fmt, polestar_dtype dtype, int batch, int seq, int n, int row_start,
                                     int n_rows, const void* x, uint8_t* codes, uint8_t* scales,
                                     hipStream_t stream);

/*
 * polestar_mx_dequantize -- the values that codes and scales stand for, exact in
 * float and (but for magnitudes below 2^-126) in bf16.
 *   codes : [rows][row bytes];  scales : [rows][n / 32];  y : out [rows][n] dtype
 * rows >= 0 (0: nothing to do).  UNSUPPORTED above 2^35 channels.
 */
polestar_status polestar_mx_dequantize(int fmt, polestar_dtype dtype, long rows, int n, const uint8_t* codes,
                                       const uint8_t* scales, void* y, hipStream_t stream);

/*
 * polestar_mx_linear -- y[r][o] = sum_i x[r][i] w[o][i] over the values that the
 * codes stand for, accumulated in fp32, rounded once to dtype.
 *   x_codes : [rows][row bytes of x_fmt];  x_scales : [rows][n_in / 32]
 *   w_codes : [n_out][n_in / 2] (MXFP4);   w_scales : [n_out][n_in / 32]
 *   y : out [rows][n_out] dtype
 *   workspace : >= polestar_mx_linear_workspace_size(...) bytes (no init; may be
 *               NULL where that is 0)
 * The matrix instruction on MXFP8 rows adds eight neighbouring products at a
 * time with about 14 bits below the largest of them; that error is far below
 * bf16's, and fp32 outputs of MXFP8 rows are computed on bf16 matrix instructions
 * from the decoded values instead, with exact products (but for channels of blocks
 * with scale bytes 0 to 2, which are rounded to multiples of 2^-133).  Results of a
 * magnitude below 2^-126 may be 0.
 * A NaN block makes NaN of every output it takes part in.
 * UNSUPPORTED unless n_in % 128 == 0, n_out % 16 == 0, both at most 2^22, rows at
 * most 2^24, and codes, y and the workspace are 16-byte aligned, scales 4-byte
 * aligned.  rows >= 0.
 */
size_t polestar_mx_linear_workspace_size(int x_fmt, polestar_dtype dtype, long rows, int n_out, int n_in);
polestar_status polestar_mx_linear(int x_fmt, polestar_dtype dtype, long rows, int n_in, int n_out,
                                   const uint8_t* x_codes, const uint8_t* x_scales, const uint8_t* w_codes,
                                   const uint8_t* w_scales, void* y, void* workspace, size_t workspace_bytes,
                                   hipStream_t stream);

/*
 * polestar_mx_quantize_linear -- polestar_mx_quantize of the rows [row_start,
 * row_start + n_rows) of every sequence, then polestar_mx_linear of them.  The rows
 * multiplied are the same, bit for bit; the sums may be taken in another order than
 * polestar_mx_linear's.  The quantized rows stay in the workspace or on chip.
 *   x : [batch][seq][n_in] dtype;  y : out [batch][n_rows][n_out] dtype
 *   workspace : >= polestar_mx_quantize_linear_workspace_size(...) bytes
 * UNSUPPORTED under the conditions of both calls.
 */
size_t polestar_mx_quantize_linear_workspace_size(int x_fmt, polestar_dtype dtype, int batch, int n_rows,
                                                  int n_out, int n_in);
polestar_status polestar_mx_quantize_linear(int x_fmt, polestar_dtype dtype, int batch, int seq, int n_in,
                                            int n_out, int row_start, int n_rows, const void* x,
                                            const uint8_t* w_codes, const uint8_t* w_scales, void* y,
                                            void* workspace, size_t workspace_bytes, hipStream_t stream);

/*
 * polestar_residual_rmsnorm_mx -- polestar_residual_rmsnorm with quantized rows:
 *   x_out[r] = x[r] + y[r] in fp32;
 *   v = x_out[r] / sqrt(mean_c x_out[r]^2 + eps) * gain;  codes, scales of v.
 * The norm is taken in 64 bits and rounded once, to the codes, so that the codes
 * do not depend on the order of the sum.
 *   x : [rows][d] float;  y : [rows][d] dtype, or NULL (nothing is added)
 *   gain : [d] float, or NULL (unit gain)
 *   x_out : out [rows][d] float, may be x; may be NULL where y is NULL
 *   codes : out [rows][row bytes];  scales : out [rows][d / 32]
 * UNSUPPORTED unless d % 32 == 0, d <= 16384, rows < 2^24 and every pointer but
 * scales is 16-byte aligned.  rows >= 0.
 */
polestar_status polestar_residual_rmsnorm_mx(int fmt, polestar_dtype dtype, long rows, int d, const float* x,
                                             const void* y, const float* gain, float eps, float* x_out,
                                             uint8_t* codes, uint8_t* scales, hipStream_t stream);

/*
 * K/V caches in MXFP4, blocks along the head's channels, a head's positions one
 * after another (a head's keys are one stream, and its row a whole number of
 * 16-byte chunks):
 *   k_codes, v_codes   : [batch][n_kv_heads][seq][head_dim / 2]
 *   k_scales, v_scales : [batch][n_kv_heads][seq][head_dim / 32]
 *
 * polestar_mx_store_kv -- quantize new rows into the caches:
 *   row r of sequence b goes to position idx[b][r] for r < count[b] (entries
 *   outside [0, seq) are skipped; of equal entries the last one counts), or,
 *   where idx is NULL, to row_start + r for r < n_rows.  Other positions keep
 *   their bytes.
 *   k, v : row (b, r) starts at element (b * n_rows + r) * row_stride and holds
 *          [n_kv_heads][head_dim] dtype, so that they may lie inside the rows of
 *          a joint product
 *   idx : [batch][n_rows] int32 or NULL;  count : [batch] int32, clamped to
 *         [0, n_rows] (NULL with idx: n_rows)
 * Requires 0 <= n_rows, row_start + n_rows <= seq without idx, row_stride >=
 * n_kv_heads * head_dim.  UNSUPPORTED unless head_dim is 64 or 128, n_rows <
 * 2^23, batch and n_kv_heads < 2^16, a stride is whole 16-byte chunks, and k, v and
 * the codes are 16-byte, the scales 4-byte aligned (head_dim 64: 2-byte).
 */
polestar_status polestar_mx_store_kv(polestar_dtype dtype, int batch, int seq, int n_kv_heads, int head_dim,
                                     int n_rows, const void* k, const void* v, long row_stride,
                                     const int32_t* idx, const int32_t* count, int row_start, uint8_t* k_codes,
                                     uint8_t* k_scales, uint8_t* v_codes, uint8_t* v_scales, hipStream_t stream);

/*
 * polestar_mx_attend -- attention of n_rows query rows per sequence over the
 * first kv_len[b] positions of such caches (polestar_attend's definition on the
 * values the codes stand for):
 *     l_j = scale * q . k_j,  out = sum_j softmax(l)_j v_j,  lse = log sum_j e^l_j
 * with KV head h / (n_heads / n_kv_heads).  A sequence of length 0 gives zeros
 * and an lse of -infinity.  Positions at and past kv_len[b] are not used,
 * whatever they hold.  scale <= 0 selects 1/sqrt(head_dim).
 *   q   : row (b, r) starts at element (b * n_rows + r) * q_stride and holds
 *         [n_heads][head_dim] dtype
 *   kv_len : [batch] int32, clamped to [0, seq], or NULL (seq)
 *   out : [batch][n_rows][n_heads][head_dim] dtype
 *   lse : [batch][n_heads][n_rows] float or NULL
 *   workspace : >= polestar_mx_attend_workspace_size(...) bytes (no init)
 * Products are bf16 matrix instructions on the exact key and value numbers;
 * probabilities are rounded to bf16 for bf16 outputs, and for fp32 queries both
 * they and the probabilities are taken as three bf16 terms (24 bits).  Results of
 * a magnitude below 2^-126 may be 0.
 * UNSUPPORTED unless head_dim is 64 or 128, n_heads % n_kv_heads == 0 is given
 * (INVALID otherwise), seq <= 2^24, batch and n_kv_heads < 2^16, the query heads'
 * rows fit 2^23 groups of 32 in all, q_stride is a whole number of 16-byte chunks,
 * and q, out, the codes and the workspace are 16-byte, the scales 4-byte aligned
 * (head_dim 64: 2-byte).
 */
size_t polestar_mx_attend_workspace_size(polestar_dtype dtype, int batch, int seq, int n_heads, int n_kv_heads,
                                         int head_dim, int n_rows);
polestar_status polestar_mx_attend(polestar_dtype dtype, int batch, int seq, int n_heads, int n_kv_heads,
                                   int head_dim, int n_rows, const void* q, long q_stride,
                                   const uint8_t* k_codes, const uint8_t* k_scales, const uint8_t* v_codes,
                                   const uint8_t* v_scales, const int32_t* kv_len, float scale, void* out,
                                   float* lse, void* workspace, size_t workspace_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif
