/*
 * libspqt - the prompt side of a decoder in 8-bit integers: rows of 16-bit values to codes, the norms before and after a block,
 * and the product of codes and weights, from one row to many thousands.  Beside the sparse GEMVs, which take 1 to 4 rows, and
 * the attention of spqt_kv.h, which takes any number.  All calls are DEVICE, async, and follow the conventions of spqt.h
 * (status codes, streams, the current device).
 *
 * Codes.  A row of numbers x is held as int8 codes and one fp32 scale, with a = the largest |x|, or 2^-100 if that is more:
 *   scale = a / 127,   code = x * (127 / a) to the nearest integer, ties to even
 * each quotient and the product rounded to fp32 first.  Codes are from -127 to 127.  A row that has an infinity or a NaN has codes 0 and the
 * scale NaN, so that every product with it is NaN.  Tokens are rows of activations, output channels are rows of weights: the
 * same call quantizes both.
 *
 * Tensors are [rows][...] with the stride of a row in elements, which is at least the row's width for what is written and 0 or more
 * for what is read; elements of a row are dense.  16-bit and 32-bit tensors need the alignment of their elements only.
 * Codes and weights begin at a multiple of 16 bytes and their strides are multiples of 16; a row's bytes from its width to the next
 * multiple of 16 may be anything, and are read but have no effect.  Writes leave what is behind a row's last element as it was.
 * Products read rows fastest that begin at multiples of 128 bytes: 777 rows by 1111 channels, K 5003, in rows of 5008 bytes 24.6 us, of 5120 bytes 20.0.
 *
 * A tensor that is written overlaps no other tensor of the call, except where it is said that it may be another one.
 */
#ifndef SPQT_I8_H
#define SPQT_I8_H

#include "spqt.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SPQT_I8_FP16 0
#define SPQT_I8_BF16 1
#define SPQT_I8_FP32 2           /* outputs of spqt_i8_gemm only */
#define SPQT_I8_MAX_ROWS (1 << 24)
#define SPQT_I8_MAX_NORM 65536   /* widest row of spqt_i8_norm and spqt_i8_quantize */
#define SPQT_I8_MAX_K 131071     /* widest row of spqt_i8_gemm and spqt_i8_read: sums of products of any two codes are less than 2^31 */

/* codes and scales of x [rows][K] of the 16-bit type; 1 <= K <= SPQT_I8_MAX_NORM. */
int spqt_i8_quantize(const void *x, int64_t x_row, int64_t rows, int64_t K, int type, int8_t *codes, int64_t codes_row, float *scales, void *stream);

/* out = code * scale in the 16-bit type, at most its largest number. */
int spqt_i8_read(const int8_t *codes, int64_t codes_row, const float *scales, int64_t rows, int64_t K, int type, void *out, int64_t out_row, void *stream);

/* The norms around a block.  With r(v) = 1 / sqrt(mean of v^2 + eps), the mean over a row's K numbers:
 *
 *   z = block * r(block) * (offset + block_gain)      or block itself without block_gain
 *   z = z * gate                                      with a gate
 *   s = residual * h + z                              or h itself without block
 *   x = s * r(s) * (offset + gain)
 *
 * h_out = s, out = x in the 16-bit type, codes and scales those of x: all arithmetic is fp32, x is made of s and codes are made of x as they are before
 * they are rounded.  h_out may be h or block, and out may be h or block, element for element (with several rows, of the same stride); h_out and out are two tensors. */
typedef struct {
    const void *h;          /* [rows][K]: the residual stream */
    const void *block;      /* [rows][K] or NULL: what a block has made */
    const void *block_gain; /* [K] or NULL; with block */
    const void *gate;       /* [rows][K] or NULL; with block.  gate_row 0: one row for all */
    const void *gain;       /* [K] */
    void *h_out;            /* [rows][K]; with block, else NULL */
    void *out;              /* [rows][K] or NULL */
    int8_t *codes;          /* [rows][K] or NULL */
    float *scales;          /* [rows], with codes */
    int64_t h_row, block_row, gate_row, h_out_row, out_row, codes_row;
    int64_t rows, K;        /* 1 <= K <= SPQT_I8_MAX_NORM */
    float residual, eps, offset; /* finite; eps >= 1e-30 */
    int type;               /* of all 16-bit tensors */
} spqt_i8_norm_call;
int spqt_i8_norm(const spqt_i8_norm_call *call, void *stream);

/* y[r][n] = (sum over k of codes[r][k] * weights[n][k]) * scales[r] * weight_scales[n] + bias[n]
 * The sum is exact; it is rounded to fp32, so is each step after it, and the result to y's type.
 * gated: weights, weight_scales and bias are those of N / 2 rows of a gate and, behind them, N / 2 rows of an up projection (N even), and with v the above
 *   y[r][f] = v[r][f] / (1 + exp(-v[r][f])) * v[r][N / 2 + f],   f < N / 2
 * in fp32, rounded once. Exponential and quotient are the hardware's: v / (1 + exp(-v)) is off by 2^-24 times 8 relative at most (12 where v < -87.3) for 32-bit
 * outputs, by 2^-24 times 1.3 |v| + 11 for 16-bit ones. */
typedef struct {
    const int8_t *codes;    /* [rows][K] */
    const float *scales;    /* [rows] */
    const int8_t *weights;  /* [N][K] */
    const float *weight_scales; /* [N] */
    const float *bias;      /* [N] or NULL */
    void *y;                /* [rows][N], gated [rows][N / 2] */
    int64_t codes_row, weights_row, y_row;
    int64_t rows, N, K;     /* 1 <= N <= 2^24, 1 <= K <= SPQT_I8_MAX_K */
    int y_type, gated;
} spqt_i8_product;

/* Bytes of the workspace with which spqt_i8_gemm may divide K where rows and channels alone do not fill the chip: a bound that depends on rows, N and K only, no less for
 * more of any of them, so that a workspace for more serves less, and at most 64 MiB and 256 bytes. 0 for up to 16 rows and for K up to 128; sizes that fill the chip
 * by themselves have the bound of smaller ones, of which they use nothing (NULL serves them as well). */
int spqt_i8_workspace_bytes(int64_t rows, int64_t N, int64_t K, size_t *out_bytes);

/* workspace: 256-byte aligned, at least spqt_i8_workspace_bytes, or NULL, with which K is not divided and y is the same.  It needs no preparation and
 * holds nothing between calls: calls of one stream may share one, whatever their shapes, calls that may overlap in time may not.
 * Not with GEMVs, whose workspace has to be all zeros: a call raises the flag that makes them yield NaN on its workspace
 * until spqt_workspace_init. */
int spqt_i8_gemm(const spqt_i8_product *product, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif
