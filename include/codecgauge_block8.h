/*
 * codecgauge_block8.h -- matrices in 8-bit floating point with a scale for each block of 128 channels: the
 * projections before and after the paged operators, coded in the manner of the cache.
 *
 * A coded matrix [R][K] is
 *   codes  : e4m3 [R][K] (4 exponent bits, 3 mantissa bits, largest 448), rows `stride` bytes apart
 *   scales : fp32 [ceil(R / rows)][ceil(K / 128)], contiguous; rows = 1 (activations) or 128 (weights)
 * and stands for codes[r][k] * scales[r / rows][k / 128]. The last block of a row, and of rows, may be short.
 *
 * The conventions of codecgauge.h hold: device pointers owned by the caller, asynchronous on `stream`, an int
 * status, a message in cg_last_error(), device status bits in cg_get_status(). No call waits for the GPU or
 * allocates; all can be captured in a CUDA graph.
 */
#ifndef CODECGAUGE_BLOCK8_H
#define CODECGAUGE_BLOCK8_H

#include "codecgauge_paged.h"

#ifdef __cplusplus
extern "C" {
#endif

#define CG_BLOCK8 128

/* codes and scales of x [R][K] (CG_BF16 or CG_FP16, rows x_stride elements apart). Per block: scale = (largest
 * |x|) / 448, code = e4m3(x / scale), quotients in fp32, every rounding to nearest even. A block of zeros has
 * scale 0 and codes 0. A block that holds an infinity or NaN raises CG_FLAG_NONFINITE_INPUT and has scale NaN and
 * codes NaN.
 *   rows : 1 or 128;  K : a multiple of 16, >= 16;  R >= 0
 *   x 16-byte aligned, x_stride >= K (unless R < 2) a multiple of 8;  codes 16-byte aligned, stride >= K
 *   (unless R < 2) a multiple of 16. The outputs must not overlap x or one another (rows may lie between another
 *   matrix's rows). One launch. */
int cg_block8_encode(int32_t dtype, int64_t R, int64_t K, int32_t rows, const void* x, int64_t x_stride, void* codes,
                     int64_t stride, float* scales, void* stream);

/* out = x w^T: out[m][n] = sum_k x[m][k] w[n][k] of the matrices that the codes stand for; x [M][K] with
 * rows = 1, w [N][K] with rows = 128. A block's products are summed in fp32 on the tensor cores; the block's sum times
 * the product of its two scales (rounded to fp32: it should be a normal number, or 0) is added in fp32; the total is
 * rounded once to dtype (CG_BF16 or CG_FP16; beyond its range it becomes infinite). NaN codes and scales reach the
 * outputs that they enter, and no others.
 *   M, N >= 0;  K : a multiple of 16, >= 16;  M, N, K <= 2^30
 *   codes 16-byte aligned, strides in bytes >= K (unless one row) and multiples of 16, below 2^40;  out_stride in
 *   elements, >= N (unless M < 2);  out aligned to 2 bytes (16 with out_stride a multiple of 8 is fastest).
 *   out must not overlap the inputs (its rows may lie between theirs). One launch. The same call gives the same bits each time. */
int cg_block8_matmul(int32_t dtype, int64_t M, int64_t N, int64_t K, const void* x, int64_t x_stride, const float* x_scales,
                     const void* w, int64_t w_stride, const float* w_scales, void* out, int64_t out_stride, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* CODECGAUGE_BLOCK8_H */
