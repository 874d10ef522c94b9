/*
 * ssd_mx.h - microscaled operators of the SSD library: quantisation to 4 and 8 bits, RMSNorm with an 8-bit
 * output, and the product of 8-bit rows with a 4-bit matrix.  A forward of a masked-diffusion model (ssd.h) is bound by
 * the weights that it streams; in microscaled form they take 4.25 bits instead of 16.  A context whose ssd_config says
 * SSD_MXFP4 runs its layers on these operators; a program with a forward of its own calls them one by one.
 *
 * Microscaled form of a matrix [rows, cols], cols a multiple of 32: every 32 consecutive values of a row, a block, share a
 * scale 2^(s - 127), one byte s (s = 255: the block is not a number).
 *   codes   row-major.  SSD_MX_FP8: a byte per value, sign, 4 bits exponent, 3 bits mantissa (largest 448).
 *           SSD_MX_FP4: two values to a byte, the first in the low half; sign, 2 bits exponent, 1 bit mantissa:
 *           0, 0.5, 1, 1.5, 2, 3, 4, 6.
 *   scales  in groups of four blocks (128 columns): byte b % 4 of word [b / 4][row], rows rounded up to 32:
 *           ssd_mx_scale_bytes(rows, cols) bytes.  Rows and blocks that only fill up hold 127; readers pay no heed to them.
 * The scale of a block is the smallest power of two for which its largest value, rounded, is not past the largest
 * element: every value is off by at most half a step of the element's format.  An infinity or a NaN makes its block NaN.
 * (Producers that take the exponent of the largest value as it is, and saturate, give a block whose largest is in [7, 8) times a power
 * of two, with 8 bits in (464, 512), half this scale.  Such matrices are read like any other; their codes are not these.)
 *
 * Conventions: those of ssd.h (return codes, host-side validation, nothing launched by a call that fails).  All pointers
 * are device pointers; the calls need no context, run asynchronously on `hip_stream` (NULL = the default stream) and
 * allocate nothing, so they may be captured into a graph; ssd_last_error(NULL) gives the detail of the last failure on
 * the calling thread.  The current device must be the stream's.  codes, scales and out start on 16-byte
 * boundaries; outputs must not overlap inputs except where said.
 */
#ifndef SSD_MX_H
#define SSD_MX_H

#include "ssd.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SSD_MX_FP4 4
#define SSD_MX_FP8 8

#define SSD_MX_MAX_ROWS (1 << 20)
#define SSD_MX_MAX_COLS (1 << 20)
#define SSD_MX_MAX_OUT  (1ll << 33)   /* outputs of a product */

/* Bytes of the scales of a microscaled matrix (0 on a bad size). */
size_t ssd_mx_scale_bytes(int rows, int cols);

/* Quantisation.  src [rows, cols] row-major in `dtype` (SSD_F32 or SSD_BF16; 16-byte aligned) -> codes and scales in
 * `format`; values (may be NULL; [rows, cols] in dtype) = the rounded values, i.e. what codes and scales stand for.
 * Errors: SSD_EINVAL, SSD_ERANGE (a size beyond SSD_MX_MAX_ROWS or SSD_MX_MAX_COLS). */
int ssd_mx_quantize(const void* src, int dtype, int rows, int cols, int format, void* codes, void* scales, void* values,
                    void* hip_stream);

/* Residual + RMSNorm (the step in front of every projection of Section 3.1's f_theta), output in SSD_MX_FP8:
 * h_out (fp32 [rows, cols]) = h + the n_part partial sums `partials` (fp32 [n_part, rows, cols], the first half's sum, then the
 * second's; n_part 0 .. 8); codes, scales = h_out / sqrt(mean(h_out^2) + eps) * gain (fp32 [cols]).  h_out may be h (the
 * residual stream is updated in place) or NULL (it is not kept).  cols at most 8192.  Errors: SSD_EINVAL, SSD_ERANGE. */
int ssd_mx_norm(const float* h, const float* partials, int n_part, const float* gain, float eps, int rows, int cols, float* h_out,
                void* codes, void* scales, void* hip_stream);

/* Results of ssd_mx_linear. */
#define SSD_MX_OUT_F32    0   /* out fp32 [M, N]                                                                  */
#define SSD_MX_OUT_BF16   1   /* out bf16 [M, N]                                                                  */
#define SSD_MX_OUT_SWIGLU 2   /* W = N/2 gate rows, then N/2 up rows (N a multiple of 64): silu(gate) * up in
                                 SSD_MX_FP8, out = its codes [M, N/2], out_scales = its scales; silu is 0 for
                                 gates below about -87, where 1 / (1 + e^-gate) ends among the normal floats        */

/* Bytes of workspace of a product: the partial sums of all k-slices of its matrix (0 where that has one slice, and on a bad
 * size).  Proportional to M: a workspace for the most rows serves every call with fewer.  Calls that add their slices in
 * one launch, a matter of speed, leave it as it is. */
size_t ssd_mx_linear_workspace(int M, int N, int K, int result);

/* Product: X W^T of x [M, K] in SSD_MX_FP8 and w [N, K] in SSD_MX_FP4, K a multiple of 32, on the matrix cores.  A row's result
 * does not depend on the other rows nor on M.  Products and sums are the hardware's: the 64 products of a step are
 * added with about 18 bits below the largest of them, steps in fp32.  `workspace` (16-byte aligned, at least
 * ssd_mx_linear_workspace bytes) holds partial sums during the call: calls that can overlap in time need one each.
 * Errors: SSD_EINVAL, SSD_ERANGE (M or N beyond SSD_MX_MAX_ROWS, K beyond
 * SSD_MX_MAX_COLS, M * N beyond SSD_MX_MAX_OUT), SSD_ENOMEM (workspace too small). */
int ssd_mx_linear(const void* x_codes, const void* x_scales, int M, const void* w_codes, const void* w_scales, int N, int K,
                  int result, void* out, void* out_scales, void* workspace, size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* SSD_MX_H */
