// Microscaled form (include/ssd_mx.h): scales, conversions and the launchers of its kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "mx_rules.h"

typedef uint16_t bf16_t;

// Exponent code of a block's scale from the bits of its largest magnitude: the smallest power of two for which that value
// rounds to a finite element.  e2m1: largest 6 = 1.5 x 2^2, and from 7 = 1.75 x 2^2 on the nearest would be 8 (the tie goes
// to the even code); e4m3: largest 448 = 1.75 x 2^8, and past 464 = 1.8125 x 2^8 the nearest would be 480.  So the
// exponent less that of the largest element, one more where the fraction is past the border, which an addition to the bits does.
// Maxima are taken on the bits, as integers: exact, and a NaN stays.
template <int BITS>
__device__ __forceinline__ unsigned mx_scale_code(unsigned top) {
    constexpr unsigned past = BITS == 4 ? 0x200000u : 0x17ffffu;
    constexpr int emax = BITS == 4 ? 2 : 8;
    const int e = (int)((top + past) >> 23) - emax;
    return top >= 0x7f800000u ? 255u : (unsigned)(e < 0 ? 0 : e);
}
// 2^(code - 127) as a float (code 255: not reached, such blocks hold zeros under any scale)
__device__ __forceinline__ float mx_scale_value(unsigned code) {
    return __uint_as_float(code == 0 ? 0x400000u : (code > 254 ? 127u : code) << 23);
}

typedef short short2_t __attribute__((ext_vector_type(2)));
// Conversions of eight values in units of `scale`, to nearest even (v_cvt_scalef32_*: one instruction for two values; the
// scale keeps them in range, so nothing saturates).
__device__ __forceinline__ unsigned mx_pack4(const float* v, float scale) {
    unsigned o = 0;
    o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, v[0], v[1], scale, 0);
    o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, v[2], v[3], scale, 1);
    o = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, v[4], v[5], scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(o, v[6], v[7], scale, 3);
}
__device__ __forceinline__ unsigned mx_pack8(const float* v, float scale) {       // four values
    short2_t o = {0, 0};
    o = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(o, v[0], v[1], scale, false);
    o = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(o, v[2], v[3], scale, true);
    return __builtin_bit_cast(unsigned, o);
}

// Word [group][row] of the scales of a matrix of `rows` rows.
__host__ __device__ inline size_t mx_scale_word(int group, int row, int rows) { return (size_t)group * mx_pad_rows(rows) + row; }

// The product's operands, as the kernels take them.
struct MxArgs {
    const uint8_t *x, *w;              // codes [M, K], [N, K / 2]
    const uint32_t *xs, *ws;           // scale words
    void* out;                         // fp32 sums [parts][M, N], bf16 [M, N] or codes [M, N / 2]
    uint32_t* out_s;                   // scales of the codes
    size_t part_stride;                // fp32 elements between two partial sums
    int M, N, K;
    int split;                         // k-slices
    hipStream_t st;
};

// Launchers (asynchronous on a.st / st); arguments have been checked.
void mx_launch_quantize(const void* src, int dtype, int rows, int cols, int format, void* codes, void* scales, void* values, hipStream_t st);
void mx_launch_norm(const float* h, const float* partials, int n_part, size_t part_stride, const float* gain, float eps, int rows, int cols,
                    float* h_out, void* codes, void* scales, hipStream_t st);
// The product; fp32 results are *n_part partial sums for the consumer to add by halves (a.split > 1 yields no other result).  False if a
// kernel could not be set up.
bool mx_launch_gemm(const MxArgs& a, int result, int* n_part);
// the same sums by a wave per 32 x 32 outputs
void mx_launch_gemm_plain(const MxArgs& a, int result, int* n_part);
bool mx_gemm_f32(const MxArgs& a, int kind, int* n_part);
bool mx_gemm_f32_large(const MxArgs& a, int kind, int* n_part);
bool mx_gemm_bf16(const MxArgs& a, int kind, int* n_part);
bool mx_gemm_bf16_large(const MxArgs& a, int kind, int* n_part);
bool mx_gemm_swiglu(const MxArgs& a, int kind, int* n_part);
bool mx_gemm_swiglu_large(const MxArgs& a, int kind, int* n_part);
// the product of three or four slices in one launch (mx_choose_all's kind)
bool mx_gemm_all_f32(const MxArgs& a, int kind);
bool mx_gemm_all_bf16(const MxArgs& a, int kind);
// out (bf16 or fp32, [M, N]) = the sum of the n_part partial sums, by halves
void mx_launch_join(const float* part, int n_part, size_t part_stride, int result, void* out, size_t n, hipStream_t st);
