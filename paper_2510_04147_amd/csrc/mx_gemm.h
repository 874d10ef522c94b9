// What the kernels of the microscaled product share.
#pragma once
#include "../../include/ssd_mx.h"
#include "mx.h"

typedef int mx_int8 __attribute__((ext_vector_type(8)));
typedef float mx_floatx16 __attribute__((ext_vector_type(16)));

// One step of v_mfma_scale_f32_32x32x64_f8f6f4: 32 weight rows (A, e2m1) x 32 activation rows (B, e4m3) x 64 columns.  Lane (lm = lane
// % 32, lh = lane / 32) holds of weight row lm the columns 32 lh .. + 31 (16 bytes), of activation row lm the columns 16 lh .. + 15 and
// 32 + 16 lh .. + 15 (twice 16 bytes), and in one byte of a word each the scales of column block lh of its two rows.  It
// gets the outputs of activation row lm and weight rows 8 (i / 4) + 4 lh + i % 4, i = 0 .. 15.  BYTE: which byte of the words.
template <int BYTE>
__device__ __forceinline__ mx_floatx16 mx_mfma(uint4 w, uint4 x0, uint4 x1, unsigned sw, unsigned sx, mx_floatx16 acc) {
    const mx_int8 a = {(int)w.x, (int)w.y, (int)w.z, (int)w.w, 0, 0, 0, 0};
    const mx_int8 b = {(int)x0.x, (int)x0.y, (int)x0.z, (int)x0.w, (int)x1.x, (int)x1.y, (int)x1.z, (int)x1.w};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, acc, 4, 0, BYTE, (int)sw, BYTE, (int)sx);
}

__device__ __forceinline__ float mx_silu_mul(float g, float u) { return g * __builtin_amdgcn_rcpf(1.0f + __expf(-g)) * u; }

// Activated channels of 32 channels x 32 rows (gate and up sums of one tile each) as e4m3 codes and one scale per row.  Lane (lm,
// lh) holds channels 8 g + 4 lh + j of row lm; the block's maximum is that of both halves.  Writes row m = lm's codes at `codes` (of the
// row, at the block's channel 0) and returns the scale's code, the same in both halves.
__device__ __forceinline__ unsigned mx_store_channels(const mx_floatx16& gate, const mx_floatx16& up, int lh, uint8_t* codes, bool store) {
    float o[16];
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        o[i] = mx_silu_mul(gate[i], up[i]);
        const unsigned b = __float_as_uint(o[i]) & 0x7fffffffu;
        top = b > top ? b : top;
    }
    const auto both = __builtin_amdgcn_permlane32_swap(top, top, false, false);
    top = both[0] > both[1] ? both[0] : both[1];
    const unsigned code = mx_scale_code<8>(top);
    const float scale = mx_scale_value(code);
    if (store)
#pragma unroll
        for (int g = 0; g < 4; ++g) *(uint32_t*)(codes + 8 * g + 4 * lh) = code == 255 ? 0u : mx_pack8(o + 4 * g, scale);
    return code;
}

// fp32 or bf16 outputs of four consecutive columns n .. n + 3 of a row of N columns; `whole`: rows start on 16 (8) bytes
__device__ __forceinline__ unsigned mx_bf16_pair(float a, float b) {
    typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
    const bf2 v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(unsigned, v);
}
__device__ __forceinline__ void mx_store4(float* p, const float* v, int left, bool whole) {
    if (whole) { if (left > 0) *(float4*)p = make_float4(v[0], v[1], v[2], v[3]); }
    else
#pragma unroll
        for (int j = 0; j < 4; ++j) if (j < left) p[j] = v[j];
}
__device__ __forceinline__ void mx_store4(bf16_t* p, const float* v, int left, bool whole) {
    const unsigned a = mx_bf16_pair(v[0], v[1]), b = mx_bf16_pair(v[2], v[3]);
    if (whole) { if (left > 0) *(uint2*)p = make_uint2(a, b); }
    else {
        const unsigned u[4] = {a & 0xffff, a >> 16, b & 0xffff, b >> 16};
#pragma unroll
        for (int j = 0; j < 4; ++j) if (j < left) p[j] = (bf16_t)u[j];
    }
}
