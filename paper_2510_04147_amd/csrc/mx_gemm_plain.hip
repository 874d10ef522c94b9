// The microscaled product, plainly: a wave per 32 x 32 outputs, operands straight from memory.  Kernel path 0 of a context; the other kernels'
// sums are these, bit for bit.
#include "mx_gemm.h"

// One k-slice of 32 weight rows x 32 activation rows: a chain of matrix instructions over [k0, k1).  Rows past the end read the last
// one (their outputs are never stored); a last step of 32 columns takes zeros for the other 32.
__device__ __forceinline__ mx_floatx16 mx_plain_slice(const uint8_t* w, const uint32_t* ws, int n, int wpad, const uint8_t* x, const uint32_t* xs, int m, int xpad,
                                                      int K, int k0, int k1, int lh) {
    mx_floatx16 acc;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0.f;
    const uint8_t *wr = w + (size_t)n * (K / 2), *xr = x + (size_t)m * K;
    for (int k = k0; k < k1; k += 64) {
        const bool half = k + 32 >= k1;                      // 32 columns are left
        uint4 a = make_uint4(0, 0, 0, 0), b0, b1 = a;
        if (!half || lh == 0) a = *(const uint4*)(wr + k / 2 + 16 * lh);
        b0 = *(const uint4*)(xr + k + 16 * lh);
        if (!half) b1 = *(const uint4*)(xr + k + 32 + 16 * lh);
        const int shift = (((k >> 5) & 3) + lh) * 8;
        unsigned sw = ws[(size_t)(k >> 7) * wpad + n] >> shift & 255, sx = xs[(size_t)(k >> 7) * xpad + m] >> shift & 255;
        if (half && lh) sw = sx = 127;
        acc = mx_mfma<0>(a, b0, b1, sw, sx, acc);
    }
    return acc;
}

template <int RESULT>
__global__ __launch_bounds__(64) void k_mx_gemm_plain(MxArgs a) {
    const int lane = threadIdx.x, lm = lane & 31, lh = lane >> 5;
    const int n0 = blockIdx.x * 32, m0 = blockIdx.y * 32;
    const int wpad = mx_pad_rows(a.N), xpad = mx_pad_rows(a.M), k_len = mx_slice(a.K, a.split);
    const int m = min(m0 + lm, a.M - 1);
    if constexpr (RESULT == SSD_MX_OUT_SWIGLU) {
        const int F = a.N / 2;
        const mx_floatx16 g = mx_plain_slice(a.w, a.ws, n0 + lm, wpad, a.x, a.xs, m, xpad, a.K, 0, a.K, lh);
        const mx_floatx16 u = mx_plain_slice(a.w, a.ws, F + n0 + lm, wpad, a.x, a.xs, m, xpad, a.K, 0, a.K, lh);
        const bool in = m0 + lm < a.M;
        const unsigned code = mx_store_channels(g, u, lh, (uint8_t*)a.out + (size_t)m * F + n0, in);
        if (lh == 0) ((uint8_t*)a.out_s)[mx_scale_word(n0 >> 7, m0 + lm, a.M) * 4 + (n0 >> 5 & 3)] = (uint8_t)(in ? code : 127);
        // the blocks that only fill up the last group
        if (lh == 0 && n0 + 32 >= F)
            for (int b = (n0 >> 5 & 3) + 1; b < 4; ++b) ((uint8_t*)a.out_s)[mx_scale_word(n0 >> 7, m0 + lm, a.M) * 4 + b] = 127;
    } else {
        const int n = min(n0 + lm, a.N - 1);
        for (int s = 0; s < a.split; ++s) {
            const mx_floatx16 acc = mx_plain_slice(a.w, a.ws, n, wpad, a.x, a.xs, m, xpad, a.K, s * k_len, min((s + 1) * k_len, a.K), lh);
            if (m0 + lm < a.M) {
                using T = std::conditional_t<RESULT == SSD_MX_OUT_F32, float, bf16_t>;
                T* out = (T*)a.out + s * a.part_stride + (size_t)m * a.N;
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int c = n0 + 8 * g + 4 * lh;
                    const float v[4] = {acc[4 * g], acc[4 * g + 1], acc[4 * g + 2], acc[4 * g + 3]};
                    mx_store4(out + c, v, a.N - c, a.N % 4 == 0);
                }
            }
        }
    }
}

// The sum of the partial sums, by halves: bound by reading them, for few rows by the launch (a forward's products have no such launch:
// the norm and the attention behind them add the sums).
template <typename T>
__global__ __launch_bounds__(256) void k_mx_join(const float* __restrict__ part, int n_part, size_t stride, T* __restrict__ out, size_t n) {
    const size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= n) return;
    const int half = (n_part + 1) / 2;
    float v[4];
    const bool whole = i + 4 <= n && stride % 4 == 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = 0.f;
    if (whole) {
        float4 t[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int s0 = h ? half : 0, s1 = h ? n_part : half;
            if (s0 >= s1) { t[h] = make_float4(0.f, 0.f, 0.f, 0.f); continue; }
            t[h] = *(const float4*)(part + s0 * stride + i);
            for (int s = s0 + 1; s < s1; ++s) {
                const float4 p = *(const float4*)(part + s * stride + i);
                t[h].x += p.x; t[h].y += p.y; t[h].z += p.z; t[h].w += p.w;
            }
        }
        v[0] = t[0].x + t[1].x; v[1] = t[0].y + t[1].y; v[2] = t[0].z + t[1].z; v[3] = t[0].w + t[1].w;
        mx_store4(out + i, v, 4, true);
    } else {
        for (int j = 0; j < 4 && i + j < n; ++j) {
            float a = part[i + j], b = 0.f;
            for (int s = 1; s < half; ++s) a += part[s * stride + i + j];
            for (int s = half; s < n_part; ++s) b = s == half ? part[s * stride + i + j] : b + part[s * stride + i + j];
            v[0] = a + b;
            mx_store4(out + i + j, v, 1, false);
        }
    }
}

void mx_launch_join(const float* part, int n_part, size_t stride, int result, void* out, size_t n, hipStream_t st) {
    const dim3 grid((unsigned)((n + 1023) / 1024));
    if (result == SSD_MX_OUT_F32) k_mx_join<float><<<grid, 256, 0, st>>>(part, n_part, stride, (float*)out, n);
    else k_mx_join<bf16_t><<<grid, 256, 0, st>>>(part, n_part, stride, (bf16_t*)out, n);
}

void mx_launch_gemm_plain(const MxArgs& a, int result, int* n_part) {
    const dim3 grid(((result == SSD_MX_OUT_SWIGLU ? a.N / 2 : a.N) + 31) / 32, (a.M + 31) / 32);
    *n_part = a.split;
    if (result == SSD_MX_OUT_F32) k_mx_gemm_plain<SSD_MX_OUT_F32><<<grid, 64, 0, a.st>>>(a);
    else if (result == SSD_MX_OUT_BF16) k_mx_gemm_plain<SSD_MX_OUT_BF16><<<grid, 64, 0, a.st>>>(a);
    else k_mx_gemm_plain<SSD_MX_OUT_SWIGLU><<<grid, 64, 0, a.st>>>(a);
}

bool mx_launch_gemm(const MxArgs& a, int result, int* n_part) {
    const int kind = mx_choose(a.M, a.N, a.K, a.split, result == SSD_MX_OUT_SWIGLU);
    if (result == SSD_MX_OUT_F32) return mx_gemm_f32(a, kind, n_part) || mx_gemm_f32_large(a, kind, n_part);
    if (result == SSD_MX_OUT_BF16) return mx_gemm_bf16(a, kind, n_part) || mx_gemm_bf16_large(a, kind, n_part);
    return mx_gemm_swiglu(a, kind, n_part) || mx_gemm_swiglu_large(a, kind, n_part);
}
