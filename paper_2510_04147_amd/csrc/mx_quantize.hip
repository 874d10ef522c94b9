// Microscaled quantisation, and RMSNorm with an 8-bit output.
#include "../../include/ssd_mx.h"
#include "mx.h"

__device__ __forceinline__ void mx_load8(const float* p, float* v) {
    const float4 a = ((const float4*)p)[0], b = ((const float4*)p)[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void mx_load8(const bf16_t* p, float* v) {
    const uint4 a = *(const uint4*)p;
    const unsigned w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ void mx_store8(float* p, const float* v) {
    ((float4*)p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    ((float4*)p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void mx_store8(bf16_t* p, const float* v) {      // rounded values have at most four significant bits
    unsigned w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (__float_as_uint(v[2 * i]) >> 16) | (__float_as_uint(v[2 * i + 1]) & 0xffff0000u);
    *(uint4*)p = make_uint4(w[0], w[1], w[2], w[3]);
}

// The other lanes' values, by DPP: lane ^ 1, lane ^ 2; then of the other four lanes of eight, the other eight of sixteen.
template <int CTRL>
__device__ __forceinline__ unsigned mx_dpp(unsigned v) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true); }
__device__ __forceinline__ unsigned mx_max(unsigned a, unsigned b) { return a > b ? a : b; }

// Quantisation.  A work-group of four waves takes 32 rows x 512 columns: a wave reads 512 columns of a row in one go, eight values
// to a lane, so a block is four lanes and a scale word (four blocks) sixteen; a wave has its eight rows' loads in flight together.
// They are neighbours (37888 x 3584 bf16 to 4 bits and values, us, neighbours / every fourth row: 132.6 / 135.6), but for calls of at most 32 rows, where
// every fourth keeps all waves busy (8 x 4096: 4.1 / 3.4).
// The tile's scale words meet in LDS and leave as whole lines.  Reads every value once: bound by memory (37888 x 3584 bf16 to 4 bits 72.4 us,
// 4.75 TB/s read and written; 4097 x 1504 fp32 to 8 bits 5.7 us, 5.4 TB/s; few rows by the launch and one trip to memory).
template <typename T, int BITS, bool VALUES>
__global__ __launch_bounds__(256) void k_mx_quantize(const T* __restrict__ src, int rows, int cols, uint8_t* __restrict__ codes,
                                                     uint32_t* __restrict__ scales, T* __restrict__ values) {
    __shared__ uint32_t words[4][32];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int row0 = blockIdx.x * 32, col = blockIdx.y * 512 + lane * 8;
    const bool in = col < cols;                              // whole blocks are in or out
    const int step = rows <= 32 ? 4 : 1, first = rows <= 32 ? wave : wave * 8;
    float v[8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int row = row0 + first + i * step;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
        if (in && row < rows) mx_load8(src + (size_t)row * cols + col, v[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int row = row0 + first + i * step;
        unsigned top = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) top = mx_max(top, __float_as_uint(v[i][j]) & 0x7fffffffu);
        top = mx_max(top, mx_dpp<0xB1>(top));
        top = mx_max(top, mx_dpp<0x4E>(top));
        unsigned code = mx_scale_code<BITS>(top);
        const float scale = mx_scale_value(code);
        if (code == 255)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
        if (in && row < rows) {
            const size_t at = (size_t)row * cols + col;
            if constexpr (BITS == 4) {
                const unsigned o = mx_pack4(v[i], scale);
                *(uint32_t*)(codes + at / 2) = o;
                if constexpr (VALUES) {
                    float r[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        // sign, two bits of exponent, one of mantissa, to a float: the exponent in place, or half the mantissa
                        const unsigned c = o >> (4 * j), e = c >> 1 & 3, m = c & 1;
                        const float mag = e ? __uint_as_float((126 + e) << 23 | m << 22) : m * 0.5f;
                        r[j] = code == 255 ? NAN : (c & 8 ? -mag : mag) * scale;
                    }
                    mx_store8(values + at, r);
                }
            } else {
                const unsigned a = mx_pack8(v[i], scale), b = mx_pack8(v[i] + 4, scale);
                *(uint2*)(codes + at) = make_uint2(a, b);
                if constexpr (VALUES) {
                    float r[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const unsigned c = (j < 4 ? a : b) >> (8 * (j & 3)), e = c >> 3 & 15, m = c & 7;
                        const float mag = e ? __uint_as_float((120 + e) << 23 | m << 20) : m * 0x1p-9f;
                        r[j] = code == 255 ? NAN : (c & 128 ? -mag : mag) * scale;
                    }
                    mx_store8(values + at, r);
                }
            }
        }
        if (!in || row >= rows) code = 127;                  // what only fills up
        // the word: four blocks of four lanes
        unsigned word = code << ((lane >> 2 & 3) * 8);
        word |= mx_dpp<0x141>(word);
        word |= mx_dpp<0x140>(word);
        if ((lane & 15) == 0) words[lane >> 4][first + i * step] = word;
    }
    __syncthreads();
    const int group = blockIdx.y * 4 + (threadIdx.x >> 5);
    if (threadIdx.x < 128 && group < mx_groups(cols)) scales[(size_t)group * mx_pad_rows(rows) + row0 + (threadIdx.x & 31)] = words[threadIdx.x >> 5][threadIdx.x & 31];
}

void mx_launch_quantize(const void* src, int dtype, int rows, int cols, int format, void* codes, void* scales, void* values, hipStream_t st) {
    const dim3 grid((rows + 31) / 32, (cols + 511) / 512);
    auto run = [&](auto t, auto bits, auto with) {
        using T = decltype(t);
        k_mx_quantize<T, decltype(bits)::value, decltype(with)::value><<<grid, 256, 0, st>>>((const T*)src, rows, cols, (uint8_t*)codes, (uint32_t*)scales, (T*)values);
    };
    auto typed = [&](auto t) {
        if (format == SSD_MX_FP4) values ? run(t, std::integral_constant<int, 4>{}, std::true_type{}) : run(t, std::integral_constant<int, 4>{}, std::false_type{});
        else values ? run(t, std::integral_constant<int, 8>{}, std::true_type{}) : run(t, std::integral_constant<int, 8>{}, std::false_type{});
    };
    if (dtype == SSD_F32) typed(0.f);
    else typed(bf16_t(0));
}

// The sum of the wave's 64 values, in every lane, without trips through LDS.
__device__ __forceinline__ double mx_wave_sum(double v) {
    auto both = [](double a, unsigned lo, unsigned hi) { return a + __hiloint2double((int)hi, (int)lo); };
    auto lo = [](double a) { return (unsigned)__double2loint(a); };
    auto hi = [](double a) { return (unsigned)__double2hiint(a); };
    v = both(v, mx_dpp<0xB1>(lo(v)), mx_dpp<0xB1>(hi(v)));
    v = both(v, mx_dpp<0x4E>(lo(v)), mx_dpp<0x4E>(hi(v)));
    v = both(v, mx_dpp<0x141>(lo(v)), mx_dpp<0x141>(hi(v)));
    v = both(v, mx_dpp<0x140>(lo(v)), mx_dpp<0x140>(hi(v)));
    auto l = __builtin_amdgcn_permlane16_swap(lo(v), lo(v), false, false), h = __builtin_amdgcn_permlane16_swap(hi(v), hi(v), false, false);
    v = __hiloint2double((int)h[0], (int)l[0]) + __hiloint2double((int)h[1], (int)l[1]);
    l = __builtin_amdgcn_permlane32_swap(lo(v), lo(v), false, false);
    h = __builtin_amdgcn_permlane32_swap(hi(v), hi(v), false, false);
    return __hiloint2double((int)h[0], (int)l[0]) + __hiloint2double((int)h[1], (int)l[1]);
}

// RMSNorm behind the residual's addition, output in 8 bits.  One work-group per row, four values to a lane: a block is eight lanes, a
// scale word 32.  The row and all its partial sums are in flight at once; the row stays in registers between the two passes over it
// (mean square, then scale and conversion).  Squares, their sum and the normed values are held in 64 bits, which costs nothing beside
// the loads: a value that falls on the other side of a border between two 8-bit codes is off by a step of 2^-3 to 2^-4.
// Bound by memory for many rows (2304 x 3584, two partial sums, 24.7 us: 5.7 TB/s); 8 x 4096 without partial sums 3.3 us and 160 x 4096
// with four 4.3 us are a launch, one trip to memory and the sum over the work-group.
template <int NP>
__device__ __forceinline__ float4 mx_sum_partials(float4 v, const float* p, size_t stride, int i4) {
    // the first half's sum, then the second's
    auto add = [](float4& x, const float4& y) { x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w; };
    float4 pv[NP > 0 ? NP : 1];
#pragma unroll
    for (int s = 0; s < NP; ++s) pv[s] = ((const float4*)(p + s * stride))[i4];
    constexpr int HALF = (NP + 1) / 2;
    if constexpr (NP > 0) {
        float4 t = pv[0];
#pragma unroll
        for (int s = 1; s < HALF; ++s) add(t, pv[s]);
        add(v, t);
    }
    if constexpr (NP > 1) {
        float4 t = pv[HALF];
#pragma unroll
        for (int s = HALF + 1; s < NP; ++s) add(t, pv[s]);
        add(v, t);
    }
    return v;
}

template <int NP, int T, int J>                              // T lanes, J groups of four columns of a lane
__global__ __launch_bounds__(T) void k_mx_norm(const float* h, const float* part, size_t part_stride, const float* gain, float eps, int rows,
                                                      int cols, float* h_out, uint8_t* codes, uint32_t* scales) {
    const int row = blockIdx.x, n4 = cols >> 2, lane = threadIdx.x & 63;
    const size_t at = (size_t)row * cols;
    float4 v[J], g[J];
    double ss = 0.;
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int i4 = threadIdx.x + j * T;
        v[j] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (i4 < n4) {
            v[j] = ((const float4*)(h + at))[i4];
            g[j] = ((const float4*)gain)[i4];
            v[j] = mx_sum_partials<NP>(v[j], part + at, part_stride, i4);
            if (h_out && (NP > 0 || h_out != h)) ((float4*)(h_out + at))[i4] = v[j];
            ss += (double)v[j].x * v[j].x + (double)v[j].y * v[j].y + (double)v[j].z * v[j].z + (double)v[j].w * v[j].w;
        }
    }
    __shared__ double red[T / 64];
    ss = mx_wave_sum(ss);
    if (lane == 0) red[threadIdx.x >> 6] = ss;
    __syncthreads();
    double tot = 0.;
#pragma unroll
    for (int w = 0; w < T / 64; ++w) tot += red[w];
    const double r = 1.0 / sqrt(tot / cols + (double)eps);
    const int groups = mx_groups(cols), pad = mx_pad_rows(rows);
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int i4 = threadIdx.x + j * T;
        const bool in = i4 < n4;
        float y[4] = {0.f, 0.f, 0.f, 0.f};
        if (in) { y[0] = (float)(v[j].x * r * g[j].x); y[1] = (float)(v[j].y * r * g[j].y); y[2] = (float)(v[j].z * r * g[j].z); y[3] = (float)(v[j].w * r * g[j].w); }
        unsigned top = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) top = mx_max(top, __float_as_uint(y[i]) & 0x7fffffffu);
        top = mx_max(top, mx_dpp<0xB1>(top));
        top = mx_max(top, mx_dpp<0x4E>(top));
        top = mx_max(top, mx_dpp<0x141>(top));
        unsigned code = mx_scale_code<8>(top);
        if (code == 255)
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = 0.f;
        if (in) *(uint32_t*)(codes + at + 4 * i4) = mx_pack8(y, mx_scale_value(code));
        if (!in) code = 127;
        // the word: four blocks of eight lanes
        unsigned word = code << ((lane >> 3 & 3) * 8);
        word |= mx_dpp<0x140>(word);                         // the other eight of sixteen lanes, the other sixteen of 32
        const auto halves = __builtin_amdgcn_permlane16_swap(word, word, false, false);
        word = halves[0] | halves[1];
        const int group = i4 >> 5;
        if ((lane & 31) == 0 && group < groups) scales[(size_t)group * pad + row] = word;
        if (row == rows - 1 && group < groups && rows + (lane & 31) < pad) scales[(size_t)group * pad + rows + (lane & 31)] = 0x7f7f7f7fu;
    }
}

void mx_launch_norm(const float* h, const float* partials, int n_part, size_t part_stride, const float* gain, float eps, int rows, int cols,
                    float* h_out, void* codes, void* scales, hipStream_t st) {
    // Four waves where they hold the row (2304 rows of 512 columns, one partial sum, us, sixteen waves / four: 15.4 / 5.0); longer rows
    // take sixteen, whose loads are all in flight at once.
    auto run = [&](auto np) {
        constexpr int NP = decltype(np)::value;
        if (cols <= 1024) k_mx_norm<NP, 256, 1><<<rows, 256, 0, st>>>(h, partials, part_stride, gain, eps, rows, cols, h_out, (uint8_t*)codes, (uint32_t*)scales);
        else if (cols <= 4096) k_mx_norm<NP, 1024, 1><<<rows, 1024, 0, st>>>(h, partials, part_stride, gain, eps, rows, cols, h_out, (uint8_t*)codes, (uint32_t*)scales);
        else k_mx_norm<NP, 1024, 2><<<rows, 1024, 0, st>>>(h, partials, part_stride, gain, eps, rows, cols, h_out, (uint8_t*)codes, (uint32_t*)scales);
    };
    switch (n_part) {
        case 0: return run(std::integral_constant<int, 0>{});
        case 1: return run(std::integral_constant<int, 1>{});
        case 2: return run(std::integral_constant<int, 2>{});
        case 3: return run(std::integral_constant<int, 3>{});
        case 4: return run(std::integral_constant<int, 4>{});
        case 5: return run(std::integral_constant<int, 5>{});
        case 6: return run(std::integral_constant<int, 6>{});
        case 7: return run(std::integral_constant<int, 7>{});
        default: return run(std::integral_constant<int, 8>{});
    }
}
