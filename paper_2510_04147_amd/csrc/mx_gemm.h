// What the kernels of the microscaled product share.
#pragma once
#include "../../include/ssd_mx.h"
#include "gemm_mfma.h"
#include "mx.h"

typedef int mx_int8 __attribute__((ext_vector_type(8)));
typedef float mx_floatx16 __attribute__((ext_vector_type(16)));

// One step of v_mfma_scale_f32_32x32x64_f8f6f4: 32 weight rows (A, e2m1) x 32 activation rows (B, e4m3) x 64 columns.  Lane (lm = lane
// % 32, lh = lane / 32) holds of weight row lm the columns 32 lh .. + 31 (16 bytes), of activation row lm the columns 16 lh .. + 15 and
// 32 + 16 lh .. + 15 (twice 16 bytes), and in one byte of a word each the scales of column block lh of its two rows.  It
// gets the outputs of activation row lm and weight rows 8 (i / 4) + 4 lh + i % 4, i = 0 .. 15.  BYTE: which byte of the words.
// 64 cycles.  Products are exact; the instruction lines the 64 of a step up with the largest of them and keeps about 18 bits below it, then
// adds to the accumulator in fp32.  Measured against 64 bits: 4e-6 to 1.2e-5 of an output's size on ordinary rows, 1.6e-4 of the sum of the magnitudes
// on codes and scales drawn evenly from all there are.  That is finer than bf16's half step (2^-9 to 2^-8 of the value) and than what rounding to 4 and 8
// bits did before; instructions that add in full fp32 (bf16 operands) take twice the cycles for a step and four times the
// operand bytes of the weights.  An activated channel beside a border between two 8-bit codes can land on the other side, and a
// block whose largest is beside the border of its scale gets the scale's other value: the same values, rounded to the other grid.
template <int BYTE>
__device__ __forceinline__ mx_floatx16 mx_mfma(uint4 w, uint4 x0, uint4 x1, unsigned sw, unsigned sx, mx_floatx16 acc) {
    const mx_int8 a = {(int)w.x, (int)w.y, (int)w.z, (int)w.w, 0, 0, 0, 0};
    const mx_int8 b = {(int)x0.x, (int)x0.y, (int)x0.z, (int)x0.w, (int)x1.x, (int)x1.y, (int)x1.z, (int)x1.w};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, acc, 4, 0, BYTE, (int)sw, BYTE, (int)sx);
}

// silu(g) u, within (|g| + 4) 2^-23 of its size (the exponent |g| log2 e is rounded twice), finer than the sums that it is given; 0 below
// about -87, where the reciprocal is no normal float.
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

// ------------------------------------------------------------------------
// The product's kernel.  Work-group = WN x WM waves, wave (wn, wm) owns TN tiles of 32 weight rows x TM tiles of 32 activation rows and
// walks every column of the work-group's k-slice: one chain of matrix instructions per output, the same in every shape of this
// template and in the plain kernel, so a row's bits do not depend on the shape that a call takes.
//
// Codes and scales go global -> LDS without passing through registers, in chunks of KC columns: weight rows of KC / 2
// bytes, activation rows of KC bytes, 16-byte piece s of row r in slot s ^ f(r), so that the 32 rows of a fragment spread over all LDS banks, and
// per tile and group of 128 columns a line of 32 scale words, into a ring of NST stages.  From the barrier in front of chunk c on, whose
// stage has landed and with which everyone has read chunk c - 1, chunk c - 1 + NST is loaded into the stage of chunk c - 1.
//
// A matrix instruction takes 64 cycles, in which its wave can issue whatever is no matrix instruction: the reads of the next step's fragments
// and the loads stand between the products one by one (160 rows of the 8B shape's gate/up in tiles of 192 x 96 27.0 us with all of them
// in front of the products of a step, 24.7 so; 2304 rows of the 7B class's, 256 x 192, 302 and 278; both in turn on one card).  The last step of
// a chunk runs behind the next barrier.
//
// What bounds it, by rows: up to 32 the weights' stream (12288 x 4096 in 10 us, 2.8 TB/s: the launch, the first chunks' way from memory and
// the sums' way back are half of it); 64 to 300 the requests of a CU, a cache line of weights taking 5.3 ns and one of activations,
// which the L2 holds, 1.2 ns (24576 x 4096, 160 rows, 192 x 96: 22 to 25 us by card; where it took 23 the matrix instructions and barriers alone
// took 15, with the reads of LDS 17.4.  Its two row blocks fetch every line of weights twice and cover 192 rows, and its three waves leave a SIMD
// of every CU without matrix instructions); thousands the matrix cores (37888 x 3584, 2304 rows: 237 to 279 us by card and load before it,
// 2.2 to 2.6 PFLOP/s, where the instruction alone reaches 3.5 on such codes).
//
// HALVES: the work-group walks two slices and adds their sums (two of four slices: what the consumer adds first).
// A last chunk that ends inside KC runs as many steps as it has, the other half of a last half step as zeros.
// ------------------------------------------------------------------------
// A work-group that yields the sum of three or four slices, added as the consumers of partial sums add them, without partial sums in memory and a
// second launch: MX_BESIDE: its waves are the slices (WN = WM = TN = 1), each with a ring of its own, and meet when the sums do, in LDS.  MX_BEHIND: it
// walks one slice after the other and keeps the sum of those before the last two, the last but one and the one at hand in registers.
template <int WN, int WM, int TN, int TM, int KC, int NST, int RESULT, bool HALVES, bool NT, int JOIN = MX_APART>
struct MxShape {
    static constexpr bool ALL = JOIN == MX_BESIDE;
    static_assert(JOIN == MX_APART || !HALVES, "all slices or two");
    static_assert(!ALL || (WN * WM * TN == 1 && !HALVES && RESULT != SSD_MX_OUT_SWIGLU), "one wave to a slice");
    static constexpr int WAVES = ALL ? 4 : WN * WM;
    static constexpr int NW = WN * WM, BN = WN * TN * 32, BM = WM * TM * 32, G = KC / 128, Q = KC / 64;
    static constexpr int WROW = KC / 2, XROW = KC, WP = BN * WROW / 1024, XP = BM * XROW / 1024;     // pieces of 1 KB of a chunk
    // scales: pieces of eight lines, the weights' first; every wave loads equally many pieces of each kind
    static constexpr int SWP = (BN / 32 * G + 7) / 8, SXP = (BM / 32 * G + 7) / 8, SJ = (SWP + SXP + NW - 1) / NW;
    static_assert(WP % NW == 0 && XP % NW == 0, "equal shares");
    static constexpr int WJ = WP / NW, XJ = XP / NW, PER = WJ + XJ + SJ, STAGE = (WP + XP + SJ * NW) * 1024;
    static_assert(NST >= 2 && PER * (NST - 1) < 64, "ring depth");
    static constexpr int OUT = 4096;                                         // of a wave: a tile in row order
    static constexpr int RING = NST * STAGE, LDS = ALL ? 4 * (RING > TM * OUT ? RING : TM * OUT) : RING > NW * OUT ? RING : NW * OUT;
};

// At most N of this wave's loads outstanding and none of its LDS accesses: for a ring that no other wave reads.
template <int N>
__device__ __forceinline__ void wait_own() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory"); }

__device__ __forceinline__ int mx_swizzle16(int r, int pieces) { return (r / (16 / pieces)) & (pieces - 1); }

template <int WN, int WM, int TN, int TM, int KC, int NST, int RESULT, bool HALVES, bool NT, int JOIN>
__global__ __launch_bounds__((JOIN == MX_BESIDE ? 4 : WN * WM) * 64) void k_mx_gemm(MxArgs a, int n_blocks, int m_blocks, int parts) {
    using S = MxShape<WN, WM, TN, TM, KC, NST, RESULT, HALVES, NT, JOIN>;
    constexpr bool ALL = S::ALL, BEHIND = JOIN == MX_BEHIND;
    constexpr int BN = S::BN, BM = S::BM, G = S::G, Q = S::Q, WROW = S::WROW, XROW = S::XROW, WP = S::WP, SWP = S::SWP, SXP = S::SXP;
    constexpr int NW = S::NW, STAGE = S::STAGE, XAT = WP * 1024, SAT = XAT + S::XP * 1024;           // a stage: weights, activations, scales
    constexpr int WJ = S::WJ, XJ = S::XJ, SJ = S::SJ, PER = S::PER;
    constexpr bool CHANNELS = RESULT == SSD_MX_OUT_SWIGLU;
    static_assert(!CHANNELS || TN % 2 == 0, "gate and up tiles in pairs");
    extern __shared__ uint4 smem_u4[];
    const int lane = threadIdx.x & 63, id_of_wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = ALL ? 0 : id_of_wave;
    char* const smem = (char*)smem_u4 + (ALL ? id_of_wave * S::RING : 0);    // the ring
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
    const int wn = wave % WN, wm = wave / WN, lm = lane & 31, lh = lane >> 5;

    // Work-groups go to the 8 XCDs round-robin by their id, and every XCD has an L2 of its own: an XCD takes tiles that are neighbours
    // (the k-slice slowest, then the weights, the rows of one n-block next to each other).
    int bx, by, bz;
    {
        const int total = n_blocks * m_blocks * parts, id = blockIdx.x;
        const int per = total / 8, more = total % 8, xcd = id & 7;
        const int t = xcd * per + (xcd < more ? xcd : more) + (id >> 3);
        by = t % m_blocks;
        bx = (t / m_blocks) % n_blocks;
        bz = ALL ? id_of_wave : t / (m_blocks * n_blocks);
    }
    const int K = a.K, k_len = mx_slice(K, a.split), spw = BEHIND ? a.split : HALVES ? 2 : 1;
    const int k0 = min(K, bz * spw * k_len), k1 = min(K, k0 + spw * k_len);  // a wave past the last slice: nothing
    const int nchunks = (k1 - k0 + KC - 1) / KC, tail = (k1 - k0) % KC;      // tail: columns of a last chunk that is not whole
    const int whole = tail ? nchunks - 1 : nchunks;
    const int boundary = HALVES || BEHIND ? k_len / KC : 0;                  // chunks of a slice
    const int F = a.N / 2, m0 = by * BM;
    // first weight row of the work-group's tile t; past the end: the last tile (never stored)
    auto tile_row = [&](int t) SSD_INLINE {
        if constexpr (CHANNELS) {
            const int c = min(bx * (BN / 64) + t / 2, F / 32 - 1) * 32;
            return t % 2 ? F + c : c;
        } else
            return min(bx * (BN / 32) + t, (a.N - 1) / 32) * 32;
    };

    floatx16 acc[TN][TM], tot[HALVES || BEHIND ? TN : 1][HALVES || BEHIND ? TM : 1], last[BEHIND ? TN : 1][BEHIND ? TM : 1];
#pragma unroll
    for (int n = 0; n < TN; ++n)
#pragma unroll
        for (int m = 0; m < TM; ++m)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                acc[n][m][i] = 0.f;
                if constexpr (BEHIND) tot[n][m][i] = last[n][m][i] = 0.f;
            }
    int ended = 0;                                                           // slices that are done
    // The end of a slice.  BEHIND: the slice before it joins the others, so that in front of the last slice's end `tot` is the sum of
    // the first two and `last` the third, or with three slices in all the first and the second.  (No sum is -0: they start from 0.)
    auto flush = [&]() SSD_INLINE {
        if constexpr (HALVES || BEHIND)
#pragma unroll
            for (int n = 0; n < TN; ++n)
#pragma unroll
                for (int m = 0; m < TM; ++m) {
                    if constexpr (BEHIND) {
                        tot[n][m] += last[n][m];
                        last[n][m] = acc[n][m];
                    } else
                        tot[n][m] = acc[n][m];
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[n][m][i] = 0.f;
                }
        ++ended;
    };
    // whether a slice ends in front of chunk c
    auto ends = [&](int c) SSD_INLINE { return HALVES ? c == boundary : BEHIND && c == (ended + 1) * boundary; };
    // Fragments of a step; its scale words are those of a group, two steps: byte 0 or 2, shifted by the lane's half, is the block's.
    struct Frags { uint4 w[TN], x[TM][2]; unsigned sw[TN], sx[TM]; };
    const int fw = mx_swizzle16(lm, WROW / 16), fx = mx_swizzle16(lm, XROW / 16), shift = lh * 8;
    constexpr int CODES = TN + 2 * TM, READS = CODES + TN + TM;              // reads of a step: codes, and scales if it is even
    auto read1 = [&](auto ec, Frags& f, int slot, int q) SSD_INLINE {        // read e of step q
        constexpr int e = decltype(ec)::value;
        const char* w = smem + slot * STAGE;
        if constexpr (e < TN)
            f.w[e] = *(const uint4*)(w + (wn * TN + e) * (32 * WROW) + lm * WROW + (((2 * q + lh) ^ fw) << 4));
        else if constexpr (e < CODES) {
            constexpr int m = (e - TN) / 2, h = (e - TN) % 2;
            f.x[m][h] = *(const uint4*)(w + XAT + (wm * TM + m) * (32 * XROW) + lm * XROW + (((4 * q + 2 * h + lh) ^ fx) << 4));
        } else {
            const char* r = w + SAT + (q / 2) * 128 + lm * 4;
            if constexpr (e < CODES + TN) f.sw[e - CODES] = *(const unsigned*)(r + (wn * TN + e - CODES) * (G * 128));
            else f.sx[e - CODES - TN] = *(const unsigned*)(r + SWP * 1024 + (wm * TM + e - CODES - TN) * (G * 128));
        }
    };
    auto multiply1 = [&](auto jc, auto odd, const Frags& f) SSD_INLINE {
        constexpr int n = decltype(jc)::value / TM, m = decltype(jc)::value % TM;
        acc[n][m] = mx_mfma<decltype(odd)::value * 2>(f.w[n], f.x[m][0], f.x[m][1], f.sw[n] >> shift, f.sx[m] >> shift, acc[n][m]);
    };
    constexpr std::integral_constant<int, 0> even{};
    constexpr std::integral_constant<int, 1> odd{};
    constexpr std::integral_constant<int, CODES> codes{};
    constexpr std::integral_constant<int, READS> all{};

    // ---- the walk over the chunks
    {
        constexpr int WL = WROW / 16, XL = XROW / 16;                        // lanes to a row
        const int wrow0 = tile_row(0), urow0 = CHANNELS ? tile_row(1) : wrow0;
        const uint64_t wbase = (uint64_t)a.w + (size_t)wrow0 * (K / 2) + k0 / 2, up_rows = (uint64_t)(urow0 - wrow0) * (K / 2);
        const uint64_t xbase = (uint64_t)a.x + (size_t)m0 * K + k0;
        unsigned off[PER];                                                   // a lane's place from the base
        uint64_t sbase[SJ];
        unsigned sstep[SJ];
#pragma unroll
        for (int j = 0; j < WJ; ++j) {
            const int r0 = (wave + NW * j) * (64 / WL), row0 = tile_row(r0 / 32), r = r0 % 32 + lane / WL;
            const int from = CHANNELS && r0 / 32 % 2 ? urow0 + 0 : wrow0 + 0;
            off[j] = (unsigned)(min(row0 + r, a.N - 1) - from) * (unsigned)(K / 2) + ((lane % WL) ^ mx_swizzle16(r, WL)) * 16;
        }
#pragma unroll
        for (int j = 0; j < XJ; ++j) {
            const int r = (wave + NW * j) * (64 / XL) + lane / XL;
            off[WJ + j] = (unsigned)(min(m0 + r, a.M - 1) - m0) * (unsigned)K + ((lane % XL) ^ mx_swizzle16(r, XL)) * 16;
        }
        // line q (tile q / G, group q % G) of the weights' or the activations' scales; past the last: the last again
        auto scale_line = [&](int j, bool& of_w) SSD_INLINE {
            const int s = min(wave + NW * j, SWP + SXP - 1);
            of_w = s < SWP;
            return min((of_w ? s : s - SWP) * 8 + lane / 8, (of_w ? BN : BM) / 32 * G - 1);
        };
#pragma unroll
        for (int j = 0; j < SJ; ++j) {
            bool of_w;
            const int q = scale_line(j, of_w), pad = of_w ? mx_pad_rows(a.N) : mx_pad_rows(a.M);
            const int row0 = of_w ? tile_row(q / G) : min(m0 / 32 + q / G, (a.M - 1) / 32) * 32;
            sbase[j] = (of_w ? (uint64_t)a.ws : (uint64_t)a.xs) + (size_t)(k0 >> 7) * pad * 4;
            sstep[j] = (unsigned)pad * (G * 4);
            off[WJ + XJ + j] = ((unsigned)(q % G) * pad + row0) * 4u + (lane & 7) * 16;
        }
        // load i of chunk `at` into stage `slot`
        auto issue = [&](auto ic, int slot, int at) SSD_INLINE {
            constexpr int i = decltype(ic)::value;
            const unsigned dst = lds0 + slot * STAGE + (wave + NW * i) * 1024;
            if constexpr (i < WJ) {
                uint64_t src = wbase + (size_t)at * WROW;
                if (CHANNELS) src += (wave + NW * i) * (64 / WL) / 32 % 2 ? up_rows + 0 : 0;
                load_to_lds<NT>(dst, off[i], (const char*)src);
            } else if constexpr (i < WJ + XJ)
                load_to_lds<false>(dst, off[i], (const char*)(xbase + (size_t)at * XROW));
            else
                load_to_lds<false>(dst, off[i], (const char*)(sbase[i - WJ - XJ] + (size_t)at * sstep[i - WJ - XJ]));
        };
        // before the last chunk, if it is not whole, is loaded: what lies past the end of the rows reads something of theirs instead
        auto shorten = [&]() SSD_INLINE {
#pragma unroll
            for (int j = 0; j < WJ; ++j) {
                const int s = (lane % WL) ^ mx_swizzle16((wave + NW * j) * (64 / WL) % 32 + lane / WL, WL);
                if (s * 32 >= tail) off[j] -= s * 16;
            }
#pragma unroll
            for (int j = 0; j < XJ; ++j) {
                const int s = (lane % XL) ^ mx_swizzle16((wave + NW * j) * (64 / XL) + lane / XL, XL);
                if (s * 16 >= tail) off[WJ + j] -= s * 16;
            }
#pragma unroll
            for (int j = 0; j < SJ; ++j) {
                bool of_w;
                const int q = scale_line(j, of_w) % G;
                if (q * 128 >= tail) off[WJ + XJ + j] -= q * (sstep[j] / G);
            }
        };
        Frags fa, fb;
        int ahead = NST, slot = 0, free = 0;                                 // chunk to load next; stage of the chunk at hand, free stage
        // A step: the products of f, between them the reads of the next step's fragments (to `to`, from step nq of the chunk at hand; an odd
        // one shares f's scale words) and the q-th share of the free stage's loads.
        auto step = [&](auto qc, auto par, const Frags& f, auto reads, Frags& to, int nq, auto load) SSD_INLINE {
            constexpr int q = decltype(qc)::value, R = decltype(reads)::value, NM = TN * TM, EARLY = NM > 3 ? NM / 2 : NM;
            constexpr int L0 = q * PER / Q, L1 = (q + 1) * PER / Q;
            static_for<0, NM>([&](auto jc) SSD_INLINE {
                constexpr int j = decltype(jc)::value;
                __builtin_amdgcn_sched_barrier(0);
                multiply1(jc, par, f);
                __builtin_amdgcn_sched_barrier(0);
                if constexpr (j < EARLY) static_for<j * R / EARLY, (j + 1) * R / EARLY>([&](auto ec) SSD_INLINE { read1(ec, to, slot, nq); });
                if constexpr (decltype(load)::value) static_for<L0 + j * (L1 - L0) / NM, L0 + (j + 1) * (L1 - L0) / NM>([&](auto ic) SSD_INLINE { issue(ic, free, ahead); });
            });
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (R == CODES) {
#pragma unroll
                for (int n = 0; n < TN; ++n) to.sw[n] = f.sw[n];
#pragma unroll
                for (int m = 0; m < TM; ++m) to.sx[m] = f.sx[m];
            }
        };
        // all but the last bc chunks
        auto landed = [&](auto bc) SSD_INLINE {
            if constexpr (ALL) wait_own<PER * decltype(bc)::value>();
            else wait_and_meet<PER * decltype(bc)::value>();
        };
        auto next_stage = [&]() SSD_INLINE {
            free = slot;
            slot = slot + 1 == NST ? 0 : slot + 1;
        };
        // the steps 0 .. Q - 2 of a chunk whose first fragments are in fa; the last step's end up in fb
        auto earlier_steps = [&](auto load) SSD_INLINE {
            step(std::integral_constant<int, 1>{}, even, fa, codes, fb, 1, load);
            if constexpr (Q == 4) {
                step(std::integral_constant<int, 2>{}, odd, fb, all, fa, 2, load);
                step(std::integral_constant<int, 3>{}, even, fa, codes, fb, 3, load);
            }
        };
#pragma unroll
        for (int u = 0; u < NST; ++u)
            if (u < nchunks) {
                if (tail && u == nchunks - 1) shorten();
                static_for<0, PER>([&](auto ic) SSD_INLINE { issue(ic, u, u); });
            }
        if (nchunks >= NST) landed(std::integral_constant<int, NST - 1>{});
        else landed(std::integral_constant<int, 0>{});
        if (whole > 0) {
            static_for<0, READS>([&](auto ec) SSD_INLINE { read1(ec, fa, 0, 0); });
            earlier_steps(std::false_type{});
            int c = 1;
            // from the barrier in front of chunk c on: the last step of the chunk before, whose stage is free, and all but the last of its own.
            // Without branches, across which the compiler would move the products together.
            auto period = [&](auto load) SSD_INLINE {
                constexpr bool LOAD = decltype(load)::value;
                landed(std::integral_constant<int, LOAD ? NST - 2 : 0>{});
                if (LOAD && tail && ahead == nchunks - 1) shorten();
                next_stage();
                step(std::integral_constant<int, 0>{}, odd, fb, all, fa, 0, load);
                if (ends(c)) flush();
                earlier_steps(load);
                if (LOAD) ++ahead;
                ++c;
            };
            const int loading = max(0, min(nchunks - NST, whole - 1)), rest = whole - 1 - loading;
            for (int i = 0; i < loading; ++i) period(std::true_type{});
            for (int i = 0; i < rest; ++i) period(std::false_type{});
            static_for<0, TN * TM>([&](auto jc) SSD_INLINE { multiply1(jc, odd, fb); });
        }
        if (tail) {
            if (whole > 0) {
                landed(std::integral_constant<int, 0>{});
                next_stage();
                if (ends(whole)) flush();
            }
            for (int q = 0; q * 64 < tail; ++q) {
                Frags f;
                static_for<0, READS>([&](auto ec) SSD_INLINE { read1(ec, f, slot, q); });
                const bool half = q * 64 + 32 >= tail;                       // 32 columns are left: blocks 1 are zeros
                const uint4 zero = make_uint4(0, 0, 0, 0);
#pragma unroll
                for (int n = 0; n < TN; ++n) {
                    if (half && lh) f.w[n] = zero;
                    f.sw[n] = half && lh ? 127u << 8 : f.sw[n] >> (q % 2 * 16);
                }
#pragma unroll
                for (int m = 0; m < TM; ++m) {
                    if (half) f.x[m][1] = zero;
                    f.sx[m] = half && lh ? 127u << 8 : f.sx[m] >> (q % 2 * 16);
                }
                static_for<0, TN * TM>([&](auto jc) SSD_INLINE { multiply1(jc, even, f); });
            }
        }
    }
    if constexpr (BEHIND)
#pragma unroll
        for (int n = 0; n < TN; ++n)
#pragma unroll
            for (int m = 0; m < TM; ++m)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float t = tot[n][m][i], l = last[n][m][i], v = acc[n][m][i];
                    acc[n][m][i] = a.split > 3 ? t + (l + v) : (t + l) + v;
                }
    if constexpr (HALVES) {
        // one slice alone, where rounding up to chunks leaves the other one empty
        if (k1 - k0 > k_len)
#pragma unroll
            for (int n = 0; n < TN; ++n)
#pragma unroll
                for (int m = 0; m < TM; ++m)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[n][m][i] = tot[n][m][i] + acc[n][m][i];
    }

    // ---- results.  Lane (lm, lh) holds, per tile, weight rows 8 g + 4 lh + j of activation row lm.  They pass through LDS, where
    // every wave has an area of its own, into row order, so that a store covers whole pieces of rows.
    __syncthreads();                                                         // the last fragments of the rings have been read
    if constexpr (ALL) {
        using T = std::conditional_t<RESULT == SSD_MX_OUT_F32, float, bf16_t>;
        float4* const t = (float4*)smem_u4;                                  // [slice][row tile]: 32 lines of 128 bytes, as below
        const bool whole4 = a.N % 4 == 0;
#pragma unroll
        for (int m = 0; m < TM; ++m)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                t[(id_of_wave * TM + m) * 256 + lm * 8 + ((g * 2 + lh) ^ (lm & 7))] = make_float4(acc[0][m][4 * g], acc[0][m][4 * g + 1], acc[0][m][4 * g + 2], acc[0][m][4 * g + 3]);
        __syncthreads();
        const bool fourth = a.split > 3;                                     // three or four slices (mx_slices)
#pragma unroll
        for (int m = 0; m < TM; ++m) {
            const int r = id_of_wave * 8 + (lane >> 3), row = m0 + m * 32 + r, col = bx * 32 + (lane & 7) * 4, at = m * 256 + r * 8 + ((lane & 7) ^ (r & 7));
            const float4 p0 = t[at], p1 = t[at + TM * 256], p2 = t[at + 2 * TM * 256], p3 = t[at + 3 * TM * 256];
            const float v[4] = {(p0.x + p1.x) + (fourth ? p2.x + p3.x : p2.x), (p0.y + p1.y) + (fourth ? p2.y + p3.y : p2.y),
                                (p0.z + p1.z) + (fourth ? p2.z + p3.z : p2.z), (p0.w + p1.w) + (fourth ? p2.w + p3.w : p2.w)};
            if (row < a.M) mx_store4((T*)a.out + (size_t)row * a.N + col, v, a.N - col, whole4);
        }
        return;
    }
    char* const area = smem + wave * S::OUT;
#pragma unroll
    for (int m = 0; m < TM; ++m) {
        const int row0 = m0 + (wm * TM + m) * 32;
        if constexpr (CHANNELS) {
            constexpr int PR = TN, LINE = PR * 16 + 16;                      // 16-byte pieces of a row; bytes of its line in LDS
            static_assert(32 * LINE <= S::OUT, "a wave's area");
            const int ch0 = (bx * (BN / 64) + wn * TN / 2) * 32, row = row0 + lm;
            wave_lds_order();                                                // every lane has read what is overwritten next
#pragma unroll
            for (int n = 0; n < TN; n += 2) {
                const int ch = ch0 + n * 16;
                const unsigned code = mx_store_channels(acc[n][m], acc[n + 1][m], lh, (uint8_t*)area + lm * LINE + n * 16, true);
                if (lh == 0 && row < mx_pad_rows(a.M) && ch < F) {
                    uint8_t* word = (uint8_t*)(a.out_s + mx_scale_word(ch >> 7, row, a.M));
                    word[ch >> 5 & 3] = (uint8_t)(row < a.M ? code : 127);
                    if (ch + 32 >= F)
                        for (int b = (ch >> 5 & 3) + 1; b < 4; ++b) word[b] = 127;   // blocks that only fill up the last group
                }
            }
            wave_lds_order();                                                // other lanes wrote what is read next
#pragma unroll
            for (int i = 0; i < PR / 2; ++i) {
                const int r = i * (64 / PR) + lane / PR, at = lane % PR * 16;
                const uint4 v = *(const uint4*)(area + r * LINE + at);
                if (row0 + r < a.M && ch0 + at < F) *(uint4*)((uint8_t*)a.out + (size_t)(row0 + r) * F + ch0 + at) = v;
            }
        } else {
            using T = std::conditional_t<RESULT == SSD_MX_OUT_F32, float, bf16_t>;
            float4* const t = (float4*)area;                                 // 32 lines of 128 bytes, piece s of line r in slot s ^ (r % 8)
            const bool whole4 = a.N % 4 == 0;
#pragma unroll
            for (int n = 0; n < TN; ++n) {
                wave_lds_order();
#pragma unroll
                for (int g = 0; g < 4; ++g) t[lm * 8 + ((g * 2 + lh) ^ (lm & 7))] = make_float4(acc[n][m][4 * g], acc[n][m][4 * g + 1], acc[n][m][4 * g + 2], acc[n][m][4 * g + 3]);
                wave_lds_order();
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int r = g * 8 + (lane >> 3), col = bx * BN + (wn * TN + n) * 32 + (lane & 7) * 4;
                    const float4 o = t[r * 8 + ((lane & 7) ^ (r & 7))];
                    const float v[4] = {o.x, o.y, o.z, o.w};
                    if (row0 + r < a.M) mx_store4((T*)a.out + (size_t)bz * a.part_stride + (size_t)(row0 + r) * a.N + col, v, a.N - col, whole4);
                }
            }
        }
    }
}

// Launches one shape; *n_part = the partial sums it leaves.
template <int WN, int WM, int TN, int TM, int KC, int NST, int RESULT, bool HALVES, bool NT, int JOIN = MX_APART>
bool mx_launch_shape(const MxArgs& a, int* n_part) {
    using S = MxShape<WN, WM, TN, TM, KC, NST, RESULT, HALVES, NT, JOIN>;
    static_assert(S::LDS <= 160 * 1024, "LDS budget");
    auto kern = k_mx_gemm<WN, WM, TN, TM, KC, NST, RESULT, HALVES, NT, JOIN>;
    static bool attr_done[64];                               // per device
    int device = 0;
    if (hipGetDevice(&device) != hipSuccess) return false;
    if (device >= 64 || !attr_done[device]) {
        if (hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, S::LDS) != hipSuccess) return false;
        if (device < 64) attr_done[device] = true;
    }
    const int slices = mx_slices(a.K, a.split), parts = JOIN != MX_APART ? 1 : HALVES ? (slices + 1) / 2 : slices;
    const int n_blocks = (a.N + S::BN - 1) / S::BN, m_blocks = (a.M + S::BM - 1) / S::BM;
    *n_part = parts;
    kern<<<dim3((unsigned)(n_blocks * m_blocks * parts)), S::WAVES * 64, S::LDS, a.st>>>(a, n_blocks, m_blocks, parts);
    return true;
}

// Launches shape `kind` if it is one of FIRST .. LAST and yields RESULT (the shapes are spread over translation units, which compile
// in parallel); false if not.
template <int RESULT, int FIRST, int LAST>
bool mx_launch_kind(const MxArgs& a, int kind, int* n_part) {
#define MX_KIND_CASE(id, wn, wm, tn, tm, kc, nst, nt, halves, results, ...)                                     \
    if constexpr (id >= FIRST && id <= LAST && ((results) & (RESULT == SSD_MX_OUT_SWIGLU ? 2 : 1)) != 0 &&       \
                  !(halves && RESULT != SSD_MX_OUT_F32))                                                         \
        if (kind == id) return mx_launch_shape<wn, wm, tn, tm, kc, nst, RESULT, halves, nt>(a, n_part);
    MX_KINDS(MX_KIND_CASE)
#undef MX_KIND_CASE
    return false;
}

// The same for the shapes with all slices in a work-group.
template <int RESULT>
bool mx_launch_all(const MxArgs& a, int kind) {
    int parts;
#define MX_ALL_CASE(id, wn, wm, tn, tm, kc, nst, nt, join, ...) \
    if (kind == id) return mx_launch_shape<wn, wm, tn, tm, kc, nst, RESULT, false, nt, join>(a, &parts);
    MX_ALL_KINDS(MX_ALL_CASE)
#undef MX_ALL_CASE
    return false;
}
