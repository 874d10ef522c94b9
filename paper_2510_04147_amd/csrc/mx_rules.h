// Sizes of the microscaled form and how a product is cut: plain C++ without HIP, so that a host compiler can check it.
#pragma once
#include <stddef.h>

__attribute__((unused)) static const int MX_STEP = 64;      // columns of a matrix instruction
__attribute__((unused)) static const int MX_CHUNK = 256;    // k-slices are whole chunks, but for the last one's end

#ifdef __HIPCC__
#define MX_HD __host__ __device__
#else
#define MX_HD
#endif
// Rows of the scales: whole tiles of 32 rows, so that a tile's scale words are one aligned line.
MX_HD inline int mx_pad_rows(int rows) { return (rows + 31) / 32 * 32; }
MX_HD inline int mx_groups(int cols) { return (cols + 127) / 128; }

// k-slices of a product: a function of the matrix alone, so that a row's order of summation is the same in every call.  A matrix
// with few rows and many columns takes four, which fill the chip when few rows of activations leave nothing else to split.
inline int mx_split(int N, int K, bool swiglu) { return swiglu || K < 2048 || N > 8192 ? 1 : 4; }
// Columns of a slice.
MX_HD inline int mx_slice(int K, int split) { return (K + split * MX_CHUNK - 1) / (split * MX_CHUNK) * MX_CHUNK; }
// Slices that hold columns: rounding up to chunks can leave the last ones empty.
MX_HD inline int mx_slices(int K, int split) { return (K + mx_slice(K, split) - 1) / mx_slice(K, split); }

// The shapes of the product's kernel (mx_gemm.h): id, waves along weight and activation rows, tiles of 32 rows of a wave, columns of a
// chunk, stages of the ring, weights loaded past the L2 (one pass streams them), k-halves, which results (1: sums, 2: activated channels),
// and the time of a call in us:
//     a + b rounds over the 256 CUs + rounds x steps of 64 columns x c + share of the chip's work-groups x steps x d
//     + weights, millions, x e + results, millions x partial sums, x f
// d on top of c because a round that fills the chip only partly finds memory and clocks less loaded.  Fitted to 3605 timings of 18
// matrices (512 to 37888 rows, 512 to 18944 columns), 1 to 2304 activation rows, every shape timed for each; one shape's time is met within 3 to
// 9 % rms.  The choice is 0.6 % slower than the fastest shape on average, 4 % at the 95th percentile and 13 % at most.
// us of some shapes by tile, weight rows x activation rows, in turn on one card: 12288 x 4096, 32 rows 64x32 9.8, 64x64 10.7,
// 32x32 11.0, 128x96 13.9; 160 rows 128x96 17.4, 128x128 20.0, 64x64 27.9; 1000 rows 192x256 52.1, 256x256 55.7, 128x128 66.6; gate/up of
// 24576 x 4096, 32 rows 128x32 13.4, 64x32 15.0, 128x64 15.2; 160 rows 192x96 24.7, 256x128 33.0, 256x64 35.6; of 37888 x 3584, 2304 rows
// 256x192 278, 256x256 279, 256x128 310.
#define MX_KINDS(X)                                                                                             \
    X(0, 1, 1, 1, 1, 256, 4, true, false, 1, 2.6162, 0.5747, 0.0466, 0.0000, 0.0266, 1.9548)                    \
    X(1, 2, 1, 1, 1, 256, 6, true, false, 1, 1.3974, 1.7863, 0.0587, 0.0149, 0.0429, 1.4530)                    \
    X(2, 2, 2, 1, 1, 256, 4, true, false, 1, 1.7568, 1.5940, 0.0822, 0.0214, 0.0243, 0.7856)                    \
    X(3, 4, 1, 1, 2, 256, 4, true, false, 1, 1.9364, 1.7508, 0.1305, 0.0185, 0.0148, 0.7602)                    \
    X(4, 4, 1, 1, 3, 256, 3, true, false, 1, 2.1455, 2.0250, 0.1460, 0.0303, 0.0015, 0.6846)                    \
    X(5, 2, 2, 2, 2, 256, 3, true, false, 3, 1.8679, 2.7029, 0.1616, 0.0230, 0.0137, 0.6465)                    \
    X(6, 2, 2, 4, 2, 128, 4, false, false, 3, 1.6124, 3.2137, 0.3056, 0.0079, 0.0369, 0.5122)                   \
    X(7, 2, 2, 3, 4, 128, 3, false, false, 1, 3.1544, 3.7368, 0.3758, 0.0958, 0.0005, 0.3694)                   \
    X(8, 2, 2, 4, 4, 128, 3, false, false, 3, 0.5452, 7.8770, 0.4636, 0.0911, 0.0060, 0.2794)                   \
    X(9, 2, 2, 1, 2, 256, 3, true, true, 1, 2.4762, 0.9289, 0.1323, 0.0288, 0.0000, 0.7424)                     \
    X(10, 2, 2, 2, 2, 128, 4, false, true, 1, 2.6675, 1.8194, 0.1472, 0.0920, 0.0658, 0.4508)                   \
    X(11, 2, 2, 2, 4, 128, 3, false, true, 1, 1.5978, 5.3398, 0.3031, 0.0407, 0.0176, 0.3375)                   \
    X(12, 1, 1, 2, 1, 256, 4, true, false, 2, 3.7295, 0.1686, 0.0684, 0.0077, 0.0423, 0.9168)                   \
    X(13, 2, 1, 2, 1, 256, 4, true, false, 2, 1.7610, 2.1913, 0.0976, 0.0000, 0.0413, 0.9342)                   \
    X(14, 2, 2, 2, 1, 256, 4, true, false, 2, 1.9830, 1.6215, 0.1484, 0.0000, 0.0192, 0.5291)                   \
    X(15, 4, 1, 2, 2, 256, 3, true, false, 2, 1.9282, 3.1649, 0.1796, 0.0205, 0.0331, 0.2163)                   \
    X(16, 3, 1, 2, 3, 256, 3, true, false, 2, 3.2515, 2.0753, 0.2205, 0.0000, 0.0175, 0.5842)                   \
    X(17, 2, 2, 4, 3, 128, 3, false, false, 2, 0.0000, 6.4031, 0.3822, 0.0780, 0.0087, 0.0548)
#define MX_N_KINDS 18

struct MxKind { int wn, wm, tn, tm, kc, nst; bool halves; int results; double t[6]; };
inline const MxKind& mx_kind(int id) {
#define MX_KIND_ROW(id, wn, wm, tn, tm, kc, nst, nt, halves, results, a, b, c, d, e, f) {wn, wm, tn, tm, kc, nst, halves, results, {a, b, c, d, e, f}},
    static const MxKind kinds[MX_N_KINDS] = {MX_KINDS(MX_KIND_ROW)};
#undef MX_KIND_ROW
    return kinds[id];
}

// The shape for a call: the least estimated time, with 0.8 us for a million partial sums that the consumer reads again.
inline int mx_choose(int M, int N, int K, int slices, bool swiglu, double* time = nullptr) {
    int best = -1;
    double least = 0;
    for (int i = 0; i < MX_N_KINDS; ++i) {
        const MxKind& k = mx_kind(i);
        if (!(k.results & (swiglu ? 2 : 1)) || (k.halves && slices < 2)) continue;
        const int bn = k.wn * k.tn * 32, bm = k.wm * k.tm * 32, parts = k.halves ? (slices + 1) / 2 : slices;
        const double wgs = (double)((N + bn - 1) / bn) * ((M + bm - 1) / bm) * parts, rounds = (double)(long long)((wgs + 255) / 256);
        const double walk = (double)mx_slice(K, slices) * (k.halves ? 2 : 1), steps = (walk < K ? walk : K) / MX_STEP;
        const double sums = (double)parts * M * N / 1e6;
        const double t = k.t[0] + k.t[1] * rounds + k.t[2] * rounds * steps + k.t[3] * wgs * steps / 256 + k.t[4] * N * K / 1e6 + k.t[5] * sums +
                         (slices > 1 ? 0.8 * sums : 0);
        if (best < 0 || t < least) { best = i; least = t; }
    }
    if (time) *time = least;
    return best;
}

// A product of three or four slices whose sum is wanted, not its parts, is one launch where that is faster (mx_gemm.h): slices beside each other, a
// work-group of four waves per 32 weight rows and each wave a slice, for few rows; slices behind each other, for many.  id, as above but for the
// result, MX_BESIDE or MX_BEHIND, and the call's time as above, with the steps of a slice or of all of them.  The launch that adds partial
// sums takes 3.5 us and 0.03 for a million outputs.  Fitted to 126 calls of 14 matrices (64 to 8192 rows, 2048 to 18944 columns), 1 to 160
// activation rows, and 195 of 13, 64 to 4000 rows, weights from memory.  The choice is 0.4 % slower than the fastest way on average, 19 % at most.
// us, one launch / two: 4096 x 4096 1 row 6.3 / 7.2, 64 rows 6.7 / 10.0, 500 rows 13.6 / 19.7, 1000 rows 21.2 / 29.8, 2304 rows 59.5 / 70.7;
// 4096 x 12288 1 row 14.3 / 10.9, 1000 rows 54.5 / 56.5; 8192 x 2048 64 rows 6.7 / 11.2, 2304 rows 65.9 / 99.5.
// Slices behind each other have tiles of at most 128 rows (three sets of sums are all that registers hold), so they read the activations more often.
// The times were fitted to activations of no more than the L2s hold, and past M K = 2^24 the slices stay apart.  Measured past it (up to 50 M values,
// 512 to 8192 weight rows; behind each other / apart, ratio by columns): 2080 0.46 to 0.84, 4096 0.62 to 0.83, 8192 0.74 to 1.05, 12288 0.89 to 1.26: at
// 12288 columns the border is right, with fewer it costs the calls of many rows (us, 10082 x 8192 x 2080 310 / 603, 8192 x 4096 x 4096 190 / 285,
// 6144 x 4096 x 8192 253 / 277, 4096 x 4096 x 12288 251 / 217).
enum { MX_APART, MX_BESIDE, MX_BEHIND };
#define MX_ALL_KINDS(X)                                                                                          \
    X(0, 1, 1, 1, 1, 256, 2, true, MX_BESIDE, 1.6333, 0.2987, 0.2191, 0.0000, 0.0442, 3.1069)                    \
    X(1, 1, 1, 1, 2, 128, 3, true, MX_BESIDE, 1.7476, 0.0000, 0.3106, 0.0320, 0.0191, 3.4893)                    \
    X(2, 2, 2, 1, 1, 256, 4, false, MX_BEHIND, 1.3649, 2.2618, 0.0941, 0.0148, 0.0000, 0.1919)                   \
    X(3, 4, 1, 1, 2, 256, 4, false, MX_BEHIND, 1.1710, 3.3180, 0.1316, 0.0210, 0.0047, 0.0494)                   \
    X(4, 2, 2, 2, 2, 256, 3, false, MX_BEHIND, 0.0914, 5.7895, 0.1891, 0.0536, 0.0165, 0.0511)
#define MX_N_ALL_KINDS 5

// Which of them a call takes, -1: none.
inline int mx_choose_all(int M, int N, int K, int slices) {
    if (slices < 3) return -1;
    struct Kind { int bn, bm, join; double t[6]; };
#define MX_ALL_ROW(id, wn, wm, tn, tm, kc, nst, nt, join, a, b, c, d, e, f) {wn * tn * 32, wm * tm * 32, join, {a, b, c, d, e, f}},
    static const Kind kinds[MX_N_ALL_KINDS] = {MX_ALL_KINDS(MX_ALL_ROW)};
#undef MX_ALL_ROW
    int best = -1;
    double least;
    mx_choose(M, N, K, slices, false, &least);
    least += 3.5 + 0.03e-6 * M * N;
    for (int i = 0; i < MX_N_ALL_KINDS; ++i) {
        const Kind& k = kinds[i];
        if (k.join == MX_BEHIND && (double)M * K > 1 << 24) continue;
        const double wgs = (double)((N + k.bn - 1) / k.bn) * ((M + k.bm - 1) / k.bm), rounds = (double)(long long)((wgs + 255) / 256);
        const double steps = (double)(k.join == MX_BESIDE ? mx_slice(K, slices) : K) / MX_STEP;
        const double t = k.t[0] + k.t[1] * rounds + k.t[2] * rounds * steps + k.t[3] * wgs * steps / 256 + k.t[4] * N * K / 1e6 + k.t[5] * M * N / 1e6;
        if (t < least) { best = i; least = t; }
    }
    return best;
}
