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
