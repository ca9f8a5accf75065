// Layouts of microscaled 4-bit rows and weights (see regione.h), shared by their conversion and their products.
#pragma once
#include "common.h"

constexpr int kMxBlock = 32;             // values that share a scale
constexpr int kMxStep = 256;             // values of a row in one K-step of the products: 128 bytes of codes, eight scales

// Scales in steps: for every step the rows one after the other, eight bytes per row, so that the rows of a tile are one piece of memory and a matrix
// instruction's lane (row l%16, block l/16 of the step's first or second 128 values) finds the scales of both halves side by side: block b at byte 2*(b%4) + b/4.
// An even number of rows keeps every step 16-byte aligned.
__host__ __device__ __forceinline__ int64_t mx_padded_rows(int64_t rows) { return (rows + 1) & ~static_cast<int64_t>(1); }
__host__ __device__ __forceinline__ int64_t mx_scale_step(int64_t row, int block, int64_t padded_rows) {
    return ((block >> 3) * padded_rows + row) * 8 + 2 * (block & 3) + ((block >> 2) & 1);
}
__host__ __device__ __forceinline__ int64_t mx_packed_bytes(int n, int k) {
    const int64_t n32 = (n + 31) & ~31, steps = (k + kMxStep - 1) / kMxStep;
    return n32 * steps * (kMxStep / 2 + 8);
}
// 2^(byte - 127), as the conversion instructions take it: they read the exponent field
__device__ __forceinline__ float mx_scale_value(unsigned byte) { return __uint_as_float(byte << 23); }
