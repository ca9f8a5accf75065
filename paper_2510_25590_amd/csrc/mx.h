// Layouts of microscaled 4-bit rows and weights (see regione.h), shared by their conversion and their products.
#pragma once
#include "common.h"

constexpr int kMxBlock = 32;             // values that share a scale
constexpr int kMxMostInputs = 1 << 20, kMxMostFeatures = 1 << 24;         // of a product: offsets inside a tile stay below 2^31 bytes
constexpr int kMxStep = 256;             // values of a row in one K-step of the products: 128 bytes of codes, eight scales

// Scales in steps: for every step the rows one after the other, eight bytes per row, so that the rows of a tile are one piece of memory.  Block b is byte 4*(b%2) + b/2: a lane of
// the 32x32x64 instruction (row l%32, block l/32 of the two) finds its scales for the step's four instructions in one word, and names them by the instruction's byte select.
// An even number of rows keeps every step 16-byte aligned.
__host__ __device__ __forceinline__ int64_t mx_padded_rows(int64_t rows) { return (rows + 1) & ~static_cast<int64_t>(1); }
__host__ __device__ __forceinline__ int64_t mx_scale_step(int64_t row, int block, int64_t padded_rows) {
    return ((block >> 3) * padded_rows + row) * 8 + 4 * (block & 1) + ((block & 7) >> 1);
}
__host__ __device__ __forceinline__ int64_t mx_packed_bytes(int n, int k) {
    const int64_t n32 = (static_cast<int64_t>(n) + 31) & ~31, steps = (static_cast<int64_t>(k) + kMxStep - 1) / kMxStep;
    return n32 * steps * (kMxStep / 2 + 8);
}
// 2^(byte - 127), as the conversion instructions take it: they read the exponent field
__device__ __forceinline__ float mx_scale_value(unsigned byte) { return __uint_as_float(byte << 23); }

// ---- products
enum { MX_BF16 = 0, MX_FP4 = 1 };

// Operands of a product: a [m, row_bytes], packed weights one after the other (w_stride bytes each).  Groups: rows [offsets[g], offsets[g + 1]) are those of weight
// use[g] (of weight g without `use`); without offsets all rows are one group.
struct MxOperands {
    const uint8_t* a; const uint8_t* a_scale; const uint8_t* w; int64_t w_stride;
    const int32_t* offsets; const int32_t* use; int n_groups, n_weights;
    int m, n, row_bytes, steps;
};

// Row tiles of R rows that a launch may have: of groups, which begin at even rows, one more each.  Groups that share rows, against their contract, can have more: those beyond are not run.
static __host__ __device__ inline int64_t mx_most_row_tiles(const MxOperands& p, int R) {
    if (!p.offsets) return (static_cast<int64_t>(p.m) + R - 1) / R;
    return p.m / R + (p.n_groups < p.m ? p.n_groups : p.m);
}

// The kernel of tiles (gemm_mx_tile.h): its code is 10 * RF + CF, for 32 * RF rows and 128 * CF columns.  REGIONE_ERR_INVALID_ARG for a code that there is no kernel of.
int rg_mx_tile_4bit(regione_ctx* ctx, int tile, const MxOperands& p, int splits, const GemmEpilogue& ep);
int rg_mx_tile_bf16(regione_ctx* ctx, int tile, const MxOperands& p, int splits, const GemmEpilogue& ep);
