// Products of microscaled 4-bit rows and weights, and products over groups of rows that have weights of their own (4-bit and bf16).
//
//   y[r, c] = act(sum_k x[r, k] w[c, k] + b[c])
//
// Both formats move the same bytes: a K-step is 128 bytes of every row, 64 bf16 or 256 E2M1 values, and a lane feeds 16 of them to a matrix instruction
// (v_mfma_f32_16x16x32_bf16, v_mfma_scale_f32_16x16x128_f8f6f4), in 4 bits together with the byte of their scale: the instruction's lane holds 32 values of one row,
// which is one block.  The instruction multiplies E2M1 values exactly and applies both powers of two; sums are float32.  The weights are the first operand, so that a
// lane ends up with eight consecutive columns of a row and the other products' epilogue serves here, too.
#pragma once
#include "gemm_epilogue.h"
#include "mx.h"

namespace {

enum { MX_BF16 = 0, MX_FP4 = 1 };

// Operands of a product: a [m, row_bytes], packed weights one after the other (w_stride bytes each).  Groups: rows [offsets[g], offsets[g + 1]) are those of weight
// use[g] (of weight g without `use`); without offsets all rows are one group.
struct MxOperands {
    const uint8_t* a; const uint8_t* a_scale; const uint8_t* w; int64_t w_stride;
    const int32_t* offsets; const int32_t* use; int n_groups, n_weights;
    int m, n, row_bytes, steps;
};

// The tile of a workgroup: rows [row0, row0 + R) below `end`, of weight `weight`.
struct MxTile { int row0, end, weight; };

// Row tile `unit` of a launch: the groups' tiles of R rows follow each other.  Every wave finds it by itself: 64 groups at a time, the tiles before each by a prefix sum.  False
// where there are fewer tiles than units.  Offsets outside [0, m] are taken as the nearer end, a group that ends before it starts is empty, and one whose
// weight does not exist is passed over.
template <int R>
__device__ __forceinline__ bool mx_find_tile(const MxOperands& p, int unit, MxTile& t) {
    if (!p.offsets) {
        t = {unit * R, p.m, 0};
        return t.row0 < p.m;
    }
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int g0 = 0; g0 < p.n_groups; g0 += 64) {
        const int g = g0 + lane;
        int lo = 0, hi = 0, w = 0;
        if (g < p.n_groups) {
            lo = p.offsets[g]; hi = p.offsets[g + 1];
            w = p.use ? p.use[g] : g;
            lo = lo < 0 ? 0 : (lo < p.m ? lo : p.m);
            hi = hi < 0 ? 0 : (hi < p.m ? hi : p.m);
            if (hi < lo || w < 0 || w >= p.n_weights) hi = lo;
        }
        const int tiles = (hi - lo + R - 1) / R;
        int upto = tiles;                                       // tiles of the groups up to this lane's
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int other = __shfl_up(upto, d);
            if (lane >= d) upto += other;
        }
        const int total = __shfl(upto, 63);
        if (unit < before + total) {
            const int first = __builtin_ctzll(__ballot(before + upto > unit));       // the group that holds the unit
            const int in_group = unit - before - __shfl(upto - tiles, first);
            t.row0 = __builtin_amdgcn_readfirstlane(__shfl(lo, first) + in_group * R);
            t.end = __builtin_amdgcn_readfirstlane(__shfl(hi, first));
            t.weight = __builtin_amdgcn_readfirstlane(__shfl(w, first));
            return true;
        }
        before += total;
    }
    return false;
}

__device__ __forceinline__ i32x8 mx_half_operand(const u32x4& v) { return i32x8{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0}; }
// one matrix instruction on half H of a step; scales: bytes H of both
template <int FMT, int H>
__device__ __forceinline__ f32x4 mx_mfma(const u32x4& w, const u32x4& a, const f32x4& acc, unsigned w_scale, unsigned a_scale) {
    if constexpr (FMT == MX_BF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, a), acc, 0, 0, 0);
    else return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(mx_half_operand(w), mx_half_operand(a), acc, 4, 4, H, static_cast<int>(w_scale), H, static_cast<int>(a_scale));
}

// 16 rows x 16*CF columns per workgroup; its waves split K, read their fragments straight from memory with the loads of CHUNK steps in flight, and meet in LDS,
// where the sums are formed in wave order.
constexpr int kMxSmallRows = 16, kMxSmallWaves = 8;

template <int FMT, int CF>
__global__ void __launch_bounds__(kMxSmallWaves * 64) __attribute__((amdgpu_waves_per_eu(2)))
gemm_mx_small_kernel(MxOperands p, GemmEpilogue ep) {
    constexpr int CHUNK = CF == 2 ? 6 : 3;
    __shared__ __attribute__((aligned(16))) f32x4 sums[kMxSmallWaves * CF * 64];
    const int n_tiles = (p.n + 16 * CF - 1) / (16 * CF), unit = static_cast<int>(blockIdx.x) / n_tiles;
    MxTile t;
    if (!mx_find_tile<kMxSmallRows>(p, unit, t)) return;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, kc = lane >> 4;
    const int n0 = (static_cast<int>(blockIdx.x) - unit * n_tiles) * (16 * CF), n32 = (p.n + 31) & ~31;
    const int per = (p.steps + kMxSmallWaves - 1) / kMxSmallWaves, s0 = wave * per, s1 = s0 + per < p.steps ? s0 + per : p.steps;

    const uint8_t* w = p.w + t.weight * p.w_stride;
    const uint8_t* wp[CF / 2];
    const uint8_t* wsp[CF];
#pragma unroll
    for (int b = 0; b < CF / 2; ++b) {
        int nb = (n0 >> 5) + b;
        nb = nb < n32 / 32 ? nb : n32 / 32 - 1;                 // blocks past N repeat the last one; their sums are not stored
        const int col = 8 * (l16 >> 2) + (l16 & 3);             // of fragment 2 b; the other one's is four further (see gemm_epilogue16)
        wp[b] = w + ((static_cast<int64_t>(nb) * p.steps * 4 + (kc >> 1)) * 64 + (kc & 1) * 32 + col) * 16;
#pragma unroll
        for (int jl = 0; jl < 2; ++jl) wsp[2 * b + jl] = w + static_cast<int64_t>(n32) * p.steps * 128 + (nb * 32 + col + 4 * jl) * 8 + 2 * kc;
    }
    int row = t.row0 + l16;
    row = row < t.end ? row : t.end - 1;                        // rows past the end repeat the last one
    const uint8_t* ap = p.a + static_cast<int64_t>(row) * p.row_bytes;
    const int64_t a_step = mx_padded_rows(p.m) * 8;
    const uint8_t* asp = FMT == MX_FP4 ? p.a_scale + static_cast<int64_t>(row) * 8 + 2 * kc : nullptr;

    f32x4 acc[CF];
#pragma unroll
    for (int j = 0; j < CF; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    u32x4 av[CHUNK][2], wv[CHUNK][2][CF];
    unsigned as[CHUNK], ws[CHUNK][CF];
    for (int base = s0; base < s1; base += CHUNK) {
#pragma unroll
        for (int i = 0; i < CHUNK; ++i) {
            const int s = base + i;
            if (s < s1) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int at = s * 128 + h * 64 + kc * 16;  // past the row's end the weights are zero, and a row's first values serve
                    av[i][h] = *reinterpret_cast<const u32x4*>(ap + (at < p.row_bytes ? at : 0));
#pragma unroll
                    for (int j = 0; j < CF; ++j)
                        wv[i][h][j] = *reinterpret_cast<const u32x4*>(wp[j >> 1] + (static_cast<int64_t>(s) * 4 + 2 * h) * 1024 + (j & 1) * 64);
                }
                if (FMT == MX_FP4) {
                    as[i] = *reinterpret_cast<const uint16_t*>(asp + s * a_step);
#pragma unroll
                    for (int j = 0; j < CF; ++j) ws[i][j] = *reinterpret_cast<const uint16_t*>(wsp[j] + static_cast<int64_t>(s) * n32 * 8);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < CHUNK; ++i)
            if (base + i < s1) {
#pragma unroll
                for (int j = 0; j < CF; ++j) acc[j] = mx_mfma<FMT, 0>(wv[i][0][j], av[i][0], acc[j], ws[i][j], as[i]);
#pragma unroll
                for (int j = 0; j < CF; ++j) acc[j] = mx_mfma<FMT, 1>(wv[i][1][j], av[i][1], acc[j], ws[i][j], as[i]);
            }
    }
#pragma unroll
    for (int j = 0; j < CF; ++j) sums[(wave * CF + j) * 64 + lane] = acc[j];
    __syncthreads();
    if (wave >= CF / 2) return;
    f32x4 sum[2];
#pragma unroll
    for (int jl = 0; jl < 2; ++jl) {
        sum[jl] = sums[(2 * wave + jl) * 64 + lane];
#pragma unroll
        for (int v = 1; v < kMxSmallWaves; ++v) sum[jl] += sums[(v * CF + 2 * wave + jl) * 64 + lane];
    }
    if (ep.bias) ep.bias += static_cast<int64_t>(t.weight) * p.n;
    const int col = n0 + 32 * wave + 8 * kc;
    if (t.row0 + l16 >= t.end || col >= p.n) return;
    if (col + 8 > p.n) { epilogue_ragged<EPI_PLAIN, false>(ep, row, col, p.n, sum[0], sum[1]); return; }
    EpiColumns<EPI_PLAIN, false> cols;
    EpiRow<EPI_PLAIN, false> r;
    Raw8 raw;
    cols.load(ep, col);
    r.load(ep, row);
    if (ep.vec_ok) epilogue_store8<EPI_PLAIN, false, true>(ep, row, col, sum[0], sum[1], cols, r, raw);
    else epilogue_store8<EPI_PLAIN, false, false>(ep, row, col, sum[0], sum[1], cols, r, raw);
}

}  // namespace
