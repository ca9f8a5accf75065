// Low-rank adapters beside a projection, in the projection's kernels: y[r] += sum over s of (weight[r, s] x[r] A_a^T) B_a^T, a = which[r, s].
//
// The inner products with A, times their weights, are there already (adapters.hip) as bf16 terms that add up to them, `blocks` blocks of 16 ranks per term, so that a row of terms times
// [B_a | B_a | ..] is the adapter's share of the result.  An adapter that a row names more than once has its weights added up.  The share is summed in the accumulators that hold the
// projection's sums: nothing is written or read in between, and the result is rounded once.
//
// Tiles (gemm_pp.h) take the terms as K-steps behind the product's own: for every adapter that a row of the tile names, in ascending order, its terms in all of the tile's rows, zeros in those
// that do not name it, in the order that a step has in LDS, the tile's steps one after the other.  As steps of the same loop they cost what K costs, and their first loads fly under the
// product's last steps: 4096 x 2048 x 2048, six steps of eight adapters behind 32, 35.7 -> 41.6 us; 820 x 12288 x 3072, up to nine behind 48, 59.1 -> 68.3.  Summed at the end of the tile, each
// wave its rows and their adapters, they waited for memory step by step, 1.7 us each.
// The plan of a tile, 32-bit words: the number of its steps, whether one of its adapters has values in B that are not finite, where its adapters stand, one unused; then for each 16 terms where
// the block of 16 ranks of B that they meet begins (64 bits), and for each 16 terms the adapter.
// Rows without the adapter must not see its values (zero times infinity): what is not finite in B is zero in the packed adapter, and the columns that hold such values are spoilt at the end,
// in the rows that name the adapter.
#pragma once
#include "gemm_epilogue.h"

namespace {

typedef const __attribute__((address_space(4))) int32_t* AdapterPlan;          // read by the scalar unit: no vector load among the counted copies
typedef __attribute__((ext_vector_type(4), aligned(8))) int64_t AdapterStep;     // where a step's four blocks of B begin, in bytes from `b`
__device__ __forceinline__ AdapterPlan adapter_plan(const AdapterRows& ad, int tile) { return (AdapterPlan)(ad.plan + static_cast<int64_t>(tile) * ad.plan_pitch); }
__device__ __forceinline__ int adapter_steps(AdapterPlan plan) { return plan[0]; }
// (a tile without adapters reads what its plan's memory holds; no copy goes there)
__device__ __forceinline__ AdapterStep adapter_step(AdapterPlan plan, int at) { return reinterpret_cast<const __attribute__((address_space(4))) AdapterStep*>(plan + 4)[at]; }
__device__ __forceinline__ const char* adapter_terms(const AdapterRows& ad, int tile) { return reinterpret_cast<const char*>(ad.t + tile * ad.tile_elems); }
// 32 columns x 16 ranks of B: block j of a step in column block nb
__device__ __forceinline__ const char* adapter_block(const AdapterRows& ad, const AdapterStep& step, int j, int nb) {
    const int64_t low = j & 1 ? step[1] : step[0], high = j & 1 ? step[3] : step[2];
    return reinterpret_cast<const char*>(ad.b) + (j & 2 ? high : low) + static_cast<int64_t>(nb) * (ad.blocks * 1024);
}
// the bits of 32 columns of an adapter
__device__ __forceinline__ uint32_t adapter_bad(const AdapterRows& ad, int id, int nb) { return ad.bad[(static_cast<int64_t>(id) * ad.stride >> 1) + nb]; }

// Rows [I0, I1) of a wave's fragments, in the layout of gemm_epilogue16: columns of adapters that hold values that are not finite, in the rows that name the adapter.
template <int I0, int I1, int RF, int CF> __device__ __forceinline__ void adapters_spoil(f32x4 (&acc)[RF][CF], int M, int N, int m0, int n0w, const AdapterRows& ad, AdapterPlan plan) {
    if (plan[1] == 0) return;
    const int lane = threadIdx.x & 63, last_block = ((N + 31) >> 5) - 1, blocks = 4 * plan[0];
    const AdapterPlan ids = plan + plan[2];
    int last = -1;
#pragma unroll 1
    for (int at = 0; at < blocks; ++at) {
        const int id = ids[at];
        if (id == last) continue;
        last = id;
        unsigned bad[CF / 2], any = 0;                            // of the lane's eight columns
#pragma unroll
        for (int b = 0; b < CF / 2; ++b) {
            const int nb = (n0w >> 5) + b;
            bad[b] = adapter_bad(ad, id, nb < last_block ? nb : last_block) >> (8 * (lane >> 4));
            any |= bad[b] & 0xffu;
        }
        if (!__ballot(any != 0)) continue;
#pragma unroll
        for (int i = I0; i < I1; ++i) {
            const int row = m0 + 16 * i + (lane & 15);
            bool named = false;
            if (row < M)
                for (int s = 0; s < ad.sel; ++s) named = named || ad.which[static_cast<int64_t>(row) * ad.sel + s] == id;
#pragma unroll
            for (int j = 0; j < CF; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][e] = named && (bad[j >> 1] >> (4 * (j & 1) + e)) & 1 ? __builtin_nanf("") : acc[i][j][e];
        }
    }
}

// Weight fragment j of a lane: column 8*(l16/4) + 4*(j%2) + l16%4 of the 32 columns' block j / 2, as the epilogue expects it, and the 16 terms of its half of a step, from `block0` on.
template <int CF> __device__ __forceinline__ void adapter_weights(const AdapterRows& ad, int a, int N, int n0, int block0, bf16x8 (&w)[CF]) {
    const int lane = threadIdx.x & 63, l16 = lane & 15, kc = lane >> 4, last_block = ((N + 31) >> 5) - 1;
    int block = block0 + (kc >> 1);
    block = block < ad.blocks ? block : block - ad.blocks;
    const int at = block * 512 + ((kc & 1) * 32 + 8 * (l16 >> 2) + (l16 & 3)) * 8;
#pragma unroll
    for (int b = 0; b < CF / 2; ++b) {
        int nb = __builtin_amdgcn_readfirstlane(n0 >> 5) + b;
        nb = nb < last_block ? nb : last_block;                   // blocks past N repeat the last one; their sums are not stored
        const bf16_t* const from = ad.b + static_cast<int64_t>(a) * ad.stride + static_cast<int64_t>(nb) * ad.blocks * 512;
        w[2 * b] = *reinterpret_cast<const bf16x8*>(from + at);
        w[2 * b + 1] = *reinterpret_cast<const bf16x8*>(from + at + 32);
    }
}
// rows of terms, all of them within 64 MB; what lies outside, such as no place at all, is zero by the resource's size
__device__ __forceinline__ auto adapter_terms_rsrc(const AdapterRows& ad, int M) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(ad.t), 0, M * ad.sel * ad.cols * 2, 0x00027000); }
constexpr unsigned kNoTerms = 0xfffffff0u;

// For the 16 rows that several waves share (gemm_small.h): t [rows, sel, cols], each adapter's terms at the first of the row's places that name it.  A unit of work is a step of 32 terms of an
// adapter that no earlier row or place of the tile names; wave `turn` of `turns` takes every unit that is its turn.  The tile's list of adapters is asked for ahead of the product's first loads
// (ask) and looked at behind them, when it has come and they have not; the first units' operands fly under the product (fetch, then add behind it).  Lists of up to 64 places stay in a register.
template <int CF> struct AdapterUnits {
    static constexpr int AHEAD = 2;
    bf16x8 wf[AHEAD][CF];
    u32x4 tf[AHEAD];
    unsigned bad[AHEAD][CF / 2];                                  // of the lane's columns, where its row names the adapter
    bool there[AHEAD];
    int next, ids;

    __device__ __forceinline__ void ask(const AdapterRows& ad, int M, int m0) {
        const int lane = threadIdx.x & 63, entries = (M - m0 < 16 ? M - m0 : 16) * ad.sel;
        ids = ad.which[static_cast<int64_t>(m0) * ad.sel + (lane < entries ? lane : 0)];
    }

    __device__ __forceinline__ void load(const AdapterRows& ad, int M, int N, int m0, int n0, int q, int unit, int units, int turns) {
        const int lane = threadIdx.x & 63, l16 = lane & 15, kc = lane >> 4, steps = ad.cols >> 5;
        there[q] = false;
        const int rows = M - m0 < 16 ? M - m0 : 16;
        const int32_t* const which = ad.which + static_cast<int64_t>(m0) * ad.sel;
        if (unit >= units) return;
        const int entry = unit / steps, st = unit - entry * steps;
        const bool held = rows * ad.sel <= 64;
        const int a = held ? __builtin_amdgcn_readlane(ids, entry) : __builtin_amdgcn_readfirstlane(which[entry]);
        if (a < 0 || a >= ad.count) return;
        if (held) {
            if (__ballot(lane < entry && ids == a)) return;       // named before
        } else {
            for (int i = 0; i < entry; i += 64)
                if (__ballot(i + lane < entry && which[i + lane < entry ? i + lane : 0] == a)) return;
        }
        unsigned at = kNoTerms;
        for (int s = ad.sel - 1; s >= 0; --s) {
            const int of = l16 * ad.sel + s;
            const int id = held ? __builtin_amdgcn_ds_bpermute(of * 4, ids) : l16 < rows ? which[of] : -1;
            if (l16 < rows && id == a) at = (static_cast<unsigned>(m0 + l16) * ad.sel + s) * (ad.cols * 2u) + 64u * st + 16u * kc;
        }
        there[q] = true;
        tf[q] = __builtin_amdgcn_raw_buffer_load_b128(adapter_terms_rsrc(ad, M), at, 0, 0);
        adapter_weights<CF>(ad, a, N, n0, 2 * st % ad.blocks, wf[q]);
        const int last_block = ((N + 31) >> 5) - 1;
#pragma unroll
        for (int b = 0; b < CF / 2; ++b) {
            const int nb = (n0 >> 5) + b;
            bad[q][b] = adapter_bad(ad, a, nb < last_block ? nb : last_block);
            bad[q][b] = st == 0 && at != kNoTerms ? bad[q][b] >> (8 * kc) : 0u;
        }
    }
    __device__ __forceinline__ void use(f32x4 (&acc)[CF], int q) {
        if (!there[q]) return;
#pragma unroll
        for (int j = 0; j < CF; ++j) {
            acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[q][j], __builtin_bit_cast(bf16x8, tf[q]), acc[j], 0, 0, 0);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[j][e] = (bad[q][j >> 1] >> (4 * (j & 1) + e)) & 1 ? __builtin_nanf("") : acc[j][e];
        }
    }
    __device__ __forceinline__ void fetch(const AdapterRows& ad, int M, int N, int m0, int n0, int turn, int turns) {
        const int units = (M - m0 < 16 ? M - m0 : 16) * ad.sel * (ad.cols >> 5);
#pragma unroll
        for (int q = 0; q < AHEAD; ++q) load(ad, M, N, m0, n0, q, turn + q * turns, units, turns);
        next = turn + AHEAD * turns;
    }
    __device__ __forceinline__ void add(f32x4 (&acc)[CF], const AdapterRows& ad, int M, int N, int m0, int n0, int turns) {
        const int units = (M - m0 < 16 ? M - m0 : 16) * ad.sel * (ad.cols >> 5);
#pragma unroll
        for (int q = 0; q < AHEAD; ++q) use(acc, q);
        for (int unit = next; unit < units; unit += turns) {
            load(ad, M, N, m0, n0, 0, unit, units, turns);
            use(acc, 0);
        }
    }
};

}  // namespace
