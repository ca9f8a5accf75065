// Low-rank adapters beside a projection, at the end of the projection's tiles: y[r] += sum over s of (weight[r, s] x[r] A_a^T) B_a^T, a = which[r, s].
//
// The inner products with A, times their weights, are there already (adapters.hip): rows t[r, s] of bf16 terms that add up to them, `blocks` blocks of 16 ranks per term, so that a row of
// t times [B_a | B_a | ..] is the adapter's share of the result.  A wave multiplies the rows of its fragments with one adapter after the other, those of other adapters as zeros, into the
// accumulators that hold the projection's sums: nothing is written or read in between, and the result is rounded once.
#pragma once
#include "gemm_epilogue.h"

namespace {

// the smallest of a value's 16 lanes, in all of them
__device__ __forceinline__ int lanes16_min(int v) {
    auto less = [](int a, int b) { return a < b ? a : b; };
    v = less(v, __builtin_amdgcn_update_dpp(v, v, 0x121, 0xf, 0xf, false));       // row_ror 1, 2, 4, 8
    v = less(v, __builtin_amdgcn_update_dpp(v, v, 0x122, 0xf, 0xf, false));
    v = less(v, __builtin_amdgcn_update_dpp(v, v, 0x124, 0xf, 0xf, false));
    return less(v, __builtin_amdgcn_update_dpp(v, v, 0x128, 0xf, 0xf, false));
}
constexpr int kNoAdapter = 0x7fffffff;

// Rows [I0, I1) of a wave's fragments, in the layout of gemm_epilogue16.  turn, turns: of the steps of 32 terms, counted over all adapters, this wave takes those numbered turn modulo turns
// (where several waves add up the same fragments).
// Rows without the adapter must not see its values (zero times infinity): the fragments that hold such rows take the instruction's result for their own rows only.
template <int I0, int I1, int RF, int CF>
__device__ __forceinline__ void adapters_add(f32x4 (&acc)[RF][CF], int M, int N, int m0, int n0w, const AdapterRows& ad, int turn = 0, int turns = 1) {
    constexpr int R = I1 - I0;
    const int lane = threadIdx.x & 63, l16 = lane & 15, kc = lane >> 4;
    const int last_block = ((N + 31) >> 5) - 1, steps = ad.cols >> 5;
    // weight fragment j of a lane: column 8*(l16/4) + 4*(j%2) + l16%4 of block j / 2, as the epilogue expects it
    int64_t w_at[CF / 2];
#pragma unroll
    for (int b = 0; b < CF / 2; ++b) {
        int nb = (n0w >> 5) + b;
        nb = nb < last_block ? nb : last_block;                   // blocks past N repeat the last one; their sums are not stored
        w_at[b] = (static_cast<int64_t>(nb) * ad.blocks * 64 + (kc & 1) * 32 + 8 * (l16 >> 2) + (l16 & 3)) * 8;
    }
    // rows of terms, all of them within 32 MB; those past M are zero by the resource's size
    const auto terms = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(ad.t), 0, M * ad.sel * ad.cols * 2, 0x00027000);
    const unsigned t_rows = 16u * ad.sel * ad.cols * 2u, t_first = static_cast<unsigned>((m0 + 16 * I0 + l16) * ad.sel * ad.cols + 8 * kc) * 2u;
    // One loop over all steps of all adapters, the smallest number first: nested ones leave the compiler with a copy of the accumulators for each.
    int step_no = 0, s = 0, a = -1, st = steps - 1, first_block = 0;
    int id[R];
    auto load_ids = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int row = m0 + 16 * (I0 + i) + l16;
            id[i] = row < M ? ad.which[row * ad.sel + s] : -1;
            if (id[i] >= ad.count) id[i] = -1;
        }
    };
    load_ids();
    // the next step; false behind the last one
    auto go = [&]() __attribute__((always_inline)) {
        if (++st < steps) {
            first_block += 2;
            while (first_block >= ad.blocks) first_block -= ad.blocks;
            return true;
        }
        st = first_block = 0;
        int next = kNoAdapter;
#pragma unroll 1
        while (true) {
#pragma unroll
            for (int i = 0; i < R; ++i) next = id[i] > a && id[i] < next ? id[i] : next;
            next = __builtin_amdgcn_readfirstlane(lanes16_min(next));
            if (next != kNoAdapter || ++s >= ad.sel) break;
            load_ids();
            a = -1;
        }
        a = next;
        return next != kNoAdapter;
    };
    bool more = go();
#pragma unroll 1
    while (more) {
        if (turns == 1 || step_no++ % turns == turn) {
            const unsigned t_at = t_first + static_cast<unsigned>(s * ad.cols + 32 * st) * 2u;
            const bf16_t* const b = ad.b + static_cast<int64_t>(a) * ad.stride;
            int block = first_block + (kc >> 1);
            block = block < ad.blocks ? block : block - ad.blocks;
            bf16x8 wf[CF];
#pragma unroll
            for (int j = 0; j < CF; ++j) wf[j] = *reinterpret_cast<const bf16x8*>(b + w_at[j / 2] + block * 512 + (j & 1) * 32);
#pragma unroll
            for (int i = 0; i < R; ++i) {
                u32x4 tr = __builtin_amdgcn_raw_buffer_load_b128(terms, t_at + i * t_rows, 0, 0);
                const bool mine = id[i] == a;
#pragma unroll
                for (int e = 0; e < 4; ++e) tr[e] = mine ? tr[e] : 0u;
#pragma unroll
                for (int j = 0; j < CF; ++j) {
                    const f32x4 sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[j], __builtin_bit_cast(bf16x8, tr), acc[I0 + i][j], 0, 0, 0);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[I0 + i][j][e] = mine ? sum[e] : acc[I0 + i][j][e];
                }
#pragma unroll
                for (int j = 0; j < CF; ++j) {
                    f32x4 here = acc[I0 + i][j];              // here, and not behind all rows' instructions with all their results in registers
                    asm volatile("" : "+v"(here));
                    acc[I0 + i][j] = here;
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        more = go();
    }
}

}  // namespace
