// Products of microscaled 4-bit rows and weights, and products over groups of rows that have weights of their own (4-bit and bf16).
//
//   y[r, c] = act(sum_k x[r, k] w[c, k] + b[c])
//
// Both formats move the same bytes: a K-step is 128 bytes of every row, 64 bf16 or 256 E2M1 values, and a lane feeds 16 of them to a matrix instruction
// (16x16 or 32x32 results), in 4 bits together with the byte of their scale: the instruction's lane holds 32 values of one row, which is one block.  The instruction multiplies E2M1 values exactly and applies both powers of two; sums are float32.  The weights are the first operand, so that a
// lane ends up with consecutive columns of a row.
#pragma once
#include "gemm_pp.h"
#include "mx.h"

namespace {

// The tile of a workgroup: rows [row0, row0 + R) from `begin` up to `end`, of weight `weight`.
struct MxTile { int row0, begin, end, weight; };

// The groups' tiles of R rows follow each other.  A group's first tile starts at an even row (scales are copied by pairs of rows), which may be one row before the group.
// Every wave does the arithmetic by itself, 64 groups at a time with a group per lane.
struct MxGroupLane { int lo, hi, first, tiles, weight; };
template <int R>
__device__ __forceinline__ MxGroupLane mx_group_lane(const MxOperands& p, int g) {
    MxGroupLane t = {0, 0, 0, 0, 0};
    if (g < p.n_groups) {
        int lo = p.offsets[g], hi = p.offsets[g + 1];
        t.weight = p.use ? p.use[g] : g;
        lo = lo < 0 ? 0 : (lo < p.m ? lo : p.m);                // offsets outside [0, m]: the nearer end
        hi = hi < 0 ? 0 : (hi < p.m ? hi : p.m);
        if (hi > lo && t.weight >= 0 && t.weight < p.n_weights) {
            t.lo = lo; t.hi = hi; t.first = lo & ~1;
            t.tiles = (hi - t.first + R - 1) / R;
        }
    }
    return t;
}
__device__ __forceinline__ int mx_prefix(int v) {              // sum over the lanes up to this one
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);      // within rows of 16: from one, two, four and eight lanes below
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);     // the first row's last lane to the second row, the third's to the fourth
    return v + __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);   // the second row's last lane to both above
}
// Row tiles of a launch: of all rows, or of all groups, as many as the launch has workgroups for (groups that share rows could have so many that their number passes 32 bits).  The first 64
// groups stay in the lanes.
template <int R> struct MxTiles {
    MxGroupLane lane;
    int upto, total;
    __device__ __forceinline__ explicit MxTiles(const MxOperands& p) {
        if (!p.offsets) { total = (p.m + R - 1) / R; return; }
        lane = mx_group_lane<R>(p, threadIdx.x & 63);
        upto = mx_prefix(lane.tiles);
        const int most = static_cast<int>(mx_most_row_tiles(p, R));
        auto held = [&](int tiles) { return tiles < most ? tiles : most; };
        total = held(__builtin_amdgcn_readlane(upto, 63));
        for (int g0 = 64; g0 < p.n_groups; g0 += 64) total = held(total + __builtin_amdgcn_readlane(mx_prefix(mx_group_lane<R>(p, g0 + (threadIdx.x & 63)).tiles), 63));
    }
    __device__ __forceinline__ MxTile find(const MxOperands& p, int unit) const {
        if (!p.offsets) return {unit * R, 0, p.m, 0};
        MxGroupLane t = lane;
        int sum = upto, before = 0, here = __builtin_amdgcn_readlane(upto, 63);
        for (int g0 = 64; unit >= before + here; g0 += 64) {
            before += here;
            t = mx_group_lane<R>(p, g0 + (threadIdx.x & 63));
            sum = mx_prefix(t.tiles);
            here = __builtin_amdgcn_readlane(sum, 63);
        }
        const int at = __builtin_ctzll(__ballot(before + sum > unit));           // the group that holds the unit
        const int row0 = __builtin_amdgcn_readlane(t.first, at) + (unit - before - __builtin_amdgcn_readlane(sum - t.tiles, at)) * R;
        return {row0, __builtin_amdgcn_readlane(t.lo, at), __builtin_amdgcn_readlane(t.hi, at), __builtin_amdgcn_readlane(t.weight, at)};
    }
};

__device__ __forceinline__ i32x8 mx_half_operand(const u32x4& v) { return i32x8{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0}; }
// One 16x16 instruction on half H of a step; a lane's scales of the two halves are bytes 0 and 2 (block l/16 of the half, see mx_scale_step).
template <int FMT, int H>
__device__ __forceinline__ f32x4 mx_mfma(const u32x4& w, const u32x4& a, const f32x4& acc, unsigned w_scale, unsigned a_scale) {
    if constexpr (FMT == MX_BF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, a), acc, 0, 0, 0);
    else return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(mx_half_operand(w), mx_half_operand(a), acc, 4, 4, 2 * H, static_cast<int>(w_scale), 2 * H, static_cast<int>(a_scale));
}

// 0.5 x (1 + tanh(u)) as in gelu_tanh_f32, without the correction of its quotient: 1.5 units of the last place of float32 from the reciprocal and the product, no more than what the rounded
// argument of the exponential brings.  The end of a product in 4 bits is bound by these instructions; us with the correction / without it / without activation: 820 x 12288 x 3072
// 25.9 / 24.4 / 21.2; with / without it: 16384 x 4096 x 2048 in 16 groups 103.7 / 99.6, 2000 x 2048 x 1024 in 16 groups of bf16 21.1 / 20.6.
__device__ __forceinline__ float mx_gelu(float x) {
    constexpr float kLin = -2.0f * 0.7978845608028654f * 1.4426950408889634f, kCub = kLin * 0.044715f;
    const float e = __builtin_amdgcn_exp2f(x * __builtin_fmaf(x * x, kCub, kLin));
    return 0.25f * x * __builtin_amdgcn_rcpf(__builtin_fmaf(0.25f, e, 0.25f));
}
// The end of E consecutive columns of a row, those below N.  WIDE: all of them are, and 16-byte pieces are aligned.  STREAM: past the caches, where stores cover whole pieces of a row side by
// side: 16384 x 4096 x 2048 120 -> 114 us, 8704 x 9216 x 3072 148 -> 143; with a quantiser reading the result behind it 128.2 -> 126.7 and, 205 x 12288 x 3072, 18.1 -> 17.1.
struct MxBias {                // of eight columns; those past N, and all without a bias, are zero by the resource's size: no branches, all loads in flight together
    float v[8];
    __device__ __forceinline__ MxBias(const GemmEpilogue& ep, int col, int N) {
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(ep.bias), 0, ep.bias ? N * 4 : 0, 0x00027000);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rsrc, (col + e) * 4, 0, 0));
    }
};
template <bool STREAM, typename P> __device__ __forceinline__ void mx_put_piece(const P& v, void* to) {
    if constexpr (STREAM) __builtin_nontemporal_store(v, static_cast<P*>(to));
    else *static_cast<P*>(to) = v;
}
template <int E, bool WIDE, bool STREAM>
__device__ __forceinline__ void mx_put(const GemmEpilogue& ep, int row, int col, int N, const f32x4 (&sum)[E / 4], const MxBias& bias) {
    float val[E];
#pragma unroll
    for (int e = 0; e < E; ++e) val[e] = sum[e / 4][e & 3] + bias.v[e];
    if (ep.act == REGIONE_ACT_GELU_TANH) {
#pragma unroll
        for (int e = 0; e < E; ++e) val[e] = mx_gelu(val[e]);
    }
    const int64_t at = static_cast<int64_t>(row) * ep.ldy + col;
    if (ep.y_f32) {
        float* y = static_cast<float*>(ep.y) + at;
#pragma unroll
        for (int e = 0; e < E; e += 4)
            if constexpr (WIDE) mx_put_piece<STREAM>(f32x4{val[e], val[e + 1], val[e + 2], val[e + 3]}, y + e);
        if constexpr (!WIDE) {
#pragma unroll
            for (int e = 0; e < E; ++e) if (col + e < N) y[e] = val[e];
        }
    } else {
        __bf16* y = static_cast<__bf16*>(ep.y) + at;
        if constexpr (WIDE) {
            typedef __attribute__((ext_vector_type(E))) __bf16 Values;
            typedef __attribute__((ext_vector_type(E / 2))) unsigned Piece;
            Values o;
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = static_cast<__bf16>(val[e]);
            mx_put_piece<STREAM>(__builtin_bit_cast(Piece, o), y);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) if (col + e < N) y[e] = static_cast<__bf16>(val[e]);
        }
    }
}

// Few rows: a wave owns 16 rows x 16 * CF columns of a part of K and reads its operands straight from memory, the weights as they lie, with the loads of CHUNK steps in flight.  KW of a
// workgroup's eight waves share K and meet in LDS, where the sums are formed in wave order; the others take further columns.  Such a launch is a chain of trips to memory and the reading of
// the weights.  Where K is long and N short there are fewer workgroups than CUs, and registers for one trip only: 16 columns, eight steps at a time, two waves per SIMD; us, 32 columns and
// two steps / so, weights in the Infinity Cache: one row x 3072 x 12288 6.7 / 5.0 (from HBM 8.8 / 6.9, 3 TB/s with the launch), 16 rows x 3072 x 15360 10.7 / 8.0, but one row x 9216 x 3072
// 5.3 / 6.6, 96 rows x 2048 x 1024 of 64 experts 15.8 / 46.6.
constexpr int kMxSmallRows = 16, kMxSmallWaves = 8;

template <int FMT, int KW, int CF>
__global__ void __launch_bounds__(kMxSmallWaves * 64) __attribute__((amdgpu_waves_per_eu(CF == 1 ? 2 : 4)))
gemm_mx_small_kernel(MxOperands p, GemmEpilogue ep) {
    constexpr int CHUNK = CF == 1 ? 8 : FMT == MX_FP4 ? 2 : 3, NW = kMxSmallWaves / KW, COLS = 16 * CF;
    __shared__ __attribute__((aligned(16))) f32x4 sums[KW == 1 ? 1 : kMxSmallWaves * CF * 64];
    const int n_tiles = (p.n + COLS * NW - 1) / (COLS * NW), unit = static_cast<int>(blockIdx.x) / n_tiles;
    const MxTiles<kMxSmallRows> tiles(p);
    if (unit >= tiles.total) return;
    const MxTile t = tiles.find(p, unit);
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), kw = wave % KW;
    const int l16 = lane & 15, kc = lane >> 4;
    const int n0 = ((static_cast<int>(blockIdx.x) - unit * n_tiles) * NW + wave / KW) * COLS, n32 = (p.n + 31) & ~31;
    const int per = (p.steps + KW - 1) / KW, s0 = kw * per, s1 = s0 + per < p.steps ? s0 + per : p.steps;

    const uint8_t* w = p.w + t.weight * p.w_stride;
    int nb = n0 >> 5;
    nb = nb < n32 / 32 ? nb : n32 / 32 - 1;                     // blocks past N repeat the last one; their sums are not stored
    const int col0 = CF == 1 ? (n0 & 16) + l16 : 8 * (l16 >> 2) + (l16 & 3);   // of the first fragment; the other one's is four further: a lane's results are 4 * CF consecutive columns
    const uint8_t* wp = w + ((static_cast<int64_t>(nb) * p.steps * 4 + (kc >> 1)) * 64 + (kc & 1) * 32 + col0) * 16;
    const uint8_t* wsp = w + static_cast<int64_t>(n32) * p.steps * 128 + (nb * 32 + col0) * 8 + 4 * (kc & 1);
    int row = t.row0 + l16;
    row = row < t.end ? row : t.end - 1;                        // rows past the end repeat the last one
    const uint8_t* ap = p.a + static_cast<int64_t>(row) * p.row_bytes;
    const int64_t a_step = mx_padded_rows(p.m) * 8;
    const uint8_t* asp = FMT == MX_FP4 ? p.a_scale + static_cast<int64_t>(row) * 8 + 4 * (kc & 1) : nullptr;

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
#pragma unroll
                    for (int j = 0; j < CF; ++j) wv[i][h][j] = *reinterpret_cast<const u32x4*>(wp + (static_cast<int64_t>(s) * 4 + 2 * h) * 1024 + j * 64);
                    av[i][h] = *reinterpret_cast<const u32x4*>(ap + (at < p.row_bytes ? at : 0));
                }
                if (FMT == MX_FP4) {
#pragma unroll
                    for (int j = 0; j < CF; ++j) ws[i][j] = *reinterpret_cast<const unsigned*>(wsp + static_cast<int64_t>(s) * n32 * 8 + j * 32);
                    as[i] = *reinterpret_cast<const unsigned*>(asp + s * a_step);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < CHUNK; ++i)
            if (base + i < s1) {
                const unsigned shift = 8 * (kc >> 1);
#pragma unroll
                for (int j = 0; j < CF; ++j) acc[j] = mx_mfma<FMT, 0>(wv[i][0][j], av[i][0], acc[j], ws[i][j] >> shift, as[i] >> shift);
#pragma unroll
                for (int j = 0; j < CF; ++j) acc[j] = mx_mfma<FMT, 1>(wv[i][1][j], av[i][1], acc[j], ws[i][j] >> shift, as[i] >> shift);
            }
    }
    if (KW > 1) {
#pragma unroll
        for (int j = 0; j < CF; ++j) sums[(wave * CF + j) * 64 + lane] = acc[j];
        __syncthreads();
        if (kw) return;
#pragma unroll
        for (int v = 1; v < KW; ++v)
#pragma unroll
            for (int j = 0; j < CF; ++j) acc[j] += sums[((wave + v) * CF + j) * 64 + lane];
    }
    if (ep.bias) ep.bias += static_cast<int64_t>(t.weight) * p.n;
    const int col = n0 + 4 * CF * kc;
    if (t.row0 + l16 >= t.end || t.row0 + l16 < t.begin || col >= p.n) return;
    const MxBias bias(ep, col, p.n);
    if (ep.vec_ok) mx_put<4 * CF, true, false>(ep, row, col, p.n, acc, bias);
    else mx_put<4 * CF, false, false>(ep, row, col, p.n, acc, bias);
}

}  // namespace
