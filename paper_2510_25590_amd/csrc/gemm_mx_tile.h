// The products of gemm_mx.h for many rows: tiles of 32 x 128 to 224 x 256 results.
//
// Four waves; each owns all 32 * RF rows of the tile and 32 * CF columns, in 32x32 fragments.  The weights go from their packed layout straight into the registers of the one wave that
// wants them; the rows, which all waves want, go by way of registers into LDS, a whole step (128 bytes of a row, one line of memory) at a time, two steps in LDS.  Loads are requested
// LOOK steps ahead and registers are loaded again as soon as they have been used.  A step is four phases of RF * CF instructions; while a phase's instructions run, the same wave reads the
// rows of the next phase, puts rows of the next step into LDS and requests rows, weights and scales of the steps ahead.  One barrier per step.
// Why not straight into LDS: such copies are taken at 35 bytes a clock by a CU (all tiles ended at 65 to 70 bytes a ns), where loads into registers get 64; and
// weights in LDS, shared by waves that split the rows, cost it as many bytes again.  us, tiles of the same sizes with copies into LDS / so: 820 x 3072 x 12288 30.0 / 27.6,
// 205 x 12288 x 3072 12.5 / 11.4, 64 x 9216 x 3072 6.9 / 6.2, 128 x 3072 x 12288 23.6 / 20.0, 2048 x 8192 x 12288 106 / 97.
// What bounds it.  Several rounds of tiles (8704 x 9216 x 3072, 127 us, 3.9 PFLOP/s): matrix instructions run in 63 % of the cycles in which a CU holds workgroups, at 1.6 to 1.8 GHz, where a register loop that is
// always busy holds 1.55 (6.5 PFLOP/s); in the rest the two workgroups of a CU, which run in step, start, end or wait together, and the 4.8 rounds of tiles take the time of five.  One round
// (820 x 12288 x 3072): the start and the end, which nothing hides, are half of the call.  128 columns: all four waves read all rows, so a step of 160 x 128 moves 100 KiB through LDS, 800
// clocks at 128 bytes, beside 640 of matrix instructions; the counters have each busy 52 % of the time (1382 x 3072 x 15360), and a second workgroup per CU finds nothing left to overlap.
// The 32x32 instruction reaches its rate with one wave per SIMD, which the 16x16 one does not (register-only loops in 4 bits, PFLOP/s with one, two and four waves per
// SIMD: 6.3 / 6.5 / 6.6 against 4.2 / 5.5 / 6.1).
#pragma once
#include "gemm_mx.h"
#include <type_traits>

namespace {

// A source of loads: `at` moves on by a stride per step; `left` bytes from there may be read, and none of a step that does not exist.
struct MxSource {
    uint64_t at; int left;
    __device__ __forceinline__ auto rsrc(bool there) const { return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(at), 0, there ? left : 0, 0x00027000); }
};

template <int FMT, int RF, int CF> struct MxTileShape {
    static constexpr int ROWS = 32 * RF, COLS = 128 * CF, THREADS = 256;
    static constexpr unsigned SLOT = ROWS * 128u;                                  // a step's rows
    static constexpr int ROW_SCALES = (ROWS + 127) / 128;                          // 1 KiB pieces of a step's scales: of 128 rows each, then of 128 columns each; a wave per piece
    static constexpr unsigned SCALES = FMT == MX_FP4 ? 4096u : 0u, S_BASE = 2 * SLOT;    // (a place for every wave, so that none has to ask)
    static_assert(ROW_SCALES + CF <= 4, "a wave per piece");
    static constexpr int STORE_ROWS = RF % 2 == 0 ? 2 : 1;                         // rows of fragments per wave that mx_store leaves in LDS at a time
    static constexpr unsigned STORE = STORE_ROWS * CF * 4096u, LDS_BYTES = S_BASE + 2 * SCALES > 4 * STORE ? S_BASE + 2 * SCALES : 4 * STORE;
    static_assert(LDS_BYTES <= 65536u, "more has to be granted");
    static constexpr int64_t PART_FLOATS = static_cast<int64_t>(ROWS) * COLS;
};

// One instruction on phase P of a step (64 or 16 inputs); scales: byte P of a lane's words.
template <int FMT, int P>
__device__ __forceinline__ f32x16 mx_mfma32(const u32x4& w, const u32x4& a, const f32x16& acc, unsigned w_scale, unsigned a_scale) {
    if constexpr (FMT == MX_BF16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, a), acc, 0, 0, 0);
    else return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(mx_half_operand(w), mx_half_operand(a), acc, 4, 4, P, static_cast<int>(w_scale), P, static_cast<int>(a_scale));
}
template <int I> __device__ __forceinline__ f32x4 mx_part(const f32x16& v) { return f32x4{v[4 * I], v[4 * I + 1], v[4 * I + 2], v[4 * I + 3]}; }

// this wave's LDS accesses are complete
__device__ __forceinline__ void mx_lds_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); __builtin_amdgcn_sched_barrier(0); }

// A fragment as it is from here on: without it the compiler reads all accumulators of the three ways to store them out of their registers at once, and spills.
template <bool ACC_REGISTERS> __device__ __forceinline__ f32x16 mx_here(f32x16 v) {
    if constexpr (ACC_REGISTERS) asm volatile("" : "+a"(v)); else asm volatile("" : "+v"(v));
    return v;
}

// Writes a wave's accumulators: acc[i][j] of a lane holds row 32*i + lane%32 and columns 32*j + 16*b + 8*(lane/32) + 0..7, b = 0, 1, of the wave's part.  By way of LDS (the wave's own
// part of it, IR rows of fragments at a time), so that a store covers whole rows of the part, 16 bytes per lane: straight from the accumulators, 32 bytes of 32
// rows at a time, 2048 x 8192 x 256 took 17.6 us instead of 15.1.
template <int ROWS, int CF, int E, bool ALIGNED>                                  // E columns per lane: eight of bf16, four of float32
__device__ __forceinline__ void mx_store_rows(const unsigned char* lds, const MxTile& t, int N, int row0, int col, const GemmEpilogue& ep, const MxBias& bias) {
    constexpr int PIECES = 8 * CF, KEY = (PIECES < 16 ? PIECES : 16) - 1;        // 16-byte pieces of a row; piece c of row r lies at c ^ (r & KEY)
    constexpr int GROUPS = 32 * CF / E;                                           // of E columns in a row: a lane stays with one
    const int lane = threadIdx.x & 63, group = lane % GROUPS;
    const f32x4* const from = reinterpret_cast<const f32x4*>(lds);
#pragma unroll 4
    for (int lr = lane / GROUPS; lr < ROWS; lr += 64 / GROUPS) {
        const int row = row0 + lr;
        f32x4 v[E / 4];
#pragma unroll
        for (int e = 0; e < E / 4; ++e) v[e] = from[lr * PIECES + ((E / 4 * group + e) ^ (lr & KEY))];
        if (row < t.begin || row >= t.end || col >= N) continue;
        mx_put<E, ALIGNED, ALIGNED>(ep, row, col, N, v, bias);
    }
}
template <int RF, int CF, int IR, bool ALIGNED>
__device__ __forceinline__ void mx_store(const f32x16 (&acc)[RF][CF], unsigned char* lds, const MxTile& t, int N, int m0, int n0w, const GemmEpilogue& ep) {
    constexpr int PIECES = 8 * CF, KEY = (PIECES < 16 ? PIECES : 16) - 1;
    static_assert(RF % IR == 0, "whole rounds");
    const int lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
    const int col = n0w + (ep.y_f32 ? 4 * (lane % (8 * CF)) : 8 * (lane % (4 * CF)));
    const MxBias bias(ep, col, N);
    f32x4* const to = reinterpret_cast<f32x4*>(lds) + l32 * PIECES;
    for (int i0 = 0; i0 < RF; i0 += IR) {
#pragma unroll
        for (int i = 0; i < RF; ++i) {
            if (i / IR * IR != i0) continue;
#pragma unroll
            for (int j = 0; j < CF; ++j) {
                const f32x16 v = mx_here<(RF * CF > 8)>(acc[i][j]);
                f32x4* const at = to + (i % IR) * 32 * PIECES;
                at[(8 * j + 2 * half + 0) ^ (l32 & KEY)] = mx_part<0>(v);
                at[(8 * j + 2 * half + 1) ^ (l32 & KEY)] = mx_part<1>(v);
                at[(8 * j + 2 * half + 4) ^ (l32 & KEY)] = mx_part<2>(v);
                at[(8 * j + 2 * half + 5) ^ (l32 & KEY)] = mx_part<3>(v);
            }
        }
        if (ep.y_f32) mx_store_rows<32 * IR, CF, 4, ALIGNED>(lds, t, N, m0 + 32 * i0, col, ep, bias);
        else mx_store_rows<32 * IR, CF, 8, ALIGNED>(lds, t, N, m0 + 32 * i0, col, ep, bias);
    }
}

// The end of a K split: sums of all splits, added in split order, straight from where they were left; G fragments' pieces of a split are requested together, one split ahead.
template <int RF, int CF>
__device__ __forceinline__ void mx_store_sums(float* sums, int splits, unsigned off, const MxTile& t, int N, int m0, int n0w, const GemmEpilogue& ep) {
    constexpr int F = RF * CF, G = F % 4 == 0 ? 4 : F % 3 == 0 ? 3 : F % 2 == 0 ? 2 : 1;
    constexpr unsigned bytes = RF * CF * 4u * 4096u;               // of a split
    const auto rsrc = pp_part_rsrc(sums, splits * static_cast<int64_t>(bytes / 4));
    const int l32 = threadIdx.x & 31, half = (threadIdx.x >> 5) & 1;
    for (int f0 = 0; f0 < F; f0 += G) {
        f32x4 sum[G * 4];
        u32x4 v[2][G * 4];
        auto request = [&](int b, int s) __attribute__((always_inline)) {
#pragma unroll
            for (int c = 0; c < G * 4; ++c) v[b][c] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, off + (c & 3) * 1024u, static_cast<int>(s * bytes + (f0 + c / 4) * 4096u), kDeviceScope);
        };
        auto add = [&](int b, bool first) __attribute__((always_inline)) {
#pragma unroll
            for (int c = 0; c < G * 4; ++c) sum[c] = first ? __builtin_bit_cast(f32x4, v[b][c]) : sum[c] + __builtin_bit_cast(f32x4, v[b][c]);
        };
        request(0, 0);
        for (int s = 0; s < splits; s += 2) {
            request(1, s + 1 < splits ? s + 1 : s);
            add(0, s == 0);
            request(0, s + 2 < splits ? s + 2 : s);
            if (s + 1 < splits) add(1, false);
        }
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int row = m0 + 32 * ((f0 + g) / CF) + l32;
            if (row < t.begin || row >= t.end) continue;
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const int col = n0w + 32 * ((f0 + g) % CF) + 16 * b + 8 * half;
                if (col >= N) continue;
                const MxBias bias(ep, col, N);
                const f32x4 v[2] = {sum[4 * g + 2 * b], sum[4 * g + 2 * b + 1]};
                if (ep.vec_ok) mx_put<8, true, false>(ep, row, col, N, v, bias);
                else mx_put<8, false, false>(ep, row, col, N, v, bias);
            }
        }
    }
}

template <int FMT, int RF, int CF, int LOOK, int WAVES>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(WAVES)))
gemm_mx_tile_kernel(MxOperands p, int splits, int steps_per_split, float* __restrict__ partial, int* __restrict__ arrived, GemmEpilogue ep) {
    using T = MxTileShape<FMT, RF, CF>;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds_raw[];
    const int n_tiles = (p.n + T::COLS - 1) / T::COLS;
    const MxTiles<T::ROWS> row_tiles(p);
    const int m_tiles = row_tiles.total;
    const int units = m_tiles * n_tiles * splits, per_xcd = (units + 7) >> 3;
    const int local = static_cast<int>(blockIdx.x >> 3), unit = static_cast<int>(blockIdx.x & 7) * per_xcd + local;     // each XCD a contiguous range (see pp_unit)
    if (local >= per_xcd || unit >= units) return;
    int m_tile, n_tile, split = 0;
    if (FMT == MX_BF16 || splits == 1) {               // (bf16 comes in groups, which have no K splits)
        tile_coords(unit, m_tiles, n_tiles, m_tiles > 8 ? 4 : m_tiles, m_tile, n_tile);
    } else {
        m_tile = unit % m_tiles;
        const int rest = unit / m_tiles;
        n_tile = rest / splits;
        split = rest - n_tile * splits;
    }
    // (the divisions leave these in vector registers, and everything that follows from them)
    m_tile = __builtin_amdgcn_readfirstlane(m_tile); n_tile = __builtin_amdgcn_readfirstlane(n_tile); split = __builtin_amdgcn_readfirstlane(split);
    const MxTile t = row_tiles.find(p, m_tile);
    const int n0 = n_tile * T::COLS, n32 = (p.n + 31) & ~31;
    const int lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int step0 = split * steps_per_split;
    int n_steps = p.steps - step0;
    n_steps = n_steps < steps_per_split ? n_steps : steps_per_split;

    // Rows: a load takes 8 rows' 128 bytes; 16-byte chunk c of row r lies at c ^ ((r >> 1) & 7) in LDS, so that sixteen rows' same chunk covers all banks once.  Rows past the tensor's end
    // are zero; past a row's end the next row's values are read, which meet weights of zero (bf16 rows are whole steps), and E2M1 has neither NaN nor infinity.
    unsigned a_voff[RF], a_put[2], a_get[4];
#pragma unroll
    for (int i = 0; i < RF; ++i) a_voff[i] = static_cast<unsigned>((wave * RF + i) * 8 + (lane >> 3)) * static_cast<unsigned>(p.row_bytes) + (lane & 7) * 16u;
#pragma unroll
    for (int i = 0; i < 2; ++i) {                                                  // of even and odd loads
        const int row = (wave * RF + i) * 8 + (lane >> 3);
        a_put[i] = static_cast<unsigned>(row - i * 8) * 128u + static_cast<unsigned>(((lane & 7) ^ ((row >> 1) & 7)) << 4);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) a_get[q] = l32 * 128u + static_cast<unsigned>(((2 * q + half) ^ ((l32 >> 1) & 7)) << 4);
    const int64_t a_first = static_cast<int64_t>(t.row0) * p.row_bytes + static_cast<int64_t>(step0) * 128, a_left = static_cast<int64_t>(p.m) * p.row_bytes - a_first;
    MxSource a = {reinterpret_cast<uint64_t>(p.a) + a_first, static_cast<int>(a_left < INT32_MAX ? a_left : INT32_MAX)};
    // Weights: a block's 64 inputs are one fragment; its 32 features are put in the order that leaves a lane with twice eight consecutive results beside those of the row's other lane:
    // place 8*g + 4*h + u, whose results lane half h holds in registers 4*g + u, gets feature 16*(g/2) + 8*h + 4*(g%2) + u.  Blocks past N repeat the last one.
    const unsigned feature = (l32 >> 4) * 16 + ((l32 >> 2) & 1) * 8 + ((l32 >> 3) & 1) * 4 + (l32 & 3);
    const uint8_t* w_all = p.w + t.weight * p.w_stride;
    const int last = n32 / 32 - 1;
    int nb0 = (n0 >> 5) + wave * CF;
    nb0 = nb0 < last ? nb0 : last;
    unsigned w_voff[CF];
#pragma unroll
    for (int j = 0; j < CF; ++j) w_voff[j] = static_cast<unsigned>(nb0 + j < last ? j : last - nb0) * static_cast<unsigned>(p.steps) * 4096u + ((lane & 32) + feature) * 16u;
    MxSource w = {reinterpret_cast<uint64_t>(w_all) + (static_cast<int64_t>(nb0) * p.steps + step0) * 4096, INT32_MAX};
    // Scales: 16 bytes (two rows or columns) per lane of a wave's piece; a word for each fragment straight from memory costs as many trips of the data path as the fragments themselves.
    const int64_t padded = mx_padded_rows(p.m);
    const bool of_rows = wave < T::ROW_SCALES;
    const int s_first = of_rows ? t.row0 + wave * 128 : n0 + (wave - T::ROW_SCALES) * 128;
    const int64_t s_all = of_rows ? padded : n32, s_left = s_all - s_first;       // (rows and columns past the end: nothing is read)
    MxSource scales = {(of_rows ? reinterpret_cast<uint64_t>(p.a_scale) : reinterpret_cast<uint64_t>(w_all) + static_cast<int64_t>(n32) * p.steps * 128) + (step0 * s_all + s_first) * 8,
                       wave < T::ROW_SCALES + CF && s_left > 0 ? static_cast<int>(s_left * 8) : 0};
    const unsigned as_get = T::S_BASE + l32 * 8u + half * 4u, ws_get = T::S_BASE + T::ROW_SCALES * 1024u + (wave * (CF * 32) + feature) * 8u + half * 4u;

    auto each = [&](auto from, auto to, auto f, auto self) __attribute__((always_inline)) {
        if constexpr (decltype(from)::value < decltype(to)::value) {
            f(from);
            self(std::integral_constant<int, decltype(from)::value + 1>{}, to, f, self);
        }
    };
    typedef std::integral_constant<int, 0> zero;
    typedef std::integral_constant<int, RF> rows;
    typedef std::integral_constant<int, CF> columns;
    typedef std::integral_constant<int, 4> phases;

    // What is on its way: rows and scales of the steps s + 1 .. s + LOOK, weights of the steps s .. s + LOOK - 1, in buffer number step % LOOK (weights) or one less (rows and scales).
    u32x4 put[LOOK][RF], put_scales[LOOK], wf[LOOK][4][CF], af[2][RF];
    unsigned ws[2][CF], as[2][RF];                                                 // of this step and of the next one
    int a_step = 0, w_step = 0, s_step = 0;                                       // the next step of each source
    auto load_a = [&](auto b, auto i) __attribute__((always_inline)) {
        (decltype(b)::value < 0 ? af[1] : put[decltype(b)::value < 0 ? 0 : decltype(b)::value])[decltype(i)::value] = __builtin_amdgcn_raw_buffer_load_b128(a.rsrc(a_step < n_steps), a_voff[decltype(i)::value], 0, 0);
        if constexpr (decltype(i)::value == RF - 1) {
            ++a_step;
            a.at += 128;
            asm("s_sub_i32 %0, %0, 128\n\ts_max_i32 %0, %0, 0" : "+s"(a.left) : : "scc");       // (left to itself the compiler subtracts in a vector register)
        }
    };
    auto load_w = [&](auto b, auto q, auto j) __attribute__((always_inline)) {
        wf[decltype(b)::value][decltype(q)::value][decltype(j)::value] =
            __builtin_amdgcn_raw_buffer_load_b128(w.rsrc(w_step < n_steps), w_voff[decltype(j)::value] + decltype(q)::value * 1024u, 0, 0);
        if constexpr (decltype(q)::value == 3 && decltype(j)::value == CF - 1) { ++w_step; w.at += 4096; }
    };
    auto load_scales = [&](auto b) __attribute__((always_inline)) {
        if constexpr (FMT == MX_FP4) {
            put_scales[decltype(b)::value] = __builtin_amdgcn_raw_buffer_load_b128(scales.rsrc(s_step < n_steps), lane * 16u, 0, 0);
            ++s_step;
            scales.at += s_all * 8;
        }
    };
    auto write_scales = [&](unsigned slot, auto b) __attribute__((always_inline)) {
        if constexpr (FMT == MX_FP4) *reinterpret_cast<u32x4*>(lds_raw + T::S_BASE + (slot ? T::SCALES : 0u) + wave * 1024u + lane * 16u) = put_scales[decltype(b)::value];
    };
    auto read_scales = [&](unsigned slot, auto b, auto i) __attribute__((always_inline)) {         // number i: of the rows' fragment i and, the first ones, of the columns'
        constexpr int I = decltype(i)::value, B = decltype(b)::value;
        if constexpr (FMT == MX_FP4) {
            const unsigned at = slot ? T::SCALES : 0u;
            as[B][I] = *reinterpret_cast<const unsigned*>(lds_raw + (as_get + at) + I * 256);
            if constexpr (I < CF) ws[B][I] = *reinterpret_cast<const unsigned*>(lds_raw + (ws_get + at) + I * 256);
            if constexpr (CF > RF && I == RF - 1) ws[B][CF - 1] = *reinterpret_cast<const unsigned*>(lds_raw + (ws_get + at) + (CF - 1) * 256);
        }
    };
    auto write_a = [&](unsigned slot, auto b, auto i) __attribute__((always_inline)) {
        constexpr int I = decltype(i)::value;
        *reinterpret_cast<u32x4*>(lds_raw + (a_put[I & 1] + slot) + I * 1024) = (decltype(b)::value < 0 ? af[1] : put[decltype(b)::value < 0 ? 0 : decltype(b)::value])[I];
    };
    auto read_a = [&](unsigned slot, auto q, auto i) __attribute__((always_inline)) {
        constexpr int Q = decltype(q)::value, I = decltype(i)::value;
        af[Q & 1][I] = *reinterpret_cast<const u32x4*>(lds_raw + (a_get[Q] + slot) + I * 4096);
    };

    // The first step's rows by way of registers that are not needed yet; then everything in the order in which the steps request it, so that no wait of theirs is stricter for the start's sake.
    u32x4 first_scales;
    each(zero{}, rows{}, [&](auto i) __attribute__((always_inline)) { load_a(std::integral_constant<int, -1>{}, i); __builtin_amdgcn_sched_barrier(0); }, each);
    load_scales(zero{});
    first_scales = put_scales[0];
    each(zero{}, std::integral_constant<int, LOOK>{}, [&](auto b) __attribute__((always_inline)) {
        each(zero{}, rows{}, [&](auto i) __attribute__((always_inline)) { load_a(b, i); __builtin_amdgcn_sched_barrier(0); }, each);
        load_scales(b);
        each(zero{}, phases{}, [&](auto q) __attribute__((always_inline)) { each(zero{}, columns{}, [&](auto j) __attribute__((always_inline)) { load_w(b, q, j); __builtin_amdgcn_sched_barrier(0); }, each); }, each);
    }, each);
    f32x16 acc[RF][CF];                                                            // (while the loads are on their way)
#pragma unroll
    for (int i = 0; i < RF; ++i)
#pragma unroll
        for (int j = 0; j < CF; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    __builtin_amdgcn_sched_barrier(0);
    each(zero{}, rows{}, [&](auto i) __attribute__((always_inline)) { write_a(0, std::integral_constant<int, -1>{}, i); }, each);
    if constexpr (FMT == MX_FP4) *reinterpret_cast<u32x4*>(lds_raw + T::S_BASE + wave * 1024u + lane * 16u) = first_scales;
    mx_lds_done();
    pp_barrier();
    each(zero{}, rows{}, [&](auto i) __attribute__((always_inline)) { read_a(0, zero{}, i); read_scales(0, zero{}, i); }, each);

    // Step s (in LDS slot `slot`) from buffers B: its instructions column by column, between them what is said above.
    unsigned slot = 0;
    auto phase = [&](auto bc, auto pc) __attribute__((always_inline)) {
        constexpr int P = decltype(pc)::value, COUNT = RF * CF;
        if constexpr (P == 3) {              // the next step's rows are in LDS, and all reads of this step's have been made
            mx_lds_done();
            pp_barrier();
        }
        each(zero{}, std::integral_constant<int, COUNT>{}, [&](auto qc) __attribute__((always_inline)) {
            constexpr int Q = decltype(qc)::value, I = Q % RF, J = Q / RF, B = decltype(bc)::value;
            acc[I][J] = mx_mfma32<FMT, P>(wf[B][P][J], af[P & 1][I], acc[I][J], ws[0][J], as[0][I]);
            if constexpr (Q < RF) {
                if constexpr (P == 3) { read_a(slot ^ T::SLOT, zero{}, std::integral_constant<int, Q>{}); read_scales(slot ^ T::SLOT, std::integral_constant<int, 1>{}, std::integral_constant<int, Q>{}); }
                else read_a(slot, std::integral_constant<int, (P + 1) & 3>{}, std::integral_constant<int, Q>{});
            }
            if constexpr (P < 3) {           // a third of the next step's rows
                constexpr int R0 = P * RF / 3, R = (P + 1) * RF / 3 - R0;
                each(std::integral_constant<int, R0 + Q * R / COUNT>{}, std::integral_constant<int, R0 + (Q + 1) * R / COUNT>{}, [&](auto i) __attribute__((always_inline)) {
                    write_a(slot ^ T::SLOT, bc, i);
                    load_a(bc, i);
                }, each);
            }
            if constexpr (P == 2 && Q == COUNT - 1) { write_scales(slot ^ T::SLOT, bc); load_scales(bc); }
            if constexpr (I == RF - 1) load_w(bc, pc, std::integral_constant<int, J>{});
            __builtin_amdgcn_sched_barrier(0);
        }, each);
    };
    const int turns = (n_steps + LOOK - 1) / LOOK;                                 // (steps that do not exist multiply zeros)
    for (int turn = 0; turn < turns; ++turn)
        each(zero{}, std::integral_constant<int, LOOK>{}, [&](auto b) __attribute__((always_inline)) {
            each(zero{}, phases{}, [&](auto q) __attribute__((always_inline)) { phase(b, q); }, each);
            slot ^= T::SLOT;
            if constexpr (FMT == MX_FP4) {
#pragma unroll
                for (int i = 0; i < RF; ++i) as[0][i] = as[1][i];
#pragma unroll
                for (int j = 0; j < CF; ++j) ws[0][j] = ws[1][j];
            }
        }, each);

    const int m0 = t.row0, n0w = n0 + wave * (CF * 32);
    if (ep.bias) ep.bias += static_cast<int64_t>(t.weight) * p.n;
    if (FMT == MX_FP4 && splits > 1) {
        // As in pp_finish: every split leaves its sums in register order and the workgroup that arrives last adds all of them in split order.
        const int tile = n_tile * m_tiles + m_tile;
        float* mine = partial + (static_cast<int64_t>(tile) * splits + split) * T::PART_FLOATS;
        const unsigned off = static_cast<unsigned>(wave * (RF * CF * 4) * 64 + lane) * 16u;
#pragma unroll
        for (int f = 0; f < RF * CF; ++f) {
            // (a resource per fragment, so that the pieces differ by constants; with a scalar offset a wide store's data would not be kept long enough, see pp_finish)
            const auto rsrc = pp_part_rsrc(mine + f * 1024, T::PART_FLOATS - f * 1024);
            const f32x16 v = mx_here<(RF * CF > 8)>(acc[f / CF][f % CF]);
            each(zero{}, std::integral_constant<int, 4>{}, [&](auto c) __attribute__((always_inline)) {
                constexpr int C = decltype(c)::value;
                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, mx_part<C>(v)), rsrc, off + C * 1024u, 0, kDeviceScope);
            }, each);
        }
        pp_wait<0>();
        __syncthreads();
        int* flag = reinterpret_cast<int*>(lds_raw);
        if (threadIdx.x == 0) *flag = __hip_atomic_fetch_add(arrived + tile, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        if (*flag != splits - 1) return;
        if (threadIdx.x == 0) __hip_atomic_store(arrived + tile, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        mx_store_sums<RF, CF>(partial + static_cast<int64_t>(tile) * splits * T::PART_FLOATS, splits, off, t, p.n, m0, n0w, ep);
        return;
    }
    __syncthreads();               // other waves may still be reading operands
    unsigned char* const own = lds_raw + wave * (T::STORE);
    if (ep.vec_ok) mx_store<RF, CF, T::STORE_ROWS, true>(acc, own, t, p.n, m0, n0w, ep);
    else mx_store<RF, CF, T::STORE_ROWS, false>(acc, own, t, p.n, m0, n0w, ep);
}

template <int FMT, int RF, int CF, int LOOK, int WAVES>
int launch_mx_tile(regione_ctx* ctx, const MxOperands& p, int splits, const GemmEpilogue& ep) {
    using T = MxTileShape<FMT, RF, CF>;
    const int64_t row_tiles = mx_most_row_tiles(p, T::ROWS), n_tiles = (p.n + T::COLS - 1) / T::COLS;
    const int per = (p.steps + splits - 1) / splits, used = (p.steps + per - 1) / per;
    if (used > 1 && (static_cast<size_t>(row_tiles * n_tiles * used) * T::PART_FLOATS * sizeof(float) > ctx->gemm_part_bytes || row_tiles * n_tiles > kMaxSplitTiles))
        RG_FAIL(REGIONE_ERR_WORKSPACE, "linear: %d K-splits of a %d x %d result exceed the workspace", used, p.m, p.n);
    const int64_t workgroups = (row_tiles * n_tiles * used + 7) / 8 * 8;
    if (workgroups >= (int64_t{1} << 32) / T::THREADS) RG_FAIL(REGIONE_ERR_UNSUPPORTED, "linear: a result of %d x %d", p.m, p.n);
    hipLaunchKernelGGL((gemm_mx_tile_kernel<FMT, RF, CF, LOOK, WAVES>), dim3(static_cast<unsigned>(workgroups)), dim3(T::THREADS), T::LDS_BYTES, ctx->stream, p, used, per, ctx->gemm_part, ctx->gemm_arrived, ep);
    RG_LAUNCH_CHECK();
    return REGIONE_OK;
}

template <int FMT>
int launch_mx_tile(regione_ctx* ctx, int tile, const MxOperands& p, int splits, const GemmEpilogue& ep) {
    switch (tile) {
        case 72: return launch_mx_tile<FMT, 7, 2, 1, 1>(ctx, p, splits, ep);
        case 62: return launch_mx_tile<FMT, 6, 2, 1, 1>(ctx, p, splits, ep);
        case 52: return launch_mx_tile<FMT, 5, 2, 1, 1>(ctx, p, splits, ep);
        case 42: return launch_mx_tile<FMT, 4, 2, 1, 2>(ctx, p, splits, ep);
        case 32: return launch_mx_tile<FMT, 3, 2, 1, 2>(ctx, p, splits, ep);
        case 51: return launch_mx_tile<FMT, 5, 1, 2, 2>(ctx, p, splits, ep);
        case 41: return launch_mx_tile<FMT, 4, 1, 2, 2>(ctx, p, splits, ep);
        case 31: return launch_mx_tile<FMT, 3, 1, 2, 2>(ctx, p, splits, ep);
        case 22: return launch_mx_tile<FMT, 2, 2, 2, 2>(ctx, p, splits, ep);
        case 21: return launch_mx_tile<FMT, 2, 1, 2, 3>(ctx, p, splits, ep);
        case 11: return launch_mx_tile<FMT, 1, 1, 4, 3>(ctx, p, splits, ep);
    }
    RG_FAIL(REGIONE_ERR_INVALID_ARG, "linear: no tile %d", tile);
}

}  // namespace
