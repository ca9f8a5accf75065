// The products of gemm_mx.h for many rows: tiles of 64 x 64 to 256 x 256 results through LDS.
//
// Four waves, one per SIMD, each RF x CF fragments of 32 x 32 results: at 256 x 256 a wave's 256 accumulators fill half its registers, and 8 KiB of operands from LDS
// feed 16 instructions of 32 cycles, half of what the LDS delivers in that time (a quarter more goes into the copies).  The 32x32 instruction reaches its rate with one
// wave per SIMD, which the 16x16 one does not (register-only loops in 4 bits, PFLOP/s with one, two and four waves per SIMD: 6.3 / 6.5 / 6.6 against 4.2 / 5.5 / 6.1).
//
// K goes by in half steps (64 bytes of every row), copied from global memory straight into a ring of three or four LDS slots; a half step is two phases of RF * CF instructions.
// While a phase's instructions run, the same wave reads the operands of the next phase and issues a share of the copies; one barrier per half step.
#pragma once
#include "gemm_mx.h"
#include <type_traits>

namespace {

// One or two copies of 16 bytes per lane into LDS, the second one's 1 KiB behind the first (its lane offset is 1 KiB less than its address): the counterpart of pp_copy16 through a
// buffer resource, whose size makes accesses past the end of a tensor, and all of a half step that does not exist, into reads of nothing.
__device__ __forceinline__ void mx_copy(unsigned lane_off, const u32x4& rsrc, unsigned lds_base) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" :: "v"(lane_off), "s"(rsrc), "s"(lds_base) : "memory", "m0");
}
__device__ __forceinline__ void mx_copy(unsigned lane_off, unsigned lane_off2, const u32x4& rsrc, unsigned lds_base) {
    asm volatile("s_mov_b32 m0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %2, 0 offen lds\n\tbuffer_load_dwordx4 %1, %2, 0 offen offset:1024 lds"
                 :: "v"(lane_off), "v"(lane_off2), "s"(rsrc), "s"(lds_base) : "memory", "m0");
}
// A source of copies: `at` moves on by a stride per (half) step, `left` are the bytes from there to the end of what may be read.
struct MxSource {
    uint64_t at; int left;
    __device__ __forceinline__ u32x4 rsrc(bool there) const { return u32x4{static_cast<unsigned>(at), static_cast<unsigned>(at >> 32), there ? static_cast<unsigned>(left) : 0u, 0x00027000u}; }
};

template <int FMT, int RF, int CF, int SLOTS, int KG> struct MxTileShape {
    static constexpr int ROWS = 64 * RF, COLS = 64 * CF, THREADS = 256 * KG;
    static constexpr int COPIES = RF + CF;                          // 1 KiB copies per wave and half step: RF of 16 rows, CF of a weight block's 64 inputs
    static constexpr unsigned SLOT = (ROWS + COLS) * 64u, W_BASE = ROWS * 64u;
    static constexpr unsigned SCALES = FMT == MX_FP4 ? 4096u : 0u, S_BASE = SLOTS * SLOT;       // of a whole step, 1 KiB per wave: rows 0.., 128.., columns 0.., 128..; two of them
    static constexpr unsigned GROUP = S_BASE + 2 * SCALES, LDS_BYTES = KG * GROUP;       // of a group of four waves
    static_assert(LDS_BYTES <= 163840u && (KG == 1 || (RF % 2 == 0 && LDS_BYTES >= ROWS * COLS * 4u)), "what a CU has, and the groups' exchange");
    static constexpr int STORE_ROWS = RF / KG % 2 == 0 && 2 * CF * 16384u <= GROUP ? 2 : 1;                   // rows of fragments per wave that mx_store leaves in LDS at a time
    static_assert(STORE_ROWS * CF * 16384u <= GROUP, "four waves' fragments");
    static constexpr int FIT = 163840 / LDS_BYTES, WAVES = RF * CF > 8 ? 1 : RF * CF > 2 || KG == 2 ? 2 : FIT > 4 ? 4 : FIT;    // workgroups that a CU's LDS holds; waves per SIMD that registers are kept for
    static constexpr int64_t PART_FLOATS = static_cast<int64_t>(ROWS) * COLS;
};

// One instruction on phase P of a step (64 or 16 inputs); scales: byte P of a lane's words.
template <int FMT, int P>
__device__ __forceinline__ f32x16 mx_mfma32(const u32x4& w, const u32x4& a, const f32x16& acc, unsigned w_scale, unsigned a_scale) {
    if constexpr (FMT == MX_BF16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, a), acc, 0, 0, 0);
    else return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(mx_half_operand(w), mx_half_operand(a), acc, 4, 4, P, static_cast<int>(w_scale), P, static_cast<int>(a_scale));
}
template <int I> __device__ __forceinline__ f32x4 mx_part(const f32x16& v) { return f32x4{v[4 * I], v[4 * I + 1], v[4 * I + 2], v[4 * I + 3]}; }

// A fragment as it is from here on: without it the compiler reads all accumulators of the three ways to store them out of their registers at once, and spills.
template <bool ACC_REGISTERS> __device__ __forceinline__ f32x16 mx_here(f32x16 v) {
    if constexpr (ACC_REGISTERS) asm volatile("" : "+a"(v)); else asm volatile("" : "+v"(v));
    return v;
}

// Writes a wave's accumulators: acc[i][j] of a lane holds row 32*i + lane%32 and columns 32*j + 16*b + 8*(lane/32) + 0..7, b = 0, 1, of the wave's part.  By way of LDS (the wave's own
// part of it, IR rows of fragments at a time), so that a store covers whole rows of the part, 256 bytes at 128 bf16 columns: straight from the accumulators, 32 bytes of 32
// rows at a time, 2048 x 8192 x 256 took 17.6 us instead of 15.1.
template <int RF, int CF, int IR, bool ALIGNED>
__device__ __forceinline__ void mx_store(const f32x16 (&acc)[RF][CF], unsigned char* lds, const MxTile& t, int N, int m0, int n0w, const GemmEpilogue& ep) {
    constexpr int PIECES = 8 * CF, KEY = (PIECES < 16 ? PIECES : 16) - 1;        // 16-byte pieces of a row; piece c of row r lies at c ^ (r & KEY)
    constexpr int GROUPS = 4 * CF;                                                // of eight columns in a row: a lane stays with one
    static_assert(RF % IR == 0, "whole rounds");
    const int lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
    const int group = lane % GROUPS, col = n0w + 8 * group;
    Raw8 raw;
    EpiRow<EPI_PLAIN, false> r;
    EpiColumns<EPI_PLAIN, false> cols;
    if (col + 8 <= N) cols.load(ep, col);
    f32x4* const to = reinterpret_cast<f32x4*>(lds) + l32 * PIECES;
    const f32x4* const from = reinterpret_cast<const f32x4*>(lds);
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
#pragma unroll 4
        for (int lr = lane / GROUPS; lr < 32 * IR; lr += 64 / GROUPS) {
            const int row = m0 + 32 * i0 + lr;
            const f32x4 lo = from[lr * PIECES + ((2 * group) ^ (lr & KEY))], hi = from[lr * PIECES + ((2 * group + 1) ^ (lr & KEY))];
            if (row < t.begin || row >= t.end || col >= N) continue;
            if (ALIGNED || col + 8 <= N) epilogue_store8<EPI_PLAIN, false, ALIGNED>(ep, row, col, lo, hi, cols, r, raw);
            else epilogue_ragged<EPI_PLAIN, false>(ep, row, col, N, lo, hi);
        }
    }
}

// The end of a K split: sums of all splits, added in split order, straight from where they were left; G fragments' pieces of a split are requested together, one split ahead.
template <int RF, int CF>
__device__ __forceinline__ void mx_store_sums(float* sums, int splits, unsigned off, const MxTile& t, int N, int m0, int n0w, const GemmEpilogue& ep) {
    constexpr int F = RF * CF, G = F % 4 == 0 ? 4 : F % 3 == 0 ? 3 : F % 2 == 0 ? 2 : 1;
    constexpr unsigned bytes = RF * CF * 4u * 4096u;               // of a split
    const auto rsrc = pp_part_rsrc(sums, splits * static_cast<int64_t>(bytes / 4));
    const int l32 = threadIdx.x & 31, half = (threadIdx.x >> 5) & 1;
    Raw8 raw;
    EpiRow<EPI_PLAIN, false> r;
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
                if (col + 8 <= N) {
                    EpiColumns<EPI_PLAIN, false> cols;
                    cols.load(ep, col);
                    if (ep.vec_ok) epilogue_store8<EPI_PLAIN, false, true>(ep, row, col, sum[4 * g + 2 * b], sum[4 * g + 2 * b + 1], cols, r, raw);
                    else epilogue_store8<EPI_PLAIN, false, false>(ep, row, col, sum[4 * g + 2 * b], sum[4 * g + 2 * b + 1], cols, r, raw);
                } else if (col < N) {
                    epilogue_ragged<EPI_PLAIN, false>(ep, row, col, N, sum[4 * g + 2 * b], sum[4 * g + 2 * b + 1]);
                }
            }
        }
    }
}

template <int FMT, int RF, int CF, int SLOTS, int KG>
__global__ void __launch_bounds__(256 * KG) __attribute__((amdgpu_waves_per_eu(MxTileShape<FMT, RF, CF, SLOTS, KG>::WAVES)))
gemm_mx_tile_kernel(MxOperands p, int splits, int steps_per_split, float* __restrict__ partial, int* __restrict__ arrived, GemmEpilogue ep) {
    using T = MxTileShape<FMT, RF, CF, SLOTS, KG>;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds_all[];
    const int kg = KG == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 8);
    unsigned char* const lds_raw = lds_all + kg * T::GROUP;
    const unsigned lds0 = static_cast<unsigned>(reinterpret_cast<size_t>((__attribute__((address_space(3))) void*)(lds_all))) + kg * T::GROUP;
    const int n_tiles = (p.n + T::COLS - 1) / T::COLS;
    const MxTiles<T::ROWS> row_tiles(p);
    const int m_tiles = row_tiles.total;
    const int units = m_tiles * n_tiles * splits, per_xcd = (units + 7) >> 3;
    const int local = static_cast<int>(blockIdx.x >> 3), unit = static_cast<int>(blockIdx.x & 7) * per_xcd + local;     // each XCD a contiguous range (see pp_unit)
    if (local >= per_xcd || unit >= units) return;
    int m_tile, n_tile, split = 0;
    if (splits == 1) {
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
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) & 3;
    const int wm = wave >> 1, wn = wave & 1;
    int step0 = split * steps_per_split;
    int n_steps = p.steps - step0;
    n_steps = n_steps < steps_per_split ? n_steps : steps_per_split;
    const int n_turns = KG == 1 ? n_steps : (n_steps + 1) >> 1;                    // two groups: the first takes the first half of the steps, one more where they are odd
    if (KG == 2) {
        step0 += kg * n_turns;
        n_steps = kg == 0 ? n_turns : n_steps - n_turns;
    }
    const int n_half = 2 * n_steps;

    // Copy sources.  A: a lane copies 16 bytes of a row's 64; chunk c of row r lies at c ^ ((r >> 2) & 3), so that sixteen rows' same chunk covers all banks once.  Rows past the tensor's
    // end read nothing; past a row's end the next row's values are read, which meet weights of zero (bf16 rows are whole steps), and E2M1 has neither NaN nor infinity.
    unsigned a_voff[RF];
#pragma unroll
    for (int i = 0; i < RF; ++i)
        a_voff[i] = static_cast<unsigned>((wave * RF + i) * 16 + (lane >> 2)) * static_cast<unsigned>(p.row_bytes) + static_cast<unsigned>((lane & 3) ^ ((lane >> 4) & 3)) * 16u + (i % 2 == 1 ? 0u : 1024u);
    const int64_t a_first = static_cast<int64_t>(t.row0) * p.row_bytes + static_cast<int64_t>(step0) * 128 - 1024;     // (the second copy of a pair adds 1 KiB by itself)
    const int64_t a_left = static_cast<int64_t>(p.m) * p.row_bytes - a_first;
    MxSource a = {reinterpret_cast<uint64_t>(p.a) + a_first, static_cast<int>(a_left < INT32_MAX ? a_left : INT32_MAX)};
    // W: a block's 64 inputs are one fragment; its 32 features are put in the order that leaves a lane with twice eight consecutive results beside those of the row's other lane:
    // place 8*g + 4*h + u, whose results lane half h holds in registers 4*g + u, gets feature 16*(g/2) + 8*h + 4*(g%2) + u.
    const uint8_t* w_all = p.w + t.weight * p.w_stride;
    const unsigned feature = (l32 >> 4) * 16 + ((l32 >> 2) & 1) * 8 + ((l32 >> 3) & 1) * 4 + (l32 & 3);
    unsigned w_voff[CF];
#pragma unroll
    for (int j = 0; j < CF; ++j) {
        const int piece = wave * CF + j;                                           // piece / 2: block of the tile, piece % 2: phase of the half step
        int nb = piece >> 1;
        nb = (n0 >> 5) + nb < n32 / 32 ? nb : n32 / 32 - 1 - (n0 >> 5);            // blocks past N repeat the last one
        w_voff[j] = static_cast<unsigned>(nb) * static_cast<unsigned>(p.steps) * 4096u + (piece & 1) * 1024u + ((lane & 32) + feature) * 16u + (j % 2 == 1 ? 0u : 1024u);
    }
    MxSource w = {reinterpret_cast<uint64_t>(w_all) + (static_cast<int64_t>(n0 >> 5) * p.steps + step0) * 4096 - 1024, INT32_MAX};
    // scales of a step: waves 0 and 1 copy those of the rows, waves 2 and 3 of the columns, 16 bytes (two rows) per lane
    MxSource scales = {0, INT32_MAX};
    unsigned s_voff = 0;
    int64_t s_step = 0;
    if (FMT == MX_FP4) {
        const int first = wave < 2 ? t.row0 / 2 : n0 / 2, last = (wave < 2 ? static_cast<int>(mx_padded_rows(p.m)) : n32) / 2 - 1 - first, pair = (wave & 1) * 64 + lane;
        s_voff = static_cast<unsigned>(pair < last ? pair : last) * 16u;           // pairs past the end repeat the last one
        s_step = (wave < 2 ? mx_padded_rows(p.m) : n32) * 8;
        scales.at = reinterpret_cast<uint64_t>(wave < 2 ? p.a_scale : w_all + static_cast<int64_t>(n32) * p.steps * 128) + step0 * s_step + static_cast<int64_t>(first) * 16;
    }

    // LDS addresses of the fragments
    unsigned a_off[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) a_off[q] = static_cast<unsigned>(wm * (RF * 32) + l32) * 64u + static_cast<unsigned>(((2 * q + half) ^ ((l32 >> 2) & 3)) << 4);
    const unsigned w_off = T::W_BASE + static_cast<unsigned>(wn * CF) * 2048u + lane * 16u;
    const unsigned as_off = T::S_BASE + static_cast<unsigned>(wm * (RF * 32) + l32) * 8u + half * 4u;
    const unsigned ws_off = T::S_BASE + 2048u + (static_cast<unsigned>(wn * (CF * 32)) + feature) * 8u + half * 4u;

    f32x16 acc[RF][CF];
#pragma unroll
    for (int i = 0; i < RF; ++i)
#pragma unroll
        for (int j = 0; j < CF; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

    // Copies come in pairs; sources move on with the last one of a half step.  (No branches: the accumulators' instructions would be moved across them.)
    auto copy_pair = [&](MxSource& from, const auto& voff, bool there, unsigned to, auto index, int stride) __attribute__((always_inline)) {
        constexpr int C = 2 * decltype(index)::value, N = sizeof(voff) / sizeof(voff[0]);
        if constexpr (C + 1 < N) mx_copy(voff[C], voff[C + 1], from.rsrc(there), to + C * 1024u);
        else mx_copy(voff[C], from.rsrc(there), to + C * 1024u);
        if constexpr (C + 2 >= N) from.at += static_cast<int64_t>(stride);
    };
    constexpr int A_PAIRS = (RF + 1) / 2, W_PAIRS = (CF + 1) / 2;
    constexpr int SC = FMT == MX_FP4 ? 1 : 0;
    // number C of the copies of half step h into its slot: rows; weights, and for even half steps scales behind them
    auto copy_a = [&](int h, unsigned slot, auto c) __attribute__((always_inline)) {
        copy_pair(a, a_voff, h < n_half, lds0 + slot + wave * (RF * 1024u), c, 64);
        if constexpr (decltype(c)::value == A_PAIRS - 1) asm("s_sub_i32 %0, %0, 64\n\ts_max_i32 %0, %0, 0" : "+s"(a.left) : : "scc");     // (left to itself the compiler subtracts in a vector register)
    };
    auto copy_w = [&](int h, unsigned slot, auto c) __attribute__((always_inline)) {
        if constexpr (decltype(c)::value < W_PAIRS) {
            copy_pair(w, w_voff, h < n_half, lds0 + slot + T::W_BASE + wave * (CF * 1024u), c, 2048);
        } else {
            mx_copy(s_voff, scales.rsrc(h < n_half), lds0 + T::S_BASE + ((h >> 1) & 1) * T::SCALES + wave * 1024u);
            scales.at += s_step;
        }
    };
    auto each = [&](auto from, auto to, auto f, auto self) __attribute__((always_inline)) {
        if constexpr (decltype(from)::value < decltype(to)::value) {
            f(from);
            self(std::integral_constant<int, decltype(from)::value + 1>{}, to, f, self);
        }
    };
    typedef std::integral_constant<int, 0> zero;
    typedef std::integral_constant<int, A_PAIRS> a_pairs;
    each(zero{}, std::integral_constant<int, SLOTS>{}, [&](auto hc) __attribute__((always_inline)) {
        constexpr int H = decltype(hc)::value;
        each(zero{}, a_pairs{}, [&](auto c) __attribute__((always_inline)) { copy_a(H, H * T::SLOT, c); }, each);
        if constexpr (H < SLOTS - 1) each(zero{}, std::integral_constant<int, W_PAIRS + (H % 2 == 0 ? SC : 0)>{}, [&](auto c) __attribute__((always_inline)) { copy_w(H, H * T::SLOT, c); }, each);
    }, each);
    pp_wait<(SLOTS == 4 ? 2 * T::COPIES + SC : T::COPIES) + RF>();
    pp_barrier();

    u32x4 af[2][RF], wf[2][CF];
    unsigned as[2][RF], ws[2][CF];
    // operand number F of phase Q of the half step in `slot`
    auto read = [&](unsigned slot, auto q, auto b, auto index) __attribute__((always_inline)) {
        constexpr int F = decltype(index)::value, Q = decltype(q)::value, B = decltype(b)::value;
        if constexpr (F < CF) wf[B][F] = *reinterpret_cast<const u32x4*>(lds_raw + (w_off + slot) + F * 2048 + Q * 1024);
        else af[B][F - CF] = *reinterpret_cast<const u32x4*>(lds_raw + (a_off[Q] + slot) + (F - CF) * 2048);
    };
    auto read_scale = [&](unsigned which, auto b, auto index) __attribute__((always_inline)) {
        constexpr int F = decltype(index)::value, B = decltype(b)::value;
        if constexpr (FMT == MX_FP4) {
            if constexpr (F < CF) ws[B][F] = *reinterpret_cast<const unsigned*>(lds_raw + (ws_off + which) + F * 256);
            else as[B][F - CF] = *reinterpret_cast<const unsigned*>(lds_raw + (as_off + which) + (F - CF) * 256);
        }
    };
    typedef std::integral_constant<int, 1> one;
    typedef std::integral_constant<int, RF + CF> operands;
    each(zero{}, operands{}, [&](auto f) { read(0, zero{}, zero{}, f); read_scale(0, zero{}, f); }, each);

    // Phase P (0..3) of step `s`, whose half steps lie in slots `lo` and `hi`: its instructions, between them the reads of the next phase and copies.  Copies into the slot of a half step
    // start in its second phase, behind the barrier that all waves reach with their reads of it done, and end in the phase after that; a half step's copies have landed when those
    // of the SLOTS - 2 half steps after it are in flight.
    auto phase = [&](int s, unsigned lo, unsigned hi, auto pc) __attribute__((always_inline)) {
        constexpr int P = decltype(pc)::value, B = P & 1, COUNT = RF * CF;                // operands are in buffer B
        constexpr int AHEAD = P == 0 ? SLOTS - 1 : P == 3 ? SLOTS + 1 : SLOTS;            // of half step 2 s + AHEAD the rows are copied in odd phases, the weights and scales in even ones
        constexpr int PAIRS = (P & 1) ? A_PAIRS : W_PAIRS + (AHEAD % 2 == 0 ? SC : 0);
        const int ch = 2 * s + AHEAD;
        const unsigned cslot = P == 0 ? (lo == 0 ? (SLOTS - 1) * T::SLOT : lo - T::SLOT) : P == 3 ? hi : lo;
        const unsigned next = hi == (SLOTS - 1) * T::SLOT ? 0 : hi + T::SLOT;
        if constexpr (P & 1) {
            pp_wait<SLOTS == 4 ? 2 * T::COPIES + SC : T::COPIES + (P == 1 ? SC : 0)>();
            pp_barrier();
        }
        each(zero{}, std::integral_constant<int, COUNT>{}, [&](auto qc) __attribute__((always_inline)) {
            constexpr int Q = decltype(qc)::value, I = Q / CF, J = Q % CF;
            acc[I][J] = mx_mfma32<FMT, P>(wf[B][J], af[B][I], acc[I][J], ws[0][J], as[0][I]);
            // an operand of the next phase (all of them early, since the barrier waits for them), and copies spread over the phase
            constexpr int PER = (RF + CF + COUNT - 1) / COUNT, R0 = Q * PER < RF + CF ? Q * PER : RF + CF, R1 = (Q + 1) * PER < RF + CF ? (Q + 1) * PER : RF + CF;
            each(std::integral_constant<int, R0>{}, std::integral_constant<int, R1>{}, [&](auto f) __attribute__((always_inline)) {
                if constexpr (P == 0) read(lo, one{}, one{}, f);
                else if constexpr (P == 1) read(hi, zero{}, zero{}, f);
                else if constexpr (P == 2) read(hi, one{}, one{}, f);
                else { read(next, zero{}, zero{}, f); read_scale(((s + 1) & 1) * T::SCALES, one{}, f); }
            }, each);
            each(std::integral_constant<int, Q * PAIRS / COUNT>{}, std::integral_constant<int, (Q + 1) * PAIRS / COUNT>{}, [&](auto c) __attribute__((always_inline)) {
                if constexpr (P & 1) copy_a(ch, cslot, c);
                else copy_w(ch, cslot, c);
            }, each);
            __builtin_amdgcn_sched_barrier(0);
        }, each);
    };
    typedef std::integral_constant<int, 2> two;
    typedef std::integral_constant<int, 3> three;
    unsigned lo = 0;
    for (int s = 0; s < n_steps; ++s) {
        const unsigned hi = lo == (SLOTS - 1) * T::SLOT ? 0 : lo + T::SLOT;
        phase(s, lo, hi, zero{});
        phase(s, lo, hi, one{});
        phase(s, lo, hi, two{});
        phase(s, lo, hi, three{});
        lo = hi == (SLOTS - 1) * T::SLOT ? 0 : hi + T::SLOT;
#pragma unroll
        for (int j = 0; j < CF; ++j) ws[0][j] = ws[1][j];
#pragma unroll
        for (int i = 0; i < RF; ++i) as[0][i] = as[1][i];
    }
    pp_wait<0>();                  // nothing may still be writing LDS when it is used again or the workgroup ends
    if (KG == 2 && n_steps < n_turns) {       // the barriers of the other group's odd step
        pp_barrier();
        pp_barrier();
    }

    const int m0 = t.row0 + wm * (RF * 32), n0w = n0 + wn * (CF * 32);
    if (ep.bias) ep.bias += static_cast<int64_t>(t.weight) * p.n;
    if constexpr (KG == 2) {
        // Each group leaves the half of its rows of fragments that the other one finishes, and adds what that one left of its own.
        constexpr int H = RF / 2;
        f32x4* const give = reinterpret_cast<f32x4*>(lds_all) + ((1 - kg) * 4 + wave) * (H * CF * 256) + lane;
        const f32x4* const take = reinterpret_cast<const f32x4*>(lds_all) + (kg * 4 + wave) * (H * CF * 256) + lane;
        auto finish = [&](auto first) __attribute__((always_inline)) {
            constexpr int I0 = decltype(first)::value, G0 = H - I0;                // finishes rows [I0, I0 + H), gives [G0, G0 + H)
            __syncthreads();
#pragma unroll
            for (int f = 0; f < H * CF; ++f) {
                const f32x16 v = mx_here<false>(acc[G0 + f / CF][f % CF]);
                give[f * 256] = mx_part<0>(v); give[f * 256 + 64] = mx_part<1>(v); give[f * 256 + 128] = mx_part<2>(v); give[f * 256 + 192] = mx_part<3>(v);
            }
            __syncthreads();
            f32x16 sum[H][CF];
#pragma unroll
            for (int f = 0; f < H * CF; ++f)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const f32x4 x = take[f * 256 + c * 64];
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[f / CF][f % CF][4 * c + e] = kg == 0 ? acc[I0 + f / CF][f % CF][4 * c + e] + x[e] : x[e] + acc[I0 + f / CF][f % CF][4 * c + e];
                }
            __syncthreads();
            unsigned char* const own = lds_raw + wave * (T::STORE_ROWS * CF * 4096);
            if (ep.vec_ok) mx_store<H, CF, T::STORE_ROWS, true>(sum, own, t, p.n, m0 + 32 * I0, n0w, ep);
            else mx_store<H, CF, T::STORE_ROWS, false>(sum, own, t, p.n, m0 + 32 * I0, n0w, ep);
        };
        if (kg == 0) finish(zero{}); else finish(std::integral_constant<int, H>{});
        return;
    }
    if (splits > 1) {
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
    unsigned char* const own = lds_raw + wave * (T::STORE_ROWS * CF * 4096);
    if (ep.vec_ok) mx_store<RF, CF, T::STORE_ROWS, true>(acc, own, t, p.n, m0, n0w, ep);
    else mx_store<RF, CF, T::STORE_ROWS, false>(acc, own, t, p.n, m0, n0w, ep);
}

template <int FMT, int RF, int CF, int SLOTS, int KG>
int launch_mx_tile(regione_ctx* ctx, const MxOperands& p, int splits, const GemmEpilogue& ep) {
    using T = MxTileShape<FMT, RF, CF, SLOTS, KG>;
    static std::atomic<uint64_t> granted{0};
    const int64_t row_tiles = mx_most_row_tiles(p, T::ROWS), n_tiles = (p.n + T::COLS - 1) / T::COLS;
    if (KG > 1) splits = 1;
    const int per = (p.steps + splits - 1) / splits, used = (p.steps + per - 1) / per;
    if (used > 1 && (static_cast<size_t>(row_tiles * n_tiles * used) * T::PART_FLOATS * sizeof(float) > ctx->gemm_part_bytes || row_tiles * n_tiles > kMaxSplitTiles))
        RG_FAIL(REGIONE_ERR_WORKSPACE, "linear: %d K-splits of a %d x %d result exceed the workspace", used, p.m, p.n);
    const int64_t workgroups = (row_tiles * n_tiles * used + 7) / 8 * 8;
    if (workgroups >= (int64_t{1} << 32) / T::THREADS) RG_FAIL(REGIONE_ERR_UNSUPPORTED, "linear: a result of %d x %d", p.m, p.n);
    if (int rc = rg_grant_lds(ctx, reinterpret_cast<const void*>(gemm_mx_tile_kernel<FMT, RF, CF, SLOTS, KG>), granted, T::LDS_BYTES)) return rc;
    hipLaunchKernelGGL((gemm_mx_tile_kernel<FMT, RF, CF, SLOTS, KG>), dim3(static_cast<unsigned>(workgroups)), dim3(T::THREADS), T::LDS_BYTES, ctx->stream, p, used, per, ctx->gemm_part, ctx->gemm_arrived, ep);
    RG_LAUNCH_CHECK();
    return REGIONE_OK;
}

template <int FMT>
int launch_mx_tile(regione_ctx* ctx, int tile, const MxOperands& p, int splits, const GemmEpilogue& ep) {
    switch (tile) {
        case 44: return launch_mx_tile<FMT, 4, 4, 4, 1>(ctx, p, splits, ep);
        case 842: return launch_mx_tile<FMT, 4, 2, 3, 2>(ctx, p, splits, ep);
        case 824: return launch_mx_tile<FMT, 2, 4, 3, 2>(ctx, p, splits, ep);
        case 822: return launch_mx_tile<FMT, 2, 2, 4, 2>(ctx, p, splits, ep);
        case 821: return launch_mx_tile<FMT, 2, 1, 4, 2>(ctx, p, splits, ep);
        case 324: return launch_mx_tile<FMT, 2, 4, 3, 1>(ctx, p, splits, ep);
        case 342: return launch_mx_tile<FMT, 4, 2, 3, 1>(ctx, p, splits, ep);
        case 322: return launch_mx_tile<FMT, 2, 2, 3, 1>(ctx, p, splits, ep);
        case 34: return launch_mx_tile<FMT, 3, 4, 4, 1>(ctx, p, splits, ep);
        case 24: return launch_mx_tile<FMT, 2, 4, 4, 1>(ctx, p, splits, ep);
        case 42: return launch_mx_tile<FMT, 4, 2, 4, 1>(ctx, p, splits, ep);
        case 22: return launch_mx_tile<FMT, 2, 2, 4, 1>(ctx, p, splits, ep);
        case 12: return launch_mx_tile<FMT, 1, 2, 4, 1>(ctx, p, splits, ep);
        case 21: return launch_mx_tile<FMT, 2, 1, 4, 1>(ctx, p, splits, ep);
        case 11: return launch_mx_tile<FMT, 1, 1, 4, 1>(ctx, p, splits, ep);
    }
    RG_FAIL(REGIONE_ERR_INVALID_ARG, "linear: no tile %d", tile);
}

}  // namespace
