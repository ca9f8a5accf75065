// Low-rank adapters of many requests beside a shared projection: packing, and the inner products of every row with its adapters' A.  What they bring to the result are further
// K-steps of the projection's tiles (gemm_adapters.h).
#include "gemm_adapters.h"

namespace {

constexpr int kThreads = 256;
constexpr int kNoAdapter = 0x7fffffff;
constexpr int kMostRank = 256, kMostSel = 32, kMostAdapters = 1 << 16;
constexpr size_t kTermBytes = size_t{64} << 20;          // of the inner products of the rows that go through at a time

// A packed adapter: behind A and B a bit per column of B that holds a value that is not finite (zero in B), 32 to a word, a word that is not zero if there is one, and zeros up to 16 bytes.
// A in fragments of 16 ranks x 32 inputs, 64 lanes x 8 values, lane l holding A[16 * (block) + l % 16][32 * step + 8 * (l / 16) .. +8]; behind it B as regione_pack_weight
// lays out a weight [n, rank rounded up to 16].
__host__ __device__ __forceinline__ int64_t a_elems(int k, int blocks) { return static_cast<int64_t>(blocks) * 16 * k; }
__host__ __device__ __forceinline__ int64_t b_elems(int n, int blocks) { return (static_cast<int64_t>(n) + 31) / 32 * 32 * blocks * 16; }
__host__ __device__ __forceinline__ int64_t bad_words(int n) { return ((static_cast<int64_t>(n) + 31) / 32 + 1 + 3) / 4 * 4; }
__host__ __device__ __forceinline__ int64_t adapter_elems(int n, int k, int blocks) { return a_elems(k, blocks) + b_elems(n, blocks) + 2 * bad_words(n); }

__global__ void __launch_bounds__(kThreads)
pack_adapter_kernel(const bf16_t* __restrict__ a, const bf16_t* __restrict__ b, int n, int k, int rank, int blocks, bf16_t* __restrict__ packed) {
    const int64_t a_count = a_elems(k, blocks), b_end = a_count + b_elems(n, blocks), count = adapter_elems(n, k, blocks), stride = static_cast<int64_t>(gridDim.x) * kThreads;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < count; i += stride) {
        bf16_t v = 0;
        if (i < a_count) {
            const int e = static_cast<int>(i & 7), lane = static_cast<int>(i >> 3) & 63;
            const int64_t f = i >> 9;
            const int block = static_cast<int>(f / (k >> 5)), step = static_cast<int>(f % (k >> 5));
            const int r = 16 * block + (lane & 15);
            if (r < rank) v = a[static_cast<int64_t>(r) * k + 32 * step + 8 * (lane >> 4) + e];
        } else if (i < b_end) {
            const int64_t at = i - a_count;
            const int e = static_cast<int>(at & 7), lane = static_cast<int>(at >> 3) & 63;
            const int64_t f = at >> 9;
            const int block = static_cast<int>(f % blocks);
            const int64_t col = f / blocks * 32 + (lane & 31);
            const int r = 16 * block + 8 * (lane >> 5) + e;
            if (col < n && r < rank) v = b[col * rank + r];
            v = (v & 0x7f80u) == 0x7f80u ? 0 : v;
        }
        packed[i] = v;
    }
}

// the columns' bits, a lane per column (behind pack_adapter_kernel, which has made them zeros)
__global__ void __launch_bounds__(kThreads)
pack_adapter_bad_kernel(const bf16_t* __restrict__ b, int n, int rank, uint32_t* __restrict__ bad) {
    const int64_t n_pad = (static_cast<int64_t>(n) + 63) / 64 * 64, stride = static_cast<int64_t>(gridDim.x) * kThreads;
    const int words = (n + 31) / 32;
    for (int64_t col = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; col < n_pad; col += stride) {       // (whole waves)
        bool found = false;
        if (col < n)
            for (int r = 0; r < rank; ++r) found = found || (b[col * rank + r] & 0x7f80u) == 0x7f80u;
        const uint64_t bits = __ballot(found);
        const int word = static_cast<int>(col >> 5);
        if ((threadIdx.x & 31) == 0 && word < words) {
            const uint32_t here = static_cast<uint32_t>(bits >> (threadIdx.x & 32));
            if (here) { bad[word] = here; bad[words] = 1u; }      // (whoever writes the last word writes the same)
        }
    }
}

// w * x[row] A_a^T, w the sum of the row's weights of adapter a, as kTerms bf16 values: the value rounded, what is left of it rounded, and what is left then.  Of a float32's 24 bits the first leaves at
// most 16 and the second eight, so that the three add up to it exactly.  One term would be rounded as a bf16 result is, two would leave 2^-17 of the share: where the projection cancels the
// adapter, all that is left may lie below that.  us, the whole call with a bf16 result, two terms / three: 48 rows with 32 adapters of
// rank 16, 2048 x 4096, 14.0 / 15.4; 820 rows, two of rank 32 each, 3072 x 12288, 74.3 / 77.0; 8704 rows, rank 64, 3072 x 9216, 395 / 404; 8192 rows with 500 adapters of rank 16, 2048 x 4096, 194 / 236.
constexpr int kTerms = 3;
// Four values at ranks 16 * block + 4 * kc on, where at(column) is: the terms' blocks one after the other, filled up to `cols` with zeros.
template <typename At> __device__ __forceinline__ void put_terms(const At& at, int kc, int block, int blocks, int cols, float w, const f32x4& sum, bool named = true) {
    float left[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) left[e] = named ? w * sum[e] : 0.f;
#pragma unroll
    for (int p = 0; p < kTerms; ++p) {
        bf16_t v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] = f32_to_bf16(left[e]);
            if (p == 0) v[e] -= (v[e] & 0x7fff) == 0x7f80 && __builtin_fabsf(left[e]) < INFINITY ? 1 : 0;       // (rounded up past the largest bf16, which is the first term then)
            const float r = bf16_to_f32(v[e]);
            left[e] = __builtin_fabsf(r) < INFINITY ? left[e] - r : 0.f;           // (what is not finite is one term)
        }
        *reinterpret_cast<uint2*>(at((p * blocks + block) * 16 + 4 * kc)) = make_uint2(v[0] | static_cast<unsigned>(v[1]) << 16, v[2] | static_cast<unsigned>(v[3]) << 16);
    }
    if (block == blocks - 1 && cols > kTerms * blocks * 16) *reinterpret_cast<uint2*>(at(kTerms * blocks * 16 + 4 * kc)) = make_uint2(0u, 0u);
}

constexpr int kDownWaves = 8;
struct DownCall { const bf16_t* x; const bf16_t* packed; int64_t stride; const int32_t* which; const float* weight; int count, sel, m, k, blocks, cols; bf16_t* t; };

// For the kernel of 16 rows, t [rows, sel, cols], each adapter at the first of the row's places that name it: a workgroup per block of 16 ranks of every place of 16 rows; those whose adapter an earlier place names end at once.  Its eight waves split K and meet in LDS, where the sums are
// formed in wave order.  One row, K 3072, rank 16 4.0 us, 48 rows with 32 adapters, K 2048 5.2: the launch, the row's adapter, then x and A in one trip to memory.
__global__ void __launch_bounds__(kDownWaves * 64)
adapters_down_rows_kernel(DownCall d) {
    constexpr int AHEAD = 8;
    __shared__ __attribute__((aligned(16))) f32x4 sums[kDownWaves][64];
    const int lane = threadIdx.x & 63, l16 = lane & 15, kc = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int m0 = blockIdx.x * 16, rows = d.m - m0 < 16 ? d.m - m0 : 16, entry = blockIdx.y / d.blocks, block = blockIdx.y - entry * d.blocks;
    if (entry >= rows * d.sel) return;
    const int32_t* const which = d.which + static_cast<int64_t>(m0) * d.sel;
    const int a = __builtin_amdgcn_readfirstlane(which[entry]);
    if (a < 0 || a >= d.count) return;
    const int steps = d.k >> 5, per = (steps + kDownWaves - 1) / kDownWaves;
    const int s0 = wave * per, s1 = s0 + per < steps ? s0 + per : steps;
    const bf16_t* const xp = d.x + static_cast<int64_t>(m0 + (l16 < rows ? l16 : rows - 1)) * d.k + 8 * kc;        // rows past the end repeat the last one
    const bf16_t* const wp = d.packed + static_cast<int64_t>(a) * d.stride + static_cast<int64_t>(block) * steps * 512 + lane * 8;
    bf16x8 xf[AHEAD], wf[AHEAD];
    auto request = [&](int base) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < AHEAD; ++c)
            if (base + c < s1) {
                xf[c] = *reinterpret_cast<const bf16x8*>(xp + (base + c) * 32);
                wf[c] = *reinterpret_cast<const bf16x8*>(wp + static_cast<int64_t>(base + c) * 512);
            }
    };
    request(s0);
    for (int i = 0; i < entry; i += 64)
        if (__ballot(i + lane < entry && which[i + lane < entry ? i + lane : 0] == a)) return;      // (the same for all waves)
    int place = -1;                                               // the row's first place of the adapter, and its weights
    float w = 0.f;
    if (l16 < rows)
        for (int s = d.sel - 1; s >= 0; --s)
            if (which[l16 * d.sel + s] == a) {
                place = s;
                w += d.weight ? d.weight[static_cast<int64_t>(m0 + l16) * d.sel + s] : 1.f;
            }
    f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int base = s0; base < s1; base += AHEAD) {
        if (base > s0) request(base);
#pragma unroll
        for (int c = 0; c < AHEAD; ++c)
            if (base + c < s1) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[c], xf[c], acc, 0, 0, 0);
    }
    sums[wave][lane] = acc;
    __syncthreads();
    if (wave || place < 0) return;
#pragma unroll
    for (int v = 1; v < kDownWaves; ++v) acc += sums[v][lane];
    bf16_t* const row = d.t + (static_cast<int64_t>(m0 + l16) * d.sel + place) * d.cols;
    put_terms([&](int c) { return row + c; }, kc, block, d.blocks, d.cols, w, acc);
}

// For tiles (their layout and plan: gemm_adapters.h): a workgroup owns 16 * RB rows and goes through the blocks of 16 ranks of their adapters, NB at a time; those of the tile that none of the
// rows names are zeros there.  Without a plan (many rows for the kernel of 16): the layout above, every workgroup's rows by themselves.  Workgroups of the same rows (blockIdx.y) take turns.  WAVES waves split K and meet in LDS, where the sums are formed in wave order.
// The rows come in whole lines, 8 x 128 bytes to a load, and change to fragments in a part of LDS that is the wave's own.  What bounds it is the way from L2 into a CU, 20 bytes a cycle: all of A
// for every workgroup beside its rows, so that 32 rows to a workgroup pay where there are workgroups enough.  8704 rows, K 3072, rank 64: 22 us (33 with x from HBM), 6 of them the launch and the list of the
// adapters; with A from L1 20, with x from L1 too 18.  As fragments from memory, 64 bytes of 16 rows to a load, x took half as long again.
// Steps past a wave's own are multiplied with zeros: a branch around the products lets the compiler move the loads into it, behind all that should hide them.
struct DownTiles { int rows, plan_pitch; int64_t tile_elems; int32_t* plan; int64_t bad; };      // rows of a tile; elements of an adapter ahead of its bits
template <bool PLANNED, int RB, int NB, int WAVES>
__global__ void __launch_bounds__(WAVES * 64)
adapters_down_tiles_kernel(DownCall d, DownTiles tiles) {
    constexpr int T = WAVES * 64, ROWS = 16 * RB, AHEAD = 2;
    __shared__ uint32_t named[2][kMostAdapters / 32];             // by the tile, by the workgroup's rows
    __shared__ int32_t ids[ROWS * kMostSel];
    __shared__ float weights[ROWS * kMostSel];
    // a wave's rows of a step on their way from whole lines to fragments; at the end the sums
    constexpr int TURN = 2048 * RB, SUMS = NB * 1024;
    __shared__ __attribute__((aligned(16))) unsigned char lds[WAVES * (TURN > SUMS ? TURN : SUMS)];
    static_assert(NB <= WAVES && sizeof(named) + sizeof(ids) + sizeof(weights) + sizeof(lds) <= 65536, "a wave per block at the end, and LDS");
    unsigned char (*const turn)[TURN] = reinterpret_cast<unsigned char (*)[TURN]>(lds);
    f32x4 (*const sums)[NB][64] = reinterpret_cast<f32x4 (*)[NB][64]>(lds);
    const int lane = threadIdx.x & 63, l16 = lane & 15, kc = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int pieces = PLANNED ? (tiles.rows + ROWS - 1) / ROWS : 1, tile = blockIdx.x / pieces, row0 = (blockIdx.x - tile * pieces) * ROWS;
    const int most_rows = PLANNED ? tiles.rows : ROWS, t0 = tile * most_rows, tile_rows = d.m - t0 < most_rows ? d.m - t0 : most_rows, m0 = t0 + row0;
    const int rows = tile_rows - row0 < ROWS ? tile_rows - row0 : ROWS, place_rows = most_rows - row0 < ROWS ? most_rows - row0 : ROWS;
    if (rows <= 0) return;                                        // (the last tile's end)
    const int steps = d.k >> 6, share = (steps + WAVES - 1) / WAVES, s0 = wave * share;    // of 64 inputs
    const int own = s0 + share < steps ? share : (steps > s0 ? steps - s0 : 0);
    const bf16_t* xp[2 * RB];
#pragma unroll
    for (int i = 0; i < 2 * RB; ++i) {
        const int row = 8 * i + (lane >> 3);
        xp[i] = d.x + static_cast<int64_t>(m0 + (row < rows ? row : rows - 1)) * d.k + 8 * (lane & 7);      // rows past the end repeat the last one
    }
    u32x4 xr[AHEAD][2 * RB];
    bf16x8 wf[AHEAD][2][NB];
    unsigned char* const put = turn[wave] + (lane >> 3) * 128 + (((lane & 7) ^ ((lane >> 4) & 3)) << 4);
    unsigned char* const put_odd = turn[wave] + (lane >> 3) * 128 + (((lane & 7) ^ (((lane >> 4) & 3) + 4)) << 4);       // rows 8 on of 16
    const unsigned char* const get = turn[wave] + l16 * 128;
    auto step_of = [&](int c) __attribute__((always_inline)) { const int s = s0 + c; return s < steps ? s : steps - 1; };      // (what is past the wave's steps is not multiplied)
#pragma unroll
    for (int c = 0; c < AHEAD; ++c)
#pragma unroll
        for (int i = 0; i < 2 * RB; ++i) xr[c][i] = *reinterpret_cast<const u32x4*>(xp[i] + step_of(c) * 64);

    const bool lead = PLANNED && row0 == 0 && blockIdx.y == 0;     // writes the tile's plan
    uint32_t bad = 0;                                             // (looked at here, side by side; one after the other as the list goes, 1711 rows with 23 adapters, K 320, 14.5 -> 16.1 us)
    const int words = (d.count + 31) / 32;
    for (int i = threadIdx.x; i < words; i += T) named[0][i] = named[1][i] = 0u;
    __syncthreads();
    for (int i = threadIdx.x; i < tile_rows * d.sel; i += T) {
        const int id = d.which[static_cast<int64_t>(t0) * d.sel + i], at = i - (m0 - t0) * d.sel;
        const bool counts = id >= 0 && id < d.count, here = at >= 0 && at < rows * d.sel;
        if (counts) {
            atomicOr(&named[0][id >> 5], 1u << (id & 31));
            if (here) atomicOr(&named[1][id >> 5], 1u << (id & 31));
            if (lead) bad |= *reinterpret_cast<const uint32_t*>(d.packed + static_cast<int64_t>(id) * d.stride + tiles.bad);
        }
        if (here) {
            ids[at] = counts ? id : kNoAdapter;
            weights[at] = d.weight ? d.weight[static_cast<int64_t>(m0) * d.sel + at] : 1.f;
        }
    }
    __syncthreads();

    unsigned char* const t = reinterpret_cast<unsigned char*>(d.t + (PLANNED ? tile * tiles.tile_elems : static_cast<int64_t>(m0) * d.sel * d.cols));
    auto place = [&](int row, int of, int c) __attribute__((always_inline)) {       // column c of a block of 16 terms, in the order of LDS
        return t + (static_cast<int64_t>(of >> 2) * tiles.rows + row) * 128 + ((((of & 3) * 2 + (c >> 3)) ^ ((row >> 1) & 7)) << 4) + (c & 7) * 2;
    };
    const int per = kTerms * d.blocks;                            // blocks of 16 terms of an adapter
    int32_t* const plan = tiles.plan + static_cast<int64_t>(tile) * tiles.plan_pitch;
    int64_t* const offsets = reinterpret_cast<int64_t*>(plan + 4);
    const int ids_at = 4 + (tiles.plan_pitch - 4) / 3 * 2;
    auto zeros = [&](int of, int count) __attribute__((always_inline)) {
        for (int i = threadIdx.x; i < count * (ROWS * 2); i += T)
            if (i / 2 % ROWS < place_rows) *reinterpret_cast<uint4*>(place(row0 + i / 2 % ROWS, of + i / (ROWS * 2), (i & 1) * 8)) = make_uint4(0u, 0u, 0u, 0u);
    };

    int a = -1, last = 0, pos = -1, block = d.blocks;
    bool in_rows = false;
    const uint32_t tile_word = lane < words ? named[0][lane] : 0u, rows_word = lane < words ? named[1][lane] : 0u;
    auto next_adapter = [&]() __attribute__((always_inline)) {    // the tile's next one, in order (its words from LDS one by one: 1711 rows with 23 adapters 12.5 -> 14.5 us)
        int w = (a + 1) >> 5;
        uint32_t mask = ~0u << ((a + 1) & 31);
        a = kNoAdapter;
        if (words <= 64) {                                        // all words in the wave's registers
            const uint32_t v = lane < w ? 0u : lane == w ? tile_word & mask : tile_word;
            const uint64_t some = __ballot(v != 0u);
            if (some) {
                const int first = __builtin_ctzll(some);
                a = first * 32 + __builtin_ctz(static_cast<unsigned>(__builtin_amdgcn_readlane(static_cast<int>(v), first)));
                in_rows = static_cast<unsigned>(__builtin_amdgcn_readlane(static_cast<int>(rows_word), first)) >> (a & 31) & 1u;
            }
        } else {
            while (w < words) {
                const int at = w + lane;
                uint32_t v = at < words ? named[0][at] : 0u;
                if (lane == 0) v &= mask;
                mask = ~0u;
                const uint64_t some = __ballot(v != 0u);
                if (some) {
                    const int first = __builtin_ctzll(some);
                    a = (w + first) * 32 + __builtin_ctz(static_cast<unsigned>(__builtin_amdgcn_readlane(static_cast<int>(v), first)));
                    in_rows = named[1][a >> 5] >> (a & 31) & 1u;
                    break;
                }
                w += 64;
            }
        }
        if (a == kNoAdapter) return;
        ++pos;
        last = a;
        if (lead) {
            for (int i = threadIdx.x; i < per; i += T) {
                offsets[pos * per + i] = (a * d.stride + (i % d.blocks) * 512) * 2;
                plan[ids_at + pos * per + i] = a;
            }
        }
        if (PLANNED && !in_rows && pos % gridDim.y == blockIdx.y) zeros(pos * per, per);
    };
    bool first_batch = true;
    for (unsigned batch = 0; a != kNoAdapter; ++batch) {
        int unit_a[NB], unit_block[NB], unit_pos[NB], units = 0;
#pragma unroll
        for (int q = 0; q < NB; ++q) {
            while (a != kNoAdapter && (block == d.blocks || !in_rows)) { next_adapter(); block = 0; }
            unit_a[q] = a; unit_block[q] = block; unit_pos[q] = pos;
            if (a != kNoAdapter) { ++units; ++block; }
        }
        if (units == 0 || batch % gridDim.y != blockIdx.y) continue;
        const bf16_t* wp[NB];
#pragma unroll
        for (int q = 0; q < NB; ++q) wp[q] = d.packed + static_cast<int64_t>(q < units ? unit_a[q] : unit_a[0]) * d.stride + static_cast<int64_t>(q < units ? unit_block[q] : unit_block[0]) * steps * 1024 + lane * 8;
        f32x4 acc[RB][NB];
#pragma unroll
        for (int i = 0; i < RB; ++i)
#pragma unroll
            for (int q = 0; q < NB; ++q) acc[i][q] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < AHEAD; ++c) {
            const int s = step_of(c);
            if (!first_batch)
#pragma unroll
                for (int i = 0; i < 2 * RB; ++i) xr[c][i] = *reinterpret_cast<const u32x4*>(xp[i] + s * 64);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int q = 0; q < NB; ++q) wf[c][h][q] = *reinterpret_cast<const bf16x8*>(wp[q] + static_cast<int64_t>(s) * 1024 + h * 512);
        }
        first_batch = false;
        for (int base = 0; base < own; base += AHEAD)
#pragma unroll
            for (int c = 0; c < AHEAD; ++c) {
#pragma unroll
                for (int i = 0; i < 2 * RB; ++i) *reinterpret_cast<u32x4*>(i & 1 ? put_odd + i * 1024 : put + i * 1024) = base + c < own ? xr[c][i] : u32x4{0u, 0u, 0u, 0u};
                const int s = step_of(base + c + AHEAD);
#pragma unroll
                for (int i = 0; i < 2 * RB; ++i) xr[c][i] = *reinterpret_cast<const u32x4*>(xp[i] + s * 64);
                bf16x8 xf[2][RB];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < RB; ++i) xf[h][i] = *reinterpret_cast<const bf16x8*>(get + i * 2048 + (((4 * h + kc) ^ (l16 >> 1)) << 4));
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int q = 0; q < NB; ++q)
#pragma unroll
                        for (int i = 0; i < RB; ++i) acc[i][q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[c][h][q], xf[h][i], acc[i][q], 0, 0, 0);
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int q = 0; q < NB; ++q) wf[c][h][q] = *reinterpret_cast<const bf16x8*>(wp[q] + static_cast<int64_t>(s) * 1024 + h * 512);
                __builtin_amdgcn_sched_barrier(0);
            }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < RB; ++i) {
#pragma unroll
            for (int q = 0; q < NB; ++q) sums[wave][q][lane] = acc[i][q];
            __syncthreads();
#pragma unroll
            for (int q = 0; q < NB; ++q)
                if (q == wave && q < units) {
                    f32x4 sum = sums[0][q][lane];
#pragma unroll
                    for (int v = 1; v < WAVES; ++v) sum += sums[v][q][lane];
                    const int row = 16 * i + l16, first = unit_pos[q] * per;
                    int at = -1;                                  // the row's first place of the adapter, and its weights
                    float w = 0.f;
                    if (row < rows)
                        for (int s = d.sel - 1; s >= 0; --s)
                            if (ids[row * d.sel + s] == unit_a[q]) { at = s; w += weights[row * d.sel + s]; }
                    if (!PLANNED) {
                        bf16_t* const to = reinterpret_cast<bf16_t*>(t) + (row * d.sel + at) * d.cols;
                        if (at >= 0) put_terms([&](int c) { return to + c; }, kc, unit_block[q], d.blocks, d.cols, w, sum);
                    } else if (row < place_rows) put_terms([&](int c) { return place(row0 + row, first + (c >> 4), c & 15); }, kc, unit_block[q], d.blocks, 0, w, sum, at >= 0);
                }
            __syncthreads();
        }
    }
    if (!PLANNED) return;
    const int all = (pos + 1) * per, filled = (all + 3) & ~3;     // whole steps
    if (filled > all && blockIdx.y == 0) zeros(all, filled - all);
    if (!lead) return;
    const int any = __syncthreads_or(bad != 0u);
    if (threadIdx.x == 0) {
        plan[0] = filled / 4;
        plan[1] = any;
        plan[2] = ids_at;
        for (int i = all; i < filled; ++i) { offsets[i] = last * d.stride * 2; plan[ids_at + i] = last; }
    }
}

// Places with their blocks of ranks, of all the 16 rows, up to which each has a workgroup: it fills the chip where rows name many adapters, and loads what the earlier places of its 16 rows load as well.  us, the
// whole call, a workgroup to a place (adapters_down_rows_kernel) / the other kernel: 40 rows, two of 64 adapters of rank 16 each, 3072 x 3072 (96 places) 21.9 / 29.0; 128 rows, two of eight, 2048 x 2048 (256) 14.3 / 15.9; 64 rows, one of
// four of rank 64, 3072 x 3072 (256) 16.6 / 16.2; 48 rows, two of six of rank 64 (384) 24.1 / 25.7; 820 rows, rank 16, 64 x 3072 (832) 18.7 / 12.6; 8704 rows, rank 64, 64 x 3072 (34816) 346 / 51
constexpr int64_t kDownPlaces = 512;
template <bool PLANNED, int RB, int NB, int WAVES>
void launch_down(regione_ctx* ctx, const DownCall& d, const DownTiles& tiles) {
    const int rows = PLANNED ? tiles.rows : 16 * RB, pieces = (d.m + rows - 1) / rows * ((rows + 16 * RB - 1) / (16 * RB));
    const int64_t most = static_cast<int64_t>(16 * RB) * d.sel < d.count ? static_cast<int64_t>(16 * RB) * d.sel : d.count, batches = (most * d.blocks + NB - 1) / NB;
    const int64_t room = pieces < 512 ? 512 / pieces : 1;
    hipLaunchKernelGGL((adapters_down_tiles_kernel<PLANNED, RB, NB, WAVES>), dim3(pieces, static_cast<unsigned>(batches < room ? batches : room)), dim3(WAVES * 64), 0, ctx->stream, d, tiles);
}
template <bool PLANNED> void launch_down(regione_ctx* ctx, const DownCall& d, const DownTiles& tiles) {
    // us, K 3072, a block of ranks to a workgroup / four / four of 32 rows: 820 rows, rank 16 7.0 / 8.8 / 11.1, rank 64 9.1 / 10.5 / 12.5; 2048 rows, rank 16 7.2 / 8.6 / 10.2, rank 64
    // 10.0 / 10.5 / 12.2; 4096 rows, rank 16 9.2 / 9.9 / 11.4, rank 64 19.0 / 11.9 / 14.0; 6144 rows, rank 64 29.4 / 17.3 / 14.8; 8704 rows, rank 64 45 / 23.6 / 21.6; 16384 rows 61 / 31 / 24
    // A block of ranks to a workgroup only where all that 16 rows may name have one: 1711 rows, any of 23 adapters of rank 9, K 320, four workgroups to 16 rows, 19.8 us against 13.1
    const int64_t pieces = (d.m + 15) / 16, most = static_cast<int64_t>(16) * d.sel < d.count ? static_cast<int64_t>(16) * d.sel : d.count;
    if (pieces * most * d.blocks <= kDownPlaces) launch_down<PLANNED, 1, 1, 8>(ctx, d, tiles);
    else if (pieces <= 256) launch_down<PLANNED, 1, 4, 4>(ctx, d, tiles);
    else launch_down<PLANNED, 2, 4, 4>(ctx, d, tiles);
}
int down_tiles(regione_ctx* ctx, const DownCall& d, const DownTiles& tiles) {
    launch_down<true>(ctx, d, tiles);
    RG_LAUNCH_CHECK();
    return REGIONE_OK;
}
int down_rows(regione_ctx* ctx, const DownCall& d) {
    const int64_t tiles = (d.m + 15) / 16, places = static_cast<int64_t>(d.m < 16 ? d.m : 16) * d.sel * d.blocks;
    if (tiles * places <= kDownPlaces) {
        hipLaunchKernelGGL(adapters_down_rows_kernel, dim3(static_cast<unsigned>(tiles), static_cast<unsigned>(places)), dim3(kDownWaves * 64), 0, ctx->stream, d);
    } else {
        launch_down<false>(ctx, d, DownTiles{});
    }
    RG_LAUNCH_CHECK();
    return REGIONE_OK;
}

}  // namespace

extern "C" int64_t regione_packed_adapter_elems(int32_t n, int32_t k, int32_t rank) {
    if (n <= 0 || k <= 0 || rank <= 0) return 0;
    return adapter_elems(n, k, (rank + 15) / 16);
}

static int adapter_shape(const char* who, int n, int k, int rank) {
    if (n <= 0 || k <= 0 || rank <= 0) RG_FAIL(REGIONE_ERR_INVALID_ARG, "%s: n=%d k=%d rank=%d", who, n, k, rank);
    if (k % 64 || k > (1 << 20) || n > (1 << 24)) RG_FAIL(REGIONE_ERR_BAD_SHAPE, "%s: n=%d (at most 2^24), k=%d must be a multiple of 64, at most 2^20", who, n, k);
    if (rank > kMostRank) RG_FAIL(REGIONE_ERR_UNSUPPORTED, "%s: rank %d (at most %d)", who, rank, kMostRank);
    return REGIONE_OK;
}

extern "C" int regione_pack_adapter(regione_ctx* ctx, const void* a, const void* b, int32_t n, int32_t k, int32_t rank, void* packed) {
    if (!ctx) RG_FAIL(REGIONE_ERR_INVALID_ARG, "pack_adapter: null context");
    if (ctx->f32) RG_FAIL(REGIONE_ERR_UNSUPPORTED, "pack_adapter: belongs to bf16 contexts");
    if (int rc = adapter_shape("pack_adapter", n, k, rank)) return rc;
    if (!a || !b || !packed) RG_FAIL(REGIONE_ERR_INVALID_ARG, "pack_adapter: null tensor");
    if (!rg_aligned16(packed)) RG_FAIL(REGIONE_ERR_INVALID_ARG, "pack_adapter: unaligned tensor");
    const int blocks = (rank + 15) / 16;
    int64_t grid = (adapter_elems(n, k, blocks) + kThreads - 1) / kThreads;
    if (grid > 256 * 32) grid = 256 * 32;
    ProfScope prof(ctx, REGIONE_PROF_ROWS);
    hipLaunchKernelGGL(pack_adapter_kernel, dim3(static_cast<unsigned>(grid)), dim3(kThreads), 0, ctx->stream, static_cast<const bf16_t*>(a), static_cast<const bf16_t*>(b), n, k, rank, blocks,
                       static_cast<bf16_t*>(packed));
    RG_LAUNCH_CHECK();
    grid = (static_cast<int64_t>(n) + kThreads - 1) / kThreads;
    hipLaunchKernelGGL(pack_adapter_bad_kernel, dim3(static_cast<unsigned>(grid < 256 * 32 ? grid : 256 * 32)), dim3(kThreads), 0, ctx->stream, static_cast<const bf16_t*>(b), n, rank,
                       reinterpret_cast<uint32_t*>(static_cast<bf16_t*>(packed) + a_elems(k, blocks) + b_elems(n, blocks)));
    RG_LAUNCH_CHECK();
    return REGIONE_OK;
}

extern "C" int regione_linear_adapters(regione_ctx* ctx, const void* x, const void* w_packed, const float* b_opt, const void* adapters_packed, const int32_t* adapter, const float* weight_opt,
                                       int32_t n_adapters, int32_t n_sel, int32_t rank, int32_t m, int32_t n, int32_t k, int32_t act, int32_t out_dtype, void* y) {
    if (!ctx) RG_FAIL(REGIONE_ERR_INVALID_ARG, "linear_adapters: null context");
    if (ctx->f32) RG_FAIL(REGIONE_ERR_UNSUPPORTED, "linear_adapters: belongs to bf16 contexts");
    if (m < 0) RG_FAIL(REGIONE_ERR_INVALID_ARG, "linear_adapters: m=%d", m);
    if (int rc = adapter_shape("linear_adapters", n, k, rank)) return rc;
    if (act != REGIONE_ACT_NONE && act != REGIONE_ACT_GELU_TANH) RG_FAIL(REGIONE_ERR_INVALID_ARG, "linear_adapters: bad act %d", act);
    if (out_dtype != REGIONE_BF16 && out_dtype != REGIONE_FP32) RG_FAIL(REGIONE_ERR_INVALID_ARG, "linear_adapters: bad out_dtype %d", out_dtype);
    if (n_adapters <= 0 || n_sel <= 0) RG_FAIL(REGIONE_ERR_INVALID_ARG, "linear_adapters: n_adapters=%d n_sel=%d", n_adapters, n_sel);
    if (n_adapters > kMostAdapters || n_sel > kMostSel) RG_FAIL(REGIONE_ERR_UNSUPPORTED, "linear_adapters: %d adapters (at most %d), %d per row (%d)", n_adapters, kMostAdapters, n_sel, kMostSel);
    if (m > (1 << 24)) RG_FAIL(REGIONE_ERR_BAD_SHAPE, "linear_adapters: m=%d (at most 2^24)", m);
    if (m == 0) return REGIONE_OK;
    if (!x || !w_packed || !adapters_packed || !adapter || !y) RG_FAIL(REGIONE_ERR_INVALID_ARG, "linear_adapters: null tensor");
    if (!rg_aligned16(x) || !rg_aligned16(w_packed) || !rg_aligned16(adapters_packed)) RG_FAIL(REGIONE_ERR_INVALID_ARG, "linear_adapters: operands must be 16-byte aligned");

    const bool y_f32 = out_dtype == REGIONE_FP32;
    const int blocks = (rank + 15) / 16, cols = (kTerms * blocks * 16 + 31) & ~31;
    const size_t all = ctx->gemm_part_bytes, room = all / 2 < kTermBytes ? (all / 2) & ~size_t{255} : kTermBytes;      // (a context without a workspace has none)
    // the inner products lie at the workspace's end, the sums of K splits in the rest of it
    char* const end = reinterpret_cast<char*>(ctx->gemm_part) + all - room;
    ctx->gemm_part_bytes = all - room;
    AdapterTiles tiles = rg_adapter_tiles(ctx, m, n, k);
    // the most that a tile can name: every row another adapter
    const int64_t named = static_cast<int64_t>(tiles.rows) * n_sel < n_adapters ? static_cast<int64_t>(tiles.rows) * n_sel : n_adapters, tile_steps = (named * kTerms * blocks + 3) / 4;
    const int64_t tile_bytes = tile_steps * tiles.rows * 128, plan_words = 4 + 12 * tile_steps, plan_bytes = plan_words * 4, fits = static_cast<int64_t>(room) / (tile_bytes + plan_bytes), m_tiles = (m + tiles.rows - 1) / tiles.rows;
    // More than fits goes through in passes of whole tiles; a tile that does not fit leaves the call to the kernel of 16 rows, which reads what its rows name and no more.  us, passes / that kernel, 500 adapters,
    // 4096 x 2048: 8192 rows, rank 16, a request every 64 rows 206 / 772, every row any adapter 1290 / 1210; 2048 rows, rank 64 78 / 266 and 746 / 599
    int64_t chunk = m;
    if (tiles.tile && fits < m_tiles) {
        if (fits > 0) {
            chunk = fits * tiles.rows;
            tiles.splits = 1;
        } else {
            tiles = {0, 1, 16};
        }
    }
    const size_t row_bytes = static_cast<size_t>(n_sel) * cols * 2;
    if (!tiles.tile) {
        const int64_t most = static_cast<int64_t>(room / row_bytes) & ~int64_t{15};
        chunk = m < most ? m : most;
    }
    int rc = REGIONE_OK;
    if (chunk <= 0) {
        rc = REGIONE_ERR_WORKSPACE;
        regione_set_error("linear_adapters: the inner products of a row, %zu bytes, need a workspace", row_bytes);
    }
    ProfScope prof(ctx, REGIONE_PROF_GEMM);
    for (int64_t r0 = 0; r0 < m && rc == REGIONE_OK; r0 += chunk) {
        const int rows = static_cast<int>(m - r0 < chunk ? m - r0 : chunk);
        DownCall d = {static_cast<const bf16_t*>(x) + r0 * k, static_cast<const bf16_t*>(adapters_packed), adapter_elems(n, k, blocks), adapter + r0 * n_sel, weight_opt ? weight_opt + r0 * n_sel : nullptr,
                      n_adapters, n_sel, rows, k, blocks, cols, reinterpret_cast<bf16_t*>(end)};
        GemmEpilogue ep = {};
        ep.kind = EPI_PLAIN; ep.bias = b_opt; ep.act = act; ep.act_from = 0;
        ep.y = static_cast<char*>(y) + r0 * n * (y_f32 ? 4 : 2); ep.ldy = n; ep.y_f32 = y_f32;
        const bf16_t* const b = d.packed + a_elems(k, blocks);
        ep.adapters = {d.t, d.which, b, reinterpret_cast<const uint32_t*>(b + b_elems(n, blocks)), d.stride, n_sel, n_adapters, cols, blocks, nullptr, 0, 0};
        if (tiles.tile) {
            const int64_t parts = (rows + tiles.rows - 1) / tiles.rows;
            DownTiles at = {tiles.rows, static_cast<int>(plan_words), tile_bytes / 2, reinterpret_cast<int32_t*>(end + parts * tile_bytes), a_elems(k, blocks) + b_elems(n, blocks) + 2 * ((static_cast<int64_t>(n) + 31) / 32)};
            ep.adapters.plan = at.plan; ep.adapters.plan_pitch = at.plan_pitch; ep.adapters.tile_elems = at.tile_elems;
            rc = down_tiles(ctx, d, at);
        } else {
            rc = down_rows(ctx, d);
        }
        if (rc == REGIONE_OK) rc = rg_gemm_adapters(ctx, tiles, d.x, k, w_packed, rows, n, k, ep);
    }
    ctx->gemm_part_bytes = all;
    return rc;
}
