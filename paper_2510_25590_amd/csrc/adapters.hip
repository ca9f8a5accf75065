// Low-rank adapters of many requests beside a shared projection: packing, and the inner products of every row with its adapters' A.  What they bring to the result is added at the end
// of the projection's tiles (gemm_adapters.h).
#include "gemm_adapters.h"

namespace {

constexpr int kThreads = 256;
constexpr int kMostRank = 256, kMostSel = 32, kMostAdapters = 1 << 16;
constexpr size_t kTermBytes = size_t{32} << 20;              // of the inner products of the rows that go through at a time

// A packed adapter: A in fragments of 16 ranks x 32 inputs, 64 lanes x 8 values, lane l holding A[16 * (block) + l % 16][32 * step + 8 * (l / 16) .. +8]; behind it B as regione_pack_weight
// lays out a weight [n, rank rounded up to 16].
__host__ __device__ __forceinline__ int64_t a_elems(int k, int blocks) { return static_cast<int64_t>(blocks) * 16 * k; }
__host__ __device__ __forceinline__ int64_t adapter_elems(int n, int k, int blocks) { return a_elems(k, blocks) + (static_cast<int64_t>(n) + 31) / 32 * 32 * blocks * 16; }

__global__ void __launch_bounds__(kThreads)
pack_adapter_kernel(const bf16_t* __restrict__ a, const bf16_t* __restrict__ b, int n, int k, int rank, int blocks, bf16_t* __restrict__ packed) {
    const int64_t a_count = a_elems(k, blocks), count = adapter_elems(n, k, blocks), stride = static_cast<int64_t>(gridDim.x) * kThreads;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < count; i += stride) {
        bf16_t v = 0;
        if (i < a_count) {
            const int e = static_cast<int>(i & 7), lane = static_cast<int>(i >> 3) & 63;
            const int64_t f = i >> 9;
            const int block = static_cast<int>(f / (k >> 5)), step = static_cast<int>(f % (k >> 5));
            const int r = 16 * block + (lane & 15);
            if (r < rank) v = a[static_cast<int64_t>(r) * k + 32 * step + 8 * (lane >> 4) + e];
        } else {
            const int64_t at = i - a_count;
            const int e = static_cast<int>(at & 7), lane = static_cast<int>(at >> 3) & 63;
            const int64_t f = at >> 9;
            const int block = static_cast<int>(f % blocks);
            const int64_t col = f / blocks * 32 + (lane & 31);
            const int r = 16 * block + 8 * (lane >> 5) + e;
            if (col < n && r < rank) v = b[col * rank + r];
        }
        packed[i] = v;
    }
}

// t[row, s] = weight[row, s] * x[row] A_a^T, a = which[row, s], as `terms` bf16 values that add up to it: the value rounded, what is left of it rounded, and so on (2^-9, 2^-17, 2^-25
// relative).  One rounding would be as large as that of a bf16 result, and larger where the projection and the adapter cancel.
// A workgroup owns 16 * RB rows and goes through the blocks of 16 ranks of their distinct adapters, NB at a time; its eight waves split K and meet in LDS, where the sums are formed in wave order.
// Workgroups of one row tile (blockIdx.y) take turns at the batches.
constexpr int kDownWaves = 8, kDownAhead = 4;
template <int RB, int NB>
__global__ void __launch_bounds__(kDownWaves * 64)
adapters_down_kernel(const bf16_t* __restrict__ x, const bf16_t* __restrict__ packed, int64_t stride, const int32_t* __restrict__ which, const float* __restrict__ weight, int count, int sel,
                     int m, int k, int blocks, int terms, int cols, bf16_t* __restrict__ t) {
    constexpr int ROWS = 16 * RB, F = RB * NB;
    static_assert(F <= kDownWaves, "a wave per fragment at the end");
    __shared__ int32_t ids[ROWS * kMostSel];
    __shared__ __attribute__((aligned(16))) f32x4 sums[kDownWaves - 1][F][64];     // (a wave's own fragment stays in its registers)
    const int lane = threadIdx.x & 63, l16 = lane & 15, kc = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int m0 = blockIdx.x * ROWS, rows = m - m0 < ROWS ? m - m0 : ROWS, entries = rows * sel;
    for (int i = threadIdx.x; i < entries; i += kDownWaves * 64) {
        const int id = which[static_cast<int64_t>(m0) * sel + i];
        ids[i] = id >= 0 && id < count ? id : kNoAdapter;
    }
    __syncthreads();
    const int steps = k >> 5, per = (steps + kDownWaves - 1) / kDownWaves;
    const int s0 = wave * per, s1 = s0 + per < steps ? s0 + per : steps;
    const bf16_t* xp[RB];
#pragma unroll
    for (int i = 0; i < RB; ++i) {
        int row = 16 * i + l16;
        row = row < rows ? row : rows - 1;                        // rows past the end repeat the last one
        xp[i] = x + static_cast<int64_t>(m0 + row) * k + 8 * kc;
    }
    int a = -1, block = blocks;
    for (unsigned batch = 0;; ++batch) {
        int unit_a[NB], unit_block[NB], units = 0;
#pragma unroll
        for (int q = 0; q < NB; ++q) {
            if (block == blocks && a != kNoAdapter) {             // the next adapter: the smallest above the last one
                int next = kNoAdapter;
                for (int i = lane; i < entries; i += 64) {
                    const int id = ids[i];
                    next = id > a && id < next ? id : next;
                }
                next = lanes16_min(next);
                const int n0 = __builtin_amdgcn_readlane(next, 0), n1 = __builtin_amdgcn_readlane(next, 16), n2 = __builtin_amdgcn_readlane(next, 32), n3 = __builtin_amdgcn_readlane(next, 48);
                const int lo = n0 < n1 ? n0 : n1, hi = n2 < n3 ? n2 : n3;
                a = lo < hi ? lo : hi;
                block = 0;
            }
            unit_a[q] = a;
            unit_block[q] = block;
            if (a != kNoAdapter) { ++units; ++block; }
        }
        if (units == 0) return;
        if (batch % gridDim.y != blockIdx.y) continue;
        const bf16_t* wp[NB];
#pragma unroll
        for (int q = 0; q < NB; ++q) wp[q] = packed + static_cast<int64_t>(q < units ? unit_a[q] : unit_a[0]) * stride + static_cast<int64_t>(q < units ? unit_block[q] : unit_block[0]) * steps * 512 + lane * 8;
        f32x4 acc[RB][NB];
#pragma unroll
        for (int i = 0; i < RB; ++i)
#pragma unroll
            for (int q = 0; q < NB; ++q) acc[i][q] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int base = s0; base < s1; base += kDownAhead) {
            bf16x8 xf[kDownAhead][RB], wf[kDownAhead][NB];
#pragma unroll
            for (int c = 0; c < kDownAhead; ++c)
                if (base + c < s1) {
#pragma unroll
                    for (int i = 0; i < RB; ++i) xf[c][i] = *reinterpret_cast<const bf16x8*>(xp[i] + (base + c) * 32);
#pragma unroll
                    for (int q = 0; q < NB; ++q)
                        if (q < units) wf[c][q] = *reinterpret_cast<const bf16x8*>(wp[q] + static_cast<int64_t>(base + c) * 512);
                }
#pragma unroll
            for (int c = 0; c < kDownAhead; ++c)
                if (base + c < s1) {
#pragma unroll
                    for (int q = 0; q < NB; ++q)
                        if (q < units)
#pragma unroll
                            for (int i = 0; i < RB; ++i) acc[i][q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[c][q], xf[c][i], acc[i][q], 0, 0, 0);
                }
        }
        f32x4 own = f32x4{0.f, 0.f, 0.f, 0.f};
        int own_a = kNoAdapter, own_block = 0;
#pragma unroll
        for (int f = 0; f < F; ++f) {
            if (f == wave) {
                own = acc[f / NB][f % NB];
                if (f % NB < units) { own_a = unit_a[f % NB]; own_block = unit_block[f % NB]; }
            } else {
                sums[wave < f ? wave : wave - 1][f][lane] = acc[f / NB][f % NB];
            }
        }
        __syncthreads();
        if (own_a != kNoAdapter) {
            f32x4 sum = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < kDownWaves; ++w) {
                if (w == wave) sum += own;
                else sum += sums[w < wave ? w : w - 1][wave][lane];
            }
            const int row = 16 * (wave / NB) + l16;
            if (row < rows)
                for (int s = 0; s < sel; ++s) {
                    if (ids[row * sel + s] != own_a) continue;
                    const int64_t entry = static_cast<int64_t>(m0 + row) * sel + s;
                    bf16_t* const to = t + entry * cols + 16 * own_block + 4 * kc;
                    const float w = weight ? weight[entry] : 1.f;
                    float left[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) left[e] = w * sum[e];
                    for (int p = 0; p < terms; ++p) {
                        bf16_t v[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            v[e] = f32_to_bf16(left[e]);
                            const float r = bf16_to_f32(v[e]);
                            left[e] = __builtin_fabsf(r) < INFINITY ? left[e] - r : 0.f;       // (what is not finite is one term)
                        }
                        *reinterpret_cast<uint2*>(to + p * blocks * 16) = make_uint2(v[0] | static_cast<unsigned>(v[1]) << 16, v[2] | static_cast<unsigned>(v[3]) << 16);
                    }
                    if (own_block == blocks - 1 && cols > terms * blocks * 16) *reinterpret_cast<uint2*>(t + entry * cols + terms * blocks * 16 + 4 * kc) = make_uint2(0u, 0u);
                }
        }
        __syncthreads();
    }
}

struct DownCall { const bf16_t* x; const bf16_t* packed; int64_t stride; const int32_t* which; const float* weight; int count, sel, m, k, blocks, terms, cols; bf16_t* t; };
template <int RB, int NB>
int launch_down(regione_ctx* ctx, const DownCall& d) {
    const int tiles = (d.m + 16 * RB - 1) / (16 * RB);
    const int64_t most = static_cast<int64_t>(16 * RB) * d.sel < d.count ? static_cast<int64_t>(16 * RB) * d.sel : d.count;      // adapters of a tile
    const int64_t batches = (most * d.blocks + NB - 1) / NB;
    int64_t y = (512 + tiles - 1) / tiles;
    y = y < batches ? y : batches;
    hipLaunchKernelGGL((adapters_down_kernel<RB, NB>), dim3(static_cast<unsigned>(tiles), static_cast<unsigned>(y)), dim3(kDownWaves * 64), 0, ctx->stream,
                       d.x, d.packed, d.stride, d.which, d.weight, d.count, d.sel, d.m, d.k, d.blocks, d.terms, d.cols, d.t);
    RG_LAUNCH_CHECK();
    return REGIONE_OK;
}
int down(regione_ctx* ctx, const DownCall& d) {
    if (d.m <= 512) return launch_down<1, 1>(ctx, d);
    if (d.m <= 4096) return launch_down<1, 4>(ctx, d);
    return launch_down<2, 4>(ctx, d);
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
    const int blocks = (rank + 15) / 16, terms = y_f32 ? 3 : 2, cols = (terms * blocks * 16 + 31) & ~31;
    const size_t row_bytes = static_cast<size_t>(n_sel) * cols * 2;
    int64_t most = static_cast<int64_t>(kTermBytes / row_bytes) & ~int64_t{255};             // (at least 512: 32 adapters of rank 256 in three terms)
    const int64_t chunk = m < most ? m : most;
    const size_t bytes = (static_cast<size_t>(chunk) * row_bytes + 255) & ~size_t{255}, all = ctx->gemm_part_bytes;
    if (bytes > all) RG_FAIL(REGIONE_ERR_WORKSPACE, "linear_adapters: %zu bytes of inner products exceed the workspace of %zu", bytes, all);
    ProfScope prof(ctx, REGIONE_PROF_GEMM);
    // the inner products lie at the workspace's end, the sums of K splits in the rest of it
    bf16_t* const t = reinterpret_cast<bf16_t*>(reinterpret_cast<char*>(ctx->gemm_part) + all - bytes);
    ctx->gemm_part_bytes = all - bytes;
    int rc = REGIONE_OK;
    for (int64_t r0 = 0; r0 < m && rc == REGIONE_OK; r0 += chunk) {
        const int rows = static_cast<int>(m - r0 < chunk ? m - r0 : chunk);
        DownCall d = {static_cast<const bf16_t*>(x) + r0 * k, static_cast<const bf16_t*>(adapters_packed), adapter_elems(n, k, blocks), adapter + r0 * n_sel, weight_opt ? weight_opt + r0 * n_sel : nullptr,
                      n_adapters, n_sel, rows, k, blocks, terms, cols, t};
        rc = down(ctx, d);
        if (rc != REGIONE_OK) break;
        GemmEpilogue ep = {};
        ep.kind = EPI_PLAIN; ep.bias = b_opt; ep.act = act; ep.act_from = 0;
        ep.y = static_cast<char*>(y) + r0 * n * (y_f32 ? 4 : 2); ep.ldy = n; ep.y_f32 = y_f32;
        ep.adapters = {t, d.which, d.packed + a_elems(k, blocks), d.stride, n_sel, n_adapters, cols, blocks};
        rc = rg_gemm_adapters(ctx, d.x, k, w_packed, rows, n, k, ep);
    }
    ctx->gemm_part_bytes = all;
    return rc;
}
