// Products of microscaled 4-bit operands, and products over groups of rows with weights of their own: which kernel a call gets, and the entry points.
#include "gemm_mx.h"
#include <math.h>

namespace {

template <int FMT, int KW, int CF>
int launch_small(regione_ctx* ctx, const MxOperands& p, const GemmEpilogue& ep) {
    constexpr int COLS = 16 * CF * kMxSmallWaves / KW;
    const int64_t tiles = mx_most_row_tiles(p, kMxSmallRows) * ((p.n + COLS - 1) / COLS);
    if (tiles >= (int64_t{1} << 32) / (kMxSmallWaves * 64)) RG_FAIL(REGIONE_ERR_UNSUPPORTED, "linear: a result of %d x %d", p.m, p.n);
    hipLaunchKernelGGL((gemm_mx_small_kernel<FMT, KW, CF>), dim3(static_cast<unsigned>(tiles)), dim3(kMxSmallWaves * 64), 0, ctx->stream, p, ep);
    RG_LAUNCH_CHECK();
    return REGIONE_OK;
}
template <int FMT>
int launch_small(regione_ctx* ctx, int code, const MxOperands& p, const GemmEpilogue& ep) {
    switch (code) {
        case 1: return launch_small<FMT, 1, 2>(ctx, p, ep);
        case 2: return launch_small<FMT, 2, 2>(ctx, p, ep);
        case 4: return launch_small<FMT, 4, 2>(ctx, p, ep);
        case 8: return launch_small<FMT, 8, 2>(ctx, p, ep);
    }
    return launch_small<FMT, 8, 1>(ctx, p, ep);
}

// ---- which kernel a product gets
//
// A plan's time is estimated as a start, whole and partial loads of the chip by workgroups (a fixed part and a part per step of K, which grow with the workgroups that share a CU, and the
// activation, which they do one after the other), what the weights take (the root of both squares: the longer of them, and a little for the other), and the results' way out; a K split
// adds its sums' way out and back, the kernel of 16 rows what its repeated reading of the weights takes.  The host does not know the groups' sizes: they are taken as random (exponentially distributed), a group of mean length s then has
// 1 / (1 - exp(-R / s)) tiles of R rows.  All constants are fitted to every tile, K split and number of waves of 1978 products in 4 bits and 1312 in bf16 (1-16384 rows, 64-14400 columns,
// K 256-16000, up to 64 groups, equal and random, with and without activation): over 990 / 657 others the choice is 1.9 / 2.3 % behind the best plan measured on average, 9 / 11 % in the
// twentieth of them where it is furthest, 35 % at most (groups whose sizes are far from the assumed ones).
// The products of the fit found their weights in the Infinity Cache (the 11 to 12 TB/s below), where a program that goes through many weights finds them in HBM.  Of 42 other products there the
// choice was 0.8 % behind the best plan on average without groups, 25 % at most (205 x 3072 x 12288), and 9 % with groups, 40 % at most (two of 64 rows x 12288 x 3072 in bf16: 43.2 us, 64 x 128 tiles
// 30.9); with weights in the cache 0.5 % and 7 %, 29 % at most (32 groups of three rows: equal groups are not what the estimate assumes).
// us, another tile / the choice, weights in the cache: 820 x 12288 x 3072 224 x 256 23.9 / 192 x 256 20.7; 820 x 3072 x 12288 192 x 256 48.7 / 96 x 128 22.3; 128 x 3072 x 12288 unsplit 11.9 / two K
// splits 9.9; 8704 x 12288 x 3072 128 x 128 197 / 128 x 256 165; one row x 9216 x 3072 all waves over columns 9.3 / eight over K 5.3 (four 5.2).
// Left out, a kernel would cost the products that it is best for: the one of 16 rows with one, two, four and eight waves over K 32, 7, 18 and 48 %, with 16 columns 49 %.
struct MxPlan { int tile, splits; };      // tile 1, 2, 4, 8: the kernel of 16 rows and 32 columns per wave with as many waves over K; 9: with eight, 16 columns
struct MxTileCost { int code, per_cu; double fixed, step, more; };               // us, us per step, and what each further workgroup of a CU adds to the latter (as a share)
struct MxSmallCost { int code; double fixed, step, work; };                       // us and us per step of a wave, per load of the chip; us per 1e5 steps of columns
struct MxCosts { MxTileCost tile[11]; MxSmallCost small[5]; double start, weights, out, gelu; }; // us, bytes of weights per us, results per us, us per 100 kB of a tile's sums
constexpr MxCosts kMxCosts[2] = {
    {{{72, 1, 2.82, 0.922, 0.000}, {62, 1, 2.37, 0.799, 0.000}, {52, 1, 2.46, 0.597, 0.000}, {42, 2, 1.36, 0.505, 1.118}, {32, 2, 0.90, 0.434, 1.148}, {51, 2, 0.98, 0.384, 1.119},
      {41, 2, 0.82, 0.295, 1.348}, {31, 3, 0.57, 0.243, 1.305}, {22, 2, 0.47, 0.344, 1.268}, {21, 3, 0.30, 0.202, 1.312}, {11, 3, 0.45, 0.164, 1.420}},
     {{1, 0.06, 0.317, 0.83}, {2, 0.23, 0.317, 0.74}, {4, 0.43, 0.282, 0.74}, {8, 0.70, 0.222, 0.71}, {9, 0.72, 0.186, 0.37}}, 3.47, 11.55e6, 1.00e6, 0.70},
    {{{72, 1, 2.94, 1.199, 0.000}, {62, 1, 2.28, 1.017, 0.000}, {52, 1, 2.32, 0.802, 0.000}, {42, 2, 1.30, 0.622, 1.153}, {32, 2, 1.00, 0.520, 1.200}, {51, 2, 1.02, 0.458, 1.404},
      {41, 2, 0.83, 0.342, 1.728}, {31, 3, 0.69, 0.283, 1.504}, {22, 2, 0.75, 0.394, 1.376}, {21, 3, 0.54, 0.214, 1.592}, {11, 3, 0.76, 0.174, 1.682}},
     {{1, 0.00, 0.499, 0.79}, {2, 0.25, 0.480, 0.77}, {4, 0.45, 0.421, 0.72}, {8, 0.61, 0.325, 0.83}, {9, 1.01, 0.096, 0.72}}, 3.59, 10.78e6, 1.52e6, 0.65}};

double row_tiles_expected(const MxOperands& p, int R) {
    const double most = static_cast<double>(mx_most_row_tiles(p, R)), g = p.n_groups < p.m ? p.n_groups : p.m;
    if (!p.offsets) return most;
    const double random = ceil(g / (1.0 - exp(-R * g / p.m)));
    return random < most ? random : most;
}
MxPlan choose(int fmt, const MxOperands& p, int act, size_t part_bytes) {
    const MxCosts& c = kMxCosts[fmt];
    const int groups = p.offsets ? p.n_groups : 1;
    const double weights = static_cast<double>(p.m < groups ? p.m : groups) * p.n * p.steps * (fmt == MX_FP4 ? 136.0 : 128.0) / c.weights;
    MxPlan best = {42, 1};
    double best_us = 1e30;
    auto consider = [&](int tile, int splits, double us) { if (us < best_us) { best_us = us; best = {tile, splits}; } };
    for (const MxTileCost& t : c.tile) {
        const int R = 32 * (t.code / 10), C = 128 * (t.code % 10);
        const double columns = (p.n + C - 1) / C, units = row_tiles_expected(p, R) * columns;
        const int64_t most = mx_most_row_tiles(p, R) * static_cast<int64_t>(columns);
        const double tile_kb = R * C * 4.0 / 1e3, gelu = act == REGIONE_ACT_GELU_TANH ? c.gelu * tile_kb / 100.0 : 0.0;
        for (int s : {1, 2, 3, 4, 6, 8}) {
            if (s > 1) {
                if (p.offsets || units * s > 640 || p.steps < 2 * s) break;
                if (most > kMaxSplitTiles || static_cast<size_t>(most) * s * R * C * sizeof(float) > part_bytes) break;
                const int per = (p.steps + s - 1) / s;
                if ((p.steps + per - 1) / per != s) continue;     // another split count in disguise
            }
            const int per = (p.steps + s - 1) / s;
            const double loads = floor(units * s / (256.0 * t.per_cu)), rest = units * s - loads * 256.0 * t.per_cu;
            auto load = [&](double shared) { return t.fixed + per * t.step * (1.0 + t.more * (shared - 1.0)) + gelu * shared; };
            double us = loads * load(t.per_cu) + (rest > 0.0 ? load(ceil(rest / 256.0)) : 0.0);
            us = sqrt(us * us + weights * weights) + static_cast<double>(p.m) * p.n / c.out;
            if (s > 1) us += 0.91 + 0.288 * units * s * tile_kb / 1e3 + 0.0187 * s * tile_kb;
            consider(t.code, s, c.start + us);
        }
    }
    if (p.m > 48 * static_cast<int64_t>(groups)) return best;     // (more than what the kernel of 16 rows was fitted to)
    for (const MxSmallCost& t : c.small) {
        const int waves = t.code == 9 ? 8 : t.code, C = t.code == 9 ? 16 : 32 * kMxSmallWaves / waves, slots = t.code == 9 ? 256 : 512;
        const double units = row_tiles_expected(p, kMxSmallRows) * ((p.n + C - 1) / C);
        const double us = ceil(units / slots) * (t.fixed + t.step * ((p.steps + waves - 1) / waves)) + t.work * 1e-5 * units * p.steps * C;
        consider(t.code, 1, c.start + sqrt(us * us + weights * weights));
    }
    return best;
}
// remembered per context like the other products' plans (plan_gemm in gemm.hip)
MxPlan plan(regione_ctx* ctx, int fmt, const MxOperands& p, int act) {
    const int groups = p.offsets ? p.n_groups : 0;
    const uint32_t h = (static_cast<uint32_t>(p.m) * 2654435761u) ^ (static_cast<uint32_t>(p.n) * 2246822519u) ^ (static_cast<uint32_t>(p.row_bytes) * 3266489917u) ^ (static_cast<uint32_t>(groups) * 668265263u);
    GemmPlanSlot& slot = ctx->mx_plans[(h >> 16) % kGemmPlanSlots];
    const int kind = 4 * groups + 2 * act + fmt;
    if (slot.m == p.m && slot.n == p.n && slot.k == p.row_bytes && slot.kind == kind && slot.part_bytes == ctx->gemm_part_bytes) return {slot.tile, slot.splits};
    const MxPlan best = choose(fmt, p, act, ctx->gemm_part_bytes);
    slot = {p.m, p.n, p.row_bytes, kind, best.tile, best.splits, ctx->gemm_part_bytes};
    return best;
}

int launch(regione_ctx* ctx, int fmt, const MxOperands& p, const GemmEpilogue& ep) {
    ProfScope prof(ctx, REGIONE_PROF_GEMM);
    MxPlan to = plan(ctx, fmt, p, ep.act);
    if (ctx->mx_force_tile) to = {ctx->mx_force_tile, 1};
    if (ctx->mx_force_splits > 0 && !p.offsets) to.splits = ctx->mx_force_splits;
    if (to.tile < 10) return fmt == MX_FP4 ? launch_small<MX_FP4>(ctx, to.tile, p, ep) : launch_small<MX_BF16>(ctx, to.tile, p, ep);
    return fmt == MX_FP4 ? rg_mx_tile_4bit(ctx, to.tile, p, to.splits, ep) : rg_mx_tile_bf16(ctx, to.tile, p, to.splits, ep);
}

// What the three products have in common.  groups: offsets, use, n_groups and n_weights are looked at.
int linear(regione_ctx* ctx, const char* who, int fmt, bool groups, const void* x, const void* x_scale, const void* w_packed, const float* b_opt,
           const int32_t* offsets, const int32_t* use, int32_t n_groups, int32_t n_weights, int32_t m, int32_t n, int32_t k, int32_t act, int32_t out_dtype, void* y) {
    if (!ctx) RG_FAIL(REGIONE_ERR_INVALID_ARG, "%s: null context", who);
    if (ctx->f32) RG_FAIL(REGIONE_ERR_UNSUPPORTED, "%s: belongs to bf16 contexts", who);
    if (m < 0 || n <= 0 || k <= 0) RG_FAIL(REGIONE_ERR_INVALID_ARG, "%s: m=%d n=%d k=%d", who, m, n, k);
    if (act != REGIONE_ACT_NONE && act != REGIONE_ACT_GELU_TANH) RG_FAIL(REGIONE_ERR_INVALID_ARG, "%s: bad act %d", who, act);
    if (out_dtype != REGIONE_BF16 && out_dtype != REGIONE_FP32) RG_FAIL(REGIONE_ERR_INVALID_ARG, "%s: bad out_dtype %d", who, out_dtype);
    const int unit = fmt == MX_FP4 ? kMxBlock : 64;
    if (k % unit || k > kMxMostInputs) RG_FAIL(REGIONE_ERR_BAD_SHAPE, "%s: k=%d must be a multiple of %d, at most 2^20", who, k, unit);
    if (n > kMxMostFeatures || m > (1 << 24)) RG_FAIL(REGIONE_ERR_BAD_SHAPE, "%s: m=%d n=%d (at most 2^24)", who, m, n);
    if (groups && (n_groups < 0 || n_weights <= 0 || n_groups > (1 << 16) || (!use && n_groups > n_weights)))
        RG_FAIL(REGIONE_ERR_INVALID_ARG, "%s: %d groups (at most 65536), %d weights", who, n_groups, n_weights);
    if (m == 0 || (groups && n_groups == 0)) return REGIONE_OK;
    if (!x || (fmt == MX_FP4 && !x_scale) || !w_packed || !y || (groups && !offsets)) RG_FAIL(REGIONE_ERR_INVALID_ARG, "%s: null tensor", who);
    if (!rg_aligned16(x) || !rg_aligned16(x_scale) || !rg_aligned16(w_packed)) RG_FAIL(REGIONE_ERR_INVALID_ARG, "%s: operands must be 16-byte aligned", who);
    MxOperands p = {};
    p.a = static_cast<const uint8_t*>(x); p.a_scale = static_cast<const uint8_t*>(x_scale); p.w = static_cast<const uint8_t*>(w_packed);
    p.w_stride = fmt == MX_FP4 ? mx_packed_bytes(n, k) : 2 * regione_packed_weight_elems(n, k);
    if (groups) { p.offsets = offsets; p.use = use; p.n_groups = n_groups; p.n_weights = n_weights; }
    p.m = m; p.n = n; p.row_bytes = fmt == MX_FP4 ? k / 2 : 2 * k; p.steps = (p.row_bytes + 127) / 128;
    GemmEpilogue ep = {};
    ep.kind = EPI_PLAIN; ep.bias = b_opt; ep.act = act; ep.act_from = 0;
    ep.y = y; ep.ldy = n; ep.y_f32 = out_dtype == REGIONE_FP32;
    ep.vec_ok = n % 8 == 0 && rg_aligned16(y);
    return launch(ctx, fmt, p, ep);
}

}  // namespace

extern "C" int regione_linear_mxfp4(regione_ctx* ctx, const void* xq, const void* x_scale, const void* w_packed, const float* b_opt,
                                    int32_t m, int32_t n, int32_t k, int32_t act, int32_t out_dtype, void* y) {
    return linear(ctx, "linear_mxfp4", MX_FP4, false, xq, x_scale, w_packed, b_opt, nullptr, nullptr, 0, 1, m, n, k, act, out_dtype, y);
}

extern "C" int regione_linear_mxfp4_grouped(regione_ctx* ctx, const void* xq, const void* x_scale, const void* w_packed, const float* b_opt, const int32_t* group_offsets,
                                            const int32_t* group_weight_opt, int32_t n_groups, int32_t n_weights, int32_t m, int32_t n, int32_t k, int32_t act, int32_t out_dtype, void* y) {
    return linear(ctx, "linear_mxfp4_grouped", MX_FP4, true, xq, x_scale, w_packed, b_opt, group_offsets, group_weight_opt, n_groups, n_weights, m, n, k, act, out_dtype, y);
}

extern "C" int regione_linear_grouped(regione_ctx* ctx, const void* x, const void* w_packed, const float* b_opt, const int32_t* group_offsets,
                                      const int32_t* group_weight_opt, int32_t n_groups, int32_t n_weights, int32_t m, int32_t n, int32_t k, int32_t act, int32_t out_dtype, void* y) {
    return linear(ctx, "linear_grouped", MX_BF16, true, x, nullptr, w_packed, b_opt, group_offsets, group_weight_opt, n_groups, n_weights, m, n, k, act, out_dtype, y);
}

extern "C" int regione_tune_mx(regione_ctx* ctx, int32_t tile, int32_t k_splits) {
    if (!ctx) RG_FAIL(REGIONE_ERR_INVALID_ARG, "tune_mx: null context");
    bool known = tile == 0;
    for (int t : {1, 2, 4, 8, 9, 72, 62, 52, 42, 32, 51, 41, 31, 22, 21, 11}) known = known || t == tile;
    if (!known || k_splits < 0 || k_splits > 16) RG_FAIL(REGIONE_ERR_INVALID_ARG, "tune_mx: no tile %d, or k_splits=%d is not in 0..16", tile, k_splits);
    ctx->mx_force_tile = tile;
    ctx->mx_force_splits = k_splits;
    return REGIONE_OK;
}
