// Products of microscaled 4-bit operands, and products over groups of rows with weights of their own: which kernel a call gets, and the entry points.
#include "gemm_mx.h"

namespace {

template <int FMT, int KW>
int launch_small(regione_ctx* ctx, const MxOperands& p, const GemmEpilogue& ep) {
    constexpr int COLS = 32 * kMxSmallWaves / KW;
    const int64_t tiles = mx_most_row_tiles(p, kMxSmallRows) * ((p.n + COLS - 1) / COLS);
    if (tiles >= (int64_t{1} << 32) / (kMxSmallWaves * 64)) RG_FAIL(REGIONE_ERR_UNSUPPORTED, "linear: a result of %d x %d", p.m, p.n);
    hipLaunchKernelGGL((gemm_mx_small_kernel<FMT, KW>), dim3(static_cast<unsigned>(tiles)), dim3(kMxSmallWaves * 64), 0, ctx->stream, p, ep);
    RG_LAUNCH_CHECK();
    return REGIONE_OK;
}
template <int FMT>
int launch_small(regione_ctx* ctx, int waves, const MxOperands& p, const GemmEpilogue& ep) {
    return waves == 1 ? launch_small<FMT, 1>(ctx, p, ep) : waves == 2 ? launch_small<FMT, 2>(ctx, p, ep) : waves == 4 ? launch_small<FMT, 4>(ctx, p, ep) : launch_small<FMT, 8>(ctx, p, ep);
}

struct MxPlan { int tile, splits; };      // tile 1, 2, 4, 8: the kernel of 16 rows with as many waves over K

MxPlan choose(const MxOperands& p) {
    if (p.m <= 64) return {8, 1};
    return {82, 1};
}

int launch(regione_ctx* ctx, int fmt, const MxOperands& p, const GemmEpilogue& ep) {
    ProfScope prof(ctx, REGIONE_PROF_GEMM);
    MxPlan plan = choose(p);
    if (ctx->mx_force_tile) plan = {ctx->mx_force_tile, ctx->mx_force_splits > 0 && !p.offsets ? ctx->mx_force_splits : 1};
    if (plan.tile <= 8) return fmt == MX_FP4 ? launch_small<MX_FP4>(ctx, plan.tile, p, ep) : launch_small<MX_BF16>(ctx, plan.tile, p, ep);
    return fmt == MX_FP4 ? rg_mx_tile_4bit(ctx, plan.tile, p, plan.splits, ep) : rg_mx_tile_bf16(ctx, plan.tile, p, plan.splits, ep);
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
    if (k % unit || k > (1 << 20)) RG_FAIL(REGIONE_ERR_BAD_SHAPE, "%s: k=%d must be a multiple of %d, at most 2^20", who, k, unit);
    if (n > (1 << 24) || m > (1 << 24)) RG_FAIL(REGIONE_ERR_BAD_SHAPE, "%s: m=%d n=%d (at most 2^24)", who, m, n);
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
    for (int t : {1, 2, 4, 8, 82, 62, 42, 81, 41, 22, 21, 11}) known = known || t == tile;
    if (!known || k_splits < 0 || k_splits > 16) RG_FAIL(REGIONE_ERR_INVALID_ARG, "tune_mx: no tile %d, or k_splits=%d is not in 0..16", tile, k_splits);
    ctx->mx_force_tile = tile;
    ctx->mx_force_splits = k_splits;
    return REGIONE_OK;
}
