// The wide tiles of the two-group GEMM with low-rank adapters' K-steps behind the product's (gemm_adapters.h).
#include "gemm_launch.h"

#define RG_TILE_ADAPTERS(CODE, LAUNCH, ...) if (tile == CODE) return LAUNCH<__VA_ARGS__, EPI_ADAPTERS>(ctx, a, lda, wp, m, n, k, splits, ep);
int rg_gemm_tile_adapters(regione_ctx* ctx, int tile, const bf16_t* a, int lda, const bf16_t* wp, int m, int n, int k, int splits, const GemmEpilogue& ep) {
    RG_TILE_ADAPTERS(44, launch_pp, 4, 4)
    RG_TILE_ADAPTERS(64, launch_pp, 6, 4)
    RG_TILE_ADAPTERS(74, launch_pp, 7, 4)
    RG_TILE_ADAPTERS(84, launch_pp, 8, 4)
    RG_TILE_ADAPTERS(266, launch_kg, 6, 6, 2)
    RG_TILE_ADAPTERS(276, launch_kg, 7, 6, 2)
    return rg_gemm_tile_adapters_narrow(ctx, tile, a, lda, wp, m, n, k, splits, ep);
}
