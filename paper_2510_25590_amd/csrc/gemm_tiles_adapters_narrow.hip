// The 64-, 96- and 128-column tiles of the two-group GEMM with low-rank adapters' K-steps behind the product's (gemm_adapters.h).
#include "gemm_launch.h"

#define RG_TILE_ADAPTERS(CODE, ...) if (tile == CODE) return launch_kg<__VA_ARGS__, EPI_ADAPTERS>(ctx, a, lda, wp, m, n, k, splits, ep);
int rg_gemm_tile_adapters_narrow(regione_ctx* ctx, int tile, const bf16_t* a, int lda, const bf16_t* wp, int m, int n, int k, int splits, const GemmEpilogue& ep) {
    RG_TILE_ADAPTERS(222, 2, 2, 2)
    RG_TILE_ADAPTERS(224, 2, 4, 2)
    RG_TILE_ADAPTERS(242, 4, 2, 2)
    RG_TILE_ADAPTERS(244, 4, 4, 2)
    RG_TILE_ADAPTERS(274, 7, 4, 2)
    RG_TILE_ADAPTERS(284, 8, 4, 2)
    RG_TILE_ADAPTERS(426, 2, 6, 4)
    RG_TILE_ADAPTERS(436, 3, 6, 4)
    RG_TILE_ADAPTERS(446, 4, 6, 4)
    RG_FAIL(REGIONE_ERR_INVALID_ARG, "gemm: no tile %d here", tile);
}
