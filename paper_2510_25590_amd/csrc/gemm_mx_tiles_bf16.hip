// The tiles of bf16 products over groups of rows.
#include "gemm_mx_tile.h"

int rg_mx_tile_bf16(regione_ctx* ctx, int tile, const MxOperands& p, int splits, const GemmEpilogue& ep) { return launch_mx_tile<MX_BF16>(ctx, tile, p, splits, ep); }
