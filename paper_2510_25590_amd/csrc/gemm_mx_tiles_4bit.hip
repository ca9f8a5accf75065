// The tiles of 4-bit products.
#include "gemm_mx_tile.h"

int rg_mx_tile_4bit(regione_ctx* ctx, int tile, const MxOperands& p, int splits, const GemmEpilogue& ep) { return launch_mx_tile<MX_FP4>(ctx, tile, p, splits, ep); }
