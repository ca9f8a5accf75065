"""Weights and rows converted for a context whose stream is busy and is not the caller's: temporaries, dropped inputs and results have to be right although the caller goes on allocating."""
import pytest
import torch

from paper_2510_25590_amd import binding as rg

pytestmark = pytest.mark.gpu

N, K = 768, 512
CALLS = {
    "quantize_rows_mxfp4": lambda ctx, w: rg.quantize_rows_mxfp4(ctx, w),
    "pack_weight_mxfp4": lambda ctx, w: (rg.pack_weight_mxfp4(ctx, w),),
    "pack_weight": lambda ctx, w: (rg.pack_weight(ctx, w),),
    "make_stream_weights_fp8": lambda ctx, w: rg.make_stream_weights_fp8(ctx, {"w_o": w})[1]["w_o"],
}


def weight(i):
    return torch.randn(K, N, generator=torch.Generator(device="cuda").manual_seed(i), device="cuda").to(torch.bfloat16).t()       # not contiguous: a further temporary


@pytest.mark.parametrize("name", CALLS)
def test_a_context_of_another_stream(name):
    plain = rg.Context(256, 4, 64, 1024, 64, 64)
    want = [[t.cpu() for t in CALLS[name](plain, weight(i))] for i in range(4)]
    plain.close()
    side = torch.cuda.Stream()
    ctx = rg.Context(256, 4, 64, 1024, 64, 64, stream=side)
    work = torch.randn(2048, 2048, device="cuda")
    torch.cuda.synchronize()
    got = []
    for i in range(4):
        with torch.cuda.stream(side):
            for _ in range(20):
                work = (work @ work).clamp_(-1.0, 1.0)
        got.append(CALLS[name](ctx, weight(i)))                                             # the input is dropped at once
        for size in (N * K * 2, N * K, N * K // 2, N * K // 32, N * 4):                      # the sizes of the inputs and the temporaries
            torch.full((size,), 255, dtype=torch.uint8, device="cuda")
    got = [[t.cpu() for t in g] for g in got]                                               # on the caller's stream
    ctx.close()
    for a, b in zip(got, want):
        assert all(torch.equal(s, t) for s, t in zip(a, b))
