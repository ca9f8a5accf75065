"""What quantize_rows_mxfp4 and pack_weight_mxfp4 of the binding refuse, without a GPU: the library is never asked."""
import types

import pytest
import torch

from paper_2510_25590_amd import binding as rg


@pytest.mark.parametrize("call", [rg.quantize_rows_mxfp4, rg.pack_weight_mxfp4])
@pytest.mark.parametrize("dtype,shape,device", [
    (torch.float16, (4, 64), "meta"), (torch.float64, (4, 64), "meta"), (torch.int16, (4, 64), "meta"), (torch.uint8, (4, 64), "meta"), (torch.float8_e4m3fn, (4, 64), "meta"),
    (torch.bfloat16, (4, 2, 64), "meta"), (torch.float32, (64,), "meta"), (torch.bfloat16, (4, 64), "cpu"), (torch.float32, (4, 64), "cpu")])
def test_refusals(monkeypatch, call, dtype, shape, device):
    """The meta device stands for the context's own."""
    ctx = types.SimpleNamespace(handle=None, stream=types.SimpleNamespace(device=torch.device("meta")), torch_dtype=torch.bfloat16)
    asked = []
    monkeypatch.setattr(rg, "lib", lambda: asked.append(1))
    monkeypatch.setattr(rg, "_on_stream_of", lambda *a: asked.append(1), raising=False)
    with pytest.raises(rg.RegionEError) as e:
        call(ctx, torch.empty(shape, dtype=dtype, device=device))
    assert e.value.code == rg.ERR_INVALID_ARG and call.__name__ in str(e.value) and not asked
