"""Calls of the binding that make tensors themselves, on a context whose stream is not the caller's: what is allocated where and what waits for what, without a GPU."""
import contextlib

import pytest
import torch

from paper_2510_25590_amd import binding as rg


class Stream:
    def __init__(self, log, name):
        self.log, self.name, self.device = log, name, torch.device("cuda", 0)

    def wait_stream(self, other):
        self.log.append(("wait", self.name, other.name))


class Tensor:
    """As much of a CUDA tensor as the binding looks at."""
    is_cuda, device = True, torch.device("cuda", 0)

    def __init__(self, world, shape, dtype, where=None):
        self.world, self.shape, self.dtype, self.ndim = world, shape, dtype, len(shape)
        self.stream, self.address = where or world.current.name, len(world.tensors) + 1
        world.tensors.append(self)

    def dim(self):
        return self.ndim

    def contiguous(self):
        return Tensor(self.world, self.shape, self.dtype)

    def record_stream(self, stream):
        self.world.log.append(("keep", self.address, stream.name))

    def data_ptr(self):
        return self.address


class World:
    """Streams, the allocator and the library, all of which only write down what is asked of them."""

    def __init__(self, monkeypatch, same):
        self.log, self.tensors = [], []
        self.caller = self.current = Stream(self.log, "caller")
        self.ctx = rg.Context.__new__(rg.Context)
        self.ctx.handle, self.ctx.torch_dtype, self.ctx.stream = None, torch.bfloat16, self.caller if same else Stream(self.log, "context")
        make = lambda shape, dtype=None, device=None: Tensor(self, shape if isinstance(shape, tuple) else (shape,), dtype)
        monkeypatch.setattr(torch, "empty", make)
        monkeypatch.setattr(torch, "zeros", make)
        monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: self.current)
        monkeypatch.setattr(torch.cuda, "stream", self.use)
        monkeypatch.setattr(rg, "lib", lambda: self)

    @contextlib.contextmanager
    def use(self, stream):
        before, self.current = self.current, stream
        yield
        self.current = before

    def __getattr__(self, name):
        def call(*args):
            if name.endswith(("_bytes", "_elems")):
                return 64
            self.log.append(("call", name, [a for a in args if isinstance(a, int)]))
            return 0
        return call


CALLS = {
    "quantize_rows_mxfp4": lambda ctx, w: rg.quantize_rows_mxfp4(ctx, w),
    "pack_weight_mxfp4": lambda ctx, w: (rg.pack_weight_mxfp4(ctx, w),),
    "pack_weight": lambda ctx, w: (rg.pack_weight(ctx, w),),
    "make_stream_weights_fp8": lambda ctx, w: rg.make_stream_weights_fp8(ctx, {"w_o": w})[1]["w_o"],
}


@pytest.mark.parametrize("name", CALLS)
def test_tensors_belong_to_the_stream_that_works_on_them(monkeypatch, name):
    world = World(monkeypatch, same=False)
    w = Tensor(world, (64, 256), torch.bfloat16, where="caller")
    results = CALLS[name](world.ctx, w)
    assert all(t.stream == "context" for t in world.tensors[1:]), [(t.address, t.stream) for t in world.tensors]
    calls = [i for i, entry in enumerate(world.log) if entry[0] == "call"]
    assert calls and world.log.index(("wait", "context", "caller")) < calls[0]                              # the input is ready
    assert len(world.log) - 1 - world.log[::-1].index(("wait", "caller", "context")) > calls[-1]           # so are the results
    assert ("keep", w.address, "context") in world.log and all(("keep", r.address, "caller") in world.log for r in results)
    assert world.current is world.caller


@pytest.mark.parametrize("name", CALLS)
def test_on_the_caller_s_own_stream_nothing_waits(monkeypatch, name):
    world = World(monkeypatch, same=True)
    CALLS[name](world.ctx, Tensor(world, (64, 256), torch.bfloat16))
    assert all(entry[0] == "call" for entry in world.log)
