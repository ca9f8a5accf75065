"""What the 4-bit and the grouped products refuse, what calls with nothing to do launch, and how large their tensors are: without a GPU, underneath a stand-in for the HIP runtime."""
import os
import re
import shutil
import subprocess

import pytest

from oracle import mx_reference as mx
from paper_2510_25590_amd import binding as rg
import launch_recorder

BF = f"context 256 4 64 1024 64 64 {rg.BF16}"
F32 = f"context 256 4 64 1024 64 64 {rg.FP32}"
ARG, SHAPE, UNSUPPORTED = rg.ERR_INVALID_ARG, rg.ERR_BAD_SHAPE, rg.ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no host C++ compiler here")
    exe = str(tmp_path_factory.mktemp("recorder") / "mx_recorder")
    root = launch_recorder.ROOT
    subprocess.run([gxx, "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(root, "include"), "-I", os.path.join(root, "tests"), "-isystem", "/opt/rocm/include",
                    os.path.join(root, "tests", "mx_recorder.cpp"), "-rdynamic", "-ldl", "-o", exe], check=True)

    def answers(commands):
        """(code, launches, message) of each command."""
        p = subprocess.run([exe, launch_recorder.LIB], input="\n".join(commands) + "\n", capture_output=True, text=True, timeout=120)
        assert p.returncode == 0, p.stderr
        out, launches = [], []
        for line in p.stdout.splitlines():
            if line.startswith("launch "):
                x, y, z, lds, kernel = line.split(" ", 5)[1:]
                launches.append(((int(x), int(y), int(z)), int(lds), kernel))
            elif line.startswith("rc "):
                code, message = re.match(r"rc (-?\d+) ?(.*)", line).groups()
                out.append((int(code), launches, message))
                launches = []
        assert len(out) == len(commands)
        return out
    return answers


def linear(four=1, groups=-1, weights=1, given=0, m=4, n=64, k=256, act=0, out=0, null=0, off=0):
    return f"linear {four} {groups} {weights} {given} {m} {n} {k} {act} {out} {null} {off}"


@pytest.mark.parametrize("command,code,word", [
    ("quantize 0 4 33 0 0 0", SHAPE, "multiple of 32"), ("quantize 0 4 0 0 0 0", SHAPE, "cols"), ("quantize 0 -1 64 0 0 0", SHAPE, "rows"), ("quantize 0 2147483648 64 0 0 0", SHAPE, "rows"),
    ("quantize 0 4 1048608 0 0 0", SHAPE, "2^20"), ("quantize 2 4 64 0 0 0", ARG, "dtype"), ("quantize 0 4 64 2 0 0", ARG, "layout"), ("quantize 0 4 64 0 1 0", ARG, "null"),
    ("quantize 0 4 64 1 2 0", ARG, "null"), ("quantize 1 4 64 1 3 0", ARG, "null"), ("quantize 0 4 64 0 0 8", ARG, "unaligned"),
    ("dequantize 3 4 64 0 0 0", ARG, "dtype"), ("dequantize 0 4 48 0 0 0", SHAPE, "cols"), ("dequantize 0 4 64 -1 0 0", ARG, "layout"), ("dequantize 0 4 64 0 3 0", ARG, "null"), ("dequantize 0 4 64 0 0 2", ARG, "unaligned"),
    ("pack 64 40 0 0", SHAPE, "multiple of 32"), ("pack 0 64 0 0", SHAPE, "n=0"), ("pack 16777217 64 0 0", SHAPE, "2^24"), ("pack 2147483647 64 0 0", SHAPE, "2^24"), ("pack 64 1048608 0 0", SHAPE, "2^20"), ("pack 64 64 2 0", ARG, "null"), ("pack 64 64 0 4", ARG, "unaligned"),
    (linear(k=48), SHAPE, "multiple of 32"), (linear(m=-1), ARG, "m=-1"), (linear(n=0), ARG, "n=0"), (linear(k=0), ARG, "k=0"), (linear(act=2), ARG, "act"), (linear(out=2), ARG, "out_dtype"),
    (linear(null=1), ARG, "null"), (linear(null=2), ARG, "null"), (linear(null=3), ARG, "null"), (linear(null=4), ARG, "null"), (linear(null=6), ARG, "null context"), (linear(off=8), ARG, "aligned"),
    (linear(k=1048608), SHAPE, "2^20"), (linear(m=16777217), SHAPE, "2^24"), (linear(n=16777217), SHAPE, "2^24"),
    (linear(groups=2, weights=2, null=5), ARG, "null"), (linear(groups=-2, weights=2), ARG, "groups"), (linear(groups=2, weights=0, given=1), ARG, "weights"), (linear(groups=3, weights=2), ARG, "groups"),
    (linear(groups=65537, weights=2, given=1), ARG, "groups"), (linear(four=0, groups=1, k=96), SHAPE, "multiple of 64"), (linear(four=0, groups=1, null=3), ARG, "null"),
])
def test_refusals(run, command, code, word):
    _, (got, launches, message) = run([BF, command])
    assert got == code and word in message and not launches, (got, message, launches)


@pytest.mark.parametrize("command", ["pack 64 64 0 0", linear(), linear(groups=1), linear(four=0, groups=1)])
def test_float32_contexts_have_no_such_products(run, command):
    _, (got, launches, message) = run([F32, command])
    assert got == UNSUPPORTED and "bf16 context" in message and not launches


@pytest.mark.parametrize("command", ["quantize 0 0 64 0 1 0", "dequantize 1 0 64 1 1 0", linear(m=0, null=1), linear(groups=0, null=5), linear(four=0, groups=2, weights=2, m=0, null=4)])
def test_nothing_to_do(run, command):
    _, (got, launches, _) = run([BF, command])
    assert got == rg.OK and not launches


@pytest.mark.parametrize("command", ["quantize 1 1 32 0 0 0", "quantize 0 2147483647 64 1 0 0", "dequantize 1 2147483647 1048576 1 0 0", "pack 65 288 0 0", linear(m=1, n=1, k=32), linear(m=16777216, n=8, k=32),
                                     linear(m=3, n=16777216, k=32), linear(groups=65536, weights=1, given=1, m=1 << 24), linear(four=0, groups=65536, weights=1, given=1, m=70000, k=64), linear(groups=65536, weights=65536, m=1)])
def test_the_largest_and_smallest_calls_launch(run, command):
    """One launch each, within what a grid may have."""
    _, (got, launches, message) = run([BF, command])
    assert got == rg.OK and len(launches) == 1, message
    (x, y, z), lds, _ = launches[0]
    assert 0 < x * 512 < 2 ** 32 and 0 < y <= 65535 and 0 < z <= 65535


@pytest.mark.parametrize("rows,cols", [(1, 32), (2, 256), (7, 288), (820, 3072), (33, 12288)])
def test_tensor_sizes(rows, cols):
    blocks = cols // 32
    assert rg.regione_mxfp4_scale_bytes(rows, cols, rg.MX_SCALE_ROWS) == rows * blocks
    import numpy as np
    assert rg.regione_mxfp4_scale_bytes(rows, cols, rg.MX_SCALE_STEPS) == mx.scale_steps(np.zeros((rows, blocks), np.uint8)).size
    n32, k256 = -(-rows // 32) * 32, -(-cols // 256) * 256
    assert rg.regione_packed_weight_mxfp4_bytes(rows, cols) == n32 * k256 // 2 + n32 * k256 // 32
    assert rg.regione_packed_weight_mxfp4_bytes(2 ** 31 - 1, cols) == 2 ** 31 // 2 * k256 + 2 ** 31 // 32 * k256
    assert rg.regione_packed_weight_mxfp4_bytes(0, cols) == 0 and rg.regione_mxfp4_scale_bytes(0, cols, 1) == 0


def test_every_choice_covers_its_result(run):
    """Whatever kernel a call gets, its grid has a workgroup for every tile that the result, or the worst sizes of its groups, can have; and every kernel is chosen for some call."""
    import itertools
    shapes = list(itertools.product((1, 4, 16, 40, 64, 130, 205, 300, 410, 820, 1382, 2048, 8704), (64, 768, 1000, 3072, 7568, 9216, 12288), (64, 128, 256, 1024, 3072, 12288, 15360)))
    calls = [(four, groups, m, n, k) for m, n, k in shapes for four, groups in ((1, -1), (1, 2), (1, 16), (1, 64), (0, 1), (0, 4), (0, 16), (0, 64))]
    answers = run([BF] + [linear(four=f, groups=g, weights=max(g, 1), m=m, n=n, k=k) for f, g, m, n, k in calls])[1:]
    seen = set()
    for (four, groups, m, n, k), (code, launches, message) in zip(calls, answers):
        assert code == rg.OK and len(launches) == 1, message
        (x, _, _), lds, kernel = launches[0]
        kind, numbers = re.search(r"gemm_mx_(small|tile)_kernel<([\d, ]+)>", kernel).groups()
        args = tuple(int(v) for v in numbers.split(", "))
        seen.add((kind,) + args)
        assert args[0] == four
        rows, cols = (16, 16 * args[2] * 8 // args[1]) if kind == "small" else (32 * args[1], 128 * args[2])
        tiles = -(-m // rows) if groups == -1 else m // rows + min(groups, m)
        assert x >= tiles * -(-n // cols) and lds <= 65536, (kernel, m, n, k, groups)
    assert len({s for s in seen if s[1] == 1}) == len({s for s in seen if s[1] == 0}) == 16, sorted(seen)
