"""What routing, the sort by expert, the weighted sum and the low-rank adapters refuse, what calls with nothing to do launch, and how large launches get: without a GPU, underneath a
stand-in for the HIP runtime."""
import os
import re
import shutil
import subprocess
import types

import pytest
import torch

from paper_2510_25590_amd import binding as rg
import launch_recorder

BF = f"context 256 4 64 1024 64 64 {rg.BF16}"
F32 = f"context 256 4 64 1024 64 64 {rg.FP32}"
NO_ROWS = f"context 256 4 64 1024 0 64 {rg.BF16}"
ARG, SHAPE, UNSUPPORTED, WORKSPACE = rg.ERR_INVALID_ARG, rg.ERR_BAD_SHAPE, rg.ERR_UNSUPPORTED, rg.ERR_WORKSPACE


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no host C++ compiler here")
    exe = str(tmp_path_factory.mktemp("recorder") / "expert_recorder")
    root = launch_recorder.ROOT
    subprocess.run([gxx, "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(root, "include"), "-I", os.path.join(root, "tests"), "-isystem", "/opt/rocm/include",
                    os.path.join(root, "tests", "expert_recorder.cpp"), "-rdynamic", "-ldl", "-o", exe], check=True)

    def answers(commands):
        """(code, launches, grants, message) of each command."""
        p = subprocess.run([exe, launch_recorder.LIB], input="\n".join(commands) + "\n", capture_output=True, text=True, timeout=120)
        assert p.returncode == 0, p.stderr
        out, launches, grants = [], [], {}
        for line in p.stdout.splitlines():
            if line.startswith("launch "):
                x, y, z, lds, kernel = line.split(" ", 5)[1:]
                launches.append(((int(x), int(y), int(z)), int(lds), kernel))
            elif line.startswith("grant "):
                grants[line.split(" ", 2)[2]] = int(line.split(" ", 2)[1])
            elif line.startswith("rc "):
                code, message = re.match(r"rc (-?\d+) ?(.*)", line).groups()
                out.append((int(code), launches, dict(grants), message))
                launches = []
        assert len(out) == len(commands)
        return out
    return answers


def route(dtype=1, tokens=5, experts=64, score=0, groups=1, top_groups=1, best=1, k=4, renorm=1, scale=1.0, given=0, null=0, off=0):
    return f"route {dtype} {tokens} {experts} {score} {groups} {top_groups} {best} {k} {renorm} {scale} {given} {null} {off}"


def slots(tokens=5, k=2, experts=8, null=0, off=0):
    return f"slots {tokens} {k} {experts} {null} {off}"


def combine(rows_t=0, rows=10, tokens=5, k=2, cols=64, out_t=0, null=0, off=0):
    return f"combine {rows_t} {rows} {tokens} {k} {cols} {out_t} {null} {off}"


def adapters(count=3, sel=1, rank=16, m=5, n=64, k=128, act=0, out=0, null=0, off=0):
    return f"adapters {count} {sel} {rank} {m} {n} {k} {act} {out} {null} {off}"


@pytest.mark.parametrize("command,code,word", [
    (route(dtype=2), ARG, "dtype"), (route(score=2), ARG, "score"), (route(tokens=-1), ARG, "n_tokens"), (route(experts=0), ARG, "n_experts"), (route(k=0), ARG, "top_k"), (route(groups=0), ARG, "n_groups"),
    (route(best=0), ARG, "group_best"), (route(best=3), ARG, "group_best"), (route(scale="nan"), ARG, "scale"), (route(scale="inf"), ARG, "scale"), (route(experts=1025), UNSUPPORTED, "1024"),
    (route(k=33), UNSUPPORTED, "32"), (route(experts=650, groups=65), UNSUPPORTED, "64"), (route(tokens=(1 << 22) + 1), UNSUPPORTED, "2^24"), (route(tokens=1 << 62, k=4), UNSUPPORTED, "2^24"),
    (route(experts=60, groups=8), SHAPE, "groups"), (route(groups=8, top_groups=0), SHAPE, "groups"), (route(groups=8, top_groups=9), SHAPE, "groups"), (route(experts=16, groups=8, top_groups=1), SHAPE, "groups"),
    (route(experts=3), SHAPE, "experts"), (route(null=1), ARG, "null"), (route(null=2), ARG, "null"), (route(null=3), ARG, "null"), (route(null=9), ARG, "null context"), (route(off=4), ARG, "aligned"),
    (slots(tokens=-1), ARG, "n_tokens"), (slots(k=0), ARG, "top_k"), (slots(experts=0), ARG, "n_experts"), (slots(experts=1025), UNSUPPORTED, "1024"), (slots(k=33), UNSUPPORTED, "32"),
    (slots(tokens=(1 << 23) + 1), UNSUPPORTED, "2^24"), (slots(tokens=1 << 62), UNSUPPORTED, "2^24"), (slots(null=1), ARG, "null"), (slots(null=2), ARG, "null"), (slots(null=3), ARG, "null"),
    (slots(null=4), ARG, "null"), (slots(null=9), ARG, "null context"), (slots(tokens=0, null=2), ARG, "null"),
    (combine(rows_t=2), ARG, "dtype"), (combine(out_t=-1), ARG, "dtype"), (combine(rows=-1), ARG, "n_rows"), (combine(tokens=-1), ARG, "n_tokens"), (combine(k=0), ARG, "top_k"), (combine(cols=0), ARG, "cols"),
    (combine(k=33), UNSUPPORTED, "32"), (combine(tokens=1 << 24), UNSUPPORTED, "2^24"), (combine(cols=(1 << 24) + 1), UNSUPPORTED, "2^24"), (combine(null=1), ARG, "null"), (combine(null=2), ARG, "null"),
    (combine(null=3), ARG, "null"), (combine(null=9), ARG, "null context"),
    ("pack 0 64 16 0 0", ARG, "n=0"), ("pack 64 0 16 0 0", ARG, "k=0"), ("pack 64 64 0 0 0", ARG, "rank=0"), ("pack 64 96 16 0 0", SHAPE, "multiple of 64"), ("pack 64 64 257 0 0", UNSUPPORTED, "256"),
    ("pack 16777217 64 16 0 0", SHAPE, "2^24"), ("pack 64 1048640 16 0 0", SHAPE, "2^20"), ("pack 64 64 16 1 0", ARG, "null"), ("pack 64 64 16 2 0", ARG, "null"), ("pack 64 64 16 3 0", ARG, "null"),
    ("pack 64 64 16 9 0", ARG, "null context"), ("pack 64 64 16 0 8", ARG, "unaligned"),
    (adapters(m=-1), ARG, "m=-1"), (adapters(n=0), ARG, "n=0"), (adapters(k=0), ARG, "k=0"), (adapters(rank=0), ARG, "rank=0"), (adapters(k=96), SHAPE, "multiple of 64"), (adapters(rank=257), UNSUPPORTED, "256"),
    (adapters(count=0), ARG, "n_adapters"), (adapters(sel=0), ARG, "n_sel"), (adapters(count=65537), UNSUPPORTED, "65536"), (adapters(sel=33), UNSUPPORTED, "32"), (adapters(m=16777217), SHAPE, "2^24"),
    (adapters(act=2), ARG, "act"), (adapters(out=2), ARG, "out_dtype"), (adapters(null=1), ARG, "null"), (adapters(null=2), ARG, "null"), (adapters(null=3), ARG, "null"), (adapters(null=4), ARG, "null"),
    (adapters(null=5), ARG, "null"), (adapters(null=9), ARG, "null context"), (adapters(off=8), ARG, "aligned"),
])
def test_refusals(run, command, code, word):
    _, (got, launches, _, message) = run([BF, command])
    assert got == code and word in message and not launches, (got, message, launches)


@pytest.mark.parametrize("command", ["pack 64 64 16 0 0", adapters()])
def test_float32_contexts_have_no_adapters(run, command):
    _, (got, launches, _, message) = run([F32, command])
    assert got == UNSUPPORTED and "bf16 context" in message and not launches


def test_contexts_without_workspace(run):
    _, a, b, c = run([NO_ROWS, adapters(), slots(tokens=1 << 20, k=8, experts=64), slots()])
    assert a[0] == WORKSPACE and b[0] == WORKSPACE and not a[1] and not b[1] and c[0] == rg.OK


@pytest.mark.parametrize("command,launches", [(route(tokens=0, null=1), 0), (combine(tokens=0, null=2), 0), (adapters(m=0, null=4), 0), (slots(tokens=0, null=1), 1), (combine(rows=0, null=1), 1)])
def test_nothing_to_do(run, command, launches):
    """An empty sort still writes its offsets, a sum over no rows its base."""
    _, (got, made, _, message) = run([BF, command])
    assert got == rg.OK and len(made) == launches, message


@pytest.mark.parametrize("command", [
    route(tokens=1, experts=1, k=1), route(tokens=1 << 24, experts=1024, k=1), route(tokens=1 << 19, k=32), route(experts=1024, groups=64, top_groups=64, best=2, k=32), route(experts=990, groups=33, top_groups=1, given=1),
    slots(tokens=1, k=1, experts=1), slots(tokens=1 << 24, k=1, experts=1024), slots(tokens=1 << 19, k=32, experts=1024), slots(tokens=100, experts=1024),
    combine(tokens=1 << 24, k=1, cols=4096, rows=1 << 40), combine(tokens=1, k=32, cols=1 << 24), combine(cols=7), "pack 1 64 1 0 0", "pack 16777216 64 256 0 0", "pack 9216 1048576 256 0 0",
    adapters(m=1, n=1, k=64, rank=1, count=1), adapters(m=1, n=9216, k=15360, rank=256, count=65536, sel=32), adapters(m=8704, n=9216, k=3072, rank=64, sel=4), adapters(m=70000, n=64, k=64, rank=256, sel=32, out=1),
    adapters(m=1 << 24, n=64, k=64, rank=1), adapters(m=3, n=1 << 24, k=64),
])
def test_the_largest_and_smallest_calls_launch(run, command):
    _, (got, launches, grants, message) = run([BF, command])
    assert got == rg.OK and launches, message
    for (x, y, z), lds, kernel in launches:
        assert 0 < x * 1024 <= 2 ** 42 and x < 2 ** 31 and 0 < y <= 65535 and z == 1
        assert lds <= 65536 or grants.get(kernel, 0) >= lds, (kernel, lds)


def test_every_adapter_product_covers_its_result(run):
    """Whatever kernel the product gets, its grid has a workgroup for every tile of the result, behind one launch for the inner products; rows go through in parts that fit the workspace."""
    import itertools
    shapes = list(itertools.product((1, 16, 40, 130, 410, 820, 2048, 8704), (64, 768, 1000, 3072, 9216, 12288), (64, 256, 1024, 3072, 12288)))
    answers = run([BF] + [adapters(m=m, n=n, k=k) for m, n, k in shapes])[1:]
    seen = set()
    for (m, n, k), (code, launches, _, message) in zip(shapes, answers):
        assert code == rg.OK and len(launches) == 2, message
        (dx, dy, _), _, down = launches[0]
        (x, y, _), lds, kernel = launches[1]
        kind, numbers = re.search(r"gemm_(small|pp|kg)_kernel<([\d, a-z]+)>", kernel).groups()
        args = [int(v) for v in re.findall(r"\d+", numbers)]
        seen.add((kind,) + tuple(args))
        assert lds <= 163840
        if kind == "small":
            of_pieces = re.search(r"adapters_down_tiles_kernel<false, (\d+), ", down)
            assert of_pieces or "adapters_down_rows" in down
            assert dx == -(-m // (16 * int(of_pieces.group(1)) if of_pieces else 16)) and dy >= 1
            assert x == -(-n // (16 * args[0])) and y == -(-m // 16)
        else:
            tile = (32 * args[0], 64 * args[1]) if kind == "pp" else (16 * args[0] * args[2], 16 * args[1] * (4 // args[2]))
            assert x >= -(-m // tile[0]) * -(-n // tile[1]) and y == 1
            rows = 16 * int(re.search(r"adapters_down_tiles_kernel<true, (\d+), ", down).group(1))
            assert dx == -(-m // tile[0]) * -(-tile[0] // rows) and dy >= 1
    assert {s[0] for s in seen} == {"small", "pp", "kg"}
    many = run([BF, adapters(m=2000, n=64, k=64, rank=256, sel=32, out=1)])[1]
    assert len(many[1]) == 2 * 2                                         # 1360 rows at a time
    # where every row of a tile may name another adapter: passes of as many tiles as the workspace holds, or the kernel of 16 rows where a tile does not fit
    passes, single = run([BF, adapters(m=20000, n=2304, k=128, rank=8, count=600), adapters(m=4200, n=2304, k=128, rank=8, count=20000, sel=32)])[1:]
    assert len(passes[1]) > 2 and len(passes[1]) % 2 == 0 and all(re.search("gemm_(pp|kg)", kernel) for _, _, kernel in passes[1][1::2])
    assert len(single[1]) == 2 and "gemm_small" in single[1][1][2]


@pytest.mark.parametrize("rows,cols,rank", [(1, 64, 1), (33, 128, 16), (9216, 3072, 64), (40, 64, 17)])
def test_tensor_sizes(rows, cols, rank):
    r16, n32 = -(-rank // 16) * 16, -(-rows // 32) * 32
    assert rg.regione_packed_adapter_elems(rows, cols, rank) == r16 * cols + n32 * r16 + -(-(n32 // 32 + 1) // 4) * 8
    assert rg.regione_packed_adapter_elems(0, cols, rank) == rg.regione_packed_adapter_elems(rows, 0, rank) == rg.regione_packed_adapter_elems(rows, cols, 0) == 0


@pytest.mark.parametrize("a,b", [
    (((2, 16, 64), torch.float16, "meta"), ((2, 40, 16), torch.bfloat16, "meta")), (((2, 16, 64), torch.bfloat16, "meta"), ((2, 40, 16), torch.float32, "meta")),
    (((16, 64), torch.bfloat16, "meta"), ((40, 16), torch.bfloat16, "meta")), (((2, 16, 64), torch.bfloat16, "meta"), ((3, 40, 16), torch.bfloat16, "meta")),
    (((2, 16, 64), torch.bfloat16, "meta"), ((2, 16, 40), torch.bfloat16, "meta")), (((2, 16, 64), torch.bfloat16, "cpu"), ((2, 40, 16), torch.bfloat16, "meta")),
])
def test_pack_adapters_refuses_other_tensors(monkeypatch, a, b):
    """The meta device stands for the context's own; the library is never asked."""
    ctx = types.SimpleNamespace(handle=None, stream=types.SimpleNamespace(device=torch.device("meta")))
    asked = []
    monkeypatch.setattr(rg, "lib", lambda: asked.append(1))
    with pytest.raises(rg.RegionEError) as e:
        rg.pack_adapters(ctx, *(torch.empty(s, dtype=t, device=d) for s, t, d in (a, b)))
    assert e.value.code == rg.ERR_INVALID_ARG and "pack_adapters" in str(e.value) and not asked
