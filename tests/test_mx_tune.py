"""Forced tiles and K splits of the 4-bit and the grouped products: what they launch, without a GPU, underneath a stand-in for the HIP runtime."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2510_25590_amd import binding as rg
import launch_recorder

CONTEXT = f"context 256 4 64 1024 64 64 {rg.BF16}"
TILE, SMALL = "gemm_mx_tile_kernel", "gemm_mx_small_kernel"


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no host C++ compiler here")
    exe = str(tmp_path_factory.mktemp("recorder") / "mx_tune_recorder")
    root = launch_recorder.ROOT
    subprocess.run([gxx, "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(root, "include"), "-I", os.path.join(root, "tests"), "-isystem", "/opt/rocm/include",
                    os.path.join(root, "tests", "mx_tune_recorder.cpp"), "-rdynamic", "-ldl", "-o", exe], check=True)

    def answers(*commands):
        """(code, workgroups, kernel) of each command; the last two 0 and "" where nothing is launched."""
        p = subprocess.run([exe, launch_recorder.LIB], input="\n".join((CONTEXT,) + commands) + "\n", capture_output=True, text=True, timeout=120)
        assert p.returncode == 0, p.stderr
        out, launch = [], (0, "")
        for line in p.stdout.splitlines():
            if line.startswith("launch "):
                x, _, _, _, kernel = line.split(" ", 5)[1:]
                found = re.search(r"gemm_mx_\w+<[\d, ]+>", kernel)             # (a context clears memory by kernels of its own)
                launch = (int(x), found.group()) if found else launch
            elif line.startswith("rc "):
                out.append((int(line.split()[1]),) + launch)
                launch = (0, "")
        return out[1:]
    return answers


@pytest.mark.parametrize("m,n,k", [(820, 12288, 3072), (1382, 3072, 15360), (300, 520, 1536)])
def test_splits_alone_split_the_tile_that_the_product_gets(run, m, n, k):
    (_, plain, kernel), _, (rc, two, same), _, (_, one, _), _, (_, again, last) = run(
        "linear -1 %d %d %d" % (m, n, k), "tune 0 2", "linear -1 %d %d %d" % (m, n, k), "tune 0 1", "linear -1 %d %d %d" % (m, n, k), "tune 0 0", "linear -1 %d %d %d" % (m, n, k))
    tile = [int(v) for v in re.findall(r"\d+", kernel.split("<")[1])]
    units = -(-m // (32 * tile[1])) * -(-n // (128 * tile[2]))
    assert rc == rg.OK and kernel.startswith(TILE) and same == last == kernel
    assert two == -(-2 * units // 8) * 8 and one == -(-units // 8) * 8 and again == plain


def test_a_split_that_does_not_fit_fails(run):
    _, (rc, launched, _) = run("tune 0 16", "linear -1 8704 9216 3072")
    assert rc == rg.ERR_WORKSPACE and not launched


def test_what_takes_no_splits_stays_as_it_is(run):
    """Groups, and the kernels of 16 rows, chosen or forced."""
    plain = run("linear 4 1332 9216 3072", "linear -1 1 9216 3072", "tune 8 0", "linear -1 1 9216 3072")
    forced = run("tune 0 4", "linear 4 1332 9216 3072", "linear -1 1 9216 3072", "tune 8 4", "linear -1 1 9216 3072")
    assert plain[1][2].startswith(SMALL) and [plain[0], plain[1], plain[3]] == [forced[1], forced[2], forced[4]]


@pytest.mark.parametrize("command", ["tune 3 0", "tune 82 1", "tune -1 0", "tune 0 -1", "tune 0 17"])
def test_refusals(run, command):
    assert run(command)[0][0] == rg.ERR_INVALID_ARG
