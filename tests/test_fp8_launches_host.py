"""Launches of the 8-bit products without a GPU, through a stand-in for the HIP calls of a launch (tests/fake_hip.cpp):
grids at the ends of the sizes, how many launches a call takes, and workspaces where they are needed."""
import ctypes
import json
import os
import subprocess
import sys

import pytest

import paper_2407_01378_amd as thc
from paper_2407_01378_amd import binding
from test_train_ops_host import NUL, ODD, gradient, linear, matmul

TESTS = os.path.dirname(os.path.abspath(__file__))

CHILD = """
import ctypes, json, sys
fake = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
lib = ctypes.CDLL(sys.argv[2])
u64, vp, at = ctypes.c_uint64, ctypes.c_void_p, ctypes.c_void_p(0x10000)   # (an address that only a launch would use)
seen = []
for kind, M, N, K, out in json.loads(sys.argv[3]):
    before = fake.fake_launches()
    if kind == "product":
        rc = lib.thc_fp8_matmul(at, at, 0, at, at, 0, u64(M), u64(N), u64(K), 0, out, at, u64(N), at, u64(1 << 60), None)
    else:
        rc = lib.thc_fp8_linear(at, 1, u64(M), u64(K), u64(K), 0, at, at, 0, u64(N), out, at, u64(N), at, u64(1 << 60), None)
    seen.append([rc, fake.fake_grid(), fake.fake_block(), fake.fake_launches() - before])
print(json.dumps(seen))
"""


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    thc.lib()
    fake = str(tmp_path_factory.mktemp("fake") / "libfake_hip.so")
    res = subprocess.run(["hipcc", "-O1", "-std=c++17", "-fPIC", "-shared", "-o", fake, os.path.join(TESTS, "fake_hip.cpp")],
                         stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert res.returncode == 0, res.stdout[-3000:]

    def calls(*sequence):
        res = subprocess.run([sys.executable, "-c", CHILD, fake, binding.LIB_PATH, json.dumps(sequence)],
                             stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True, timeout=120)
        assert res.returncode == 0, res.stderr[-3000:]
        return json.loads(res.stdout.splitlines()[-1])
    return calls


MOST = 1 << 26   # rows of an operand


def test_grids_at_the_ends_of_the_sizes(run):
    sizes = [(1, 1), (1, 24575), (16, 24575), (17, 4096), (32, 4096), (1, MOST), (16, MOST), (33, MOST), (128, MOST), (300, MOST), (1920, MOST),
             (MOST, 1), (MOST, 33), (MOST, 300), (MOST, 1920), (MOST, 1 << 13), ((1 << 26) - 127, 8129), ((1 << 20) + 1, (1 << 19) - 1)]
    for K in (1, 1 << 22):
        seen = run(*((kind, M, N, K, out) for kind in ("product", "linear") for M, N in sizes for out in (0, 1)))
        for rc, grid, block, launches in seen:
            assert rc == 0 and 0 < grid and grid * block <= 1 << 31 and 1 <= launches <= 3


def test_results_beyond_2_to_the_39_are_refused(run):
    """As sizes, by the entry point, and with nothing started."""
    for M, N in ((MOST, MOST), (1 << 20, 1 << 20), (MOST, (1 << 13) + 1), (MOST, 1 << 14)):
        assert thc.thc_fp8_matmul_workspace_bytes(M, N, 128) == 0 and thc.thc_fp8_linear_workspace_bytes(M, N, 128) == 0
        for rc, _, _, launches in run(*((kind, M, N, 128, out) for kind in ("product", "linear") for out in (0, 1))):
            assert (rc, launches) == (-6, 0)


def test_launches_of_a_call(run):
    for (kind, M, N, K, out), launches in (
            (("linear", 1, 8192, 2048, 1), 1), (("linear", 16, 24575, 900, 0), 1),
            (("linear", 24, 2048, 8192, 1), 3),          # quantizer, product, join of two halves of k
            (("product", 24, 2048, 8192, 1), 2), (("product", 24, 2048, 1024, 1), 1),
            (("product", 777, 520, 1000, 0), 1), (("product", 4096, 4096, 2048, 0), 1),
            (("product", 1003, 50257, 1024, 1), 2),      # large tiles, and the last columns in small ones
            (("product", 128, 128, 70000, 0), 2)):
        rc, _, _, n = run((kind, M, N, K, out))[0]
        assert (rc, n) == (0, launches), (kind, M, N, K)


@pytest.mark.parametrize("M,N,K", [(64, 64, 4096), (24, 2048, 8192), (300, 300, 200), (20, 40, 1), (8, 16, 1 << 16)])
def test_workspaces_of_a_layer(M, N, K):
    """The rows' codes and scales, and the parts where k is divided."""
    L, need = thc.lib(), thc.thc_fp8_linear_workspace_bytes(M, N, K)
    parts = thc.thc_fp8_matmul_workspace_bytes(M, N, K)
    assert need > 0 and need - parts in ((M * thc.thc_fp8_row_bytes(K) + thc.thc_fp8_scale_bytes(M, K) + 15) // 16 * 16, 0 if M <= 16 else -1)
    size = dict(M=M, N=N, K=K, ldx=K, ldo=N)
    assert linear(L, wb=need - 1, **size) == -6 and linear(L, wb=0, **size) == -6
    assert linear(L, ws=NUL, **size) == -1 and linear(L, ws=ODD, **size) == -8


def test_workspaces_of_divided_sums_and_gradients():
    L = thc.lib()
    for M, N, K in ((24, 2048, 8192), (64, 64, 1 << 16), (256, 256, 1 << 20)):
        need = thc.thc_fp8_matmul_workspace_bytes(M, N, K)
        assert need >= 2 * M * N * 4
        assert matmul(L, M=M, N=N, K=K, ldc=N, wb=need - 1) == -6
        assert matmul(L, M=M, N=N, K=K, ldc=N, ws=NUL) == -1 and matmul(L, M=M, N=N, K=K, ldc=N, ws=ODD) == -8
    for count in (4, 7000):
        need = thc.thc_embed_backward_workspace_bytes(count, 10, 8)
        assert need > 8 * count
        assert gradient(L, count=count, wb=need - 1) == -6
        assert gradient(L, count=count, ws=NUL) == -1 and gradient(L, count=count, ws=ctypes.c_void_p(0x1004)) == -8
