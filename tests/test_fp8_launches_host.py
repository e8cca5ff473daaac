"""Launches of the 8-bit products without a GPU, through a stand-in for the HIP calls of a launch (tests/fake_hip.cpp):
grids at the ends of the sizes."""
import json
import os
import subprocess
import sys

import pytest

import paper_2407_01378_amd as thc
from paper_2407_01378_amd import binding

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
