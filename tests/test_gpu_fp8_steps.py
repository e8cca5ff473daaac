"""8-bit products by large tiles: every remainder of the steps along k by five, below and beyond two rounds of them; and fp32
results whose terms are further apart than the bits that the 8-bit matrix instruction keeps."""
import pytest
import torch

import paper_2407_01378_amd as thc
from test_gpu_fp8_sizes import _operand

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
STEPS = [300, 512, 513, 640, 1100, 1280, 1400, 1536, 1650, 1791, 1920, 2048, 8192]   # 3, 4, 5, 5, 9, 10, 11, 12, 13, 14, 15, 16, 64


@pytest.mark.parametrize("K", STEPS)
@pytest.mark.parametrize("M,N", [(4090, 4000), (5632, 5888)])   # a tile to a workgroup; several, whole and ragged
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_large_tiles(M, N, K, out):
    _check(M, N, K, out)


@pytest.mark.parametrize("K", [200, 512, 1100, 2048])
@pytest.mark.parametrize("M,N", [(4096, 13312), (4090, 13301)])   # the last columns in small tiles, fp32 results too
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_large_and_small_tiles(M, N, K, out):
    _check(M, N, K, out)


def _check(M, N, K, out):
    a, b = _operand(M, K, thc.THC_E5M2, 1), _operand(N, K, thc.THC_E4M3, 2)
    assert K * 64 < 2 ** 24                      # every partial sum is a whole number that fp32 holds
    want = (a[2].double() @ b[2].double().t()).float()
    n = thc.thc_fp8_matmul_workspace_bytes(M, N, K)
    ws = torch.full((n,), 0xCD, dtype=torch.uint8, device=DEV) if n else None
    c = torch.full((M, N), float("nan"), dtype=out, device=DEV)
    thc.thc_fp8_matmul(a[0], a[1], thc.THC_E5M2, b[0], b[1], thc.THC_E4M3, K, c, ws)
    assert torch.equal(c, want.to(out))
    start = c.clone().float()
    thc.thc_fp8_matmul(a[0], a[1], thc.THC_E5M2, b[0], b[1], thc.THC_E4M3, K, c, ws, True)
    assert torch.equal(c, (start + want).to(out))


@pytest.mark.parametrize("M,N,K", [(1, 700, 2048), (16, 300, 4096), (24, 512, 900), (640, 640, 1000), (130, 260, 1100), (128, 128, 8000),
                                   (4090, 4000, 512), (4090, 4000, 1280), (5632, 5888, 640), (4096, 13312, 400)])
def test_terms_far_apart_in_fp32(M, N, K):
    """One entry of A in eight or fewer is +-256, the others are +-1/64; B is +-1 and +-2.  The products are whole multiples of 2^-6 up to 2^9,
    2^15 apart among neighbours; every partial sum is held by fp32, so that sums of exact products are exact in any order."""
    g = torch.Generator(device=DEV)
    g.manual_seed(M + K)
    blocks = thc.thc_fp8_row_bytes(K) // 128

    def sides(rows):
        return torch.randint(0, 2, (rows, K), generator=g, device=DEV).to(torch.uint8) << 7

    large = torch.rand(M, K, generator=g, device=DEV) < min(0.125, 400 / K)
    two = torch.rand(N, K, generator=g, device=DEV) < 0.5
    ops = []
    # e4m3: 256 = 2^8 has exponent field 15, 1/64 = 2^-6 has 1; 1 and 2 have 7 and 8
    for rows, field in ((M, torch.where(large, 15, 1)), (N, torch.where(two, 8, 7))):
        sign = sides(rows)
        codes = torch.zeros(rows, blocks * 128, dtype=torch.uint8, device=DEV)
        codes[:, :K] = (field << 3).to(torch.uint8) | sign
        scales = torch.full((thc.thc_fp8_scale_bytes(rows, K),), 127, dtype=torch.uint8, device=DEV)
        ops.append((codes.reshape(-1), scales, torch.exp2(field.double() - 7.0) * torch.where(sign != 0, -1.0, 1.0)))
    size = ops[0][2].abs() @ ops[1][2].abs().t()
    assert float(size.max()) < 2.0 ** 24 * 2.0 ** -6
    want = ops[0][2] @ ops[1][2].t()
    n = thc.thc_fp8_matmul_workspace_bytes(M, N, K)
    ws = torch.full((n,), 0xCD, dtype=torch.uint8, device=DEV) if n else None
    c = torch.full((M, N), float("nan"), device=DEV)
    thc.thc_fp8_matmul(ops[0][0], ops[0][1], thc.THC_E4M3, ops[1][0], ops[1][1], thc.THC_E4M3, K, c, ws)
    assert torch.equal(c.double(), want)
