"""8-bit products where how they are done changes with their sizes: many tiles, few rows, long sums; exactly, on whole numbers."""
import pytest
import torch

import paper_2407_01378_amd as thc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _operand(rows, cols, fmt, seed):
    """Whole numbers from -2 to 2 with scales of 1, 2 and 4: (codes, scales, values)."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    blocks = (cols + 127) // 128
    ones, twos = {thc.THC_E4M3: (0x38, 0x40), thc.THC_E5M2: (0x3C, 0x40)}[fmt]      # 1.0 and 2.0
    table = torch.tensor([0x80 | twos, 0x80 | ones, 0, ones, twos], dtype=torch.uint8, device=DEV)
    v = torch.randint(0, 5, (rows, cols), generator=g, device=DEV)
    codes = torch.zeros(rows, blocks * 128, dtype=torch.uint8, device=DEV)
    codes[:, :cols] = table[v]
    e = torch.randint(0, 3, (rows, blocks), generator=g, device=DEV)
    scales = torch.zeros((blocks + 3) // 4, rows, 4, dtype=torch.uint8, device=DEV)
    for j in range(blocks):
        scales[j // 4, :, j % 4] = (127 + e[:, j]).to(torch.uint8)
    assert scales.numel() == thc.thc_fp8_scale_bytes(rows, cols) and codes.numel() == rows * thc.thc_fp8_row_bytes(cols)
    values = (v - 2).float() * torch.exp2(e.float()).repeat_interleave(128, 1)[:, :cols]
    return codes.reshape(-1), scales.reshape(-1), values


@pytest.mark.parametrize("M,N,K", [
    (5600, 5800, 100), (5600, 5800, 130), (5632, 5888, 700), (9000, 4200, 1000),        # several large tiles to a compute unit
    (600, 50257, 300), (130, 50257, 256), (1003, 50257, 200), (4608, 4096, 300), (4500, 4111, 700), (9216, 4096, 260),   # a rest in small ones
    (16, 24575, 260), (16, 24576, 260), (17, 24575, 1100), (1, 50257, 900), (3, 70001, 128),    # few rows
    (32, 4096, 300), (33, 4096, 300), (17, 4097, 5000), (32, 33, 6000), (29, 2048, 8192),
    (16, 4096, 4096), (17, 300, 8000), (128, 128, 70000), (40, 5000, 9000),              # long sums
    (640, 640, 1536), (639, 641, 1537), (900, 1000, 1664), (4082, 18, 1443), (2722, 25, 1472), (777, 520, 1000)])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_exact(M, N, K, out):
    a, b = _operand(M, K, thc.THC_E5M2, 1), _operand(N, K, thc.THC_E4M3, 2)
    assert K * 64 < 2 ** 24                      # every partial sum is a whole number that fp32 holds
    want = (a[2].double() @ b[2].double().t()).float()
    ws = torch.full((thc.thc_fp8_matmul_workspace_bytes(M, N, K),), 0xCD, dtype=torch.uint8, device=DEV)
    whole = torch.full((M + 2, N + 5), 7.0, dtype=out, device=DEV)
    c = whole[1:M + 1, 2:N + 2]
    c.fill_(float("nan"))
    thc.thc_fp8_matmul(a[0], a[1], thc.THC_E5M2, b[0], b[1], thc.THC_E4M3, K, c, ws)
    assert torch.equal(c, want.to(out))
    start = c.clone().float()
    thc.thc_fp8_matmul(a[0], a[1], thc.THC_E5M2, b[0], b[1], thc.THC_E4M3, K, c, ws, True)
    assert torch.equal(c, (start + want).to(out))
    c.fill_(7.0)
    assert (whole == 7.0).all()                  # nothing beside it


@pytest.mark.parametrize("M,N,K", [(5632, 5888, 384), (9000, 4200, 1000), (4608, 4096, 1000)])
def test_same_bits_on_every_run(M, N, K):
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    ops = []
    for rows in (M, N):
        q = torch.empty(rows * thc.thc_fp8_row_bytes(K), dtype=torch.uint8, device=DEV)
        s = torch.empty(thc.thc_fp8_scale_bytes(rows, K), dtype=torch.uint8, device=DEV)
        thc.thc_fp8_quantize(torch.randn(rows, K, generator=g, device=DEV), thc.THC_E4M3, q, s)
        ops.append((q, s))
    ws = torch.empty(thc.thc_fp8_matmul_workspace_bytes(M, N, K), dtype=torch.uint8, device=DEV)
    first = None
    for i in range(4):
        c = torch.full((M, N), float(i), device=DEV)
        thc.thc_fp8_matmul(*ops[0], thc.THC_E4M3, *ops[1], thc.THC_E4M3, K, c, ws)
        first = c if first is None else first
        assert torch.equal(c, first)


@pytest.mark.parametrize("M,N", [(2, 5), (20, 36), (40, 36), (300, 200)])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_longest_sums(M, N, out):
    """2^22 along k, all but 5000 of them zero."""
    K = 1 << 22
    g = torch.Generator(device=DEV)
    g.manual_seed(M)
    at = torch.randperm(K - 1, generator=g, device=DEV)[:4999]
    at = torch.cat([at, torch.tensor([K - 1], device=DEV)])
    table = torch.tensor([0xC0, 0xB8, 0, 0x38, 0x40], dtype=torch.uint8, device=DEV)     # -2 .. 2 in e4m3
    ops = []
    for rows in (M, N):
        v = torch.randint(0, 5, (rows, 5000), generator=g, device=DEV)
        codes = torch.zeros(rows, K, dtype=torch.uint8, device=DEV)
        codes[:, at] = table[v]
        scales = torch.full((thc.thc_fp8_scale_bytes(rows, K),), 127, dtype=torch.uint8, device=DEV)
        ops.append((codes.reshape(-1), scales, (v - 2).double()))
    want = (ops[0][2] @ ops[1][2].t()).float()
    ws = torch.full((thc.thc_fp8_matmul_workspace_bytes(M, N, K),), 0xCD, dtype=torch.uint8, device=DEV)
    c = torch.full((M, N), float("nan"), dtype=out, device=DEV)
    thc.thc_fp8_matmul(ops[0][0], ops[0][1], thc.THC_E4M3, ops[1][0], ops[1][1], thc.THC_E4M3, K, c, ws)
    assert torch.equal(c, want.to(out))
