"""8-bit products over the values that codes and scales can stand for: blocks with the lowest scales, blocks that are marked,
codes that are not finite, zeros of both signs; in each of the forms in which a product is done."""
import numpy as np
import pytest
import torch

import paper_2407_01378_amd as thc
from oracle import fp8 as O

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
CODE = {"e4m3": thc.THC_E4M3, "e5m2": thc.THC_E5M2}
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
K = 640
# straight from memory: one row, few rows, tiles of 64 (fp32 results; bf16: 128); through LDS: tiles of 128, tiles of 256
FORMS = [(1, 300), (20, 300), (640, 640), (130, 260), (4090, 4000)]


def _operand(rows, fmt, numbers, seed, scales):
    """(codes, scale bytes of every block, values) of rows x K; `numbers` has a code for each entry."""
    rng = np.random.default_rng(seed)
    table = O.code_values(fmt)
    which = np.array([int(np.flatnonzero(table == v)[0]) for v in numbers], dtype=np.uint8)
    codes = which[rng.integers(0, len(which), (rows, K))]
    e = rng.choice(np.array(scales, dtype=np.uint8), (rows, K // 128))
    return codes, e


def _on_gpu(codes, e, fmt):
    values = torch.tensor(O.code_values(fmt), device=DEV)[torch.tensor(codes, device=DEV).long()]
    scale = np.where(e == 255, np.nan, 2.0 ** (e.astype(float) - 127.0))
    return (torch.tensor(codes.reshape(-1), device=DEV), torch.tensor(O.pack_scales(e), device=DEV),
            values * torch.tensor(scale, device=DEV).repeat_interleave(128, 1))


def _product(a, fa, b, fb, out, M, N):
    c = torch.full((M, N), 7.0, dtype=DT[out], device=DEV)
    n = thc.thc_fp8_matmul_workspace_bytes(M, N, K)
    ws = torch.full((n,), 0xCD, dtype=torch.uint8, device=DEV) if n else None
    return thc.thc_fp8_matmul(a[0], a[1], CODE[fa], b[0], b[1], CODE[fb], K, c, ws)


@pytest.mark.parametrize("fa,fb", [("e4m3", "e4m3"), ("e5m2", "e4m3")])
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("M,N", FORMS)
def test_lowest_scales(M, N, out, fa, fb):
    """Scale bytes 0 and 1 stand for 2^-127 and 2^-126: codes of 2 and more are normal fp32 numbers there."""
    for low, high in ((0, 1), (1, 0)):   # which operand has them
        ops = []
        for side, (rows, fmt) in enumerate(((M, fa), (N, fb))):
            mine = (low, high)[side] == 0
            ops.append(_on_gpu(*_operand(rows, fmt, (2, -2, 3, -3, 4, -4, 0) if mine else (1, -1, 2, -2, 0), 5 + side,
                                         (0, 1) if mine else (227, 228)), fmt))
        want = ops[0][2] @ ops[1][2].t()
        # whole multiples of 2^-27, every sum of magnitudes below 2^-27 * 2^24: exact in fp32
        assert float((ops[0][2].abs() @ ops[1][2].abs().t()).max()) < 2.0 ** -3 and torch.equal(want.float().double(), want)
        assert want.any()
        assert torch.equal(_product(ops[0], fa, ops[1], fb, out, M, N), want.float().to(DT[out]))


@pytest.mark.parametrize("fa,fb", [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2")])
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("M,N", FORMS)
def test_blocks_that_are_marked(M, N, out, fa, fb):
    """Scale byte 255 stands for NaN whatever the block's codes are: the row's and the column's results, and no other."""
    numbers, scales = (1, -1, 2, -2, 0), (126, 127, 128)
    (ca, ea), (cb, eb) = _operand(M, fa, numbers, 1, scales), _operand(N, fb, numbers, 2, scales)
    ea[M // 2, 2] = 255
    eb[7, 4] = eb[N - 1, 0] = 255
    cb[7, 512:] = 0
    cb[N - 1, :128] = O.NAN_CODE
    a, b = _on_gpu(ca, ea, fa), _on_gpu(cb, eb, fb)
    want = torch.zeros(M, N, dtype=torch.bool, device=DEV)
    want[M // 2], want[:, 7], want[:, N - 1] = True, True, True
    c = _product(a, fa, b, fb, out, M, N)
    assert torch.equal(c.isnan(), want)
    exact = (a[2].nan_to_num(nan=0.0) @ b[2].nan_to_num(nan=0.0).t()).float().to(DT[out])
    assert torch.equal(c[~want], exact[~want])


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("M,N", FORMS)
@pytest.mark.parametrize("tile", [False, True])
def test_quantized_values_that_are_not_finite(M, N, out, tile):
    """As they come from the quantizer: a NaN or an infinity takes its block (tile) with it."""
    x = torch.randn(M, K, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV)
    w = torch.randn(N, K, generator=torch.Generator(device=DEV).manual_seed(2), device=DEV)
    x[M // 2, 600] = -float("inf")
    w[N // 2, 3] = float("nan")
    ops = []
    for m in (x, w):
        q = torch.empty(m.shape[0] * thc.thc_fp8_row_bytes(K), dtype=torch.uint8, device=DEV)
        s = torch.empty(thc.thc_fp8_scale_bytes(m.shape[0], K), dtype=torch.uint8, device=DEV)
        thc.thc_fp8_quantize(m, thc.THC_E4M3, q, s, None, None, tile)
        ops.append((q, s))
    want = torch.zeros(M, N, dtype=torch.bool, device=DEV)
    for i, rows in ((0, M), (1, N)):
        first = rows // 2 // 128 * 128
        hit = slice(first, first + 128) if tile else slice(rows // 2, rows // 2 + 1)
        if i:
            want[:, hit] = True
        else:
            want[hit] = True
    assert torch.equal(_product(ops[0], "e4m3", ops[1], "e4m3", out, M, N).isnan(), want)
    if not tile:
        n = thc.thc_fp8_linear_workspace_bytes(M, N, K)
        y = torch.full((M, N), 7.0, dtype=DT[out], device=DEV)
        thc.thc_fp8_linear(x, thc.THC_E4M3, *ops[1], thc.THC_E4M3, y, torch.empty(n, dtype=torch.uint8, device=DEV) if n else None)
        assert torch.equal(y.isnan(), want)


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("M,N", FORMS)
def test_codes_that_are_not_finite(M, N, out):
    """e5m2 has infinities, both formats have NaN codes."""
    numbers, scales = (1, -1, 2, -2, 0), (126, 127, 128)
    (ca, ea), (cb, eb) = _operand(M, "e5m2", numbers, 1, scales), _operand(N, "e4m3", numbers, 2, scales)
    ca[M // 2, 300] = 0x7C          # infinity; times zero it is a NaN
    ca[M - 1, 301] = 0xFC
    if M > 2:
        ca[0, 5] = 0x7D             # NaN
    cb[N // 3, 639] = 0xFF
    a, b = _on_gpu(ca, ea, "e5m2"), _on_gpu(cb, eb, "e4m3")
    fine = a[2].isfinite(), b[2].isfinite()
    want = torch.where(fine[0], a[2], 0.0) @ torch.where(fine[1], b[2], 0.0).t()
    for i, k in (~fine[0]).nonzero().tolist():
        want[i] += a[2][i, k] * b[2][:, k]
    for j, k in (~fine[1]).nonzero().tolist():
        want[:, j] += a[2][:, k] * b[2][j, k]
    assert want.isinf().any() and want.isnan().any() and (M == 1 or want.isfinite().any())
    assert torch.equal(_product(a, "e5m2", b, "e4m3", out, M, N).double().nan_to_num(nan=0.5),
                       want.float().to(DT[out]).double().nan_to_num(nan=0.5))


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_every_code_and_scale_back(fmt, out):
    """Every code at every scale, zeros with their signs."""
    codes = np.tile(np.arange(256, dtype=np.uint8), (256, 1))
    e = np.repeat(np.arange(256, dtype=np.uint8)[:, None], 2, 1)
    v = torch.empty(256, 256, dtype=DT[out], device=DEV)
    thc.thc_fp8_dequantize(torch.tensor(codes.reshape(-1), device=DEV), torch.tensor(O.pack_scales(e), device=DEV), CODE[fmt], v)
    with np.errstate(over="ignore", invalid="ignore"):
        want = torch.tensor(O.values(codes, e, fmt, 256).astype(np.float32)).to(DT[out])
    got = v.cpu()
    assert torch.equal(got.isnan(), want.isnan())
    bits = torch.int32 if out == "f32" else torch.int16
    assert torch.equal(got.view(bits)[~want.isnan()], want.view(bits)[~want.isnan()])
