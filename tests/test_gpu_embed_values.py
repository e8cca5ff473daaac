"""Embedding lookup and gradient: zeros keep their sign, infinities stay infinities."""
import pytest
import torch

import paper_2407_01378_amd as thc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BITS = {torch.float32: torch.int32, torch.bfloat16: torch.int16}


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dim", [1, 7, 8, 13, 64, 1001])
@pytest.mark.parametrize("scale", [1.0, -2.5, 0.0])
def test_lookup_bit_by_bit(dt, out, dim, scale):
    g = torch.Generator(device=DEV)
    g.manual_seed(dim)
    table = torch.randn(30, dim, generator=g, device=DEV)
    table[::2] = 0.0
    table[4::4] = -0.0
    table[7, ::3] = -0.0
    table = table.to(dt)
    tokens = torch.randint(-2, 32, (200,), generator=g, device=DEV)
    y = torch.full((200, dim), 9.0, dtype=out, device=DEV)
    thc.thc_embed_forward(table, tokens, scale, y)
    want = table[tokens.clamp(0, 29)].float() * torch.tensor(scale, device=DEV)
    want[(tokens < 0) | (tokens >= 30)] = 0.0
    assert torch.equal(y.view(BITS[out]), want.to(out).view(BITS[out]))


@pytest.mark.parametrize("dim", [3, 8, 13, 1001])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_zeros_that_are_added_to(dim, out):
    """old + scale * sum, a sum of zeros being +0: -0 where both are -0, in every column alike."""
    for count in (50, 7000):
        g, tokens = torch.zeros(count, dim, device=DEV), torch.arange(count, device=DEV) % 5
        ws = torch.empty(thc.thc_embed_backward_workspace_bytes(count, 9, dim), dtype=torch.uint8, device=DEV)
        for old in (-0.0, 0.0):
            for scale in (-1.0, 1.0):
                grad = torch.full((9, dim), old, dtype=out, device=DEV)
                thc.thc_embed_backward(g, tokens, scale, grad, ws, True)
                want = torch.full((9, dim), old, dtype=out, device=DEV)
                want[:5] = old + scale * 0.0
                assert torch.equal(grad.view(BITS[out]), want.view(BITS[out]))


@pytest.mark.parametrize("dim", [5, 16, 1001])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_values_that_are_not_finite(dim, out):
    inf, nan = float("inf"), float("nan")
    table = torch.ones(12, dim, device=DEV)
    table[1, 0], table[2, dim - 1], table[3, 1] = inf, -inf, nan
    tokens = torch.tensor([3, 2, 1, 0, -1, 12], device=DEV)
    y = torch.empty(6, dim, dtype=out, device=DEV)
    thc.thc_embed_forward(table, tokens, -2.0, y)
    want = table[tokens.clamp(0, 11)] * -2.0
    want[4:] = 0.0
    assert torch.equal(y.isnan(), want.isnan()) and torch.equal(y.float().nan_to_num(nan=0.5), want.nan_to_num(nan=0.5))
    for count in (40, 7000):                                # both ways to sort
        g = torch.ones(count, dim, device=DEV)
        tokens = torch.arange(count, device=DEV) % 10
        g[13, 0], g[24, dim - 1], g[37, 1], g[17, 1] = inf, -inf, inf, -inf
        g[15, 0] = nan
        grad = torch.empty(12, dim, dtype=out, device=DEV)
        ws = torch.empty(thc.thc_embed_backward_workspace_bytes(count, 12, dim), dtype=torch.uint8, device=DEV)
        thc.thc_embed_backward(g, tokens, -1.0, grad, ws)
        want = torch.zeros(12, dim, device=DEV)
        want[:10] = -float(count // 10)
        want[3, 0], want[4, dim - 1], want[7, 1], want[5, 0] = -inf, inf, nan, nan
        want = want.to(out)
        assert torch.equal(grad.isnan(), want.isnan())
        assert torch.equal(grad.float().nan_to_num(nan=0.5), want.float().nan_to_num(nan=0.5))
