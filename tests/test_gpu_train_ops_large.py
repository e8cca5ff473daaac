"""Embedding and 8-bit matrices beyond the sizes at which a grid, the sort's tiles and passes or the pieces of the sums change;
exactly, on whole numbers."""
import pytest
import torch

import paper_2407_01378_amd as thc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _ws(count, vocab, dim):
    return torch.full((thc.thc_embed_backward_workspace_bytes(count, vocab, dim),), 0xCD, dtype=torch.uint8, device=DEV)


def _tokens(count, vocab, kind, seed):
    g = _gen(seed)
    if kind == "uniform":
        return torch.randint(0, vocab, (count,), generator=g, device=DEV)
    if kind == "padded":
        t = torch.randint(0, vocab, (count,), generator=g, device=DEV)
        t[torch.rand(count, generator=g, device=DEV) < 0.6] = -1
        return t
    if kind == "mostly one":     # a padding mark that is a row of the table
        t = torch.randint(0, vocab, (count,), generator=g, device=DEV)
        t[torch.rand(count, generator=g, device=DEV) < 0.95] = vocab // 3
        return t
    if kind == "one":
        return torch.full((count,), vocab - 1, device=DEV)
    far = torch.tensor([-2 ** 63, 2 ** 63 - 1, -2 ** 31, 2 ** 31, 2 ** 32, 0, vocab - 1, vocab], device=DEV)   # "far"
    return far[torch.randint(0, 8, (count,), generator=g, device=DEV)]


@pytest.mark.parametrize("kind", ["uniform", "padded", "mostly one", "one", "far"])
@pytest.mark.parametrize("count,vocab,dim", [
    (32768, 3000, 24), (32769, 3000, 24),               # pieces of 16 entries, and of 17
    (65536, 70000, 17), (65537, 70000, 17),             # tiles of the sort of 256 keys, and of 512
    (300001, 2047, 8), (300001, 2048, 8),               # one pass of the sort, and two
    (7000, (1 << 22) - 1, 5), (7000, 1 << 22, 5),       # two passes, and three
    (70001, (1 << 25) + 77, 3), (900, (1 << 25) + 77, 3),   # more rows than workgroups that look after them
    (40000, 300, 1030)])
def test_gradient(kind, count, vocab, dim):
    g = torch.randint(-4, 5, (count, dim), generator=_gen(1), device=DEV).float()   # (sums below 2^24)
    tokens = _tokens(count, vocab, kind, 2)
    valid = (tokens >= 0) & (tokens < vocab)
    want = torch.zeros(vocab, dim, device=DEV).index_add_(0, tokens[valid], g[valid])   # (exact too)
    table = torch.full((vocab, dim), float("nan"), device=DEV)
    thc.thc_embed_backward(g.bfloat16(), tokens, 2.0, table, _ws(count, vocab, dim))
    assert torch.equal(table, 2 * want)
    thc.thc_embed_backward(g, tokens, -1.0, table, _ws(count, vocab, dim), True)
    assert torch.equal(table, want)


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_lookup_of_many(dt):
    """More than 2^28 pieces of 8 values, a result beyond 4 GiB; tokens far outside the table."""
    vocab, dim, count = 50, 1024, (1 << 21) + 3
    table = torch.randn(vocab, dim, generator=_gen(3), device=DEV)
    tokens = _tokens(count, vocab, "far", 4)
    tokens[::2] = torch.randint(0, vocab, (tokens[::2].numel(),), generator=_gen(5), device=DEV)
    y = torch.full((count, dim), 9.0, dtype=dt, device=DEV)
    thc.thc_embed_forward(table, tokens, 0.5, y)
    rows = torch.cat([(table * 0.5).to(dt), torch.zeros(1, dim, dtype=dt, device=DEV)])
    at = torch.where((tokens < 0) | (tokens >= vocab), vocab, tokens)
    for i in range(0, count, 1 << 18):
        assert torch.equal(y[i:i + (1 << 18)], rows[at[i:i + (1 << 18)]])


def test_a_table_without_rows():
    y = torch.full((3, 40), 9.0, device=DEV)
    thc.thc_embed_forward(torch.empty(0, 40, device=DEV), torch.tensor([0, -1, 5], device=DEV), 1.0, y)
    assert not y.any()
    grad = torch.empty(0, 40, device=DEV)
    thc.thc_embed_backward(y, torch.tensor([0, -1, 5], device=DEV), 1.0, grad, None)


@pytest.mark.parametrize("fmt", [thc.THC_E4M3, thc.THC_E5M2])
def test_many_rows_there_and_back(fmt):
    """More rows than workgroups take at a time, both ways; values that 8 bits hold."""
    for rows, cols, back in (((1 << 23) + 5, 3, torch.float32), ((1 << 21) + 5, 1024, torch.bfloat16)):
        x = torch.randint(-4, 5, (rows, cols), generator=_gen(cols), device=DEV, dtype=torch.int8).to(torch.bfloat16)
        q = torch.full((rows * thc.thc_fp8_row_bytes(cols),), 0xAB, dtype=torch.uint8, device=DEV)
        s = torch.full((thc.thc_fp8_scale_bytes(rows, cols),), 0xAB, dtype=torch.uint8, device=DEV)
        v = torch.full((rows, cols), 9.0, dtype=back, device=DEV)
        thc.thc_fp8_quantize(x, fmt, q, s)
        thc.thc_fp8_dequantize(q, s, fmt, v)
        assert torch.equal(v, x.to(back))
        assert not q.view(rows, -1)[:, cols:].any()


@pytest.mark.parametrize("tile", [False, True])
def test_a_long_row_transposed(tile):
    """2^20 tiles and two more: q_t has a row of 128 codes for each of x's columns."""
    cols = (1 << 27) + 200
    x = torch.randint(-4, 5, (1, cols), generator=_gen(6), device=DEV, dtype=torch.int8).to(torch.bfloat16)
    q = torch.empty(cols * 128, dtype=torch.uint8, device=DEV)
    s = torch.empty(4 * cols, dtype=torch.uint8, device=DEV)
    thc.thc_fp8_quantize(x, thc.THC_E4M3, None, None, q, s, tile)
    v = torch.empty(cols, 1, dtype=torch.bfloat16, device=DEV)
    thc.thc_fp8_dequantize(q, s, thc.THC_E4M3, v)
    assert torch.equal(v.view(-1), x.view(-1))


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_empty_sums_of_many(out):
    e = torch.empty(0, dtype=torch.uint8, device=DEV)
    c = torch.full((3000, 1001), 3.0, dtype=out, device=DEV)
    thc.thc_fp8_matmul(e, e, 0, e, e, 0, 0, c[:, :1000], None)
    assert not c[:, :1000].any() and (c[:, 1000] == 3.0).all()
