"""The entry points of the training step without a GPU: sizes, refusals of the library (dummy addresses are never
used) and of the binding."""
import ctypes

import pytest
import torch

import paper_2407_01378_amd as thc

P, NUL, ODD = ctypes.c_void_p(0x1000), ctypes.c_void_p(0), ctypes.c_void_p(0x1008)
E4M3, E5M2, F32, BF16, I32, I64 = thc.THC_E4M3, thc.THC_E5M2, thc.THC_F32, thc.THC_BF16, thc.THC_I32, thc.THC_I64
BIG = 1 << 31


@pytest.fixture(scope="module")
def L():
    return thc.lib()


def test_sizes(L):
    assert [thc.thc_fp8_row_bytes(n) for n in (0, 1, 128, 129, 1 << 22, (1 << 22) + 1)] == [0, 128, 128, 256, 1 << 22, 0]
    assert thc.thc_fp8_scale_bytes(0, 100) == 0 and thc.thc_fp8_scale_bytes(3, 0) == 0
    assert thc.thc_fp8_scale_bytes(3, 512) == 12 and thc.thc_fp8_scale_bytes(3, 513) == 24
    assert thc.thc_fp8_scale_bytes(BIG, 1) == 0 and thc.thc_fp8_scale_bytes(1, (1 << 22) + 1) == 0
    for fn in (thc.thc_fp8_matmul_workspace_bytes, thc.thc_fp8_linear_workspace_bytes):
        assert fn(BIG, 1, 1) == 0 and fn(1, BIG, 1) == 0 and fn(1, 1, (1 << 22) + 1) == 0
    assert thc.thc_embed_backward_workspace_bytes(BIG, 1, 1) == 0
    assert thc.thc_embed_backward_workspace_bytes(1 << 24, 10, 1 << 20) == 0


def quantize(L, x=P, dt=F32, rows=4, cols=200, ld=200, fmt=E4M3, tile=0, q=P, s=P, qt=NUL, st=NUL):
    return L.thc_fp8_quantize(x, dt, rows, cols, ld, fmt, tile, q, s, qt, st, NUL)


def dequantize(L, q=P, s=P, fmt=E4M3, rows=4, cols=200, dt=F32, out=P, ld=200):
    return L.thc_fp8_dequantize(q, s, fmt, rows, cols, dt, out, ld, NUL)


def matmul(L, a=P, sa=P, fa=E4M3, b=P, sb=P, fb=E4M3, M=4, N=8, K=200, dt=F32, c=P, ldc=8, ws=P, wb=1 << 60):
    return L.thc_fp8_matmul(a, sa, fa, b, sb, fb, M, N, K, 0, dt, c, ldc, ws, wb, NUL)


def linear(L, x=P, dt=F32, M=4, K=200, ldx=200, fx=E4M3, b=P, sb=P, fb=E4M3, N=8, odt=F32, out=P, ldo=8, ws=P,
           wb=1 << 60):
    return L.thc_fp8_linear(x, dt, M, K, ldx, fx, b, sb, fb, N, odt, out, ldo, ws, wb, NUL)


def lookup(L, table=P, dt=F32, vocab=10, dim=8, ld=8, tokens=P, index=I64, count=4, odt=F32, out=P, ldo=8):
    return L.thc_embed_forward(table, dt, vocab, dim, ld, tokens, index, count, 1.0, odt, out, ldo, NUL)


def gradient(L, g=P, dt=F32, ld=8, tokens=P, index=I64, count=4, vocab=10, dim=8, add=0, odt=F32, table=P, ldt=8, ws=P,
             wb=1 << 60):
    return L.thc_embed_backward(g, dt, ld, tokens, index, count, vocab, dim, 1.0, add, odt, table, ldt, ws, wb, NUL)


def test_library_refuses(L):
    for bad in (dict(dt=2), dict(fmt=2), dict(fmt=-1)):
        assert quantize(L, **bad) == -5
    for bad in (dict(ld=199), dict(rows=BIG), dict(cols=BIG, ld=BIG), dict(cols=(1 << 22) + 1, ld=1 << 23),
                dict(q=NUL, s=NUL, qt=P, st=P, rows=(1 << 22) + 1), dict(ld=1 << 63)):
        assert quantize(L, **bad) == -6, bad
    for bad in (dict(x=NUL), dict(q=NUL), dict(s=NUL), dict(qt=P), dict(st=P), dict(q=NUL, s=NUL)):
        assert quantize(L, **bad) == -1, bad
    for bad in (dict(x=ctypes.c_void_p(0x1002)), dict(dt=BF16, x=ctypes.c_void_p(0x1001)), dict(q=ODD), dict(s=ODD),
                dict(qt=ODD, st=P), dict(qt=P, st=ODD)):
        assert quantize(L, **bad) == -8, bad
    for bad, status in ((dict(fmt=2), -5), (dict(dt=2), -5), (dict(q=NUL), -1), (dict(s=NUL), -1), (dict(out=NUL), -1),
                        (dict(ld=199), -6), (dict(rows=BIG), -6), (dict(cols=(1 << 22) + 1, ld=1 << 23), -6),
                        (dict(q=ODD), -8), (dict(s=ODD), -8), (dict(out=ctypes.c_void_p(0x1002)), -8)):
        assert dequantize(L, **bad) == status, bad
    for bad, status in ((dict(fa=2), -5), (dict(fb=-1), -5), (dict(dt=2), -5), (dict(a=NUL), -1), (dict(sa=NUL), -1),
                        (dict(b=NUL), -1), (dict(sb=NUL), -1), (dict(c=NUL), -1), (dict(ldc=7), -6), (dict(M=BIG), -6),
                        (dict(N=BIG, ldc=BIG), -6), (dict(K=(1 << 22) + 1), -6), (dict(a=ODD), -8), (dict(sa=ODD), -8),
                        (dict(b=ODD), -8), (dict(sb=ODD), -8), (dict(c=ctypes.c_void_p(0x1002)), -8)):
        assert matmul(L, **bad) == status, bad
    for bad, status in ((dict(dt=2), -5), (dict(odt=2), -5), (dict(fx=2), -5), (dict(fb=2), -5), (dict(x=NUL), -1),
                        (dict(b=NUL), -1), (dict(sb=NUL), -1), (dict(out=NUL), -1), (dict(ldx=199), -6),
                        (dict(ldo=7), -6), (dict(M=BIG), -6), (dict(K=(1 << 22) + 1, ldx=1 << 23), -6), (dict(b=ODD), -8),
                        (dict(x=ctypes.c_void_p(0x1002)), -8), (dict(out=ctypes.c_void_p(0x1001), odt=BF16), -8)):
        assert linear(L, **bad) == status, bad
    for bad, status in ((dict(dt=2), -5), (dict(odt=2), -5), (dict(index=2), -5), (dict(table=NUL), -1),
                        (dict(tokens=NUL), -1), (dict(out=NUL), -1), (dict(ld=7), -6), (dict(ldo=7), -6),
                        (dict(count=BIG), -6), (dict(vocab=BIG), -6), (dict(dim=BIG, ld=BIG, ldo=BIG), -6),
                        (dict(tokens=ctypes.c_void_p(0x1004)), -8), (dict(table=ctypes.c_void_p(0x1002)), -8)):
        assert lookup(L, **bad) == status, bad
    for bad, status in ((dict(dt=2), -5), (dict(odt=2), -5), (dict(index=-1), -5), (dict(g=NUL), -1),
                        (dict(tokens=NUL), -1), (dict(table=NUL), -1), (dict(ld=7), -6), (dict(ldt=7), -6),
                        (dict(count=BIG), -6), (dict(vocab=BIG), -6), (dict(count=1 << 24, dim=1 << 20, ld=1 << 20, ldt=1 << 20), -6),
                        (dict(tokens=ctypes.c_void_p(0x1004)), -8), (dict(g=ctypes.c_void_p(0x1002)), -8)):
        assert gradient(L, **bad) == status, bad


def test_workspaces_are_checked(L):
    need = thc.thc_fp8_linear_workspace_bytes(4, 8, 200)
    if need:
        assert linear(L, wb=need - 1) == -6 and linear(L, ws=NUL) == -1 and linear(L, ws=ODD) == -8
    for M, N, K in ((4, 8, 200), (64, 64, 1 << 16), (256, 256, 1 << 20)):
        need = thc.thc_fp8_matmul_workspace_bytes(M, N, K)
        if need:
            assert matmul(L, M=M, N=N, K=K, ldc=N, wb=need - 1) == -6
            assert matmul(L, M=M, N=N, K=K, ldc=N, ws=NUL) == -1 and matmul(L, M=M, N=N, K=K, ldc=N, ws=ODD) == -8
    need = thc.thc_embed_backward_workspace_bytes(4, 10, 8)
    if need:
        assert gradient(L, wb=need - 1) == -6 and gradient(L, ws=NUL) == -1 and gradient(L, ws=ODD) == -8


def test_nothing_to_do(L):
    assert quantize(L, rows=0, x=NUL) == 0 and quantize(L, cols=0, x=NUL, q=NUL, s=NUL) == 0
    assert dequantize(L, rows=0, q=NUL) == 0 and dequantize(L, cols=0, out=NUL) == 0
    assert matmul(L, M=0, a=NUL, c=NUL) == 0 and matmul(L, N=0, b=NUL, c=NUL) == 0
    assert linear(L, M=0, x=NUL, out=NUL) == 0 and linear(L, N=0, b=NUL, out=NUL) == 0
    assert lookup(L, count=0, tokens=NUL, out=NUL) == 0 and lookup(L, dim=0, table=NUL, out=NUL) == 0
    assert gradient(L, vocab=0, table=NUL) == 0 and gradient(L, dim=0, table=NUL) == 0
    assert gradient(L, count=0, add=1, table=NUL) == 0


def _u8(n):
    return torch.zeros(n, dtype=torch.uint8)


def test_binding_refuses():
    x, q, s = torch.zeros(4, 200), _u8(4 * 256), _u8(16)
    fine = dict(x=x, format=E4M3, q=q, scales=s)
    for bad, error in ((dict(x=x.double()), TypeError), (dict(x=x[0]), ValueError), (dict(x=x.t()), ValueError),
                       (dict(x=x[:1].expand(4, 200)), ValueError), (dict(q=_u8(1023)), ValueError),
                       (dict(scales=_u8(15)), ValueError), (dict(scales=None), ValueError),
                       (dict(q=torch.zeros(1024)), TypeError), (dict(q_t=_u8(1 << 16)), ValueError),
                       (dict(q_t=_u8(200 * 128 - 1), scales_t=_u8(800)), ValueError), (dict(), ValueError)):
        with pytest.raises(error):   # (the last: not on a GPU)
            thc.thc_fp8_quantize(**dict(fine, **bad))
    c = torch.zeros(4, 8)
    fine = dict(a=q, a_scales=s, a_format=E4M3, b=_u8(8 * 256), b_scales=_u8(32), b_format=E4M3, K=200, c=c)
    for bad, error in ((dict(a=_u8(1023)), ValueError), (dict(b=_u8(2047)), ValueError), (dict(b_scales=_u8(31)), ValueError),
                       (dict(c=c[:, ::2]), ValueError), (dict(c=c.half()), TypeError), (dict(K=400), ValueError),
                       (dict(workspace=_u8(64)[::2]), ValueError), (dict(), ValueError)):
        with pytest.raises(error):
            thc.thc_fp8_matmul(**dict(fine, **bad))
    fine = dict(x=x, x_format=E4M3, b=_u8(8 * 256), b_scales=_u8(32), b_format=E4M3, out=c)
    for bad, error in ((dict(out=c[:3]), ValueError), (dict(out=c[0]), ValueError), (dict(b=_u8(2047)), ValueError),
                       (dict(x=x.half()), TypeError), (dict(), ValueError)):
        with pytest.raises(error):
            thc.thc_fp8_linear(**dict(fine, **bad))
    out = torch.zeros(4, 200)
    for bad, error in ((dict(q=_u8(1)), ValueError), (dict(out=out.long()), TypeError), (dict(), ValueError)):
        with pytest.raises(error):
            thc.thc_fp8_dequantize(**dict(dict(q=q, scales=s, format=E4M3, out=out), **bad))
    table, tokens = torch.zeros(10, 8), torch.zeros(4, dtype=torch.int64)
    for bad, error in ((dict(tokens=tokens.float()), TypeError), (dict(tokens=tokens[::2]), ValueError),
                       (dict(out=c[:3]), ValueError), (dict(table=table.t()), ValueError), (dict(), ValueError)):
        with pytest.raises(error):
            thc.thc_embed_forward(**dict(dict(table=table, tokens=tokens, scale=1.0, out=c), **bad))
    fine = dict(grad_out=c, tokens=tokens, scale=1.0, grad_table=table, workspace=_u8(1 << 16))
    for bad, error in ((dict(grad_out=c[:3]), ValueError), (dict(grad_out=c[:1].expand(4, 8)), ValueError),
                       (dict(grad_table=torch.zeros(10, 7)), ValueError), (dict(tokens=tokens.view(2, 2)), ValueError),
                       (dict(), ValueError)):
        with pytest.raises(error):
            thc.thc_embed_backward(**dict(fine, **bad))
