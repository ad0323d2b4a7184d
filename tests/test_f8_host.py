"""The 8-bit products on the host, without a GPU: calls that are refused before
any GPU work, the workspace sizes, and the plain form's own rounding."""

import ctypes

import pytest
import torch

from oracle import f8_blocks as plain
from paper_2608_06812_amd import ozfp4

P = 1 << 20            # an address that a refused call does not touch
EINVAL, EK, EWS = ozfp4.OZFP4_EINVAL, ozfp4.OZFP4_EKBOUND, ozfp4.OZFP4_EWORKSPACE


def mat(rs, cs, srs=1, scs=1, fmt=0, tile=0, values=P, scales=P):
    return ctypes.byref(ozfp4.F8Matrix(values, rs, cs, scales, srs, scs, fmt, tile))


def gemm(m=70, n=80, k=256, A=None, B=None, kind=0, C=P, ctype=1, c_rs=80, c_cs=1, add=0, ws=None, nbytes=0):
    A = mat(k, 1) if A is None else A
    B = mat(1, k) if B is None else B
    return ozfp4.ozfp4_gemm_f8(m, n, k, A, B, kind, C, ctype, c_rs, c_cs, add, ws, nbytes)


@pytest.mark.parametrize("kw,code", [
    (dict(m=-1), EINVAL), (dict(n=-1), EINVAL), (dict(k=-1), EINVAL),
    (dict(k=ozfp4.OZFP4_MAX_K_F8 + 1), EK),
    (dict(m=1 << 25, n=1 << 25, c_rs=1 << 25), EINVAL),
    (dict(m=1 << 20, n=1 << 20, c_rs=1 << 20), EINVAL),
    (dict(A=mat(255, 1)), EINVAL), (dict(A=mat(2, 2)), EINVAL), (dict(B=mat(1, 255)), EINVAL),
    (dict(A=mat(256, 1, fmt=2)), EINVAL), (dict(A=mat(256, 1, fmt=-1)), EINVAL),
    (dict(A=mat(256, 1, tile=2)), EINVAL), (dict(A=mat(256, 1, srs=-1)), EINVAL),
    (dict(A=mat(256, 1, srs=(1 << 22) + 1)), EINVAL), (dict(B=mat(1, 256, scs=(1 << 22) + 1)), EINVAL),
    (dict(A=mat(256, 1, values=None)), EINVAL), (dict(B=mat(1, 256, scales=None)), EINVAL),
    (dict(A=ctypes.POINTER(ozfp4.F8Matrix)()), EINVAL),
    (dict(kind=2), EINVAL), (dict(kind=-1), EINVAL), (dict(C=None), EINVAL),
    (dict(ctype=3), EINVAL), (dict(ctype=-1), EINVAL), (dict(c_rs=79), EINVAL), (dict(c_rs=2, c_cs=2), EINVAL),
    (dict(add=1), EINVAL), (dict(add=1, ctype=2), EINVAL),
    (dict(ws=P + 64, nbytes=1 << 20), EINVAL),
    (dict(A=mat(257, 1)), EWS), (dict(B=mat(88, 1)), EWS), (dict(A=mat(256, 1, values=P + 1)), EWS),
    (dict(B=mat(88, 1), ws=P, nbytes=80 * 256 - 1), EWS),
    (dict(m=0), 0), (dict(n=0), 0), (dict(k=0, A=mat(1, 1), B=mat(1, 1), ctype=0, add=1), 0),
])
def test_gemm_refusals(kw, code):
    assert gemm(**kw) == code


def test_workspace_sizes():
    """Nothing for operands that are read in place (the one along which C is
    adjacent in either order), the packed lines of the others (beside few lines
    on the other side only those whose k values are not adjacent)."""
    ask = lambda A, B, n=80: ozfp4.ozfp4_gemm_f8_workspace(100, n, 300, A, B, n, 1)
    assert ask(mat(304, 1), mat(1, 304)) == 0
    assert ask(mat(300, 1), mat(1, 304)) == 100 * 384
    assert ask(mat(304, 1), mat(80, 1)) == 0
    assert ask(mat(304, 1), mat(88, 1)) == 80 * 384
    assert ask(mat(1, 100), mat(80, 1)) == 100 * 384
    assert ask(mat(1, 112), mat(88, 1)) == 180 * 384
    assert ask(mat(300, 1), mat(1, 301), 30) == 0
    assert ask(mat(300, 1), mat(30, 1), 30) == 30 * 384
    assert ask(mat(304, 1, values=P + 8), mat(1, 304)) == 100 * 384
    with pytest.raises(ozfp4.OzFP4Error):
        ask(mat(10, 1), mat(1, 304))


def quantize(rows=10, cols=200, X=P, t=1, rs=200, cs=1, kind=0, one=None, two=None):
    return ozfp4.ozfp4_quantize_f8(rows, cols, X, t, rs, cs, kind, one, two)


@pytest.mark.parametrize("kw,code", [
    (dict(), EINVAL), (dict(one=mat(208, 1), X=None), EINVAL), (dict(one=mat(208, 1), t=3), EINVAL),
    (dict(one=mat(208, 1), kind=2), EINVAL), (dict(one=mat(208, 1), rs=199), EINVAL),
    (dict(one=mat(200, 1)), EINVAL), (dict(one=mat(192, 1)), EINVAL), (dict(one=mat(1, 208)), EINVAL),
    (dict(one=mat(208, 1, values=P + 8)), EINVAL), (dict(one=mat(208, 1, fmt=2)), EINVAL),
    (dict(one=mat(208, 1, scales=None)), EINVAL), (dict(two=mat(1, 10)), EINVAL), (dict(two=mat(16, 1)), EINVAL),
    (dict(one=mat(208, 1), two=mat(1, 16, fmt=1)), EINVAL), (dict(one=mat(208, 1), two=mat(1, 16, tile=1)), EINVAL),
    (dict(rows=-1, one=mat(208, 1)), EINVAL), (dict(rows=1 << 32, one=mat(208, 1)), EINVAL),
    (dict(rows=0, one=mat(208, 1)), 0),
])
def test_quantize_refusals(kw, code):
    assert quantize(**kw) == code


def linear(m=10, n=64, k=256, X=P, t=1, rs=256, cs=1, fmt=0, W=None, kind=0, Y=P, yt=1, yrs=64, ycs=1, ws=P,
           nbytes=1 << 30):
    return ozfp4.ozfp4_linear_f8(m, n, k, X, t, rs, cs, fmt, W or mat(k, 1), kind, Y, yt, yrs, ycs, ws, nbytes)


@pytest.mark.parametrize("kw,code", [
    (dict(m=-1), EINVAL), (dict(k=ozfp4.OZFP4_MAX_K_F8 + 1, rs=1 << 23), EK), (dict(X=None), EINVAL), (dict(t=4), EINVAL),
    (dict(rs=255), EINVAL), (dict(fmt=2), EINVAL), (dict(W=mat(255, 1)), EINVAL), (dict(kind=3), EINVAL),
    (dict(Y=None), EINVAL), (dict(yt=5), EINVAL), (dict(yrs=63), EINVAL), (dict(ws=P + 1), EINVAL),
    (dict(m=500, ws=None), EWS), (dict(m=500, nbytes=500 * 256), EWS), (dict(m=0), 0), (dict(n=0), 0),
])
def test_linear_refusals(kw, code):
    assert linear(**kw) == code


def backward(m=10, n=64, k=256, dY=P, X=P, t=1, yf=0, xf=0, W=None, kind=0, dX=P, dxt=1, dxs=(256, 1), dW=P,
             dws=(256, 1), add=0, ws=P, nbytes=1 << 30, ys=(64, 1), xs=(256, 1)):
    W = mat(k, 1, tile=1) if W is None else W
    return ozfp4.ozfp4_linear_f8_backward(m, n, k, dY, *ys, yf, X, *xs, xf, t, W, kind, dX, dxt, *dxs, dW, *dws, add,
                                          ws, nbytes)


@pytest.mark.parametrize("kw,code", [
    (dict(m=-1), EINVAL), (dict(m=ozfp4.OZFP4_MAX_K_F8 + 1), EK), (dict(W=mat(256, 1)), EINVAL),
    (dict(dY=None), EINVAL), (dict(X=None), EINVAL), (dict(t=3), EINVAL), (dict(yf=2), EINVAL), (dict(xf=2), EINVAL),
    (dict(dxt=3), EINVAL), (dict(dxs=(255, 1)), EINVAL), (dict(dws=(255, 1)), EINVAL), (dict(ys=(63, 1)), EINVAL),
    (dict(xs=(255, 1)), EINVAL), (dict(kind=2), EINVAL), (dict(nbytes=1000), EWS), (dict(ws=None), EWS),
    (dict(dX=None, dW=None), 0),
])
def test_backward_refusals(kw, code):
    assert backward(**kw) == code


def test_torch_helpers_refuse():
    x = torch.zeros((4, 256))
    q = torch.zeros((4, 256), dtype=torch.uint8).view(torch.float8_e4m3fn)
    s = torch.ones((4, 2))
    for call in (lambda: ozfp4.quantize_f8(x), lambda: ozfp4.quantize_f8_both(x), lambda: ozfp4.gemm_f8(q, s, q.t(), s.t()),
                 lambda: ozfp4.linear_f8(x, q, s), lambda: ozfp4.linear_f8_backward(x, x, q, s)):
        with pytest.raises(ValueError, match="device tensor"):
            call()
    for call in (lambda: ozfp4.quantize_f8([1.0]), lambda: ozfp4.quantize_f8(x[0]), lambda: ozfp4.gemm_f8(q[0], s, q, s)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError, match="dim"):
        ozfp4.quantize_f8(x, 2)
    with pytest.raises(TypeError, match="format"):
        ozfp4.quantize_f8(x, format=torch.int8)
    with pytest.raises(TypeError, match="scale"):
        ozfp4.quantize_f8(x, scale=torch.float64)


@pytest.mark.parametrize("fmt", [torch.float8_e4m3fn, torch.float8_e5m2])
def test_plain_rounding(fmt):
    """The plain form's table is torch's format, its rounding torch's cast
    where that rounds once (FP32 values), and its errors are at most half a
    step."""
    t = plain.table(fmt)
    assert torch.equal(t.to(fmt).double(), t) and float(t[-1]) == torch.finfo(fmt).max
    v = torch.randn(20000, dtype=torch.float32) * torch.exp(3 * torch.randn(20000))
    v = v.clamp(-float(t[-1]), float(t[-1]))
    q = plain.nearest(v.double(), fmt)
    assert torch.equal(q, v.to(fmt).double())
    half = torch.finfo(fmt).eps / 2
    least = float(t[1])
    assert ((q - v.double()).abs() <= torch.maximum(half * v.double().abs(), torch.tensor(least / 2))).all()


@pytest.mark.parametrize("pow2", [False, True])
def test_plain_scales(pow2):
    """Scales are the least (a power of two, or FP32 to a rounding) that bring
    a block to the format's range."""
    x = torch.randn(300, 500).double().float() * torch.exp(5 * torch.randn(300, 1))
    for fmt in (torch.float8_e4m3fn, torch.float8_e5m2):
        top = float(plain.table(fmt)[-1])
        for dim, tile in ((0, False), (1, False), (0, True)):
            q, s = plain.quantize(x, dim, tile, fmt, pow2)
            off = (plain.spread(s, x.shape) * q - x.double()).abs()
            least = float(plain.table(fmt)[1])
            bound = torch.maximum(torch.finfo(fmt).eps / 2 * x.double().abs() * (1 + 2.0 ** -20),
                                  plain.spread(s, x.shape) * least / 2)
            assert (off <= bound).all() and q.abs().max() <= top
            assert q.abs().max() > (top / 2 if pow2 else top * 0.99)
