"""Plain 64-bit forms of the 8-bit floating-point products with a scale for
each block of 128 (the independent checks of the HIP kernels; torch tensors on
any device).

Values are rounded by nearest-value search in the table of a format's values,
products are formed in float64 from the values that quantised matrices stand
for.
"""

from __future__ import annotations

import math

import torch

BLOCK = 128
_SPEC = {torch.float8_e4m3fn: (3, -6, 448.0), torch.float8_e5m2: (2, -14, 57344.0)}


def table(fmt):
    """Nonnegative finite values of a format in order of their codes."""
    bits, least, top = _SPEC[fmt]
    ones = 1 << bits
    t = []
    for c in range(128):
        v = math.ldexp(c, least - bits) if c < ones else math.ldexp(ones + c % ones, c // ones - 1 + least - bits)
        if v <= top:
            t.append(v)
    return torch.tensor(t, dtype=torch.float64)


def nearest(v, fmt):
    """v (float64, |v| at most the largest value and a little) rounded to the
    format, ties to the even code; NaN and infinities as the conversion has
    them."""
    t = table(fmt).to(v.device)
    mid = (t[1:] + t[:-1]) / 2
    a = v.abs()
    finite = torch.isfinite(a)
    code = torch.searchsorted(mid, torch.where(finite, a, torch.zeros_like(a)))
    tie = (code < mid.numel()) & (mid[code.clamp(max=mid.numel() - 1)] == a)
    code = torch.where(tie & (code % 2 == 1), code + 1, code)
    q = torch.copysign(t[code], v)
    inf = v if fmt == torch.float8_e5m2 else torch.full_like(v, math.nan)
    return torch.where(finite, q, torch.where(torch.isnan(a), torch.full_like(v, math.nan), inf))


def _per_block(x, hr, hc):
    """Largest finite |x| of every hr x hc block."""
    r, c = x.shape
    a = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x))
    a = torch.nn.functional.pad(a, (0, -c % hc, 0, -r % hr))
    return a.reshape(a.shape[0] // hr, hr, a.shape[1] // hc, hc).amax((1, 3))


def spread(s, shape):
    """Scales (blocks of 128 where a dimension is shorter) for every element."""
    for d in (0, 1):
        if s.shape[d] != shape[d]:
            s = s.repeat_interleave(BLOCK, dim=d).narrow(d, 0, shape[d])
    return s


def quantize(x, dim, tile, fmt, pow2):
    """(values, scales) in float64 of x for blocks along dim."""
    top = _SPEC[fmt][2]
    x = x.double()
    a = _per_block(x, BLOCK if tile or dim == 0 else 1, BLOCK if tile or dim == 1 else 1)
    if pow2:
        powers = torch.tensor([math.ldexp(1.0, e) for e in range(-126, 128)], dtype=torch.float64, device=x.device)
        s = powers[torch.searchsorted(powers * top, a).clamp(max=253)]
    else:
        # a 24-bit number over 7 2^j is never half-way between two FP32 values,
        # nor within 2^-50 of it, so rounding twice is rounding once
        s = (a / torch.full_like(a, top)).float().double().clamp(min=2.0 ** -126)
    s = torch.where(a == 0, torch.ones_like(s), s)
    return nearest(x / spread(s, x.shape), fmt), s


def dequantize(q, s):
    return q.float().double() * spread(s.float().double(), q.shape)


def gemm(a, sa, b, sb):
    """(A B, |A| |B|) in float64: the product and the sum of its terms'
    magnitudes, which error bounds go by."""
    x, y = dequantize(a, sa), dequantize(b, sb).contiguous()
    return torch.matmul(x, y), torch.matmul(x.abs(), y.abs())


def sum_bound(k):
    """Relative to the sum of the terms' magnitudes, how far a sum of k terms
    in FP32 can be off, in any order, with every addition off by at most one
    unit (2^-23): one addition a term, and for every block a scale product, a
    multiplication and an addition."""
    blocks = (k + BLOCK - 1) // BLOCK
    return (k + 3 * blocks + 3) * 2.0 ** -23
