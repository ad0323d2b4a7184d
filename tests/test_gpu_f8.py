"""The 8-bit floating-point products on the GPU against plain 64-bit forms
(oracle/f8_blocks.py): quantisation value for value, products within a bound
that counts the roundings, at the sizes, layouts, types and special values
where the kernels' paths differ; streams, graphs and untouched memory around
the outputs.

Tolerances: a product of k terms is off by at most sum_bound(k) times the sum
of its terms' magnitudes (every FP32 addition by one unit), with outputs of 16
bits by EIGHTS more (the 8-bit matrix instruction cuts eight products at less
than 2^-13 of the largest of them), then rounded once to its type (half a
step), or, where the value is subnormal in fp16, by half of fp16's least
step."""

import pytest
import torch

from gpu_util import announce
from oracle import f8_blocks as plain

pytestmark = pytest.mark.gpu

E4, E5 = torch.float8_e4m3fn, torch.float8_e5m2
F32, E8 = torch.float32, torch.float8_e8m0fnu
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}

EIGHTS = 8 * 2.0 ** -13


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def rand(shape, seed, dtype=torch.float32):
    g = gen(seed)
    x = torch.randn(shape, device="cuda", generator=g)
    x *= torch.exp(2 * torch.randn((shape[0], 1), device="cuda", generator=g))
    return (x * torch.exp(torch.randn((1, shape[1]), device="cuda", generator=g))).to(dtype)


def same_values(got, want):
    """8-bit values against the float64 ones: equal, zeros with their signs,
    NaN in the same places."""
    got = got.float().double()
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan)
    got, want = got[~nan], want[~nan]
    assert torch.equal(got, want)
    assert torch.equal(torch.signbit(got), torch.signbit(want))


def close(got, want, mags, k, before=None):
    """got against the float64 product `want` whose terms' magnitudes sum to
    `mags`, added to `before`."""
    slack = (plain.sum_bound(k) + (0 if got.dtype == torch.float32 else EIGHTS)) * mags
    if before is not None:
        want = want + before.double()
        slack = slack + 2.0 ** -24 * want.abs()
    slack = slack + HALF_STEP[got.dtype] * (want.abs() + slack)
    if got.dtype == torch.float16:
        slack = slack + 2.0 ** -25
    off = (got.double() - want).abs()
    assert torch.isfinite(got).all()
    worst = (off - slack).max().item() if off.numel() else -1.0
    assert worst <= 0, f"off by {off.max().item()}, {worst} more than allowed"


# ------------------------------------------------------------ quantisation

def check_quantize(lib, x, dim, tile, fmt, scale):
    announce(f"quantize {tuple(x.shape)} {x.dtype} strides {x.stride()} dim {dim} tile {tile} {fmt} {scale}")
    if dim == 2:
        q1, s1, q0, s0 = lib.quantize_f8_both(x, tile, fmt, scale)
        pairs = ((1, q1, s1), (0, q0, s0))
    else:
        q, s = lib.quantize_f8(x, dim, tile, fmt, scale)
        pairs = ((dim, q, s),)
    for d, q, s in pairs:
        assert q.dtype == fmt and s.dtype == scale and q.shape == x.shape
        assert q.shape[d] < 2 or q.stride(d) == 1
        want_q, want_s = plain.quantize(x, d, tile, fmt, scale == E8)
        assert torch.equal(s.float().double(), want_s)
        same_values(q, want_q)


@pytest.mark.parametrize("shape", [(1, 1), (1, 7), (3, 127), (1, 4096), (5, 128), (129, 129), (128, 256), (300, 1),
                                   (257, 1000), (1, 130), (640, 77)])
@pytest.mark.parametrize("dim", [0, 1, 2])
def test_quantize_sizes(gpu_lib, shape, dim):
    n = 0
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        for tile in (False, True):
            n += 1
            fmt, scale = ((E4, F32), (E5, E8), (E4, E8), (E5, F32))[(n + dim) % 4]
            check_quantize(gpu_lib, rand(shape, n, dtype).to(dtype), dim, tile, fmt, scale)


@pytest.mark.parametrize("fmt", [E4, E5])
@pytest.mark.parametrize("scale", [F32, E8])
@pytest.mark.parametrize("tile", [False, True])
def test_quantize_borders(gpu_lib, fmt, scale, tile):
    """Elements that divide to a border between two values, or one FP32 unit
    beside it: the quotient's rounding decides."""
    t = plain.table(fmt)
    mids = ((t[1:] + t[:-1]) / 2).float().cuda()
    amax = torch.tensor([448.0, 57344.0, 1.0, 0.1, 3.3e-30, 1e30, 7.0, 447.99], device="cuda")
    rows = []
    for a in amax.tolist():
        top = float(t[-1])
        v = (mids.double() * (a / top)).float()
        v = v[v <= a]
        both = torch.cat([v, torch.nextafter(v, torch.full_like(v, 1e38)), torch.nextafter(v, torch.zeros_like(v)),
                          -v])
        for i in range(0, both.numel(), 127):
            piece = both[i:i + 127].clamp(-a, a)
            rows.append(torch.cat([torch.tensor([a], device="cuda"), piece,
                                   torch.zeros(127 - piece.numel(), device="cuda")]))
    x = torch.stack(rows)
    for dtype in (torch.float32, torch.bfloat16):
        check_quantize(gpu_lib, x.to(dtype), 1, tile, fmt, scale)
        check_quantize(gpu_lib, x.to(dtype).t().contiguous(), 0, tile, fmt, scale)


@pytest.mark.parametrize("fmt", [E4, E5])
@pytest.mark.parametrize("scale", [F32, E8])
def test_quantize_extremes(gpu_lib, fmt, scale):
    """Zero blocks, subnormals, the largest values, infinities and NaN: the
    scale goes by the finite elements."""
    big = torch.finfo(torch.float32).max
    x = torch.zeros((16, 256), device="cuda")
    x[1, 3] = 1e-45
    x[2, :130] = 2.0 ** -126
    x[3] = big
    x[4, ::2] = -big
    x[4, 1] = 1e-45
    x[5, 0] = float("inf")
    x[6, 5] = float("nan")
    x[7] = float("-inf")
    x[8] = float("nan")
    x[9] = rand((1, 256), 5)[0] * 1e-38
    x[9, 7] = float("-inf")
    x[10, 0], x[10, 1] = -0.0, 1.0
    x[11] = torch.linspace(-3e-39, 3e-39, 256, device="cuda")
    x[12] = rand((1, 256), 6)[0] * 1e30
    x[12, 200] = float("nan")
    for dim in (1, 0, 2):
        check_quantize(gpu_lib, x, dim, False, fmt, scale)
        check_quantize(gpu_lib, x, dim, True, fmt, scale)
    h = rand((20, 140), 8, torch.float16)
    h[3, 3], h[4, 4], h[5, 5] = float("inf"), float("nan"), 65504.0
    h[6] = 6e-8
    check_quantize(gpu_lib, h, 2, False, fmt, scale)


@pytest.mark.parametrize("fmt", [E4, E5])
def test_quantize_every_significand(gpu_lib, fmt):
    """The FP32 scale of every 24-bit significand, in the middle of the range and
    where the scale becomes the least: the quotient rounded once."""
    m = torch.arange(1 << 23, dtype=torch.int32, device="cuda")
    top = float(plain.table(fmt)[-1])
    for exponent in (127, 10):
        a = (m | (exponent << 23)).view(torch.float32)
        x = torch.zeros((1 << 12, 1 << 11, 128), device="cuda")
        x[:, :, 77] = -a.view(1 << 12, 1 << 11)
        announce(f"scales of every significand, exponent {exponent}, {fmt}")
        q, s = gpu_lib.quantize_f8(x.view(1 << 12, 1 << 18), 1, False, fmt, F32)
        want = (a.double() / torch.full_like(a, top, dtype=torch.float64)).float().clamp(min=2.0 ** -126)
        assert torch.equal(s, want.view(1 << 12, 1 << 11))
        del x, q


def test_quantize_layouts(gpu_lib):
    """Column-major inputs, views whose rows are not 16-byte aligned, strides
    that have to be copied, and an expanded row."""
    x = rand((301, 403), 3, torch.bfloat16)
    for v in (x.t(), x[1:, 3:], x[:, 1:200].t(), x[::2, ::3], x[:1].expand(70, 403), x[5:6, ::2], x[::3, 7:8]):
        for dim in (0, 1, 2):
            check_quantize(gpu_lib, v, dim, False, E4, F32)


def test_quantize_empty(gpu_lib):
    for shape in ((0, 5), (5, 0), (0, 0)):
        q, s = gpu_lib.quantize_f8(torch.empty(shape, device="cuda"), 1)
        assert q.shape == shape and s.shape == (shape[0], (shape[1] + 127) // 128)


# ---------------------------------------------------------------- products

def values(shape, fmt, seed, order="row"):
    """Random finite codes of a format, in row- or column-major order."""
    g = gen(seed)
    r, c = shape if order == "row" else shape[::-1]
    code = torch.randint(0, 256, (r, c), device="cuda", generator=g, dtype=torch.int32)
    bad = (code & 127) == 127 if fmt == E4 else (code & 127) >= 124
    q = torch.where(bad, torch.full_like(code, 60), code).to(torch.uint8).view(fmt)
    return q if order == "row" else q.t()


def scales(shape, kind, seed):
    g = gen(seed)
    if kind == E8:
        return torch.randint(110, 141, shape, device="cuda", generator=g, dtype=torch.int32).to(torch.uint8).view(E8)
    return torch.exp(4 * torch.randn(shape, device="cuda", generator=g))


def blocks(v):
    return (v + 127) // 128


def operands(m, n, k, kind, a_fmt=E4, b_fmt=E4, a_tile=False, b_tile=True, a_order="row", b_order="col", seed=1):
    A, B = values((m, k), a_fmt, seed, a_order), values((k, n), b_fmt, seed + 1, b_order)
    SA = scales((blocks(m) if a_tile else m, blocks(k)), kind, seed + 2)
    SB = scales((blocks(k), blocks(n) if b_tile else n), kind, seed + 3)
    return A, SA, B, SB


def check_gemm(lib, ops, out_dtype=torch.float32, out=None, accumulate=False):
    A, SA, B, SB = ops
    (m, k), n = A.shape, B.shape[1]
    announce(f"gemm {m}x{n}x{k} {A.dtype} {A.stride()} {tuple(SA.shape)} {B.dtype} {B.stride()} {tuple(SB.shape)} "
             f"{SA.dtype} -> {out_dtype} {None if out is None else out.stride()} add {accumulate}")
    before = out.clone() if accumulate else None
    C = lib.gemm_f8(A, SA, B, SB, out_dtype, out=out, accumulate=accumulate)
    assert C.dtype == out_dtype and C.shape == (m, n) and (out is None or C is out)
    want, mags = plain.gemm(A, SA, B, SB)
    if out_dtype == torch.float16:   # beyond fp16: infinite
        inf = want.abs() > 65520 + (plain.sum_bound(k) + EIGHTS) * mags
        assert torch.isinf(C[inf]).all()
        keep = want.abs() + (plain.sum_bound(k) + EIGHTS) * mags < 65504
        close(C[keep], want[keep], mags[keep], k)
        return C
    close(C, want, mags, k, before)
    return C


SIZES = [(1, 1, 1), (1, 128, 128), (2, 3, 5), (16, 16, 128), (17, 33, 129), (64, 64, 256), (65, 130, 384),
         (100, 1, 300), (1, 100, 300), (128, 128, 15), (256, 256, 512), (257, 255, 640), (300, 500, 1000),
         (48, 700, 144), (513, 129, 131), (40, 1040, 1300), (2, 5000, 1024),
         (5000, 30, 1111), (64, 3000, 2048), (20, 17000, 515), (3, 9000, 1021), (31, 40, 2049),
         (20, 17000, 2000), (17000, 9, 2000)]


@pytest.mark.parametrize("kind", [F32, E8])
@pytest.mark.parametrize("size", SIZES)
def test_gemm_sizes(gpu_lib, size, kind):
    for a_tile, b_tile in ((False, True), (False, False), (True, True), (True, False)):
        check_gemm(gpu_lib, operands(*size, kind, a_tile=a_tile, b_tile=b_tile))


@pytest.mark.parametrize("kind", [F32, E8])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gemm_large(gpu_lib, dtype, kind):
    """Enough tiles for the large block tile, ragged ones among them."""
    for m, n, k in ((3500, 3601, 300), (3585, 3590, 128), (4096, 3592, 515)):
        for a_tile, b_tile in ((False, True), (False, False), (True, False)):
            check_gemm(gpu_lib, operands(m, n, k, kind, E5, E4, a_tile, b_tile), dtype)
    for m, n, k in ((3500, 3600, 300), (3600, 3488, 129), (2000, 2000, 640)):
        check_gemm(gpu_lib, operands(m, n, k, kind, E5, E4, b_order="row"), dtype)
        check_gemm(gpu_lib, operands(m, n, k, kind, E4, E5, b_tile=False, a_order="col", b_order="row"), dtype)
    room = torch.full((3503, 3611), 7.0, device="cuda", dtype=dtype)
    check_gemm(gpu_lib, operands(3500, 3601, 300, kind), dtype, out=room[1:3501, :3601])
    room[1:3501, :3601] = 7.0
    assert (room == 7.0).all()
    ops = operands(3500, 3600, 1000, kind, b_tile=False)
    first = gpu_lib.gemm_f8(*ops, dtype)
    for _ in range(3):
        assert torch.equal(first, gpu_lib.gemm_f8(*ops, dtype))


MIDDLE = [(2000, 2030, 300), (1950, 2048, 515)]


@pytest.mark.parametrize("kind", [F32, E8])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_gemm_middle(gpu_lib, dtype, kind):
    """Sizes of the middle block tile, both orders of B."""
    for m, n, k in MIDDLE:
        for b_order, b_tile in (("col", True), ("col", False), ("row", True), ("row", False)):
            A, SA, B, SB = operands(m, n, k, F32, E4, E5, b_tile=b_tile, b_order=b_order)
            check_gemm(gpu_lib, (A, (SA * 1e-3).to(kind), B, (SB * 1e-2).to(kind)), dtype)


# 128 x 128 tiles with k ranges, of FP32 and of 16-bit outputs, and 256 x 256 tiles
RANGES = [(677, 965, 5669, torch.float32), (674, 1520, 5828, torch.bfloat16), (1460, 1801, 12623, torch.bfloat16)]


@pytest.mark.parametrize("kind", [F32, E8])
@pytest.mark.parametrize("m,n,k,dtype", RANGES)
def test_gemm_ranges(gpu_lib, m, n, k, dtype, kind):
    """k ranges of the larger block tiles, both orders of B."""
    for b_order, b_tile in (("col", True), ("row", False)):
        check_gemm(gpu_lib, operands(m, n, k, kind, E4, E4, b_tile=b_tile, b_order=b_order), dtype)


@pytest.mark.parametrize("kind", [F32, E8])
@pytest.mark.parametrize("a_fmt,b_fmt", [(E4, E5), (E5, E4), (E5, E5)])
def test_gemm_formats(gpu_lib, a_fmt, b_fmt, kind):
    for m, n, k in ((3, 200, 260), (130, 140, 390), (300, 300, 256)):
        for b_tile in (False, True):
            check_gemm(gpu_lib, operands(m, n, k, kind, a_fmt, b_fmt, b_tile=b_tile))


@pytest.mark.parametrize("a_order", ["row", "col"])
@pytest.mark.parametrize("b_order", ["row", "col"])
def test_gemm_orders(gpu_lib, a_order, b_order):
    """Every storage order of the operands and of the output, aligned lines and
    others, new and given outputs."""
    for m, n, k in ((5, 300, 256), (144, 160, 272), (131, 77, 259), (272, 16, 400), (9, 1024, 640), (80, 96, 128),
                    (512, 96, 1101), (208, 208, 2048)):
        for kind in (F32, E8):
            ops = operands(m, n, k, kind, a_order=a_order, b_order=b_order)
            check_gemm(gpu_lib, ops, torch.bfloat16)
            check_gemm(gpu_lib, ops, F32, out=torch.empty((n, m), device="cuda").t())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_gemm_outputs(gpu_lib, dtype):
    """Types and strides of the output; memory between and behind its lines
    stays as it was."""
    for m, n, k in ((7, 50, 200), (130, 150, 300), (260, 300, 128)):
        A, SA, B, SB = operands(m, n, k, F32)
        SA, SB = SA * 1e-3, SB * 1e-2
        check_gemm(gpu_lib, (A, SA, B, SB), dtype)
        for pad in (1, 4, 9):
            room = torch.full((m + 2, n + pad), 7.0, device="cuda", dtype=dtype)
            C = check_gemm(gpu_lib, (A, SA, B, SB), dtype, out=room[1:m + 1, :n])
            kept = room.clone()
            kept[1:m + 1, :n] = 7.0
            assert (kept == 7.0).all() and C.data_ptr() == room[1:].data_ptr()
            room = torch.full((n + 2, m + pad), 7.0, device="cuda", dtype=dtype)
            check_gemm(gpu_lib, (A, SA, B, SB), dtype, out=room[1:n + 1, :m].t())
            room[1:n + 1, :m] = 7.0
            assert (room == 7.0).all()


@pytest.mark.parametrize("kind", [F32, E8])
def test_gemm_accumulate(gpu_lib, kind):
    for m, n, k in ((4, 100, 256), (140, 150, 300), (257, 300, 1024)):
        ops = operands(m, n, k, kind, E5, E4, b_tile=False)
        C = torch.randn((m, n), device="cuda", generator=gen(9))
        check_gemm(gpu_lib, ops, F32, out=C, accumulate=True)
        check_gemm(gpu_lib, ops, F32, out=torch.randn((n, m), device="cuda").t(), accumulate=True)


def test_gemm_scale_strides(gpu_lib):
    """Scales of any strides: transposed storage, every second one, one for
    all."""
    for m, n, k in ((6, 200, 400), (200, 260, 700)):
        for kind in (F32, E8):
            A, SA, B, SB = operands(m, n, k, kind, b_tile=False)
            wide = scales((2 * m, 2 * blocks(k)), kind, 77)
            for sa in (SA.t().contiguous().t(), wide[::2, ::2], wide[:1, :1].expand(m, blocks(k))):
                check_gemm(gpu_lib, (A, sa, B, SB.t().contiguous().t()))


def test_gemm_padding_is_not_read(gpu_lib):
    """What lies behind a line's k values (NaN here), behind the last line and
    between the lines does not reach the product."""
    for m, n, k in ((3, 40, 200), (150, 140, 200), (1, 300, 133), (257, 300, 77)):
        for lines_a, lines_b in ((208, 208), (224, 256), (211, 209)):
            room_a = torch.full((m + 3, lines_a), 0x7f, dtype=torch.uint8, device="cuda")
            room_b = torch.full((n + 3, lines_b), 0x7f, dtype=torch.uint8, device="cuda")
            A, SA, B, SB = operands(m, n, k, F32)
            room_a[:m, :k] = A.view(torch.uint8)
            room_b[:n, :k] = B.t().view(torch.uint8)
            got = check_gemm(gpu_lib, (room_a[:m, :k].view(E4), SA, room_b[:n, :k].view(E4).t(), SB))
            assert torch.isfinite(got).all()


@pytest.mark.parametrize("kind", [F32, E8])
def test_gemm_special_values(gpu_lib, kind):
    """NaN and infinities reach the outputs of their line and no other."""
    for m, n, k in ((4, 70, 300), (140, 260, 300)):
        A, SA, B, SB = operands(m, n, k, kind, E5, E4)
        A, B = A.clone(), B.clone()
        A.view(torch.uint8)[1, 3] = 0x7f       # NaN
        A.view(torch.uint8)[2, 140] = 0x7c     # infinity
        B.view(torch.uint8)[140, :] = 0x38     # times 1
        B.view(torch.uint8)[7, 5] = 0x7f       # NaN
        A.view(torch.uint8)[2, 7] = 0x3c
        announce(f"special values {m}x{n}x{k} {kind}")
        C = gpu_lib.gemm_f8(A, SA, B, SB, F32)
        want, mags = plain.gemm(A, SA, B, SB)
        assert torch.equal(torch.isnan(C), torch.isnan(want))
        assert torch.isinf(C[2]).sum() == n - 1 and (C[2][torch.isinf(C[2])] > 0).all()
        keep = torch.isfinite(want)
        close(C[keep], want[keep], mags[keep], k)


def test_gemm_extreme_scales(gpu_lib):
    """Scales far apart, their products within FP32's normal range."""
    for kind in (F32, E8):
        for m, n, k in ((5, 64, 384), (140, 150, 384)):
            A, SA, B, SB = operands(m, n, k, kind)
            up, down = 2.0 ** 100, 2.0 ** -110
            SA, SB = torch.ones(SA.shape, device="cuda") * up, torch.ones(SB.shape, device="cuda") * down
            SA[::2, 1] = 2.0 ** 90
            SB[2] = 2.0 ** -100
            check_gemm(gpu_lib, (A, SA.to(kind), B, SB.to(kind)))


def test_gemm_zeros(gpu_lib):
    """No terms: zeros, or C as it was; no lines: nothing."""
    A, SA, B, SB = operands(20, 30, 0, F32)
    C = gpu_lib.gemm_f8(A, SA, B, SB, F32, out=torch.full((20, 30), 3.0, device="cuda"))
    assert (C == 0).all()
    C = gpu_lib.gemm_f8(A, SA, B, SB, F32, out=torch.full((20, 30), 3.0, device="cuda"), accumulate=True)
    assert (C == 3).all()
    for m, n in ((0, 5), (5, 0)):
        A, SA, B, SB = operands(m, n, 256, F32)
        assert gpu_lib.gemm_f8(A, SA, B, SB).shape == (m, n)


def test_gemm_long_k(gpu_lib):
    for m, n, k in ((1, 40, 70000), (3, 20, 200001), (200, 130, 33000), (16, 300, 20000)):
        for kind in (F32, E8):
            ops = operands(m, n, k, kind, b_tile=False)
            check_gemm(gpu_lib, ops)
            check_gemm(gpu_lib, ops, torch.bfloat16, out=torch.empty((n, m), device="cuda", dtype=torch.bfloat16).t())
            check_gemm(gpu_lib, ops, F32, out=torch.randn((m, n + 3), device="cuda")[:, :n], accumulate=True)


def test_gemm_nan_scale(gpu_lib):
    """An E8M0 byte of 255 is NaN, for its line's block and no other."""
    for m, n, k in ((5, 64, 384), (140, 150, 384)):
        for dtype in (torch.float32, torch.bfloat16):
            A, SA, B, SB = operands(m, n, k, E8, b_tile=False)
            SA.view(torch.uint8)[3, 1] = 255
            SB.view(torch.uint8)[2, 7] = 255
            announce(f"NaN scales {m}x{n}x{k} {dtype}")
            C = gpu_lib.gemm_f8(A, SA, B, SB, dtype)
            nan = torch.zeros((m, n), dtype=torch.bool, device="cuda")
            nan[3], nan[:, 7] = True, True
            assert torch.equal(torch.isnan(C), nan)


def test_gemm_offsets_beyond_32_bits(gpu_lib):
    """An output and operands of more than 2^32 bytes, checked in samples."""
    m, n, k = 66000, 66000, 128
    A, SA, B, SB = operands(m, n, k, F32)
    announce("gemm 66000 x 66000 x 128")
    C = gpu_lib.gemm_f8(A, SA * 1e-3, B, SB, torch.bfloat16)
    i = torch.tensor([0, 1, 4097, 32767, 32768, 65535, 65536, 65999], device="cuda")
    want, mags = plain.gemm(A[i].contiguous(), SA[i] * 1e-3, B, SB)
    close(C[i], want, mags, k)
    del C, want, mags
    m, n, k = 130, 70, 40_000_000 // 16
    A = values((m, 32), E4, 3).repeat(1, k // 32)          # 2^32 bytes in 130 lines of 33 MB
    big = torch.empty((m, k * 14), dtype=torch.uint8, device="cuda")
    big[:, :k] = A.view(torch.uint8)
    B = values((n, 32), E4, 4).repeat(1, k // 32)
    SA, SB = torch.ones((m, blocks(k)), device="cuda"), torch.ones((blocks(k), n), device="cuda")
    announce(f"gemm {m} x {n} x {k}, lines {k * 14} bytes apart")
    C = gpu_lib.gemm_f8(big[:, :k].view(E4), SA, B.t(), SB, F32)
    one = A[:, :32].float().double() @ B[:, :32].float().double().t().contiguous()
    mags = A[:, :32].float().double().abs() @ B[:, :32].float().double().abs().t().contiguous()
    close(C, one * (k // 32), mags * (k // 32), k)


def test_gemm_repeats_bit_for_bit(gpu_lib):
    for m, n, k in ((1, 500, 3000), (300, 200, 5000), (700, 900, 1000)):
        ops = operands(m, n, k, F32, b_tile=False)
        announce(f"repeat {m}x{n}x{k}")
        first = gpu_lib.gemm_f8(*ops, F32)
        for _ in range(3):
            assert torch.equal(first, gpu_lib.gemm_f8(*ops, F32))


# ------------------------------------------------------------------ layers

def quantized(x, dim, tile, fmt, kind):
    q, s = plain.quantize(x, dim, tile, fmt, kind == E8)
    return q * plain.spread(s, q.shape)


def weights(n, k, kind, seed):
    w = torch.randn((n, k), device="cuda", generator=gen(seed)) / k ** 0.5
    q, s = plain.quantize(w, 1, True, E4, kind == E8)
    return q.float().to(E4), s.float().to(kind), q * plain.spread(s, q.shape)


def check_linear(lib, X, W, SW, wd, out_dtype, fmt=E4, out=None):
    announce(f"linear {tuple(X.shape)} {X.dtype} {X.stride()} -> {W.shape[0]} {SW.dtype} {fmt} {out_dtype}")
    Y = lib.linear_f8(X, W, SW, out_dtype, fmt, out=out)
    xd = quantized(X, 1, False, fmt, SW.dtype)
    close(Y, xd @ wd.t().contiguous(), xd.abs() @ wd.abs().t().contiguous(), X.shape[1])
    return Y


@pytest.mark.parametrize("kind", [F32, E8])
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 128, 256), (1, 1000, 300), (4, 512, 1024), (9, 77, 500),
                                   (16, 640, 4096), (17, 256, 2000), (33, 130, 257), (64, 512, 640), (65, 300, 129),
                                   (300, 260, 700)])
def test_linear(gpu_lib, m, n, k, kind):
    W, SW, wd = weights(n, k, kind, 5)
    for dtype, out_dtype in ((torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32),
                             (torch.float16, torch.bfloat16)):
        check_linear(gpu_lib, rand((m, k), 3, dtype), W, SW, wd, out_dtype)
    check_linear(gpu_lib, rand((k, m), 4, torch.bfloat16).t(), W, SW, wd, torch.float32, E5)
    check_linear(gpu_lib, rand((m, k + 3), 4, torch.bfloat16)[:, 1:k + 1], W, SW, wd, torch.bfloat16)
    check_linear(gpu_lib, rand((m, k), 4), W.t().contiguous().t(), SW, wd, torch.float32,
                 out=torch.empty((n, m), device="cuda").t())


def test_linear_line_scales(gpu_lib):
    """Weights with a scale per line."""
    for m, n, k in ((2, 300, 500), (150, 300, 500)):
        q, s = gpu_lib.quantize_f8(torch.randn((n, k), device="cuda"), 1)
        check_linear(gpu_lib, rand((m, k), 6, torch.bfloat16), q, s, plain.dequantize(q, s), torch.float32)


def test_linear_is_quantize_and_gemm(gpu_lib):
    """The layer gives what its two steps give, bit for bit, where both take
    the same path."""
    W, SW, _ = weights(700, 900, F32, 8)
    for m in (1, 5, 40, 200):
        X = rand((m, 900), 7, torch.bfloat16)
        announce(f"linear as two calls, m = {m}")
        Y = gpu_lib.linear_f8(X, W, SW, F32)
        q, s = gpu_lib.quantize_f8(X, 1)
        Z = gpu_lib.gemm_f8(q, s, W.t(), SW.t(), F32)
        want, mags = plain.gemm(q, s, W.t(), SW.t())
        close(Y, want, mags, 900)
        close(Z, want, mags, 900)


def test_linear_special_rows(gpu_lib):
    """A row of zeros gives zeros, a row with NaN gives NaN and only there."""
    W, SW, wd = weights(200, 300, F32, 8)
    for m in (3, 100):
        X = rand((m, 300), 7, torch.bfloat16)
        X[0] = 0
        X[2, 5] = float("nan")
        announce(f"linear with special rows, m = {m}")
        Y = gpu_lib.linear_f8(X, W, SW, F32)
        assert (Y[0] == 0).all() and torch.isnan(Y[2]).all()
        assert torch.isfinite(Y[1]).all() and torch.isfinite(Y[3:]).all()


def check_backward(lib, dY, X, W, SW, wd, fmt=E4, out_dtype=torch.float32, **kw):
    m, k = X.shape
    n = W.shape[0]
    announce(f"backward m {m} n {n} k {k} {X.dtype} {SW.dtype} {fmt} {out_dtype} {sorted(kw)}")
    before = kw["dW"].clone() if kw.get("accumulate") else None
    dX, dW = lib.linear_f8_backward(dY, X, W, SW, fmt, out_dtype, **kw)
    assert dX.shape == X.shape and dW.shape == W.shape and dW.dtype == F32
    y1 = quantized(dY, 1, False, fmt, SW.dtype)
    y0 = quantized(dY, 0, False, fmt, SW.dtype).t().contiguous()
    x0 = quantized(X, 0, False, E4, SW.dtype)
    close(dX, y1 @ wd, y1.abs() @ wd.abs(), n)
    close(dW, y0 @ x0, y0.abs() @ x0.abs(), m, before)


@pytest.mark.parametrize("kind", [F32, E8])
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 130, 70), (5, 128, 256), (130, 200, 300), (256, 384, 128),
                                   (300, 77, 515), (1000, 256, 384)])
def test_backward(gpu_lib, m, n, k, kind):
    W, SW, wd = weights(n, k, kind, 5)
    for dtype, fmt, out in ((torch.bfloat16, E5, torch.bfloat16), (torch.float32, E4, torch.float32)):
        X, dY = rand((m, k), 1, dtype), rand((m, n), 2, dtype) * 1e-3
        check_backward(gpu_lib, dY, X, W, SW, wd, fmt, out)
        check_backward(gpu_lib, dY, X, W, SW, wd, fmt, out, dW=torch.randn((n, k), device="cuda"), accumulate=True)
    check_backward(gpu_lib, rand((n, m), 2, torch.bfloat16).t(), rand((k, m), 1, torch.bfloat16).t(), W, SW, wd,
                   dX=torch.empty((k, m), device="cuda").t(), dW=torch.empty((k, n), device="cuda").t())


def test_backward_without_tokens(gpu_lib):
    W, SW, _ = weights(20, 30, F32, 5)
    X, dY = torch.empty((0, 30), device="cuda"), torch.empty((0, 20), device="cuda")
    dX, dW = gpu_lib.linear_f8_backward(dY, X, W, SW)
    assert dX.shape == (0, 30) and (dW == 0).all()
    kept = torch.randn((20, 30), device="cuda")
    before = kept.clone()
    gpu_lib.linear_f8_backward(dY, X, W, SW, dW=kept, accumulate=True)
    assert torch.equal(kept, before)


def test_gradients_against_differences(gpu_lib):
    """Small whole numbers quantise without loss (a block's largest is the
    format's, so its scale is 1), which makes the layer linear, and its
    gradients the differences of sum(dY Y) exactly."""
    m, n, k = 130, 70, 140
    g = gen(4)

    def whole(shape):
        x = torch.randint(-4, 5, shape, device="cuda", generator=g).float()
        for i in range(0, shape[0], 1):
            x[i, ::128] = 448.0
        for j in range(0, shape[1], 1):
            x[::128, j] = 448.0
        return x

    X, dY, w = whole((m, k)), whole((m, n)), whole((n, k))
    W, SW = gpu_lib.quantize_f8(w, 1, True)
    assert (SW == 1).all()
    announce("gradients against differences")
    dX, dW = gpu_lib.linear_f8_backward(dY, X, W, SW, out_dtype=F32)
    loss = lambda x, ww: (gpu_lib.linear_f8(x, ww, SW, F32).double() * dY.double()).sum()
    base = loss(X, W)
    for i, j in ((3, 5), (129, 139), (64, 127), (1, 130)):
        step = X.clone()
        step[i, j] += 1
        assert (loss(step, W) - base).item() == dX[i, j].item()
    for i, j in ((3, 5), (69, 139), (64, 127)):
        step = W.float()
        step[i, j] += 1
        assert (loss(X, step.to(E4)) - base).item() == dW[i, j].item()


def test_a_training_step(gpu_lib):
    """The operators in the order of their use: weights quantised, two layers
    forward, both backward with main gradients added up over two microbatches,
    against the same steps in 64 bits."""
    m, d, h = 260, 300, 520
    for kind, fmt in ((F32, E4), (E8, E5)):
        w1, w2 = torch.randn((h, d), device="cuda") / d ** 0.5, torch.randn((d, h), device="cuda") / h ** 0.5
        W1, S1 = gpu_lib.quantize_f8(w1, 1, True, E4, kind)
        W2, S2 = gpu_lib.quantize_f8(w2, 1, True, E4, kind)
        G1, G2 = torch.zeros((h, d), device="cuda"), torch.zeros((d, h), device="cuda")
        d1, d2 = plain.dequantize(W1, S1), plain.dequantize(W2, S2)
        E1, E2 = torch.zeros_like(G1).double(), torch.zeros_like(G2).double()
        B1, B2 = E1.clone(), E2.clone()
        for step in (1, 2):
            X, dY = rand((m, d), step, torch.bfloat16), rand((m, d), step + 5, torch.bfloat16) * 1e-3
            announce(f"training step {step} {kind}")
            H = gpu_lib.linear_f8(X, W1, S1)
            Y = gpu_lib.linear_f8(H, W2, S2)
            dH, _ = gpu_lib.linear_f8_backward(dY, H, W2, S2, fmt, dW=G2, accumulate=True)
            dX, _ = gpu_lib.linear_f8_backward(dH, X, W1, S1, fmt, dW=G1, accumulate=True)
            x1 = quantized(X, 1, False, E4, kind)
            close(H, x1 @ d1.t().contiguous(), x1.abs() @ d1.abs().t().contiguous(), d)
            h1 = quantized(H, 1, False, E4, kind)
            close(Y, h1 @ d2.t().contiguous(), h1.abs() @ d2.abs().t().contiguous(), h)
            for grad, act, wd, dIn, E, B in ((dY, H, d2, dH, E2, B2), (dH, X, d1, dX, E1, B1)):
                g1 = quantized(grad, 1, False, fmt, kind)
                close(dIn, g1 @ wd, g1.abs() @ wd.abs(), grad.shape[1])
                g0, a0 = quantized(grad, 0, False, fmt, kind).t().contiguous(), quantized(act, 0, False, E4, kind)
                E += g0 @ a0
                B += g0.abs() @ a0.abs()
        close(G1, E1, B1, 2 * m)
        close(G2, E2, B2, 2 * m)


# ------------------------------------------------------- streams and graphs

def test_side_stream(gpu_lib):
    """The calls run on torch's current stream, behind what produces their
    inputs there."""
    A, SA, B, SB = operands(200, 300, 1001, F32)
    X = rand((70, 500), 4, torch.bfloat16)
    W, SW, wd = weights(200, 500, F32, 5)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    announce("8-bit products on a side stream")
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        A2, X2 = A.clone(), X.clone()
        C = gpu_lib.gemm_f8(A2, SA, B, SB, F32)
        Y = gpu_lib.linear_f8(X2, W, SW, F32)
        C2, Y2 = C.clone(), Y.clone()
    torch.cuda.synchronize()
    want, mags = plain.gemm(A, SA, B, SB)
    close(C2, want, mags, 1001)
    xd = quantized(X, 1, False, E4, F32)
    close(Y2, xd @ wd.t().contiguous(), xd.abs() @ wd.abs().t().contiguous(), 500)


def test_two_graphs_share_nothing(gpu_lib):
    """Two captured calls that both need a workspace, replayed at the same time
    on two streams and with eager calls between: every replay gives the eager
    result."""
    m, n, k = 300, 260, 1003           # lines that are not 16-byte aligned
    W, SW, _ = weights(n, k, F32, 5)
    xs = [rand((m, k), 10 + i, torch.bfloat16) for i in range(2)]
    dys = [rand((m, n), 20 + i, torch.bfloat16) for i in range(2)]
    call = lambda i: (gpu_lib.linear_f8(xs[i], W, SW, F32),) + gpu_lib.linear_f8_backward(dys[i], xs[i], W, SW)
    eager = [[t.clone() for t in call(i)] for i in range(2)]
    graphs, outs = [], []
    announce("two captured layers")
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(call(i))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for rep in range(4):
        torch.cuda.synchronize()
        for i in range(2):
            for t in outs[i]:
                t.zero_()
        torch.cuda.synchronize()
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                graphs[i].replay()
        other = call(rep % 2)
        torch.cuda.synchronize()
        for i in range(2):
            for got, want in zip(outs[i], eager[i]):
                assert torch.equal(got, want)
        for got, want in zip(other, eager[rep % 2]):
            assert torch.equal(got, want)


def test_between_the_other_products(gpu_lib):
    """The exact products and the 8-bit ones, called in turn, give what each
    gives alone."""
    a = torch.randn((200, 300), device="cuda", dtype=torch.float64)
    b = torch.randn((300, 100), device="cuda", dtype=torch.float64)
    first = gpu_lib.dgemm(a, b).clone()
    ops = operands(200, 300, 1001, F32)
    alone = gpu_lib.gemm_f8(*ops, F32).clone()
    announce("dgemm and gemm_f8 in turn")
    for _ in range(3):
        assert torch.equal(gpu_lib.gemm_f8(*ops, F32), alone)
        assert torch.equal(gpu_lib.dgemm(a, b), first)
