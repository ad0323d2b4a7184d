"""The performance cases of the 8-bit floating-point products: matrices of
e4m3 or e5m2 values with one scale per block of 128, through the torch entry
points of paper_2608_06812_amd.ozfp4, over the sizes that they are called with.

A case's "op" is one of
  quantize   X -> values and scales along one axis ("dim" 0 or 1) or along both
             in one call (dim 2), one scale per line of 128 or per 128 x 128
             tile ("tile")
  gemm       C (m x n) = A B of quantised operands; A has a scale per line,
             B per tile or ("tile" false) per line; "order" says how B is held:
             "k", adjacent along the contraction as weights are in the forward
             product, or "n", across it, as the same weights are in the product
             with an output gradient; "add": the product is added to C
  linear     Y (m x n) = quantised X (m x k) times the transposed weights (n x k)
  backward   the gradients dX (m x k) and dW (n x k) of that layer; "add":
             dW is added to

"src" is the type of the high-precision input, "fmt" the 8-bit format (of A in a
gemm, of dY in a backward pass; every other operand is e4m3), "pow2" whether
scales are powers of two in 8 bits (else FP32), "out" the output type.
"""

import math

import torch

own = False

BLOCK = 128
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
FORMATS = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
# mantissa bits, exponent of the least normal number, largest finite value
GRID = {"e4m3": (3, -6, 448.0), "e5m2": (2, -14, 57344.0)}
EIGHT = torch.float8_e8m0fnu


def _case(name, op, m, n, k, src="bf16", fmt="e4m3", pow2=False, tile=True, out="bf16", dim=1, order="k",
          add=False):
    return {"name": name, "op": op, "m": m, "n": n, "k": k, "src": src, "fmt": fmt, "pow2": pow2, "tile": tile,
            "out": out, "dim": dim, "order": order, "add": add}


def listed():
    return [
        # the activations of one token before a layer: latency only
        _case("quantize_token", "quantize", 1, 1, 4096, tile=False),
        # an output gradient on its way into both products of a backward pass
        _case("quantize_both", "quantize", 8192, 1, 8192, fmt="e5m2", tile=False, dim=2),
        # FP32 weights of odd sizes, laid out for both directions
        _case("quantize_weights", "quantize", 5001, 1, 4099, src="f32", pow2=True, dim=2),
        # one token times a weight matrix, operands quantised before
        _case("gemm_token", "gemm", 1, 8192, 8192),
        # a decoding batch
        _case("gemm_batch", "gemm", 24, 16384, 4096, pow2=True),
        # sizes that no tile divides
        _case("gemm_ragged", "gemm", 1500, 777, 3001, out="f16"),
        # a large layer with FP32 scales
        _case("gemm_8192", "gemm", 8192, 8192, 8192),
        # the weight gradient of a layer over many tokens, added to the main gradient
        _case("gemm_wgrad", "gemm", 4096, 4096, 16384, fmt="e5m2", tile=False, out="f32", add=True),
        # a few sequences' next tokens through a layer
        _case("linear_tokens", "linear", 4, 4096, 4096),
        # a prompt through a layer
        _case("linear_prompt", "linear", 2048, 8192, 8192, pow2=True),
        # a training step's backward pass, a small layer on a ragged batch
        _case("backward_small", "backward", 1000, 1024, 2048, out="f32"),
        # the same at full size, weight gradients added up over microbatches
        _case("backward_large", "backward", 8192, 8192, 4096, fmt="e5m2", pow2=True, add=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size of the range: a multiple of 128, of 16, or any."""
    v = _log(rng, lo, hi)
    step = rng.choice((1, 16, 128, 128))
    return max(lo, v // step * step) if v >= step else v


def draw(rng):
    op = rng.choice(("quantize", "gemm", "gemm", "linear", "backward"))
    c = _case("", op, 1, 1, 1)
    del c["name"]
    c["src"] = rng.choice(("bf16", "bf16", "f16", "f32"))
    c["pow2"] = rng.random() < 0.4
    c["out"] = rng.choice(("bf16", "bf16", "f16", "f32"))
    if op == "quantize":
        c["m"], c["k"] = _size(rng, 1, 8192), _size(rng, 64, 8192)
        c["fmt"], c["tile"], c["dim"] = rng.choice(("e4m3", "e5m2")), rng.random() < 0.4, rng.choice((0, 1, 2))
        return c
    c["n"], c["k"] = _size(rng, 128, 8192), _size(rng, 128, 8192)
    if op == "backward":
        c["m"], c["fmt"], c["add"] = _size(rng, 128, 8192), rng.choice(("e4m3", "e5m2")), rng.random() < 0.5
        return c
    c["m"] = rng.choice((_log(rng, 1, 64), _size(rng, 64, 8192)))
    if op == "gemm":
        c["fmt"], c["tile"] = rng.choice(("e4m3", "e4m3", "e5m2")), rng.random() < 0.7
        c["order"] = rng.choice(("k", "k", "n"))
        c["add"] = rng.random() < 0.25
        if c["add"]:
            c["out"] = "f32"
    return c


# ---------------------------------------------------------------- inputs

def _rows(m, k, dtype, gen):
    """Activations: channels of different sizes, a few large ones, rows of
    different norms."""
    x = torch.randn((m, k), device="cuda", generator=gen)
    x *= torch.exp(torch.randn((1, k), device="cuda", generator=gen))
    x *= torch.exp(0.5 * torch.randn((m, 1), device="cuda", generator=gen))
    return x.to(dtype)


def _gradient(m, n, dtype, gen):
    """An output gradient: small, of a wide range, with rows of zeros where a
    batch is padded."""
    x = 1e-3 * torch.randn((m, n), device="cuda", generator=gen)
    x *= torch.exp(1.5 * torch.randn((m, 1), device="cuda", generator=gen))
    if m >= 64:
        x[m - m // 32:] = 0
    return x.to(dtype)


def _weights(n, k, gen):
    return torch.randn((n, k), device="cuda", generator=gen) / math.sqrt(k)


def _sources(case, seed):
    """The high-precision matrices that a case starts from."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    m, n, k, src = case["m"], case["n"], case["k"], TYPES[case["src"]]
    if case["op"] == "quantize":
        return {"X": (_gradient if case["fmt"] == "e5m2" else _rows)(m, k, src, gen)}
    s = {"X": _rows(m, k, src, gen), "W": _weights(n, k, gen)}
    if case["op"] == "backward":
        s["dY"] = _gradient(m, n, src, gen)
    if case["add"]:
        shape = (n, k) if case["op"] == "backward" else (m, n)
        s["C"] = torch.randn(shape, device="cuda", generator=gen)
    return s


# ----------------------------------------------------------- plain forms

def _widen(s, shape):
    """Scales of blocks (rows x cols of them, whole lines where they match)
    for every element of `shape`."""
    for d in (0, 1):
        if s.shape[d] != shape[d]:
            s = s.repeat_interleave(BLOCK, dim=d).narrow(d, 0, shape[d])
    return s


def _plain_quantize(x, dim, tile, fmt, pow2):
    """Values (8-bit floating point) and scales of x for blocks along dim."""
    bits, least, top = GRID[fmt]
    r, c = x.shape
    br, bc = (BLOCK, BLOCK) if tile else ((1, BLOCK) if dim == 1 else (BLOCK, 1))
    a = torch.nn.functional.pad(x.float().abs(), (0, -c % bc, 0, -r % br))
    a = a.reshape(a.shape[0] // br, br, a.shape[1] // bc, bc).amax((1, 3))
    # in 64 bits: a scale that is one unit off, or a value next to a border
    # that is rounded twice, is another 8-bit value
    s = a.double() / torch.full_like(a, top, dtype=torch.float64)
    if pow2:   # the least power of two that is not below
        f = torch.frexp(s)[0]
        s = torch.where(f == 0.5, s, s / f)
    s = torch.where(a == 0, torch.ones_like(s), s.clamp(min=2.0 ** -126)).float()
    v = x.double() / _widen(s, x.shape).double()
    # the power of two below a value (a quotient by its fraction: exact, as
    # powers of a device's pow() are not) and the spacing of its neighbours
    p = torch.where(v == 0, torch.zeros_like(v), v / torch.frexp(v)[0] / 2)
    step = p.clamp(min=2.0 ** least) * 2.0 ** -bits
    q = (torch.round(v / step) * step).clamp(-top, top).to(FORMATS[fmt])
    return q, s.to(EIGHT) if pow2 else s


def _dequantize(q, s):
    return q.float() * _widen(s.float(), q.shape)


def _plain(state):
    case = state["case"]
    op, fmt, pow2, out = case["op"], case["fmt"], case["pow2"], TYPES[case["out"]]
    if op == "quantize":
        got = []
        for dim in ((1, 0) if case["dim"] == 2 else (case["dim"],)):
            got += _plain_quantize(state["X"], dim, case["tile"], fmt, pow2)
        return got
    if op == "gemm":
        c = torch.matmul(_dequantize(state["A"], state["SA"]), _dequantize(state["B"], state["SB"]))
        return state["C"].add_(c) if case["add"] else c.to(out)
    w = _dequantize(state["W"], state["SW"])
    x = _dequantize(*_plain_quantize(state["X"], 1 if op == "linear" else 0, False, "e4m3", pow2))
    if op == "linear":
        return torch.matmul(x, w.t()).to(out)
    dy1 = _dequantize(*_plain_quantize(state["dY"], 1, False, fmt, pow2))
    dy0 = _dequantize(*_plain_quantize(state["dY"], 0, False, fmt, pow2))
    dx, dw = torch.matmul(dy1, w).to(out), torch.matmul(dy0.t(), x)
    return [dx, state["C"].add_(dw) if case["add"] else dw]


# ------------------------------------------------------------- the cases

def prepare(case, seed):
    s = _sources(case, seed)
    state = {"case": dict(case)}
    fmt, pow2, tile = case["fmt"], case["pow2"], case["tile"]
    if case["op"] == "quantize":
        state["X"] = s["X"]
    elif case["op"] == "gemm":
        state["A"], state["SA"] = _plain_quantize(s["X"], 1, False, fmt, pow2)
        w, sw = _plain_quantize(s["W"], 1, tile, "e4m3", pow2)
        # "n": the transposed weights are adjacent across the contraction
        state["B"] = w.t() if case["order"] == "k" else w.t().contiguous()
        state["SB"] = sw.t()
    else:
        state["X"] = s["X"]
        state["W"], state["SW"] = _plain_quantize(s["W"], 1, True, "e4m3", pow2)
        if case["op"] == "backward":
            state["dY"] = s["dY"]
    if case["add"]:
        state["C"] = s["C"]
    return state


def run(state):
    if not own:
        return _plain(state)
    from paper_2608_06812_amd import ozfp4
    case = state["case"]
    op, out = case["op"], TYPES[case["out"]]
    if op == "quantize":
        scale = EIGHT if case["pow2"] else torch.float32
        if case["dim"] == 2:
            return ozfp4.quantize_f8_both(state["X"], case["tile"], FORMATS[case["fmt"]], scale)
        return ozfp4.quantize_f8(state["X"], case["dim"], case["tile"], FORMATS[case["fmt"]], scale)
    if op == "gemm":
        return ozfp4.gemm_f8(state["A"], state["SA"], state["B"], state["SB"], out, out=state.get("C"),
                             accumulate=case["add"])
    if op == "linear":
        return ozfp4.linear_f8(state["X"], state["W"], state["SW"], out)
    return ozfp4.linear_f8_backward(state["dY"], state["X"], state["W"], state["SW"], FORMATS[case["fmt"]],
                                    out, dW=state.get("C"), accumulate=case["add"])


def work(case):
    """Every input read once, every output written once."""
    m, n, k, op = case["m"], case["n"], case["k"], case["op"]
    size = {"f32": 4, "bf16": 2, "f16": 2}
    src, out, one = size[case["src"]], size[case["out"]], 1 if case["pow2"] else 4

    def blocks(v):
        return -(-v // BLOCK)

    def scales(rows, cols, dim, tile):
        r = blocks(rows) if tile or dim == 0 else rows
        c = blocks(cols) if tile or dim == 1 else cols
        return one * r * c

    if op == "quantize":
        dims = (1, 0) if case["dim"] == 2 else (case["dim"],)
        return {"bytes": float(src * m * k + sum(m * k + scales(m, k, d, case["tile"]) for d in dims)),
                "flops": 2.0 * len(dims) * m * k}
    w = n * k + scales(n, k, 1, op != "gemm" or case["tile"])
    if op == "gemm":
        c = 8 * m * n if case["add"] else out * m * n
        return {"bytes": float(m * k + scales(m, k, 1, False) + w + c), "flops": 2.0 * m * n * k}
    if op == "linear":
        return {"bytes": float(src * m * k + w + out * m * n), "flops": 2.0 * m * n * k}
    return {"bytes": float(src * (m * n + m * k) + w + out * m * k + (8 if case["add"] else 4) * n * k),
            "flops": 4.0 * m * n * k}


# --------------------------------------------- the definition in 64 bits

def _table(fmt):
    """Every nonnegative finite value of a format in order of its code, so
    that neighbours differ by one code and ties go to the even one."""
    bits, least, top = GRID[fmt]
    ones = 1 << bits
    t = [math.ldexp(c, least - bits) if c < ones else
         math.ldexp(ones + c % ones, c // ones - 1 + least - bits) for c in range(128)]
    t = [v for v in t if v <= top]
    return torch.tensor(t, dtype=torch.float64, device="cuda")


def _exact_quantize(x, dim, tile, fmt, pow2):
    """(values, scales, scaled values) from nearest-value search in the table of the format."""
    x = x.double()
    t = _table(fmt)
    top = float(t[-1])
    mid = (t[1:] + t[:-1]) / 2
    rows, cols = x.shape
    hr = BLOCK if tile or dim == 0 else 1
    hc = BLOCK if tile or dim == 1 else 1
    i = torch.arange(rows, device="cuda")[:, None] // hr
    j = torch.arange(cols, device="cuda")[None, :] // hc
    nr, nc = -(-rows // hr), -(-cols // hc)
    at = (i * nc + j).reshape(-1)
    a = torch.zeros(nr * nc, dtype=torch.float64, device="cuda")
    a = a.scatter_reduce(0, at, x.abs().reshape(-1), "amax")
    if pow2:
        powers = torch.tensor([math.ldexp(1.0, e) for e in range(-126, 128)], dtype=torch.float64, device="cuda")
        s = powers[torch.searchsorted(powers * top, a).clamp(max=253)]
    else:
        s = (a / top).float().double().clamp(min=2.0 ** -126)   # FP32 scales: rounded as they are held
    s = torch.where(a == 0, torch.ones_like(s), s)
    per = s[at].reshape(rows, cols)
    v = x.abs() / per
    code = torch.searchsorted(mid, v)   # a value on a border: the lower neighbour
    border = (code < mid.numel()) & (mid[code.clamp(max=mid.numel() - 1)] == v)
    code = torch.where(border & (code % 2 == 1), code + 1, code)
    q = torch.copysign(t[code], x)
    return q, s.reshape(nr, nc), q * per


def exact(case, seed):
    s = _sources(case, seed)
    op, fmt, pow2, tile = case["op"], case["fmt"], case["pow2"], case["tile"]
    if op == "quantize":
        got = []
        for dim in ((1, 0) if case["dim"] == 2 else (case["dim"],)):
            got += _exact_quantize(s["X"], dim, tile, fmt, pow2)[:2]
        return got
    w = _exact_quantize(s["W"], 1, tile if op == "gemm" else True, "e4m3", pow2)[2]
    if op == "gemm":
        c = torch.matmul(_exact_quantize(s["X"], 1, False, fmt, pow2)[2], w.t().contiguous())
        return s["C"].double() + c if case["add"] else c
    x = _exact_quantize(s["X"], 1 if op == "linear" else 0, False, "e4m3", pow2)[2]
    if op == "linear":
        return torch.matmul(x, w.t().contiguous())
    dx = torch.matmul(_exact_quantize(s["dY"], 1, False, fmt, pow2)[2], w)
    dw = torch.matmul(_exact_quantize(s["dY"], 0, False, fmt, pow2)[2].t().contiguous(), x)
    return [dx, s["C"].double() + dw if case["add"] else dw]
