"""The 8-bit products' choice of tile and k ranges on the host: bounds that the
launches rest on over random sizes, and that the sizes of the GPU tests reach
every tile, with and without ranges, in both forms."""

import os
import random
import shutil
import subprocess

import pytest

import test_gpu_f8 as gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TILE = ((64, 64), (128, 128), (256, 256))


@pytest.fixture(scope="module")
def route(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no host C++ compiler")
    exe = str(tmp_path_factory.mktemp("f8") / "f8_routes")
    subprocess.run([gxx, "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2608_06812_amd", "csrc"),
                    os.path.join(ROOT, "tests", "f8_routes_host.cpp"), "-o", exe], check=True, timeout=120)

    def ask(cases):
        text = "".join(f"{p} {q} {k} {int(e)}\n" for p, q, k, e in cases)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True, timeout=120).stdout
        return [tuple(int(v) for v in line.split()) for line in out.splitlines()]
    return ask


def test_bounds(route):
    rng = random.Random(5)
    log = lambda hi: int(round(2 ** rng.uniform(0, hi)))
    cases = [(log(17), log(17), log(22), rng.random() < 0.5) for _ in range(4000)]
    cases += [((1 << 30) - 1, 1, 128, e) for e in (False, True)] + [(1, 1, 1 << 22, e) for e in (False, True)]
    for (p, q, k, exact), (tile, ranges) in zip(cases, route(cases)):
        a, b = TILE[tile]
        assert not (exact and tile == 2)                 # the exact form has the first two
        stages = -(-k // 128)
        assert 1 <= ranges <= 16 and (ranges == 1 or stages // ranges >= 4)
        blocks = -(-p // a) * -(-q // b) * ranges
        if -(-p // 64) * -(-q // 64) < 1 << 24:
            assert blocks < 1 << 24                      # fewer than 2^32 threads in a launch
        if ranges > 1:
            assert p * q * ranges * 4 < 1 << 38          # partial sums stay small beside the operands' memory


def test_gpu_cases_reach_every_tile(route):
    sizes = [(n, m, k) for m, n, k in gpu.SIZES if min(m, n) > 32] + [(3601, 3500, 300), (130, 200, 33000)]
    for exact in (False, True):
        got = {(t, r > 1) for t, r in route([(*s, exact) for s in sizes])}
        assert {(0, False), (0, True), (1 if exact else 2, False)} <= got
    # the 128 x 128 tile: sizes of test_gemm_middle
    for exact in (False, True):
        assert [t for t, _ in route([(n, m, k, exact) for m, n, k in gpu.MIDDLE])] == [1] * len(gpu.MIDDLE)
    # k ranges of the larger tiles: sizes of test_gemm_ranges
    got = route([(n, m, k, dtype.itemsize == 4) for m, n, k, dtype in gpu.RANGES])
    assert [(t, r > 1) for t, r in got] == [(1, True), (1, True), (2, True)]
