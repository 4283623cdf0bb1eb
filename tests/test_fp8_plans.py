"""Which tiles the products in 8-bit floating point take, by the host code that chooses them (tests/fp8_plans_driver.cpp, which
includes its unit).  No device call, so no GPU is needed."""
import math
import os
import random
import subprocess

import pytest

from paper_2008_12336_amd import build as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plans") / "driver")
    cmd = [B.hipcc(), "--offload-arch=gfx950", "-O1", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-I" + os.path.join(ROOT, "include"), "-I" + B.CSRC, "-x", "hip", os.path.join(ROOT, "tests", "fp8_plans_driver.cpp"),
           "-o", exe, "-L" + B.HERE, "-lgosh", "-Wl,-rpath," + B.HERE]
    made = subprocess.run(cmd, capture_output=True, text=True)
    assert made.returncode == 0, made.stderr[-2000:]

    def ask(lines):
        run = subprocess.run([exe], input="".join(f"{line}\n" for line in lines), capture_output=True, text=True, timeout=120)
        assert run.returncode == 0, run.stderr[-2000:]
        out = [[int(v) for v in line.split()] for line in run.stdout.splitlines()]
        assert len(out) == len(lines)
        return out

    return ask


def test_exact_products_take_tiles_that_they_have(ask):
    """Those of the forward pass and of dx: 32, 64 or 128."""
    rng = random.Random(1)
    log_int = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    some = [(log_int(1, 1 << 23), log_int(1, 65536), log_int(1, 65536)) for _ in range(20000)]
    tiles = [t for (t,) in ask([f"tile {m} {n} {k} 1" for m, n, k in some])]
    assert set(tiles) == {32, 64, 128}
    assert 256 in [t for (t,) in ask([f"tile {m} {n} {k} 0" for m, n, k in some])]


def test_the_shapes_of_the_tests_take_the_tiles_that_they_are_for(ask):
    from tests.test_gpu_fp8_tiles import LARGE, LARGE_DX, PAST, SMALL, SMALL_DX, WHOLE_DW

    def forward(shape, exact=0):
        rows, k, n = shape
        return ask([f"tile {rows} {n} {k} {exact}"])[0][0]

    def dw(shape):
        rows, k, n = shape
        return ask([f"dw {rows} {k} {n} 0"])[0]

    assert forward(LARGE) == 256 and 2 * LARGE[0] * LARGE[2] < 256 << 20
    assert forward(PAST) == 256 and 2 * PAST[0] * PAST[2] >= 256 << 20
    assert forward(PAST, 1) == 128  # the layer with ReLU
    assert forward((LARGE_DX[0], LARGE_DX[2], LARGE_DX[1])) == 256
    tile, splits, blocks = dw(LARGE)
    assert tile == 256 and splits > 1 and blocks % 4 != 0
    assert dw(WHOLE_DW)[:2] == [256, 1]
    for exact in (0, 1):
        assert forward(SMALL, exact) == forward((SMALL_DX[0], SMALL_DX[2], SMALL_DX[1]), exact) == 64
    # and the shapes of test_gpu_fp8.py those of the other sizes, in either kind of products
    from tests.test_gpu_fp8 import SHAPES

    for exact in (0, 1):
        assert {forward(s[:3], exact) for s in SHAPES} | {forward((20011, 512, 1024), exact), forward((70001, 300, 520), exact)} >= {32, 128}
    assert {dw(s[:3])[0] for s in SHAPES} | {dw((20011, 512, 1024))[0]} >= {32, 64, 128}
