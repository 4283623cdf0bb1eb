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
