"""The loads of the products in 8-bit floating point that go straight to LDS, held to the same rules as those of the 16-bit
products: five wait states before each, m0 set for each by the compiler.  (Device pass only, no GPU needed.)"""
import os
import subprocess

import pytest

from paper_2008_12336_amd import build as B
from tests.test_asm_product import ROOT, violations


@pytest.mark.timeout(900)
def test_loads_to_lds_have_their_wait_states(tmp_path):
    jobs = []
    for unit in ("gosh_fp8_f32.hip", "gosh_fp8_bf16.hip", "gosh_fp8_f16.hip"):
        out = str(tmp_path / (unit + ".s"))
        flags = [f for f in B.FLAGS if f not in ("-shared", "-fPIC")]
        cmd = [B.hipcc(), *flags, "--cuda-device-only", "-S", "-I" + os.path.join(ROOT, "include"), "-I" + B.CSRC,
               "-x", "hip", os.path.join(B.CSRC, unit), "-o", out]
        jobs.append((out, subprocess.Popen(cmd, stdout=subprocess.DEVNULL, stderr=subprocess.PIPE)))
    for out, job in jobs:
        _, err = job.communicate()
        assert job.returncode == 0, err.decode()[-2000:]
        loads, bad = violations(open(out))
        assert not bad, "\n".join(bad[:20])
        assert loads >= 100  # three sizes of tiles, two products or more
