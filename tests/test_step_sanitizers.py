"""The host code of the 8-bit layers, the optimiser and the loss under AddressSanitizer and UndefinedBehaviorSanitizer:
tests/sanitize_step_driver.cpp with their units and those that they need, the sanitizers on the host pass only.  No device
call, so no GPU is needed."""
import os
import subprocess

import pytest

from paper_2008_12336_amd import build as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
UNITS = ["gosh_host.cpp", "gosh_place.hip", "gosh_device_pool.cpp", "gosh_train.hip", "gosh_head.hip", "gosh_fp8.hip", "gosh_fp8_f32.hip",
         "gosh_fp8_bf16.hip", "gosh_fp8_f16.hip", "gosh_loss.hip", "gosh_adamw.hip"]


@pytest.mark.timeout(900)
def test_host_code_of_a_step_is_clean_under_asan_and_ubsan(tmp_path):
    san = []
    for flag in ("-fsanitize=address", "-fsanitize=undefined", "-fno-omit-frame-pointer"):
        san += ["-Xarch_host", flag]
    flags = ["--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fopenmp", "-munsafe-fp-atomics",
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", *san]
    sources = [os.path.join(B.CSRC, unit) for unit in UNITS] + [os.path.join(ROOT, "tests", "sanitize_step_driver.cpp")]
    objects, jobs = [], []
    for source in sources:
        objects.append(str(tmp_path / (os.path.basename(source) + ".o")))
        jobs.append(subprocess.Popen([B.hipcc(), *flags, "-I" + os.path.join(ROOT, "include"), "-I" + B.CSRC, "-x", "hip", "-c",
                                      source, "-o", objects[-1]], stdout=subprocess.DEVNULL, stderr=subprocess.PIPE))
    for job in jobs:
        _, err = job.communicate()
        assert job.returncode == 0, err.decode()[-2000:]
    exe = str(tmp_path / "driver")
    link = subprocess.run([B.hipcc(), *flags, *objects, "-o", exe], capture_output=True, text=True)
    assert link.returncode == 0, link.stderr[-2000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    run = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert run.returncode == 0, run.stdout[-2000:] + run.stderr[-4000:]
    assert "step driver ok" in run.stdout
    assert "runtime error" not in run.stderr and "AddressSanitizer" not in run.stderr, run.stderr[-4000:]
