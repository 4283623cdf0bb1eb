"""The loads of the matrix products that go straight to LDS are written in assembly, so the compiler adds no wait states to
them: their range needs five where a vector instruction wrote it last, and m0 (where in LDS they land) has to be set for
each, by an instruction that the compiler knows of.  This compiles the two units that have them (device pass only, no GPU
needed) and checks that every one is preceded by its s_nop 4 and that m0 was written since the load before it."""
import os
import re
import subprocess

import pytest

from paper_2008_12336_amd import build as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def violations(lines):
    """(loads seen, offending lines) of one assembly file."""
    loads, bad = 0, []
    before, m0_set, hand_written = "", False, False
    for number, line in enumerate(lines, 1):
        text = line.strip()
        if text.startswith(";;#ASMSTART"):
            hand_written = True
        elif text.startswith(";;#ASMEND"):
            hand_written = False
        if not text or text[0] in ";." or text.endswith(":"):
            continue
        if re.match(r"buffer_load_\S+ .*\blds$", text):
            loads += 1
            nop = re.match(r"s_nop (\d+)$", before)
            if not nop or int(nop.group(1)) < 4:
                bad.append(f"{number}: no five wait states: {before} / {text}")
            if not m0_set:
                bad.append(f"{number}: m0 is not set for {text}")
            m0_set = False
        elif re.match(r"s_\S+ m0,", text):
            m0_set = True
            if hand_written:
                bad.append(f"{number}: written behind the compiler's back: {text}")
        before = text
    return loads, bad


@pytest.mark.timeout(900)
def test_loads_to_lds_have_their_wait_states(tmp_path):
    jobs = []
    for unit in ("gosh_product_bf16.hip", "gosh_product_f16.hip"):
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
        assert loads >= 100  # three sizes of tiles, five products


def test_what_the_check_finds():
    load = "buffer_load_dwordx4 v5, s[12:15], 0 offen lds"
    assert violations(["s_mov_b32 m0, s1", "s_nop 4", load, "s_add_i32 m0, s1, 0x400", "s_nop 4", load]) == (2, [])
    assert len(violations(["s_mov_b32 m0, s1", "s_nop 0", load])[1]) == 1
    assert len(violations(["s_mov_b32 m0, s1", "s_nop 4", load, "s_nop 4", load])[1]) == 1
    assert len(violations([";;#ASMSTART", "s_mov_b32 m0, s1", "s_nop 4", load, ";;#ASMEND"])[1]) == 1
