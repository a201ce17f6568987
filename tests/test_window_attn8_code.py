"""The 8-bit attention's generated code, what the compiler does not look after
around the LDS loads written as text: the scalar registers that they read are
not written by a vector instruction, nor M0 by any, within the wait states that
this takes.  Compiles the source to assembly for gfx950 (no GPU needed)."""
import os
import re
import subprocess

import pytest

from paper_2512_22737_amd import build as B

SRC = "window_attn8.hip"


@pytest.fixture(scope="module")
def code(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("asm") / "k.s")
    try:
        cc = B.hipcc()
    except RuntimeError:
        pytest.skip("no hipcc")
    subprocess.run([cc, *B.HIPCC_FLAGS, *B.FILE_FLAGS[SRC], "-I", B.INCLUDE,
                    "-I", B.CSRC, "-S", "--cuda-device-only",
                    os.path.join(B.CSRC, SRC), "-o", out], check=True,
                   capture_output=True, timeout=600)
    lines = [l.split(";")[0].strip() for l in open(out)]
    return [l for l in lines if l and (not l.startswith(".") or
                                       l.endswith(":"))]


def late_scalars(code):
    """(load, instruction that writes what it reads too late), and how many
    loads there are."""
    bad, loads = [], 0
    for i, l in enumerate(code):
        m = re.match(r"buffer_load\w+ v\d+, s\[(\d+):(\d+)\], .*\blds\b", l)
        if not m:
            continue
        loads += 1
        lo, hi = int(m.group(1)), int(m.group(2))
        states = 0
        for j in range(i - 1, -1, -1):
            c = code[j]
            nop = re.match(r"s_nop (\d+)", c)
            w = re.match(r"v_\S+ s(?:(\d+)\b|\[(\d+):(\d+)\])", c)
            if w:
                a = int(w.group(1) or w.group(2))
                b = int(w.group(1) or w.group(3))
                if a <= hi and b >= lo:
                    bad.append((l, c))
            if states < 1 and re.match(r"s_\S+ m0\b", c):
                bad.append((l, c))
            states += int(nop.group(1)) + 1 if nop else 1
            if states >= 5 or c.endswith(":"):
                break
    return bad, loads


def test_the_loads_scalars_are_written_in_time(code):
    bad, loads = late_scalars(code)
    assert loads >= 40, loads
    assert not bad, bad[:4]


def test_the_check_sees_a_late_one():
    ok = ["v_readfirstlane_b32 s5, v1", "s_mov_b32 m0, s9", "s_nop 4",
          "buffer_load_dwordx4 v1, s[4:7], 0 offen nt lds"]
    assert late_scalars(ok) == ([], 1)
    assert len(late_scalars(ok[:2] + ok[3:])[0]) == 2
    assert late_scalars(["v_readlane_b32 s7, v1, 3", "s_nop 3", ok[3]])[0]


