"""The training operators' sizes over the whole range of their arguments, with
the host code compiled to trap where a signed number overflows (no GPU needed:
what the host code calls of the HIP runtime is replaced)."""
import os
import random
import re
import subprocess
import sys

import pytest

from paper_2512_22737_amd import build as B

SOURCES = ("attn_backward", "norm_backward", "token_loss", "dual_stream",
           "window_attn")

RUN = """
import ctypes, sys
call = getattr(ctypes.CDLL(sys.argv[1]), sys.argv[2])
call.restype = ctypes.c_size_t
for line in sys.stdin:
    args = [int(x) for x in line.split()]
    print(call(*(ctypes.c_int32(x) for x in args)), flush=True)
"""

EDGES = (-2**31, -1, 0, 1, 2, 3, 4, 16, 24, 64, 128, 1000, 4096, 65535, 1 << 20,
         (1 << 20) + 4, 1 << 26, 1 << 28, (1 << 30) - 1, 1 << 30, (1 << 30) + 5,
         2**31 - 256, 2**31 - 16, 2**31 - 1)


@pytest.fixture(scope="module")
def library(tmp_path_factory):
    at = tmp_path_factory.mktemp("host")
    try:
        cc = B.hipcc()
    except RuntimeError:
        pytest.skip("no hipcc")
    objects = []
    for name in SOURCES:
        o = str(at / (name + ".o"))
        subprocess.run(
            [cc, "--cuda-host-only", "--offload-arch=gfx950", "-O1",
             "-std=c++17", "-fPIC", "-Xarch_host",
             "-fsanitize=signed-integer-overflow,integer-divide-by-zero",
             "-Xarch_host", "-fsanitize-trap=all", "-I", B.INCLUDE, "-I",
             B.CSRC, "-c", os.path.join(B.CSRC, name + ".hip"), "-o", o],
            check=True, capture_output=True, timeout=120)
        objects.append(o)
    names = subprocess.run(["nm", "-u", *objects], check=True, text=True,
                           capture_output=True).stdout
    stub = at / "stub.c"
    stub.write_text("".join(f"int {x}(void) {{ return 1; }}\n" for x in sorted(
        set(re.findall(r"\b(?:__)?hip\w+", names)))))
    out = str(at / "host.so")
    subprocess.run(["gcc", "-shared", "-fPIC", "-w", str(stub), *objects, "-o",
                    out, "-lstdc++", "-lm"], check=True, capture_output=True)
    return out


def sizes(library, name, shapes):
    r = subprocess.run([sys.executable, "-c", RUN, library, name], text=True,
                       input="\n".join(" ".join(map(str, s)) for s in shapes),
                       capture_output=True, timeout=100)
    got = [int(x) for x in r.stdout.split()]
    assert r.returncode == 0, (name, shapes[len(got)], r.returncode, r.stderr)
    return got


@pytest.mark.parametrize("name,n", [
    ("wedlm_rmsnorm_backward_workspace_size", 2),
    ("wedlm_qk_norm_rope_backward_workspace_size", 4),
    ("wedlm_token_loss_workspace_size", 2),
    ("wedlm_dual_stream_attn_backward_workspace_size", 6)])
def test_sizes_do_not_overflow(library, name, n):
    rng = random.Random(n)
    shapes = [[rng.choice(EDGES) for _ in range(n)] for _ in range(4000)]
    if n == 6:                  # heads and blocks that go together
        for s in shapes[1000:]:
            s[2] = rng.choice((1, 16, 24, 64))
            s[1] = rng.choice((48, 4032, 48 * 21845, 48 * 43690))
            s[0] = rng.choice((1, 7, 300))
            s[4] = rng.choice((1, 3, 1 << 10, 1 << 20))
            s[3] = s[4] * rng.choice((1, 8, 1 << 9))
            s[5] = rng.choice((64, 128))
    got = sizes(library, name, shapes)
    assert any(got) and not all(got)


def test_rows_of_too_many_heads_are_no_shape(library):
    ws = "wedlm_qk_norm_rope_backward_workspace_size"
    shapes = [(1, Hq, Hkv, D) for Hq in (1, 4, 1 << 30, 2**31 - 1)
              for Hkv in ((1 << 30) - 1, 1 << 30, (1 << 30) + 5, 2**31 - 1)
              for D in (64, 128)]
    assert not any(sizes(library, ws, shapes))
