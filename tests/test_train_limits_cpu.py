"""The attention backward takes every shape that include/wedlm_train.h allows:
the limits are read there, and the largest shapes within them tried (sizes
only)."""
import math
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2512_22737_amd", "libwedlm.so")
HEADER = os.path.join(ROOT, "include", "wedlm_train.h")

pytestmark = pytest.mark.skipif(not os.path.exists(LIB),
                                reason="libwedlm.so not built")


def documented():
    """The header's limits beyond the forward's, as an expression."""
    text = re.sub(r"\s*\n \*\s*", " ", open(HEADER).read())
    said = re.search(r"Limits: those of the forward, (.*?)\.  ", text).group(1)
    return compile(said.replace("^", "**"), "limits", "eval")


def test_shapes_within_the_limits_are_taken():
    from paper_2512_22737_amd import wedlm
    lib, limits = wedlm.lib(), documented()

    def allowed(L, block, G, D):
        at = dict(L=L, block=block, Hq=G, Hkv=1, D=D, ceil=math.ceil)
        return eval(limits, {}, at) and \
            lib.wedlm_dual_stream_attn_workspace_size(1, L, block, G, 1, D)

    tried = 0
    for block in (1, 3, 5, 15, 16, 24, 40, 47, 48, 63, 64):
        unit = block * 16 // math.gcd(block, 16)
        for L in sorted({unit * max(1, n // unit) for n in (
                1, 64, 240, 256, 272, 1000, 4096, 30000, 1 << 18, 1 << 19,
                1 << 20, (1 << 21) - 64)}):
            for D in (64, 128):
                lo, hi = 0, 1 << 20        # the most heads that are allowed
                while hi - lo > 1:
                    mid = (lo + hi) // 2
                    lo, hi = (mid, hi) if allowed(L, block, mid, D) else (lo,
                                                                          mid)
                if lo == 0:
                    continue
                tried += 1
                for G in {lo, lo - 1, (lo + 1) // 2} - {0}:
                    assert lib.wedlm_dual_stream_attn_backward_workspace_size(
                        1, L, block, G, 1, D) > 0, (L, block, G, D)
    assert tried > 100


def test_shapes_far_beyond_are_refused():
    from paper_2512_22737_amd import wedlm
    ws = wedlm.lib().wedlm_dual_stream_attn_backward_workspace_size
    for s in ((1, 1 << 20, 64, 32, 1, 64), (1, 1 << 19, 32, 128, 1, 64)):
        assert ws(*s) == 0
