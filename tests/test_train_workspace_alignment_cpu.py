"""A workspace that does not start where its contents would (include/
wedlm_train.h) is refused by every training operator that uses one; one that
does is not."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2512_22737_amd", "libwedlm.so")

pytestmark = pytest.mark.skipif(not os.path.exists(LIB),
                                reason="libwedlm.so not built")

F = ctypes.c_void_p(0x1000)       # never dereferenced


def check(call, args, at, step):
    """Offsets that are no multiple of `step` are refused as arguments; those
    that are reach the next check, the workspace's size (one byte short)."""
    for off in (1, 2, 3, 4, 6, 8, 12, 16):
        bad = list(args)
        bad[at] = ctypes.c_void_p(0x1000 + off)
        assert call(*bad) == (-1 if off % step else -3), off


def test_qk_norm_rope_backward():
    from paper_2512_22737_amd import wedlm
    lib = wedlm.lib()
    need = lib.wedlm_qk_norm_rope_backward_workspace_size(3, 4, 2, 64)
    args = [F] * 7 + [3, 4, 2, 64, 1e6, 1e-6] + [F] * 4 + [need - 1, None]
    check(lib.wedlm_qk_norm_rope_backward, args, 16, 4)
    args[14] = None               # one gain's gradient
    check(lib.wedlm_qk_norm_rope_backward, args, 16, 4)


@pytest.mark.parametrize("logits_type", [0, 1])
def test_token_loss(logits_type):
    from paper_2512_22737_amd import wedlm
    lib = wedlm.lib()
    need = lib.wedlm_token_loss_workspace_size(3, 151936)
    assert need > 0               # rows in slices
    args = [F, logits_type, 151936, F, F, 3, 151936, F, F, F, need - 1, None]
    check(lib.wedlm_token_loss, args, 9, 8)
