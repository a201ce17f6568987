"""Host-side refusals of the training operators (include/wedlm_train.h): no
call here gets past the validation of its arguments."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2512_22737_amd", "libwedlm.so")

pytestmark = pytest.mark.skipif(not os.path.exists(LIB),
                                reason="libwedlm.so not built")

F = ctypes.c_void_p(0x1000)       # never dereferenced


def _lib():
    from paper_2512_22737_amd import wedlm
    return wedlm.lib()


def refusals(call, args, cases):
    for at, value, code in cases:
        bad = list(args)
        bad[at] = value
        assert call(*bad) == code, (at, value)


def test_attention_backward_workspace():
    ws = _lib().wedlm_dual_stream_attn_backward_workspace_size
    assert ws(1, 128, 32, 4, 2, 64) > 0
    # lse and D of 4 x 2 x 4096 rows of 32 heads, and partial sums
    assert ws(4, 4096, 32, 32, 8, 128) > 4 * 8192 * 32 * 8
    for bad in ((0, 128, 32, 4, 2, 64), (1, 100, 32, 4, 2, 64),
                (1, 128, 96, 4, 2, 64), (1, 128, 32, 4, 2, 96),
                (1, 128, 32, 5, 2, 64), (1, 128, 0, 4, 2, 64),
                (1, 24, 8, 4, 2, 64), (1, 128, 32, 0, 0, 64),
                (4, 65536, 1, 4, 2, 64)):
        assert ws(*bad) == 0, bad


def test_attention_backward_refusals():
    lib = _lib()
    need = lib.wedlm_dual_stream_attn_backward_workspace_size(1, 128, 32, 4, 2,
                                                              64)
    args = [F] * 6 + [1, 128, 32, 4, 2, 64, 0.125] + [F] * 4 + [need, None]
    refusals(lib.wedlm_dual_stream_attn_backward, args,
             [(i, None, -1) for i in (0, 1, 2, 3, 4, 5, 13, 14, 15)] +
             [(12, 0.0, -1), (12, float("nan"), -1), (12, float("inf"), -1),
              (7, 120, -2), (8, 33, -2), (9, 3, -2), (11, 32, -2),
              (16, None, -3), (17, need - 1, -3)])
    odd = ctypes.c_void_p(0x1008)
    refusals(lib.wedlm_dual_stream_attn_backward, args,
             [(i, odd, -1) for i in (0, 1, 2, 3, 5, 13, 14, 15, 16)])


def test_attention_backward_refuses_what_its_offsets_cannot_hold():
    ws = _lib().wedlm_dual_stream_attn_backward_workspace_size
    assert ws(1, 16, 16, 1 << 18, 1 << 18, 128) == 0
    assert ws(1, 1 << 20, 64, 1 << 16, 1, 64) == 0


def test_rmsnorm_backward_refusals():
    lib = _lib()
    ws = lib.wedlm_rmsnorm_backward_workspace_size
    assert ws(0, 64) == ws(4, 0) == ws(4, 66) == 0
    need = ws(3, 64)
    assert need == 3 * 64 * 4
    args = [F] * 4 + [3, 64, 1e-6, F, F, F, need, None]
    refusals(lib.wedlm_rmsnorm_backward, args,
             [(i, None, -1) for i in (0, 1, 2, 7)] +
             [(6, 0.0, -1), (6, float("nan"), -1), (4, 0, -2), (5, 2, -2),
              (5, 66, -2), (9, None, -3), (10, need - 1, -3)] +
             [(i, ctypes.c_void_p(0x1008), -1) for i in (0, 3, 7, 9)] +
             [(i, ctypes.c_void_p(0x1004), -1) for i in (1, 2)])


def test_qk_norm_rope_backward_refusals():
    lib = _lib()
    ws = lib.wedlm_qk_norm_rope_backward_workspace_size
    assert ws(0, 4, 2, 64) == ws(3, 4, 2, 96) == ws(3, 4, 0, 64) == 0
    assert ws(3, 1 << 24, 2, 128) == 0
    need = ws(3, 4, 2, 64)
    args = [F] * 7 + [3, 4, 2, 64, 1e6, 1e-6] + [F] * 4 + [need, None]
    refusals(lib.wedlm_qk_norm_rope_backward, args,
             [(i, None, -1) for i in (0, 1, 2, 3, 4, 5, 6, 13)] +
             [(11, 1.0, -1), (12, 0.0, -1), (7, 0, -2), (8, 0, -2),
              (9, -1, -2), (10, 32, -2), (16, None, -3), (17, need - 1, -3)] +
             [(i, ctypes.c_void_p(0x1008), -1) for i in (0, 1, 2, 4, 5, 6, 13)])


def test_token_loss_refusals():
    lib = _lib()
    ws = lib.wedlm_token_loss_workspace_size
    assert ws(0, 64) == ws(4, 0) == ws(-1, -1) == 0
    need = ws(3, 64)
    args = [F, 0, 64, F, F, 3, 64, F, F, F, need, None]
    refusals(lib.wedlm_token_loss, args,
             [(i, None, -1) for i in (0, 3, 7)] +
             [(1, 2, -1), (1, -1, -1), (2, 63, -2), (5, 0, -2), (6, 0, -2)])


def test_rmsnorm_backward_refuses_the_longest_rows():
    """A launch over their columns would have more than 2^32 threads."""
    lib = _lib()
    ws = lib.wedlm_rmsnorm_backward_workspace_size
    assert ws(1, 1 << 20) == 4 << 20 and ws(1, (1 << 20) + 4) == 0
    args = [F] * 4 + [1, (1 << 20) + 4, 1e-6, F, F, F, 1 << 40, None]
    assert lib.wedlm_rmsnorm_backward(*args) == -2
