"""Host-side refusals of the serving operators (include/wedlm_serve.h): no
call here gets past the validation of its arguments."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2512_22737_amd", "libwedlm.so")

pytestmark = pytest.mark.skipif(not os.path.exists(LIB),
                                reason="libwedlm.so not built")

F = ctypes.c_void_p(0x1000)       # never dereferenced
ODD = ctypes.c_void_p(0x1008)


def _lib():
    from paper_2512_22737_amd import wedlm
    return wedlm.lib()


def refusals(call, args, cases):
    for at, value, code in cases:
        bad = list(args)
        bad[at] = value
        assert call(*bad) == code, (at, value)


def test_append_refusals():
    args = [F] * 4 + [2, 3, 20, 2, 64] + [F] * 4 + [10, F, 4, None, None]
    refusals(_lib().wedlm_cache8_append, args,
             [(i, None, -1) for i in (0, 1, 2, 3, 9, 10, 11, 12, 14)] +
             [(i, 0, -2) for i in (4, 5, 6, 7, 13, 15)] +
             [(8, 96, -2), (13, 1 << 31, -2), (6, 1 << 29, -2),
              (5, 1 << 25, -2)] +
             [(i, ODD, -1) for i in (0, 1, 9, 10)])


def test_attention_refusals():
    lib = _lib()
    size = lib.wedlm_window_attn_cache8_workspace_size
    assert size(1, 16, 4, 2, 64, 100) == 0              # one split
    # 2 kv heads of 32 rows, 16 splits of at least 256 keys: fp32 sums of 64
    # values and two floats each, and how many splits there are
    need = size(1, 16, 4, 2, 64, 4096)
    assert need == 2 * 32 * 16 * (64 + 2) * 4 + 4
    # the longest prefix of one sequence: splits of 32768 keys
    assert size(1, 1, 1, 1, 64, 2**31 - 1) == 65536 * 32 * (64 + 2) * 4 + 4
    # 3 sequences, 8 heads, 128 rows, 16 splits at most
    assert size(3, 32, 32, 8, 128, 4096) == 3 * 8 * 128 * 16 * 130 * 4 + 12
    for bad in ((0, 16, 4, 2, 64, 9), (1, 65, 4, 2, 64, 9),
                (1, 16, 5, 2, 64, 9), (1, 16, 4, 2, 96, 9),
                (1, 16, 4, 2, 64, -1), (1 << 30, 64, 4, 2, 64, 9),
                (64, 64, 32, 8, 128, 2**31 - 1)):
        assert size(*bad) == 0, bad
    args = [F] * 7 + [300, F, 256, F, 1, 16, 4, 2, 64, 4096, 0.125, F, None,
                      None, F, need, None]
    refusals(lib.wedlm_window_attn_cache8, args,
             [(i, None, -1) for i in (0, 1, 2, 3, 4, 5, 6, 8, 10, 18)] +
             [(7, 0, -1), (9, 0, -1), (7, 1 << 31, -2), (11, 0, -2),
              (12, 0, -2), (12, 65, -2), (13, 5, -2), (14, 0, -2),
              (15, 32, -2), (16, -1, -2), (17, 0.0, -1),
              (17, float("nan"), -1), (17, float("inf"), -1),
              (21, None, -3), (22, need - 1, -3),
              (21, ctypes.c_void_p(0x1010), -1)] +
             [(i, ODD, -1) for i in (0, 1, 2, 3, 4, 18)])


def test_commit_refusals():
    args = ([F] * 4 + [0.9, 0.01] + [F] * 6 + [10, F, 4, 3, 16, 2, 64, 2] +
            [F] * 5 + [0, None])
    refusals(_lib().wedlm_commit_cache8, args,
             [(i, None, -1) for i in (0, 1, 2, 3, 6, 7, 8, 9, 10, 11, 13, 20,
                                      21, 22, 23, 24)] +
             [(4, float("nan"), -1), (25, 3, -1), (12, 0, -2), (14, 0, -2),
              (15, 0, -2), (16, 65, -2), (17, 0, -2), (18, 96, -2),
              (19, 0, -2), (12, 1 << 30, -2)] +
             [(i, ODD, -1) for i in (6, 7, 8, 9)])


def test_free_refusals():
    args = [F, 2, F, 4, 8, F, 100, None, None]
    refusals(_lib().wedlm_cache_free, args,
             [(i, None, -1) for i in (0, 2, 5)] +
             [(1, 0, -2), (1, 65536, -2), (3, 0, -2), (4, 0, -2), (6, 0, -2),
              (6, 1 << 31, -2)])


def _arrays(*made):
    from paper_2512_22737_amd import wedlm
    return (wedlm.PageArray * len(made))(*(wedlm.PageArray(*m) for m in made))


def test_fork_refusals():
    lib = _lib()
    size = lib.wedlm_cache_fork_workspace_size
    need = size(2, 8, 100)
    assert need > 0
    assert size(0, 8, 100) == size(65536, 8, 100) == size(2, 0, 100) == 0
    assert size(2, 8, 0) == size(2, 8, 1 << 31) == 0
    one = _arrays((0x1000, 64))
    args = [F, F, F, 2, F, F, 4, 8, F, 100, one, 1, 3, F, F, need, None]
    refusals(lib.wedlm_cache_fork, args,
             [(i, None, -1) for i in (0, 1, 2, 4, 5, 8, 10, 13)] +
             [(3, 0, -2), (3, 65536, -2), (6, 0, -2), (7, 0, -2), (9, 0, -2),
              (9, 1 << 31, -2), (11, -1, -2), (11, 9, -2), (12, 0, -2),
              (12, 8192, -2), (14, None, -3), (15, need - 1, -3),
              (14, ctypes.c_void_p(0x1004), -1),
              (10, _arrays((None, 64)), -1), (10, _arrays((0x1000, 0)), -1)])


def test_compact_refusals():
    lib = _lib()
    size = lib.wedlm_cache_compact_workspace_size
    need = size(100)
    assert need > 0 and size(0) == size(1 << 31) == 0
    one = _arrays((0x1000, 64))
    args = [F, 4, 8, F, 100, one, 1, 3, F, F, F, F, need, None]
    refusals(lib.wedlm_cache_compact, args,
             [(i, None, -1) for i in (0, 3, 5, 8, 9, 10)] +
             [(1, 0, -2), (2, 0, -2), (1, 1 << 30, -2), (4, 0, -2),
              (4, 1 << 31, -2), (6, 9, -2), (7, 0, -2), (11, None, -3),
              (12, need - 1, -3), (11, ctypes.c_void_p(0x1004), -1)])


def test_sample_refusals():
    args = [F, 0, 64, F, None, None, None, None, None, 2, 3, 64, F, None, None]
    refusals(_lib().wedlm_sample, args,
             [(i, None, -1) for i in (0, 3, 12)] +
             [(1, 2, -1), (1, -1, -1), (2, 63, -2), (9, 0, -2), (10, 0, -2),
              (11, 0, -2), (11, (1 << 22) + 1, -2), (9, 1 << 22, -2)])


def test_binding_refusals():
    """What the binding refuses before it calls the library (on the CPU every
    tensor is refused; here the sizes are)."""
    import torch
    from paper_2512_22737_amd import wedlm
    assert wedlm.wedlm_cache_compact_workspace_size(1 << 33) == 0
    x = torch.zeros(2, 3)
    with pytest.raises(wedlm.WedlmError, match="arrays"):
        wedlm._page_arrays([x], 3)
    t = torch.zeros(2, 4, dtype=torch.int32)
    with pytest.raises(wedlm.WedlmError, match="device"):
        wedlm.wedlm_cache_free(t[0], t, t[0])


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_step_refuses_a_mix_before_it_starts(cache):
    """One exponent alone is no 8-bit cache and no bf16 one; settings need
    random numbers."""
    import torch
    from paper_2512_22737_amd import wedlm
    step = wedlm.DecodeStep(1, 2, 2, 1, 64, 8, 16, device="cpu", cache=cache)
    e = torch.zeros(1, 1, dtype=torch.uint8)
    wrong = [(e, None), (None, e), (None, None) if step.eight_bits else (e, e)]
    for k, v in wrong:
        with pytest.raises(wedlm.WedlmError, match="exponents"):
            step(*[None] * 7, k_exp=k, v_exp=v)
    good = (e, e) if step.eight_bits else (None, None)
    with pytest.raises(wedlm.WedlmError, match="random"):
        step(*[None] * 7, *good, top_k=e)
