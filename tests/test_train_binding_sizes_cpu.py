"""Sizes that the library's 32-bit arguments cannot hold are refused by the
binding of the training operators, not cut to 32 bits: the call would leave
most rows as they were, without an error.  (Tensors without memory, the library
replaced by a recorder: no GPU needed.)"""
import pytest
import torch

from paper_2512_22737_amd import wedlm as W

N = 1 << 32                       # cut to 32 bits: nothing left of it


def meta(*s, dtype=torch.bfloat16):
    return torch.empty(*s, dtype=dtype, device="meta")


def f32(*s):
    return meta(*s, dtype=torch.float32)


def i32(*s):
    return meta(*s, dtype=torch.int32)


def _attention(n=1, L=32, Hq=4, Hkv=2):
    q, k = meta(n, 2 * L, Hq, 64), meta(n, 2 * L, Hkv, 64)
    W.wedlm_dual_stream_attn_backward(q, k, k, 16, q, f32(n, 2 * L, Hq), q, q,
                                      k, k)


def _rmsnorm(M=3, Hd=64):
    W.wedlm_rmsnorm_backward(f32(M, Hd), meta(Hd), 1e-6, meta(M, Hd),
                             f32(M, Hd), f32(Hd))


def _qk(M=3, Hq=4, Hkv=2):
    rows = meta(M, (Hq + 2 * Hkv) * 64)
    W.wedlm_qk_norm_rope_backward(
        rows, meta(64), meta(64), i32(M), 1e4, 1e-6, meta(M, Hq, 64),
        meta(M, Hkv, 64), meta(M, Hkv, 64), rows, f32(64))


def _loss(R=2, V=50):
    W.wedlm_token_loss(f32(R, V), i32(R), f32(R), V=V)


@pytest.fixture
def calls(monkeypatch):
    made = []

    class Recorder:
        def __getattr__(self, name):
            return lambda *a: made.append(name) or W.WEDLM_OK

    monkeypatch.setattr(W, "_load", Recorder)
    monkeypatch.setattr(W, "_stream", lambda: 0)
    monkeypatch.setattr(W, "_t", lambda x, *a, **kw: None)
    return made


@pytest.mark.parametrize("call,size", [
    (_attention, "n"), (_attention, "L"), (_attention, "Hq"),
    (_attention, "Hkv"), (_rmsnorm, "M"), (_rmsnorm, "Hd"), (_qk, "M"),
    (_qk, "Hq"), (_qk, "Hkv"), (_loss, "R"), (_loss, "V")])
def test_refused(call, size, calls):
    for n in (N + 64, 1 << 31):
        with pytest.raises(W.WedlmError, match="2\\^31"):
            call(**{size: n})
    assert not calls


@pytest.mark.parametrize("call", [_attention, _rmsnorm, _qk, _loss])
def test_usual_sizes_reach_the_library(call, calls):
    call()
    assert calls and not calls[-1].endswith("_size")


@pytest.mark.parametrize("size,n", [
    (W.wedlm_dual_stream_attn_backward_workspace_size, 6),
    (W.wedlm_rmsnorm_backward_workspace_size, 2),
    (W.wedlm_qk_norm_rope_backward_workspace_size, 4),
    (W.wedlm_token_loss_workspace_size, 2)])
def test_workspace_sizes(size, n, calls):
    """0, as for every shape that is not supported."""
    for at in range(n):
        shape = [64] * n
        shape[at] += N
        assert size(*shape) == 0
    assert not calls
