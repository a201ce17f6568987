"""What the binding of the training operators does around the library's call,
with the library replaced by a recorder: no GPU needed."""
import gc
import weakref

import pytest
import torch

from paper_2512_22737_amd import wedlm as W

bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)


def _attention():
    q, k = bf(1, 32, 4, 64), bf(1, 32, 2, 64)
    W.wedlm_dual_stream_attn_backward(q, k, k, 16, q, torch.zeros(1, 32, 4), q,
                                      q, k, k)


def _rmsnorm():
    x = torch.zeros(3, 64)
    W.wedlm_rmsnorm_backward(x, bf(64), 1e-6, bf(3, 64), x, torch.zeros(64))


def _qk():
    W.wedlm_qk_norm_rope_backward(
        bf(3, 8 * 64), bf(64), bf(64), torch.zeros(3, dtype=torch.int32), 1e4,
        1e-6, bf(3, 4, 64), bf(3, 2, 64), bf(3, 2, 64), bf(3, 8 * 64),
        torch.zeros(64))


def _loss():
    W.wedlm_token_loss(torch.zeros(2, 50), torch.zeros(2, dtype=torch.int32),
                       torch.zeros(2))


@pytest.mark.parametrize("call", [_attention, _rmsnorm, _qk, _loss])
def test_a_workspace_lives_until_the_launches_are_enqueued(call, monkeypatch):
    made, alive = [], []

    class Recorder:
        def __getattr__(self, name):
            if name.endswith("_workspace_size"):
                return lambda *a: 1 << 12

            def run(*a):
                gc.collect()
                alive.append(made[-1]() is not None)
                return W.WEDLM_OK
            return run

    def empty(*a, **kw):
        x = torch.zeros(*a, **kw)
        made.append(weakref.ref(x))
        return x

    monkeypatch.setattr(W, "_load", Recorder)
    monkeypatch.setattr(W, "_stream", lambda: 0)
    monkeypatch.setattr(W, "_t", lambda x, *a, **kw: x if x is None
                        else x.data_ptr())
    monkeypatch.setattr(W.torch, "empty", empty)
    call()
    assert len(made) == 1 and alive == [True]
