"""CPU pins of the gradients' oracle (oracle/train_oracle.py): its formulas
against central differences of the forward formulas in fp64, and its masks
against the forward's oracle."""
import numpy as np
import pytest
import torch

from oracle import train_oracle as T
from oracle import wedlm_oracle as O

H = 1e-5


def differences(f, x, g):
    """d/dx of sum(f(x) * g) by central differences, element by element."""
    d = np.empty_like(x)
    for i in np.ndindex(*x.shape):
        at = x[i]
        x[i] = at + H
        hi = (f(x) * g).sum()
        x[i] = at - H
        lo = (f(x) * g).sum()
        x[i] = at
        d[i] = (hi - lo) / (2 * H)
    return d


@pytest.mark.parametrize("L,block", [(16, 4), (12, 12), (10, 5), (6, 1)])
def test_masks_are_the_forward_oracles(L, block):
    # positions observed or not reorder rows inside a block only
    want = O.dual_stream_visible(L, block, set())
    assert (T.dual_stream_visible(L, block) == want).all()


@pytest.mark.parametrize("L,block,Hq,Hkv,D", [(6, 3, 4, 2, 4), (4, 1, 3, 1, 3),
                                              (5, 5, 2, 2, 4)])
def test_attention_backward_against_differences(L, block, Hq, Hkv, D):
    rng = np.random.default_rng(L)
    q, dout = rng.standard_normal((2, 2 * L, Hq, D))
    k, v = rng.standard_normal((2, 2 * L, Hkv, D))
    vis, s = T.dual_stream_visible(L, block), 0.7
    (dq, dk, dv), bounds = T.attn_backward(q, k, v, dout, vis, s)
    f = lambda a, b, c: T.attn_forward(a, b, c, vis, s)[0]
    # O(H^2) of a smooth function of order-one values, O(eps / H) of rounding
    for got, want in ((dq, differences(lambda x: f(x, k, v), q, dout)),
                      (dk, differences(lambda x: f(q, x, v), k, dout)),
                      (dv, differences(lambda x: f(q, k, x), v, dout))):
        assert np.abs(got - want).max() < 1e-8
    assert all((b >= 0).all() for b in bounds)


def test_rmsnorm_backward_against_differences():
    rng = np.random.default_rng(1)
    x, dy = rng.standard_normal((2, 3, 5))
    gain = rng.standard_normal(5)
    x[1] = 0.0                                # a zero row: eps alone
    (dx, dg), bounds = T.rmsnorm_backward(x, gain, dy, 0.3)
    assert np.abs(dx - differences(lambda a: T.rmsnorm(a, gain, 0.3), x,
                                   dy)).max() < 1e-8
    assert np.abs(dg - differences(lambda a: T.rmsnorm(x, a, 0.3), gain,
                                   dy)).max() < 1e-8
    assert all((b >= 0).all() for b in bounds)


def test_qk_norm_rope_backward_against_differences():
    rng = np.random.default_rng(2)
    M, heads, D, theta, eps = 3, 2, 6, 100.0, 0.01
    x, dy = rng.standard_normal((2, M, heads, D))
    gain, pos = rng.standard_normal(D), np.array([0, 7, 1000])
    f = lambda a, g: T.rotate(T.rmsnorm(a, g, eps), pos, theta)
    (dx, dg), _ = T.qk_norm_rope_backward(x, gain, pos, dy, theta, eps)
    assert np.abs(dx - differences(lambda a: f(a, gain), x, dy)).max() < 1e-8
    assert np.abs(dg - differences(lambda g: f(x, g), gain, dy)).max() < 1e-8


def test_rotation_is_the_step_oracles():
    x = np.random.default_rng(3).standard_normal((1, 1, 8))
    got = T.rotate(x, np.array([37]), 1e4)
    assert np.abs(got[0, 0] - O.rope(x[0, 0], 37, 1e4)).max() < 1e-12


def test_token_loss_against_differences():
    rng = np.random.default_rng(5)
    x = rng.standard_normal((4, 6))
    x[1, 2] = -np.inf
    target, weight = np.array([0, 3, -1, 5]), np.array([1.0, -0.5, 2.0, 0.0])
    (loss, d), _ = T.token_loss(x, target, weight)
    want = np.zeros_like(x)
    for r in range(4):
        keep = np.isfinite(x[r])
        row = x[r].copy()

        def f(part):
            row[keep] = part
            return T.token_loss(row[None], target[r:r + 1],
                                weight[r:r + 1])[0][0]
        want[r, keep] = differences(f, x[r, keep].copy(), 1.0)
    assert np.abs(d - want).max() < 1e-8
    assert loss[2] == loss[3] == 0 and (d[2:] == 0).all() and d[1, 2] == 0


def test_token_loss_is_the_library_cross_entropy():
    rng = np.random.default_rng(6)
    x, t = 5 * rng.standard_normal((7, 50)), rng.integers(0, 50, 7)
    (loss, d), _ = T.token_loss(x, t, np.ones(7))
    y = torch.from_numpy(x).requires_grad_(True)
    ref = torch.nn.functional.cross_entropy(y, torch.from_numpy(t),
                                            reduction="none")
    ref.sum().backward()
    assert np.abs(loss - ref.detach().numpy()).max() < 1e-12
    assert np.abs(d - y.grad.numpy()).max() < 1e-12
