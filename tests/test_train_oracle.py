"""CPU pins of the gradients' oracle (oracle/train_oracle.py): its formulas
against central differences of the forward formulas in fp64, and its masks
against the forward's oracle."""
import numpy as np
import pytest

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
