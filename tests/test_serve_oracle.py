"""The serving operators' oracle against independent facts: torch's e4m3
conversion, plain attention over rows that are codes, exhaustive sampling, and
what page sharing has to keep."""
import numpy as np
import pytest
import torch

from oracle import serve_oracle as O


def test_codes_are_torchs():
    c = np.arange(256, dtype=np.uint8)
    t = torch.from_numpy(c).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(np.nan_to_num(t, nan=7e7),
                          np.nan_to_num(O.VALUES, nan=7e7))
    rng = np.random.default_rng(0)
    x = np.concatenate((rng.standard_normal(4000) * 100, O.VALUES[:127],
                        (O.VALUES[:126] + O.VALUES[1:127]) / 2,
                        rng.standard_normal(500) * 2e-3, [0.0, -0.0, -448.0]))
    x = x[np.abs(x) <= 448].astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8)
    assert np.array_equal(O.encode(x), want.numpy())


@pytest.mark.parametrize("a,e", [
    (0.0, 1), (448.0, 127), (448.5, 128), (224.0, 126), (1.0, 119), (1.76, 120),
    (1.75, 119), (3.4e38, 247), (1e-38, 1), (2.0 ** -133, 1)])
def test_need_exp(a, e):
    assert O.need_exp([a, -a / 2, np.nan, np.inf]) == e


def test_append_keeps_what_it_should():
    rng = np.random.default_rng(1)
    k = rng.standard_normal((1, 1, 20, 1, 64))
    v = rng.standard_normal((1, 1, 20, 1, 64))
    k[0, 0, 10:] *= 50                      # the page's scale has to grow
    bt = np.array([[2, 0]], np.int32)
    st = [rng.integers(0, 127, (1, 3, 1, 16, 64)).astype(np.uint8),
          rng.integers(0, 127, (1, 3, 1, 64, 16)).astype(np.uint8),
          np.full((1, 3, 1), 120, np.uint8), np.full((1, 3, 1), 120, np.uint8)]
    one = O.append(k[:, :, :9], v[:, :, :9], [0], [9], *st, bt)
    two = O.append(k[:, :, 9:], v[:, :, 9:], [9], [11], *one[:4], bt)
    assert two[4][0] == 0 and two[2][0, 2, 0] > one[2][0, 2, 0]
    kk, vv = O.gather(two[0][0], two[1][0], two[2][0], two[3][0], bt, 0, 20)
    for got, want in ((kk, k), (vv, v)):
        want = want[0, 0]
        # two roundings at most, or the smallest code's half step of a page
        err = np.abs(got - want)
        top = np.abs(want).max()
        assert (err <= np.abs(want) * 2.0 ** -3 + top * 2.0 ** -15).all()
    # page 1 and the rows behind the last new one are as they were
    assert np.array_equal(two[0][0, 1], st[0][0, 1])
    assert np.array_equal(two[0][0, 0, 0, 4:], st[0][0, 0, 0, 4:])
    assert np.array_equal(two[1][0, 0, 0, :, 4:], st[1][0, 0, 0, :, 4:])


def test_attention_is_softmax():
    rng = np.random.default_rng(2)
    q = rng.standard_normal((3, 4, 64))
    kw, vw = rng.standard_normal((2, 3, 2, 64))
    kp, vp = rng.standard_normal((2, 21, 2, 64))
    out, lse, bo, bl = O.attention(q, kw, vw, kp, vp, 0.125)
    k = torch.from_numpy(np.concatenate((kp, kw))).transpose(0, 1)
    v = torch.from_numpy(np.concatenate((vp, vw))).transpose(0, 1)
    mask = torch.ones(3, 24).tril(21).bool()
    want = torch.nn.functional.scaled_dot_product_attention(
        torch.from_numpy(q).transpose(0, 1), k.repeat_interleave(2, 0),
        v.repeat_interleave(2, 0), attn_mask=mask).transpose(0, 1).numpy()
    assert np.abs(out - want).max() < 1e-12
    assert (bo > 0).all() and (bo < 0.05).all() and (bl < 1e-4).all()


def test_sample_takes_the_shares():
    rng = np.random.default_rng(3)
    x = np.array([0.0, 1.0, 1.0, -np.inf, 3.0, 1.0, np.nan])
    us = (np.arange(20000) + 0.5) / 20000
    p = np.exp(np.where(np.isnan(x), -np.inf, x) / 0.7)
    p /= p.sum()
    got = np.bincount([O.sample(x, u, 0.7)[0] for u in us], minlength=7)
    assert np.abs(got / len(us) - p).max() < 1e-3
    # ties go to the lowest ids
    assert {O.sample(x, u, 0.7, top_k=3)[0] for u in us[::50]} == {1, 2, 4}
    assert {O.sample(x, u, 0.7, top_p=p[4] + p[1] * 1.5)[0]
            for u in us[::50]} == {1, 2, 4}
    assert {O.sample(x, u, 0.7, top_p=0.0)[0] for u in us[::50]} == {4}
    assert {O.sample(x, u, 0.7, min_p=1.0)[0] for u in us[::50]} == {4}
    assert O.sample(x, 0.9, 0.0) == (4, 0.0)
    assert O.sample(np.full(5, -np.inf), 0.9) == (0, 0.0)
    t, lp = O.sample(x, 0.5, 0.7)
    assert abs(lp - np.log(p[t])) < 1e-12


def _counts(bt, P):
    return np.bincount(bt[bt >= 0], minlength=P)


def test_fork_and_compact_keep_counts_and_contents():
    rng = np.random.default_rng(4)
    P, maxp = 40, 6
    bt = np.full((6, maxp), -1, np.int32)
    plen = np.array([37, 16, 0, 0, 0, 0], np.int32)
    bt[0, :4], bt[1, :2] = [9, 30, 2, 11], [39, 5]
    ref = _counts(bt, P).astype(np.int32)
    data = rng.integers(0, 99, P)
    bt2, ref2, plen2, status, copies = O.fork(
        [0, 0, 1, -1, 0], [2, 3, 4, 5, 0], [50, 0, 0, 20, 90], plen, bt, ref)
    # the last request extends a row that is another's parent
    assert status.tolist() == [0, 0, 0, 0, O.BAD_ROW]
    assert np.array_equal(_counts(bt2, P), ref2)
    assert bt2[2].tolist() == [9, 30, 0, 1, -1, -1]
    assert bt2[3, :3].tolist() == [9, 30, 3] and bt2[4, 0] == 39
    assert copies == [(2, 0), (2, 3)] and plen2.tolist() == [37, 16, 37, 37,
                                                             16, 0]
    bt3, ref3, n, moves = O.compact(bt2, ref2)
    moved = data.copy()
    for s, d in moves:
        moved[d] = data[s]
    assert np.array_equal(_counts(bt3, P), ref3) and (ref3[n:] == 0).all()
    assert np.array_equal(moved[bt3[bt3 >= 0]], data[bt2[bt2 >= 0]])
    bt4, ref4, plen4 = O.free([2, 2, 77, 0], bt3, ref3, plen2)
    assert np.array_equal(_counts(bt4, P), ref4) and plen4[2] == plen4[0] == 0
