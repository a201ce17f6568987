"""GPU parity of wedlm_token_loss (include/wedlm_train.h) with the fp64
formulas of oracle/train_oracle.py, element by element within the bounds
derived there."""
import numpy as np
import pytest
import torch

from oracle import train_oracle as T

pytestmark = pytest.mark.gpu


def _host(x):
    return x.double().cpu().numpy()


def _inputs(R, V, stride, dtype, seed, ignored=0.25):
    """Rows of every kind: sharp, flat, with tokens ruled out, without loss."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((R, stride)) * np.exp(
        rng.uniform(-2, 2, (R, 1)))
    t = rng.integers(0, V, R)
    x[np.arange(R), t] += np.where(rng.random(R) < 0.5, 12.0, 0.0)
    x[:, V:] = np.nan                       # padding is not read
    drop = (rng.random((R, 1)) < 0.4) & (rng.random((R, stride)) < 0.5)
    x[drop] = -np.inf                       # sometimes the target too
    t[rng.random(R) < ignored] = -1
    w = rng.uniform(0.1, 3.0, R).astype(np.float32)
    return (torch.from_numpy(x).cuda().to(dtype),
            torch.from_numpy(t.astype(np.int32)).cuda(),
            torch.from_numpy(w).cuda())


def _check(x, t, w, V, loss, d, dtype):
    ww = np.ones(len(t)) if w is None else _host(w)
    (l, g), (bl, bg) = T.token_loss(_host(x[:, :V]), t.cpu().numpy(), ww)
    got = _host(loss)
    inf = np.isinf(l)
    assert (got[inf] == l[inf]).all()
    err = np.abs(got[~inf] - l[~inf])
    assert (err <= bl[~inf]).all(), (err / np.maximum(bl[~inf], 1e-300)).max()
    if d is None:
        return
    if dtype == torch.bfloat16:
        # half a step, and bf16's smallest normal number below that
        bg = bg + T.BF16 * (np.abs(g) + bg) + 2.0 ** -126
    err = np.abs(_host(d[:, :V]) - g)
    assert (err <= bg).all(), (err / np.maximum(bg, 1e-300)).max()


# rows that start on and off 16-byte boundaries, shorter than a vector, than
# a workgroup, of full vocabularies; few rows and many
@pytest.mark.parametrize("R,V,stride", [
    (1, 1, 1), (2, 3, 3), (5, 7, 8), (33, 1000, 1000), (9, 1021, 1021),
    (64, 4096, 4160), (3, 32003, 32064), (2, 151936, 151936),
    (7, 50257, 50257), (700, 513, 520), (600, 20000, 20000),
    (300, 12001, 12004)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_token_loss(R, V, stride, dtype):
    from paper_2512_22737_amd import wedlm
    print(f"token loss {R}x{V} stride {stride} {dtype}", flush=True)
    x, t, w = _inputs(R, V, stride, dtype, R + V)
    held = x.clone()
    loss = torch.full((R,), float("nan"), device="cuda")
    d = torch.full_like(x, 7.0)
    wedlm.wedlm_token_loss(x, t, loss, w, d, V=V)
    _check(x, t, w, V, loss, d, dtype)
    assert (d[:, V:] == 7.0).all()              # padding is not written
    # the loss alone, then in place: the same bits
    alone = torch.full_like(loss, float("nan"))
    wedlm.wedlm_token_loss(x, t, alone, w, None, V=V)
    assert torch.equal(loss, alone)
    bits = torch.int16 if dtype == torch.bfloat16 else torch.int32
    assert torch.equal(x.view(bits), held.view(bits))
    wedlm.wedlm_token_loss(x, t, alone, w, x, V=V)
    assert torch.equal(loss, alone)
    assert torch.equal(x[:, :V], d[:, :V])
    assert torch.equal(x[:, V:].view(bits), held[:, V:].view(bits))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_without_loss(dtype):
    """Targets outside the vocabulary, weight 0, NaN in rows that carry no
    loss, rows of nothing but -inf, infinite loss of a ruled-out target."""
    from paper_2512_22737_amd import wedlm
    R, V = 8, 300
    x = torch.randn(R, V, device="cuda").to(dtype)
    t = torch.tensor([-1, V, 2**31 - 1, -2**31, 5, 6, 7, 8],
                     dtype=torch.int32, device="cuda")
    w = torch.ones(R, device="cuda")
    w[4] = 0.0
    x[:5] = float("nan")
    x[5] = -float("inf")
    x[6, 7] = -float("inf")
    x[7] = -float("inf")
    x[7, 8] = -1e30
    loss, d = torch.full((R,), 9.0, device="cuda"), torch.full_like(x, 9.0)
    wedlm.wedlm_token_loss(x, t, loss, w, d)
    assert (loss[:5] == 0).all() and (d[:6] == 0).all()
    assert torch.isposinf(loss[5:7]).all()
    assert torch.isfinite(d).all() and d[6, 7] == -1
    assert loss[7] == 0 and (d[7] == 0).all()


def test_default_weight_and_unaligned_arrays():
    """No weights (all 1), arrays that start off 16-byte boundaries, logits
    and gradient at different ones."""
    from paper_2512_22737_amd import wedlm
    R, V = 6, 777
    for dtype in (torch.float32, torch.bfloat16):
        for a, b in ((0, 0), (1, 1), (3, 3), (1, 2), (0, 3)):
            x, t, _ = _inputs(R, V, V, dtype, 3)
            xs = torch.empty(R * V + 8, device="cuda", dtype=dtype)
            ds = torch.full((R * V + 8,), 5.0, device="cuda", dtype=dtype)
            xv, dv = xs[a:a + R * V].view(R, V), ds[b:b + R * V].view(R, V)
            xv.copy_(x)
            loss = torch.empty(R, device="cuda")
            wedlm.wedlm_token_loss(xv, t, loss, None, dv)
            _check(x, t, None, V, loss, dv, dtype)
            assert (ds[:b] == 5).all() and (ds[b + R * V:] == 5).all()


# (the rows' sum of the others from about e^-7 down to 0 beside the target's 1;
# V in one workgroup's registers, beyond them, and in slices)
@pytest.mark.parametrize("R,V", [(12, 200), (12, 30000), (12, 100000),
                                 (300, 100000)])
def test_well_predicted_tokens_keep_their_digits(R, V):
    """Loss and gradients of targets that stand 8 to 120 above the others:
    relative to themselves, not to 1."""
    from paper_2512_22737_amd import wedlm
    rng = np.random.default_rng(V)
    x = 0.1 * rng.standard_normal((R, V))
    t = rng.integers(0, V, R).astype(np.int32)
    x[np.arange(R), t] = np.linspace(np.log(V) + 8, 120, R)
    x = torch.from_numpy(x).cuda().float()
    t = torch.from_numpy(t).cuda()
    for a in (0, 1):                   # logits and gradients alike, and not
        loss = torch.empty(R, device="cuda")
        d = torch.empty(R * V + 4, device="cuda")[a:a + R * V].view(R, V)
        wedlm.wedlm_token_loss(x, t, loss, None, d)
        _check(x, t, None, V, loss, d, torch.float32)
        # not rounded away until e^-x is below 2^-126 (x = 87.3; the others
        # are within 1 of 0)
        near = x.gather(1, t[:, None].long())[:, 0] < 86
        assert near.sum() > R // 2 and (loss[near] > 0).all()
