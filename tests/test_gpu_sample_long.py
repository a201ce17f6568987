"""wedlm_sample (include/wedlm_serve.h) on the longest rows with small top_k,
and the weights' fixed point: rows whose tail lies just below half of its unit.
Against the fp64 definition of oracle/serve_oracle.py, which is given top_k's
tokens: equal tokens, logp within the bound that the header states."""
import numpy as np
import pytest
import torch

from oracle import serve_oracle as O

pytestmark = pytest.mark.gpu


def point(V):
    """Bits after the weights' point."""
    return min(46, 62 - (V - 1).bit_length())


def logp_bound(lp, V):
    """V weights off by half a unit of 2^-f each beside a total of at least 1,
    fp64 operations, and the rounding to fp32."""
    return V * 2.0 ** -(point(V) + 1) + 2.0 ** -45 + abs(lp) * 2.0 ** -24


def first(x, k):
    """Ids, rising, of the first k in falling order, equal ones by rising id."""
    cut = np.partition(x, len(x) - k)[len(x) - k]
    above = np.flatnonzero(x > cut)
    return np.sort(np.concatenate(
        (above, np.flatnonzero(x == cut)[:k - len(above)])))


def draw(x, u, V, **kw):
    from paper_2512_22737_amd import wedlm
    B = x.shape[0]
    token = torch.full((B, 1), -9, dtype=torch.int32, device="cuda")
    logp = torch.full((B, 1), 5.0, device="cuda")
    wedlm.wedlm_sample(x, u, token, **kw, logp=logp, V=V)
    return token[:, 0].tolist(), logp[:, 0].tolist()


@pytest.mark.parametrize("V,dtype", [
    (2 ** 20 + 7, torch.float32), (3 * 2 ** 20 + 5, torch.float32),
    (2 ** 22, torch.float32), (2 ** 20 + 7, torch.bfloat16),
    (2 ** 21 + 9, torch.bfloat16), (2 ** 22, torch.bfloat16)])
@pytest.mark.parametrize("kind", ["spread", "ties", "flat"])
def test_small_k_of_long_rows(V, dtype, kind):
    """The largest logits at both ends, in the vectors' remainders and in the
    last blocks; rows that start anywhere."""
    rng = np.random.default_rng(V)
    ks = [1, 7, 50, 500, 1000]
    B, stride = len(ks), V + 3
    g = torch.Generator(device="cuda").manual_seed(V)
    x = torch.randn(B, 1, stride, generator=g, device="cuda")
    x = x * 3 if kind == "spread" else x.round() if kind == "ties" else x * 0.01
    ends = np.concatenate((np.arange(6), V - 1 - np.arange(9),
                           V - 1 - rng.integers(0, 20000, 12),
                           rng.integers(0, V, 12)))
    at = torch.from_numpy(np.unique(ends)).cuda()
    for b in range(B):
        x[b, 0, at] += torch.rand(len(at), generator=g, device="cuda") * 4 + 9
    x = x.to(dtype)
    xs = x[:, 0, :V].double().cpu().numpy()
    ids = [first(xs[b], k) for b, k in enumerate(ks)]
    dk = torch.tensor(ks, dtype=torch.int32, device="cuda")
    for top_p in (1.0, 0.9):
        for T in (1.0, 4.0):
            print(f"sample V={V} {dtype} {kind} p={top_p} T={T}", flush=True)
            u = torch.rand(B, 1, generator=g, device="cuda")
            token, logp = draw(x, u, V, top_k=dk,
                               top_p=torch.full((B,), top_p, device="cuda"),
                               temperature=torch.full((B,), T, device="cuda"))
            for b in range(B):
                t, lp = O.sample(xs[b][ids[b]], float(u[b, 0]), T, 0,
                                 float(np.float32(top_p)))
                assert token[b] == ids[b][t], (b, ks[b])
                assert abs(logp[b] - lp) <= logp_bound(lp, V), (b, ks[b])


@pytest.mark.parametrize("V", [2, 1000, 151936, 2 ** 20, 2 ** 22])
@pytest.mark.parametrize("part", [0.49, 0.51])
def test_tails_near_half_a_unit(V, part):
    """One token at 0 and all others with a weight next to half a unit, which
    rounds them all to 0 or all to one unit: logp is off by the whole tail, as
    far as the header allows and no further."""
    x = torch.full((2, 1, V), float(np.log(part) - point(V) * np.log(2.0)),
                   device="cuda")
    x[0, 0, 0] = x[1, 0, V - 1] = 0.0
    u = torch.tensor([[0.25], [0.5]], device="cuda")
    token, logp = draw(x, u, V)
    assert token == [0, V - 1]
    w = np.exp(float(x[0, 0, V - 1]))
    lp = -np.log1p((V - 1) * w)
    for b in range(2):
        assert abs(logp[b] - lp) <= logp_bound(lp, V)
