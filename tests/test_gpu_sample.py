"""GPU parity of wedlm_sample (include/wedlm_serve.h) with the fp64 definition
of oracle/serve_oracle.py.  Tokens are equal: the inputs' random numbers lie
off every border by far more than fp64 (a border is met with a probability of
about V 2^-38 per row).  logp is rounded to fp32 once from fp64."""
import numpy as np
import pytest
import torch

from oracle import serve_oracle as O

pytestmark = pytest.mark.gpu

SETTINGS = [dict(), dict(T=0.7), dict(T=0.0), dict(T=5.0, top_k=3),
            dict(top_k=1), dict(top_p=0.9), dict(T=1.7, top_p=0.5, top_k=40),
            dict(min_p=0.1), dict(T=2.0, top_k=200, top_p=0.99, min_p=0.01),
            dict(T=30.0), dict(T=30.0, top_p=0.3), dict(T=1e-3, top_p=0.9),
            dict(top_p=0.0), dict(top_p=float("nan")), dict(min_p=7.0),
            dict(T=float("nan")), dict(T=-1.0), dict(top_k=-4),
            dict(top_k=10 ** 9, top_p=2.0), dict(T=float("inf"), top_p=0.6)]


def inputs(B, W, V, stride, dtype, seed, ties=False):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((B, W, stride)) * 2.5
    at = rng.integers(0, V, (B, W, 4))
    for b in range(B):
        for i in range(W):
            x[b, i, at[b, i]] += rng.random(4) * 9
    if ties:
        x = np.round(x)                        # few distinct values
    drop = (rng.random((B, W, 1)) < 0.3) & (rng.random(x.shape) < 0.5)
    x[drop] = -np.inf
    x[:, :, V:] = np.nan                       # padding is not read
    x = torch.from_numpy(x).to(dtype).cuda()
    u = rng.random((B, W)).astype(np.float32)
    return x, torch.from_numpy(u).cuda()


def settings(B):
    s = [SETTINGS[b % len(SETTINGS)] for b in range(B)]
    col = lambda n, d: [x.get(n, d) for x in s]
    return s, dict(
        temperature=torch.tensor(col("T", 1.0), device="cuda"),
        top_k=torch.tensor(col("top_k", 0), dtype=torch.int32, device="cuda"),
        top_p=torch.tensor(col("top_p", 1.0), device="cuda"),
        min_p=torch.tensor(col("min_p", 0.0), device="cuda"))


def oracle_of(x, u, s):
    f32 = lambda v: float(np.float32(v))
    return O.sample(x, u, f32(s.get("T", 1.0)), s.get("top_k", 0),
                    f32(s.get("top_p", 1.0)), f32(s.get("min_p", 0.0)))


def check(x, u, V, s, token, logp, rows=None):
    x, u = x[:, :, :V].double().cpu().numpy(), u.cpu().numpy()
    token, logp = token.cpu().numpy(), logp.cpu().numpy()
    for b in range(x.shape[0]):
        for i in range(x.shape[1]):
            if rows is not None and i < rows[b]:
                assert token[b, i] == -9 and logp[b, i] == 5.0
                continue
            t, lp = oracle_of(x[b, i], float(u[b, i]), s[b])
            assert token[b, i] == t, (b, i, s[b], token[b, i], t)
            # one rounding to fp32, and 2^-38 of a total of fixed-point weights
            assert abs(logp[b, i] - lp) <= abs(lp) * 2.0 ** -24 + 2.0 ** -36


@pytest.mark.parametrize("V,stride", [
    (1, 1), (2, 5), (3, 3), (63, 64), (64, 64), (65, 65), (1000, 1000),
    (1021, 1024), (4097, 4100), (32003, 32064), (50257, 50257)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("ties", [False, True])
def test_sample(V, stride, dtype, ties):
    from paper_2512_22737_amd import wedlm
    print(f"sample V={V} stride={stride} {dtype} ties={ties}", flush=True)
    B = len(SETTINGS)
    x, u = inputs(B, 2, V, stride, dtype, V, ties)
    s, kw = settings(B)
    token = torch.full((B, 2), -9, dtype=torch.int32, device="cuda")
    logp = torch.full((B, 2), 5.0, device="cuda")
    wedlm.wedlm_sample(x, u, token, **kw, logp=logp, V=V)
    check(x, u, V, s, token, logp)
    # without logp: the same tokens
    again = torch.full_like(token, -9)
    wedlm.wedlm_sample(x, u, again, **kw, V=V)
    assert torch.equal(token, again)


def test_rows_that_are_observed_stay():
    from paper_2512_22737_amd import wedlm
    B, W, V = 20, 5, 700
    x, u = inputs(B, W, V, V, torch.float32, 1)
    s, kw = settings(B)
    n = [b % 7 - 1 for b in range(B)]           # also negative and above W
    token = torch.full((B, W), -9, dtype=torch.int32, device="cuda")
    logp = torch.full((B, W), 5.0, device="cuda")
    wedlm.wedlm_sample(x, u, token, **kw, logp=logp, n_obs=torch.tensor(
        n, dtype=torch.int32, device="cuda"))
    check(x, u, V, s, token, logp, n)


def test_defaults():
    from paper_2512_22737_amd import wedlm
    x, u = inputs(3, 2, 501, 501, torch.float32, 2)
    token = torch.full((3, 2), -9, dtype=torch.int32, device="cuda")
    logp = torch.full((3, 2), 5.0, device="cuda")
    wedlm.wedlm_sample(x, u, token, logp=logp)
    check(x, u, 501, [{}] * 3, token, logp)


def test_odd_logits_and_numbers():
    """Rows of nothing but -inf, NaN and +inf among the logits, one value in
    all places, zeros of both signs, random numbers at and beyond the ends."""
    from paper_2512_22737_amd import wedlm
    V = 300
    x = np.zeros((8, 1, V), np.float32)
    x[0] = -np.inf
    x[1] = np.nan
    x[2, 0, ::3] = np.nan
    x[3, 0, [5, 77]] = np.inf
    x[4] = -3.0
    x[5, 0, ::2] = -0.0
    x[6] = -np.inf
    x[6, 0, 200:] = -1e30
    x[7] = np.arange(V) * 1e36
    for top_p, k in ((1.0, 0), (0.5, 0), (1.0, 7), (0.6, 100)):
        for u in (0.0, 0.3, 1 - 2.0 ** -24, 1.0, -1.0, 5.0, 1e-30):
            B = 8
            dx = torch.from_numpy(x).cuda()
            du = torch.full((B, 1), u, device="cuda")
            token = torch.full((B, 1), -9, dtype=torch.int32, device="cuda")
            logp = torch.full((B, 1), 5.0, device="cuda")
            wedlm.wedlm_sample(
                dx, du, token, None,
                torch.full((B,), k, dtype=torch.int32, device="cuda"),
                torch.full((B,), top_p, device="cuda"), None, None, logp)
            check(dx, du, V, [dict(top_p=top_p, top_k=k)] * B, token, logp)


@pytest.mark.parametrize("V", [151936, 1 << 20, 1 << 22])
@pytest.mark.parametrize("kind", ["peaked", "flat", "equal"])
def test_long_rows(V, kind):
    from paper_2512_22737_amd import wedlm
    print(f"sample V={V} {kind}", flush=True)
    B = 4
    g = torch.Generator(device="cuda").manual_seed(V)
    x = torch.randn(B, 1, V, generator=g, device="cuda")
    x = x * 4 if kind == "peaked" else x * 0.01 if kind == "flat" else x * 0
    u = torch.rand(B, 1, generator=g, device="cuda")
    s = [dict(), dict(top_p=0.9), dict(top_k=V // 3), dict(top_k=V // 2,
                                                          top_p=0.7)]
    kw = dict(top_k=torch.tensor([x.get("top_k", 0) for x in s],
                                 dtype=torch.int32, device="cuda"),
              top_p=torch.tensor([x.get("top_p", 1.0) for x in s],
                                 device="cuda"))
    token = torch.full((B, 1), -9, dtype=torch.int32, device="cuda")
    logp = torch.full((B, 1), 5.0, device="cuda")
    wedlm.wedlm_sample(x, u, token, **kw, logp=logp)
    check(x, u, V, s, token, logp)


def test_shares():
    """A row drawn many times: each token as often as its weight says."""
    from paper_2512_22737_amd import wedlm
    N = 4000
    x = torch.tensor([0.0, 1.0, 2.0, -1.0, 2.0], device="cuda")
    x = x.repeat(N, 1, 1).contiguous()
    u = ((torch.arange(N, device="cuda") + 0.5) / N).view(N, 1)
    token = torch.zeros(N, 1, dtype=torch.int32, device="cuda")
    wedlm.wedlm_sample(x, u, token)
    got = torch.bincount(token[:, 0].long(), minlength=5) / N
    want = torch.softmax(x[0, 0], 0)
    assert (got - want).abs().max() <= 1.0 / N
