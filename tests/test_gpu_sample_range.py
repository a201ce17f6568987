"""wedlm_sample (include/wedlm_serve.h) on logits whose differences pass the
largest fp32 number, at temperatures as large: such tokens have a weight, and
top-k's and top-p's runs reach them.  Against the fp64 definition of
oracle/serve_oracle.py: equal tokens, logp within the fixed-point weights'
bound."""
import numpy as np
import pytest
import torch

from oracle import serve_oracle as O

pytestmark = pytest.mark.gpu

MAX = {torch.float32: float(np.finfo(np.float32).max),
       torch.bfloat16: torch.finfo(torch.bfloat16).max}


def logp_bound(V):
    """V weights off by half a unit of 2^-f each beside a total of at least 1,
    and fp64 operations."""
    f = min(46, 62 - max(V - 1, 0).bit_length())
    return V * 2.0 ** -(f + 1) + 2.0 ** -45


def rows(V, dtype):
    """The largest number or +inf among the type's lowest, both with -inf and
    NaN between them; all of the type's range; ordinary logits with masks of
    the lowest value."""
    rng = np.random.default_rng(V)
    big = MAX[dtype]
    x = np.full((6, 1, V), -big)
    x[0, 0, V // 3] = np.inf
    x[1, 0, rng.integers(0, V, 5)] = big
    x[1, 0, ::7] = -np.inf
    x[1, 0, ::11] = np.nan
    x[2] = rng.uniform(-1, 1, V) * big
    x[3] = rng.uniform(-3e38, 1e38, V)
    x[4] = np.where(rng.random(V) < 0.5, x[4], rng.standard_normal(V) * 4)
    x[5] = np.where(rng.random(V) < 0.9, x[5], 1e36)
    return torch.from_numpy(x).to(dtype).cuda()


SETTINGS = [dict(), dict(top_p=0.9), dict(top_p=0.3), dict(top_k=3),
            dict(top_k=600), dict(top_k=600, top_p=0.9),
            dict(top_k=5000), dict(top_k=5000, top_p=0.7, min_p=0.01)]


@pytest.mark.parametrize("T", [float("inf"), 3e38, 1e38, 2e37, 1e31, 1.0])
@pytest.mark.parametrize("V", [1000, 9001])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_differences_beyond_the_largest_number(T, V, dtype):
    from paper_2512_22737_amd import wedlm
    x = rows(V, dtype)
    B = x.shape[0]
    T = float(np.float32(T))
    for n, s in enumerate(SETTINGS):
        print(f"sample T={T} V={V} {dtype} {s}", flush=True)
        u = torch.from_numpy(np.random.default_rng(n).random(
            (B, 1)).astype(np.float32)).cuda()
        col = lambda k, d, t: torch.full((B,), s.get(k, d), dtype=t,
                                         device="cuda")
        token = torch.full((B, 1), -9, dtype=torch.int32, device="cuda")
        logp = torch.full((B, 1), 5.0, device="cuda")
        wedlm.wedlm_sample(
            x, u, token, col("T", T, torch.float32),
            col("top_k", 0, torch.int32), col("top_p", 1.0, torch.float32),
            col("min_p", 0.0, torch.float32), None, logp)
        f32 = lambda v: float(np.float32(v))
        for b in range(B):
            t, lp = O.sample(x[b, 0].double().cpu().numpy(), float(u[b, 0]), T,
                             s.get("top_k", 0), f32(s.get("top_p", 1.0)),
                             f32(s.get("min_p", 0.0)))
            assert token[b, 0].item() == t, (b, s)
            assert abs(logp[b, 0].item() - lp) <= (abs(lp) * 2.0 ** -24 +
                                                   logp_bound(V)), (b, s)
