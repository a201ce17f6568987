"""Inputs of wedlm_window_attn_cache8 (include/wedlm_serve.h) that are not
finite, or large.  What is not finite makes the outputs that it reaches NaN
(or infinite), all others are what they were: to the bit, but for rows of one
wave, whose reference maxima are raised together and which stay within the
bounds of oracle/serve_oracle.py."""
import numpy as np
import pytest
import torch

from oracle import serve_oracle as O

pytestmark = pytest.mark.gpu

# one wave's keys to keys shared by eight, one split and several
SHAPES = [(1, 4, 2, 64), (16, 8, 2, 64), (9, 12, 2, 128), (32, 4, 2, 128),
          (64, 8, 2, 64), (64, 8, 2, 128)]
LENS = [37, 700, 2100]


def state(W, Hq, Hkv, D):
    rng = np.random.default_rng(W + D)
    pages = [-(-n // 16) for n in LENS]
    P = sum(pages)
    bt = np.full((len(LENS), max(pages)), -1, np.int32)
    at = 0
    for b, n in enumerate(pages):
        bt[b, :n] = np.arange(at, at + n)
        at += n
    codes = lambda *s: O.encode(np.clip(rng.standard_normal(s) * 40, -448, 448))
    bf = lambda *s: torch.from_numpy(rng.standard_normal(s)).to(
        torch.bfloat16).cuda()
    B = len(LENS)
    return dict(q=bf(B, W, Hq, D), kw=bf(B, W, Hkv, D), vw=bf(B, W, Hkv, D),
                k8=codes(P, Hkv, 16, D), v8=codes(P, Hkv, D, 16),
                ke=rng.integers(119, 123, (P, Hkv)).astype(np.uint8),
                ve=rng.integers(119, 123, (P, Hkv)).astype(np.uint8), bt=bt)


def call(s):
    from paper_2512_22737_amd import wedlm
    dev = lambda x: torch.from_numpy(x).cuda()
    out = torch.zeros_like(s["q"])
    lse = torch.zeros(s["q"].shape[:3], device="cuda")
    wedlm.wedlm_window_attn_cache8(
        s["q"], s["kw"], s["vw"], dev(s["k8"]), dev(s["v8"]), dev(s["ke"]),
        dev(s["ve"]), dev(s["bt"]),
        torch.tensor(LENS, dtype=torch.int32, device="cuda"), max(LENS), out,
        lse)
    return out, lse


def same_but(got, want, reached):
    """NaN where `reached`, else the same bits."""
    assert bool(got[reached].isnan().all())
    assert torch.equal(got[~reached], want[~reached])


def oracle(s):
    """out, lse and their bounds."""
    f64 = lambda x: x.double().cpu().numpy()
    D = s["q"].shape[3]
    per = [O.attention(f64(s["q"][b]), f64(s["kw"][b]), f64(s["vw"][b]),
                       *O.gather(s["k8"], s["v8"], s["ke"], s["ve"], s["bt"],
                                 b, n), D ** -0.5)
           for b, n in enumerate(LENS)]
    return [np.stack(x) for x in zip(*per)]


def near_but(got, want, bound, reached):
    """NaN where `reached`, else within the bound."""
    got, reached = got.double().cpu().numpy(), reached.cpu().numpy()
    assert np.isnan(got[reached]).all()
    err = np.abs(got - want)[~reached] / bound[~reached]
    assert (err <= 1).all(), err.max()


@pytest.mark.parametrize("W,Hq,Hkv,D", SHAPES)
def test_codes_of_the_prefix(W, Hq, Hkv, D):
    """One NaN code at the first, a middle and the last position of each
    sequence, in keys or values."""
    s = state(W, Hq, Hkv, D)
    out, lse = call(s)
    assert bool(out.isfinite().all()) and bool(lse.isfinite().all())
    G = Hq // Hkv
    for b, n in enumerate(LENS):
        for j in sorted({0, 31, n // 2, n // 32 * 32 - 1, n - 1}):
            p, h, d = s["bt"][b, j // 16], j % Hkv, (5 * j) % D
            print(f"NaN at sequence {b} position {j} head {h}", flush=True)
            heads = slice(h * G, (h + 1) * G)
            k8 = s["k8"].copy()
            k8[p, h, j % 16, d] = 0x7f
            o, l = call(dict(s, k8=k8))
            hit = torch.zeros_like(lse, dtype=torch.bool)
            hit[b, :, heads] = True
            same_but(l, lse, hit)
            same_but(o, out, hit[..., None].expand_as(out))
            v8 = s["v8"].copy()
            v8[p, h, d, j % 16] = 0xff
            o, l = call(dict(s, v8=v8))
            assert torch.equal(l, lse)
            hit = torch.zeros_like(out, dtype=torch.bool)
            hit[b, :, heads, d] = True
            same_but(o, out, hit)


@pytest.mark.parametrize("W,Hq,Hkv,D", SHAPES)
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_rows_of_the_window(W, Hq, Hkv, D, bad):
    """A query reaches its own row; a key the rows that see it; a value its
    element of all rows."""
    s = state(W, Hq, Hkv, D)
    out, lse = call(s)
    wo, wl, bo, bl = oracle(s)
    G = Hq // Hkv
    for i in sorted({0, W // 2, W - 1}):
        b, h, d = i % len(LENS), i % Hkv, (3 * i) % D
        q = s["q"].clone()
        q[b, i, h * G, d] = bad
        o, l = call(dict(s, q=q))
        hit = torch.zeros_like(lse, dtype=torch.bool)
        hit[b, i, h * G] = True
        near_but(l, wl, bl, hit)
        near_but(o, wo, bo, hit[..., None].expand_as(out))
        if bad != bad:
            kw = s["kw"].clone()
            kw[b, i, h, d] = bad
            o, l = call(dict(s, kw=kw))
            hit = torch.zeros_like(lse, dtype=torch.bool)
            hit[b, i:, h * G:(h + 1) * G] = True
            near_but(l, wl, bl, hit)
            near_but(o, wo, bo, hit[..., None].expand_as(out))
        vw = s["vw"].clone()
        vw[b, i, h, d] = bad
        o, l = call(dict(s, vw=vw))
        assert torch.equal(l, lse)
        hit = torch.zeros_like(out, dtype=torch.bool)
        hit[b, :, h * G:(h + 1) * G, d] = True
        rows = torch.arange(W, device="cuda")
        want = out.clone()
        if bad == bad:                       # rows that see it: infinity
            want[b, i:, h * G:(h + 1) * G, d] = bad
            hit &= (rows < i)[None, :, None, None]
        same_but(o, want, hit)


@pytest.mark.parametrize("W,Hq,Hkv,D", SHAPES)
def test_large_values(W, Hq, Hkv, D):
    """Values up to 2^43 at keys that outgrow every earlier one: the outputs
    are those of values 2^42 times smaller, times 2^42."""
    s = state(W, Hq, Hkv, D)
    for b in range(len(LENS)):
        for j in range(-(-LENS[b] // 16)):
            s["ke"][s["bt"][b, j]] = 112 + j // 12
    s["ve"] = np.full_like(s["ve"], 119)                  # |v| <= 448 * 2^-8
    s["vw"] = s["vw"] * 0.25
    out, lse = call(s)
    o, l = call(dict(s, ve=s["ve"] + 42, vw=s["vw"] * 2.0 ** 42))
    assert bool(o.isfinite().all()) and torch.equal(l, lse)
    assert torch.equal(o, out * 2.0 ** 42)
