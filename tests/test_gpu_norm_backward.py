"""GPU parity of wedlm_rmsnorm_backward and wedlm_qk_norm_rope_backward
(include/wedlm_train.h) with the fp64 formulas of oracle/train_oracle.py,
element by element within the bounds derived there."""
import numpy as np
import pytest
import torch

from oracle import train_oracle as T
from oracle import wedlm_oracle as O
from paper_2512_22737_amd import workloads as WL

pytestmark = pytest.mark.gpu

EPS = float(np.float32(1e-6))


def _bf16(rng, shape, scale=1.0, mean=0.0):
    return WL.f32_to_bf16_bits(
        (mean + scale * rng.standard_normal(shape)).astype(np.float32))


def _dev(a):
    return (torch.from_numpy(np.ascontiguousarray(a)).view(torch.int16)
            .cuda().view(torch.bfloat16))


def _host(x):
    return x.double().cpu().numpy()


def _nan(*shape, dtype=torch.float32):
    return torch.full(shape, float("nan"), device="cuda", dtype=dtype)


def _within(got, want, bound, what):
    err = np.abs(_host(got) - want)
    assert (err <= bound).all(), (what, (err / np.maximum(bound, 1e-300)).max())


# widths of one float4, of every number of chunks per thread, that leave the
# last chunks of the threads empty, and longer than the registers hold; rows
# fewer than workgroups, as many, and several per workgroup
@pytest.mark.parametrize("M,Hd", [
    (1, 4), (7, 64), (513, 252), (3, 1028), (1200, 1024), (5, 2560),
    (600, 4096), (2, 8188), (3, 12288), (2, 16384), (515, 16388), (3, 20000)])
@pytest.mark.parametrize("residual", [False, True])
def test_rmsnorm_backward(M, Hd, residual):
    from paper_2512_22737_amd import wedlm
    print(f"rmsnorm backward {M}x{Hd}", flush=True)
    rng = np.random.default_rng(M + Hd)
    x = (np.exp(rng.standard_normal((M, 1))) *
         rng.standard_normal((M, Hd))).astype(np.float32)
    x[M // 2] = 0.0
    gain, dy = _bf16(rng, (Hd,), 0.2, 1.0), _bf16(rng, (M, Hd), 0.01)
    dres = rng.standard_normal((M, Hd)).astype(np.float32)
    (dx, dg), (bx, bg) = T.rmsnorm_backward(
        x.astype(np.float64), O.bf16_to_f64(gain), O.bf16_to_f64(dy), EPS)
    if residual:
        dx = dx + dres
        bx = bx + T.F32 * (np.abs(dx) + bx)
    got, gg = _nan(M, Hd), _nan(Hd)
    wedlm.wedlm_rmsnorm_backward(
        torch.from_numpy(x).cuda(), _dev(gain), EPS, _dev(dy), got, gg,
        torch.from_numpy(dres).cuda() if residual else None)
    _within(got, dx, bx, "dx")
    _within(gg, dg, bg, "dgain")


def test_rmsnorm_backward_in_place_and_without_gain():
    """dres in place gives the same bits as apart; no dgain, no workspace;
    calls repeat bit by bit."""
    from paper_2512_22737_amd import wedlm
    for M, Hd in ((700, 1000), (2, 17000)):
        g = torch.Generator(device="cuda").manual_seed(M)
        x, dres = torch.randn(2, M, Hd, generator=g, device="cuda")
        gain = torch.ones(Hd, device="cuda", dtype=torch.bfloat16)
        dy = torch.randn(M, Hd, generator=g, device="cuda").bfloat16()
        a, b, c = _nan(M, Hd), dres.clone(), _nan(M, Hd)
        ga, gb = _nan(Hd), _nan(Hd)
        wedlm.wedlm_rmsnorm_backward(x, gain, EPS, dy, a, ga, dres)
        wedlm.wedlm_rmsnorm_backward(x, gain, EPS, dy, b, gb, b)
        wedlm.wedlm_rmsnorm_backward(x, gain, EPS, dy, c, None, dres)
        assert torch.equal(a, b) and torch.equal(a, c)
        assert torch.equal(ga, gb)


@pytest.mark.parametrize("M,Hq,Hkv,D,far", [
    (1, 1, 1, 64, 10), (3, 4, 2, 64, 1000), (9, 28, 4, 128, 40000),
    (1100, 4, 4, 64, 1100), (520, 32, 8, 128, 2000000), (2, 40, 1, 128, 5),
    (5, 100, 3, 64, 9), (513, 1, 3, 128, 300),
    (4099, 4, 2, 64, 4099)])
def test_qk_norm_rope_backward(M, Hq, Hkv, D, far):
    from paper_2512_22737_amd import wedlm
    print(f"qk norm rope backward {M} {Hq}/{Hkv}x{D}", flush=True)
    rng = np.random.default_rng(M + Hq)
    theta = 1e6
    qkv = _bf16(rng, (M, Hq + 2 * Hkv, D))
    qkv[M // 2, 0] = 0
    gq, gk = (_bf16(rng, (D,), 0.2, 1.0) for _ in range(2))
    pos = rng.integers(0, far, M).astype(np.int32)
    dq = _bf16(rng, (M, Hq, D), 0.01)
    dk, dv = (_bf16(rng, (M, Hkv, D), 0.01) for _ in range(2))
    out = _nan(M, (Hq + 2 * Hkv) * D, dtype=torch.bfloat16)
    gains = _nan(D), _nan(D)
    wedlm.wedlm_qk_norm_rope_backward(
        _dev(qkv.reshape(M, -1)), _dev(gq), _dev(gk),
        torch.from_numpy(pos).cuda(), theta, EPS, _dev(dq), _dev(dk),
        _dev(dv), out, *gains)
    out = out.view(M, -1, D)
    for x, g, d, at, gg in ((qkv[:, :Hq], gq, dq, 0, gains[0]),
                            (qkv[:, Hq:Hq + Hkv], gk, dk, Hq, gains[1])):
        (dx, dg), (bx, bg) = T.qk_norm_rope_backward(
            O.bf16_to_f64(x), O.bf16_to_f64(g), pos, O.bf16_to_f64(d), theta,
            EPS)
        _within(out[:, at:at + x.shape[1]], dx, bx, "dqkv")
        _within(gg, dg, bg, "gain")
    assert torch.equal(out[:, Hq + Hkv:], _dev(dv))


def test_qk_norm_rope_backward_without_gains():
    from paper_2512_22737_amd import wedlm
    M, Hq, Hkv, D = 600, 8, 2, 64
    g = torch.Generator(device="cuda").manual_seed(4)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()
    qkv, dq, dk, dv = (r(M, (Hq + 2 * Hkv) * D), r(M, Hq, D), r(M, Hkv, D),
                       r(M, Hkv, D))
    gq, gk = r(D), r(D)
    pos = torch.arange(M, dtype=torch.int32, device="cuda")
    runs = []
    for gains in ((None, None), (_nan(D), None), (None, _nan(D)),
                  (_nan(D), _nan(D))):
        out = torch.empty_like(qkv)
        wedlm.wedlm_qk_norm_rope_backward(qkv, gq, gk, pos, 1e4, EPS, dq, dk,
                                          dv, out, *gains)
        runs.append((out, *gains))
    assert all(torch.equal(runs[0][0], x[0]) for x in runs)
    assert torch.equal(runs[1][1], runs[3][1])
    assert torch.equal(runs[2][2], runs[3][2])
