"""GPU parity of wedlm_dual_stream_attn_backward (include/wedlm_train.h) with
the fp64 formulas of oracle/train_oracle.py, element by element within the
bounds that its roundings give (derived there): block sizes that divide no
tile, sequences shorter than a tile and with a partial last one, one to
sixteen query heads per kv head, rows that see one key only, splits of the
row walks, scores so sharp that most probabilities vanish, and the gradients
of outputs that the forward kernel wrote."""
import numpy as np
import pytest
import torch

from oracle import train_oracle as T
from oracle import wedlm_oracle as O
from paper_2512_22737_amd import workloads as WL

pytestmark = pytest.mark.gpu


def _bf16(rng, shape, scale=1.0):
    return WL.f32_to_bf16_bits(
        (scale * rng.standard_normal(shape)).astype(np.float32))


def _dev(a):
    return (torch.from_numpy(np.ascontiguousarray(a)).view(torch.int16)
            .cuda().view(torch.bfloat16))


def _host(x):
    return x.float().cpu().double().numpy()


def _inputs(n, L, Hq, Hkv, D, seed, sharp=1.0):
    rng = np.random.default_rng(seed)
    q = _bf16(rng, (n, 2 * L, Hq, D), sharp)
    k, v = (_bf16(rng, (n, 2 * L, Hkv, D)) for _ in range(2))
    return q, k, v, _bf16(rng, (n, 2 * L, Hq, D), 0.01)


def _grads(q, k, v, block, out, lse, dout, ws=None, scale=None):
    from paper_2512_22737_amd import wedlm
    g = [torch.full_like(x, float("nan")) for x in (q, k, v)]
    wedlm.wedlm_dual_stream_attn_backward(q, k, v, block, out, lse, dout, *g,
                                          workspace=ws, softmax_scale=scale)
    return g


def _check(got, want, bounds, what):
    for name, x, w, b in zip(("dq", "dk", "dv"), got, want, bounds):
        err = np.abs(x - w)
        assert np.isfinite(x).all(), (what, name)
        assert (err <= b).all(), (what, name, (err / b).max())


@pytest.mark.parametrize("n,L,block,Hq,Hkv,D,sharp", [
    (1, 16, 16, 1, 1, 64, 1.0), (1, 16, 1, 2, 1, 128, 1.0),
    (2, 48, 24, 4, 2, 64, 1.0), (1, 80, 5, 7, 1, 128, 1.0),
    (1, 256, 32, 4, 2, 128, 1.0), (3, 96, 48, 4, 4, 64, 4.0),
    (1, 320, 64, 8, 2, 64, 1.0), (1, 272, 16, 16, 1, 128, 1.0),
    (1, 528, 48, 3, 3, 128, 2.0), (2, 1040, 8, 2, 1, 64, 1.0),
    (1, 1536, 32, 2, 1, 128, 1.0)])
def test_gradients(n, L, block, Hq, Hkv, D, sharp):
    print(f"dual-stream backward {n}x{L} block {block} {Hq}/{Hkv}x{D}",
          flush=True)
    q, k, v, dout = _inputs(n, L, Hq, Hkv, D, L + block, sharp)
    vis, s = T.dual_stream_visible(L, block), D ** -0.5
    f = [O.bf16_to_f64(x) for x in (q, k, v, dout)]
    fwd = [T.attn_forward(f[0][b], f[1][b], f[2][b], vis, s) for b in range(n)]
    out = torch.from_numpy(np.stack([o for o, _ in fwd])).cuda().to(
        torch.bfloat16)
    lse = torch.from_numpy(np.stack([l for _, l in fwd])).cuda().float()
    got = [_host(x) for x in _grads(*(_dev(x) for x in (q, k, v)), block, out,
                                    lse, _dev(dout))]
    for b in range(n):
        want, bound = T.attn_backward(*(x[b] for x in f), vis, s)
        _check([x[b] for x in got], want, bound, b)


@pytest.mark.parametrize("n,L,block,Hq,Hkv,D", [(2, 128, 32, 8, 2, 128),
                                                (1, 192, 64, 4, 2, 64)])
def test_after_the_forward(n, L, block, Hq, Hkv, D):
    """The forward's own out and lse, another scale than the default."""
    from paper_2512_22737_amd import wedlm
    q, k, v, dout = _inputs(n, L, Hq, Hkv, D, 5)
    vis, s = T.dual_stream_visible(L, block), 0.05
    dq, dk, dv, do = (_dev(x) for x in (q, k, v, dout))
    out = torch.empty_like(dq)
    lse = torch.empty(n, 2 * L, Hq, device="cuda")
    wedlm.wedlm_dual_stream_attn(dq, dk, dv, block, out, lse, softmax_scale=s)
    got = [_host(x) for x in _grads(dq, dk, dv, block, out, lse, do, scale=s)]
    for b in range(n):
        f = [O.bf16_to_f64(x[b]) for x in (q, k, v, dout)]
        want, bound = T.attn_backward(
            *f, vis, s, T.attn_out_error(*f[:3], vis, s))
        _check([x[b] for x in got], want, bound, b)


def test_same_bits_every_time_and_inputs_left():
    """Two calls with workspaces of other contents, and one on another stream,
    give the same bits; inputs stay as they were."""
    n, L, block, Hq, Hkv, D = 1, 480, 24, 6, 2, 128
    from paper_2512_22737_amd import wedlm
    q, k, v, dout = (_dev(x) for x in _inputs(n, L, Hq, Hkv, D, 9))
    out = torch.empty_like(q)
    lse = torch.empty(n, 2 * L, Hq, device="cuda")
    wedlm.wedlm_dual_stream_attn(q, k, v, block, out, lse)
    held = [x.clone() for x in (q, k, v, out, lse, dout)]
    need = wedlm.wedlm_dual_stream_attn_backward_workspace_size(n, L, block,
                                                                Hq, Hkv, D)
    runs = []
    for fill in (0, 255):
        ws = torch.full((need,), fill, dtype=torch.uint8, device="cuda")
        runs.append(_grads(q, k, v, block, out, lse, dout, ws))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        runs.append(_grads(q, k, v, block, out, lse, dout))
    torch.cuda.synchronize()
    for r in runs[1:]:
        for x, y in zip(runs[0], r):
            assert torch.equal(x.view(torch.int16), y.view(torch.int16))
    for x, y in zip(held, (q, k, v, out, lse, dout)):
        assert torch.equal(x, y)


def test_captured_and_replayed():
    """A captured call, replayed with eager work in between, on new inputs."""
    n, L, block, Hq, Hkv, D = 1, 256, 32, 4, 2, 64
    from paper_2512_22737_amd import wedlm
    q, k, v, dout = (_dev(x) for x in _inputs(n, L, Hq, Hkv, D, 3))
    out = torch.empty_like(q)
    lse = torch.empty(n, 2 * L, Hq, device="cuda")
    ws = torch.empty(wedlm.wedlm_dual_stream_attn_backward_workspace_size(
        n, L, block, Hq, Hkv, D), dtype=torch.uint8, device="cuda")
    wedlm.wedlm_dual_stream_attn(q, k, v, block, out, lse)
    g = [torch.empty_like(x) for x in (q, k, v)]
    call = lambda: wedlm.wedlm_dual_stream_attn_backward(
        q, k, v, block, out, lse, dout, *g, workspace=ws)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in (11, 12, 13):
        dout.copy_(_dev(_inputs(n, L, Hq, Hkv, D, seed)[3]))
        graph.replay()
        torch.cuda.synchronize()
        replayed = [x.clone() for x in g]
        for x, y in zip(replayed, _grads(q, k, v, block, out, lse, dout)):
            assert torch.equal(x, y)


@pytest.mark.parametrize("L,D", [(16, 64), (16, 128), (64, 64), (96, 128)])
def test_rows_that_see_few_keys_lose_no_more_than_two_roundings(L, D):
    """dS's rounding and the result's, independent of each other and equally
    large, make sqrt(2) = 1.41 times the result's own; out's rounding, which
    would come in through the rows' sums of P dP, stays out.  (6% for the
    sample of some thousand values.)"""
    n, block, Hq, Hkv = 2, 16, 8, 4
    q, k, v, dout = _inputs(n, L, Hq, Hkv, D, 41, 1.5)
    vis, s = T.dual_stream_visible(L, block), D ** -0.5
    f = [O.bf16_to_f64(x) for x in (q, k, v, dout)]
    fwd = [T.attn_forward(f[0][b], f[1][b], f[2][b], vis, s) for b in range(n)]
    out = torch.from_numpy(np.stack([o for o, _ in fwd])).cuda().to(
        torch.bfloat16)
    lse = torch.from_numpy(np.stack([l for _, l in fwd])).cuda().float()
    got = [_host(x) for x in _grads(*(_dev(x) for x in (q, k, v)), block, out,
                                    lse, _dev(dout))]
    want = [np.stack(x) for x in zip(*(
        T.attn_backward(*(x[b] for x in f), vis, s)[0] for b in range(n)))]
    for name, x, w in zip(("dq", "dk", "dv"), got, want):
        own = torch.from_numpy(w).bfloat16().double().numpy() - w
        ratio = np.linalg.norm(x - w) / np.linalg.norm(own)
        assert ratio <= 1.5, (name, ratio)
