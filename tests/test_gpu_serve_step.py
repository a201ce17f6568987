"""The serving operators together, as they are used: prompts written into an
8-bit cache, forked into several samples, decoded with sampled tokens, freed
and compacted, eager and as replayed HIP graphs; calls on other streams."""
import numpy as np
import pytest
import torch

from oracle import serve_oracle as S
from oracle import wedlm_oracle as O

pytestmark = pytest.mark.gpu

B, W, HQ, HKV, D, V, P, MAXP = 6, 8, 4, 2, 64, 300, 70, 8


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def host(x):
    return x.cpu().numpy()


def bf16(x):
    t = torch.from_numpy(x).to(torch.bfloat16)
    return t.cuda(), t.double().numpy()


class Serving:
    """Two prompts, each with two samples, in one pool."""

    def __init__(self, seed):
        from paper_2512_22737_amd import wedlm
        self.w = wedlm
        rng = np.random.default_rng(seed)
        self.rng = rng
        z = dict(dtype=torch.uint8, device="cuda")
        self.cache = [torch.zeros(1, P, HKV, 16, D, **z),
                      torch.zeros(1, P, HKV, D, 16, **z),
                      torch.zeros(1, P, HKV, **z), torch.zeros(1, P, HKV, **z)]
        i32 = dict(dtype=torch.int32, device="cuda")
        self.ref = torch.zeros(P, **i32)
        self.bt = torch.full((B, MAXP), -1, **i32)
        self.plen = torch.zeros(B, **i32)
        self.win = torch.full((B, W), -1, **i32)
        self.step = wedlm.DecodeStep(B, W, HQ, HKV, D, V, MAXP * 16,
                                     cache="e4m3")
        self.settings = dict(
            temperature=torch.full((B,), 0.8, device="cuda"),
            top_k=torch.full((B,), 40, **i32),
            top_p=torch.full((B,), 0.9, device="cuda"))

    def ints(self, *v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    def start(self, prompts=(37, 50)):
        """Rows 0 and 1 get pages and the prompts; rows 2 to 5 fork them."""
        w = self.w
        st = self.ints(0, 0)
        w.wedlm_cache_fork(self.ints(-1, -1), self.ints(0, 1),
                           self.ints(*(n + 32 for n in prompts)), self.plen,
                           self.bt, self.ref, self.cache, st)
        T = max(prompts)
        (k, _), (v, _) = (bf16(self.rng.standard_normal((1, 2, T, HKV, D)))
                          for _ in range(2))
        w.wedlm_cache8_append(k, v, self.ints(0, 0), self.ints(*prompts),
                              *self.cache, self.bt[:2].contiguous())
        self.plen[:2] = self.ints(*prompts)
        st2 = torch.zeros(4, dtype=torch.int32, device="cuda")
        w.wedlm_cache_fork(self.ints(0, 0, 1, 1), self.ints(2, 3, 4, 5),
                           self.ints(*[n + 32 for n in prompts for _ in "ab"]),
                           self.plen, self.bt, self.ref, self.cache, st2)
        assert not st.any() and not st2.any()

    def inputs(self):
        qkv = bf16(self.rng.standard_normal((B, W, HQ + 2 * HKV, D)))[0]
        x = self.rng.standard_normal((B, W, V)).astype(np.float32) * 3
        u = self.rng.random((B, W)).astype(np.float32)
        return qkv, dev(x), dev(u)

    def run(self, qkv, x, u):
        c = self.cache
        self.step(self.win, self.plen, qkv, x, c[0][0], c[1][0], self.bt,
                  c[2][0], c[3][0], u, **self.settings)

    def state(self):
        return [t.clone() for t in
                (self.win, self.plen, self.step.out, self.step.argmax,
                 self.step.committed_tok, *self.cache)]


def test_step_against_the_oracles():
    s = Serving(1)
    s.start()
    assert np.array_equal(np.bincount(host(s.bt)[host(s.bt) >= 0],
                                      minlength=P), host(s.ref))
    seen = 0
    for n in range(5):
        qkv, x, u = s.inputs()
        win, plen = host(s.win), host(s.plen)
        before = [host(t) for t in s.cache]
        s.run(qkv, x, u)
        torch.cuda.synchronize()
        assert not s.step.attn_status.any() and not s.step.status.any()
        for b in range(B):
            perm, pos, _, n_o = O.reorder(list(win[b]), int(plen[b]))
            # the queries and keys as the step rotated them (its own test
            # compares those)
            q = s.step.q_phys[b].double().cpu().numpy()
            kw = s.step.k_phys[b].double().cpu().numpy()
            vw = s.step.v_phys[b].double().cpu().numpy()
            kp, vp = S.gather(*(t[0] for t in before), host(s.bt), b,
                              int(plen[b]))
            o, _, bo, _ = S.attention(q, kw, vw, kp, vp, D ** -0.5)
            assert (np.abs(s.step.out[b].double().cpu().numpy() - o) <=
                    bo).all()
            for i in range(n_o, W):
                t, _ = S.sample(host(x)[b, i], float(host(u)[b, i]),
                                float(np.float32(0.8)), 40,
                                float(np.float32(0.9)))
                assert s.step.argmax[b, i].item() == t
            got = host(s.step.n_commit)[b]
            seen += got
            assert host(s.plen)[b] == plen[b] + got
        # committed rows in the cache
        want = S.append(s.step.k_phys[None].double().cpu().numpy(),
                        s.step.v_phys[None].double().cpu().numpy(), plen,
                        host(s.step.n_commit), *before, host(s.bt))
        for a, b in zip(s.cache, want[:4]):
            assert np.array_equal(host(a), b)
    assert seen > 0


def test_samples_of_one_prompt_see_the_same_prefix():
    """Forked sequences with equal windows and inputs give equal outputs; what
    one commits does not reach the others."""
    s = Serving(2)
    s.start((37, 37))
    qkv, x, u = s.inputs()
    for b in (2, 3):
        qkv[b], x[b], u[b] = qkv[0], x[0], u[0]
    s.run(qkv, x, u)
    for b in (2, 3):
        assert torch.equal(s.step.out[b], s.step.out[0])
        assert torch.equal(s.win[b], s.win[0])
    u[2] = 1 - u[2]
    for _ in range(3):
        s.run(qkv, x, u)
        assert torch.equal(s.step.out[3], s.step.out[0])
    # free one of them, compact, and go on: the others do not notice
    t = Serving(2)
    for name in ("cache", "ref", "bt", "plen", "win"):
        v = getattr(s, name)
        setattr(t, name, [a.clone() for a in v] if name == "cache"
                else v.clone())
    gone = s.ints(2, 4)
    t.w.wedlm_cache_free(gone, t.bt, t.ref, t.plen)
    n = t.ints(0)
    t.w.wedlm_cache_compact(t.bt, t.ref, t.cache, t.bt, t.ref, n)
    assert n.item() == int((t.ref > 0).sum()) < int((s.ref > 0).sum())
    assert (t.ref[n.item():] == 0).all()
    s.run(qkv, x, u)
    t.run(qkv, x, u)
    for b in (0, 1, 3, 5):
        assert torch.equal(s.step.out[b], t.step.out[b])
        assert torch.equal(s.step.argmax[b], t.step.argmax[b])


def test_replayed_graph_is_the_eager_step():
    """The step, a fork with a free before it, and a compaction captured; each
    replay against the eager calls, other work and synchronizations between
    them."""
    eager, graph = Serving(3), Serving(3)
    for s in (eager, graph):
        s.start()
    qkv, x, u = eager.inputs()
    kw = dict(dtype=torch.int32, device="cuda")

    def turn(s, st, n, nbt, nref):
        s.run(qkv, x, u)
        s.w.wedlm_cache_free(rows, s.bt, s.ref, s.plen)
        s.w.wedlm_cache_fork(par, rows, res, s.plen, s.bt, s.ref, s.cache, st)
        s.w.wedlm_cache_compact(s.bt, s.ref, s.cache, nbt, nref, n)

    rows, par = eager.ints(3, 5), eager.ints(0, 1)
    res = eager.ints(100, 100)
    outs = [(torch.zeros(2, **kw), torch.zeros(1, **kw), s.bt.clone(),
             s.ref.clone()) for s in (eager, graph)]
    saved = [t.clone() for t in (graph.win, graph.plen, graph.bt, graph.ref,
                                 *graph.cache)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        turn(graph, *outs[1])
    torch.cuda.current_stream().wait_stream(side)
    for t, v in zip((graph.win, graph.plen, graph.bt, graph.ref,
                     *graph.cache), saved):
        t.copy_(v)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        turn(graph, *outs[1])
    for n in range(4):
        a, b, c = eager.inputs()
        qkv.copy_(a), x.copy_(b), u.copy_(c)
        turn(eager, *outs[0])
        torch.cuda.synchronize()
        g.replay()
        junk = torch.randn(500, 500, device="cuda") @ torch.randn(
            500, 500, device="cuda")
        torch.cuda.synchronize()
        assert junk.numel()
        for p, q in zip(eager.state(), graph.state()):
            assert torch.equal(p, q), n
        for p, q in zip((eager.bt, eager.ref, *outs[0]),
                        (graph.bt, graph.ref, *outs[1])):
            assert torch.equal(p, q), n


def test_calls_on_two_streams():
    """Independent servings on streams of their own, interleaved."""
    alone = [Serving(4), Serving(5)]
    both = [Serving(4), Serving(5)]
    ins = []
    for s in alone:
        s.start()
    for s in both:
        s.start()
    for s, t in zip(alone, both):
        ins.append([s.inputs() for _ in range(4)])
        for i in ins[-1]:
            s.run(*i)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for n in range(4):
        for s, st, i in zip(both, streams, ins):
            with torch.cuda.stream(st):
                s.run(*i[n])
    torch.cuda.synchronize()
    for s, t in zip(alone, both):
        for p, q in zip(s.state(), t.state()):
            assert torch.equal(p, q)


def test_bf16_step_samples_too_and_mixes_are_refused():
    from paper_2512_22737_amd import wedlm
    bf = dict(dtype=torch.bfloat16, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    step = wedlm.DecodeStep(B, W, HQ, HKV, D, V, 64)
    k, v = torch.zeros(P, HKV, 16, D, **bf), torch.zeros(P, HKV, D, 16, **bf)
    s = Serving(6)
    qkv, x, u = s.inputs()
    bt = torch.arange(B * 4, **i32).view(B, 4)
    win, start = torch.full((B, W), -1, **i32), torch.zeros(B, **i32)
    step(win, start, qkv, x, k, v, bt, u=u, **s.settings)
    for b in range(B):
        t, _ = S.sample(host(x)[b, 0], float(host(u)[b, 0]),
                        float(np.float32(0.8)), 40, float(np.float32(0.9)))
        assert step.argmax[b, 0].item() == t
    with pytest.raises(wedlm.WedlmError, match="e4m3"):
        step(win, start, qkv, x, k, v, bt, k, v)
    with pytest.raises(wedlm.WedlmError, match="random"):
        step(win, start, qkv, x, k, v, bt, top_k=bt[0])
    with pytest.raises(wedlm.WedlmError, match="e4m3"):
        s.step(s.win, s.plen, qkv, x, s.cache[0][0], s.cache[1][0], s.bt)
    with pytest.raises(wedlm.WedlmError, match="e4m3"):
        wedlm.DecodeStep(B, W, HQ, HKV, D, V, 64, cache="int8")
