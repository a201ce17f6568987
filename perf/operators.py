"""The backward operators of the decoder's training step, as cases that can be
timed: the backward pass of the dual-stream attention, of RMSNorm, of the
per-head q/k norm with RoPE, and the token loss with the gradient of its
logits.

listed() are fixed cases over the range of sizes; draw() gives more of the
same ranges.  prepare() builds what a training program holds before the call,
run() is one pass: the plain form in torch operations, or with `own` the calls
of the binding; exact() is the same in 64 bits, by differentiating the forward
formulas.
"""
from __future__ import annotations

import math

import torch

own = False

THETA, EPS = 1e6, 1e-6


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------

def _attn(n_seq, L, block, Hq, Hkv, D, sharp=1.0):
    return dict(kind="attn", n_seq=n_seq, L=L, block=block, Hq=Hq, Hkv=Hkv,
                D=D, sharp=sharp)


def _norm(M, Hd, residual=True, gain_grad=True):
    return dict(kind="norm", M=M, Hd=Hd, residual=residual,
                gain_grad=gain_grad)


def _qk(M, L, Hq, Hkv, D):
    return dict(kind="qk", M=M, L=L, Hq=Hq, Hkv=Hkv, D=D)


def _loss(R, V, half, stride=0, ignored=0.0, grad=True):
    return dict(kind="loss", R=R, V=V, half=half, stride=stride or V,
                ignored=ignored, grad=grad)


def listed():
    return [
        # one short sequence of a small model: launches are all there is
        dict(_attn(1, 256, 16, 4, 2, 64), name="attn_1x256"),
        # a document at an odd length, seven query heads to a kv head
        dict(_attn(2, 1008, 24, 28, 4, 128), name="attn_2x1008"),
        # one document: few key tiles for the whole card
        dict(_attn(1, 2048, 64, 16, 8, 128), name="attn_1x2048"),
        # the batch of documents that the forward is measured on
        dict(_attn(4, 4096, 32, 32, 8, 128), name="attn_4x4096"),
        # a small model's norm over a few rows
        dict(_norm(64, 1024), name="norm_64x1024"),
        # odd rows, the first norm of a network (no residual gradient)
        dict(_norm(8193, 2560, residual=False), name="norm_8193x2560"),
        # both streams of four documents at the Qwen3-8B width
        dict(_norm(32768, 4096), name="norm_32768x4096"),
        # q/k norm and RoPE: a small model, then the batch of documents
        dict(_qk(512, 256, 4, 2, 64), name="qk_512"),
        dict(_qk(32768, 4096, 32, 8, 128), name="qk_32768"),
        # the loss of one window of a small vocabulary
        dict(_loss(32, 1024, False), name="loss_32x1024"),
        # bf16 logits with rows that carry no loss, and padded columns
        dict(_loss(1000, 32003, True, 32064, 0.5), name="loss_1000x32003"),
        # fp32 logits of a few thousand masked positions, full vocabulary
        dict(_loss(4096, 151936, False), name="loss_4096x151936"),
    ]


HEADS = ((4, 2), (8, 2), (4, 4), (32, 8), (32, 8), (28, 4), (16, 8), (16, 2))


def _log(rng, lo, hi):
    """A whole number spread over the logarithm of lo..hi."""
    return max(lo, min(hi, int(round(math.exp(
        rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("attn", "attn", "norm", "qk", "loss"))
    Hq, Hkv = rng.choice(HEADS)
    D = rng.choice((64, 128))
    if kind == "attn":
        block = rng.choice((1, 5, 8, 16, 24, 32, 32, 48, 64))
        unit = block * 16 // math.gcd(block, 16)
        n_seq = rng.randint(1, 4)
        # the blocks of a call are numbered in 16 bits
        hi = min(4096, 65535 // (2 * n_seq) * block)
        L = unit * max(1, _log(rng, 16, hi) // unit)
        return _attn(n_seq, L, block, Hq, Hkv, D, rng.choice((0.5, 1.0, 1.5)))
    if kind == "norm":
        Hd = rng.choice((256, 1024, 2048, 4096, 4 * _log(rng, 1, 2500)))
        return _norm(_log(rng, 1, min(32768, 32768 * 4096 // Hd)), Hd,
                     rng.random() < 0.7, rng.random() < 0.8)
    if kind == "qk":
        M = _log(rng, 1, 32768)
        return _qk(M, rng.choice((M, max(1, M // 2), 40000)), Hq, Hkv, D)
    V = rng.choice((_log(rng, 1, 151936), _log(rng, 500, 151936), 151936))
    return _loss(_log(rng, 1, 4096), V, rng.random() < 0.5,
                 V + rng.choice((0, 0, rng.randint(1, 64))),
                 rng.choice((0.0, 0.3, 0.8)), rng.random() < 0.8)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * (seed + 1))
    return g


def _normal(g, *shape, scale=1.0):
    """N(0, scale^2) in bf16."""
    x = torch.randn(*shape, generator=g, device="cuda")
    return x.mul_(scale).to(torch.bfloat16)


def _gain(g, n):
    return (1.0 + 0.1 * torch.randn(n, generator=g, device="cuda")).to(
        torch.bfloat16)


def _visible(c, rows):
    """Keys (memory, then prediction) that physical rows of a sequence see."""
    L, P = c["L"], c["block"]
    r = torch.arange(rows.start, rows.stop, device="cuda")[:, None]
    j = torch.arange(L, device="cuda")[None, :]
    pred, p = r >= L, r % L
    first = p // P * P
    return torch.cat((torch.where(pred, j < first, j <= p),
                      pred & (j >= first) & (j <= p)), 1)


def _chunks(c):
    """Runs of physical rows of which the scores of one kv head fit."""
    n = max(16, min(1024, (1 << 25) // (2 * c["L"] * c["Hq"] // c["Hkv"])))
    return [slice(i, min(i + n, 2 * c["L"])) for i in range(0, 2 * c["L"], n)]


def _prepare_attn(c, g):
    n, L, Hq, Hkv, D = (c[k] for k in ("n_seq", "L", "Hq", "Hkv", "D"))
    G = Hq // Hkv
    q = _normal(g, n, 2 * L, Hq, D, scale=c["sharp"])
    k, v = _normal(g, n, 2 * L, Hkv, D), _normal(g, n, 2 * L, Hkv, D)
    dout = _normal(g, n, 2 * L, Hq, D, scale=0.01)
    # the forward's output and normaliser, which a training step has kept
    out = torch.empty_like(q)
    lse = torch.empty(n, 2 * L, Hq, device="cuda")
    for r in _chunks(c):
        hide = ~_visible(c, r).repeat_interleave(G, 0)
        for b in range(n):
            for h in range(Hkv):
                hh = slice(h * G, (h + 1) * G)
                s = (q[b, r, hh].float().reshape(-1, D) @
                     k[b, :, h].float().T) * D ** -0.5
                s.masked_fill_(hide, -math.inf)
                z = torch.logsumexp(s, 1, keepdim=True)
                lse[b, r, hh] = z.view(-1, G)
                out[b, r, hh] = (torch.exp(s - z) @ v[b, :, h].float()).view(
                    -1, G, D).to(torch.bfloat16)
    s = dict(case=c, q=q, k=k, v=v, out=out, lse=lse, dout=dout)
    if own:
        from paper_2512_22737_amd import wedlm
        s["grads"] = (torch.zeros_like(q), torch.zeros_like(k),
                      torch.zeros_like(v))
        s["ws"] = torch.empty(
            wedlm.wedlm_dual_stream_attn_backward_workspace_size(
                n, L, c["block"], Hq, Hkv, D), dtype=torch.uint8,
            device="cuda")
    return s


def _prepare_norm(c, g):
    M, Hd = c["M"], c["Hd"]
    x = torch.randn(M, Hd, generator=g, device="cuda")
    # rows of a residual stream grow at different rates
    x *= torch.exp(torch.randn(M, 1, generator=g, device="cuda"))
    s = dict(case=c, x=x, gain=_gain(g, Hd), dy=_normal(g, M, Hd, scale=0.01),
             dres=0.01 * torch.randn(M, Hd, generator=g, device="cuda")
             if c["residual"] else None)
    if own:
        from paper_2512_22737_amd import wedlm
        s["dx"] = torch.zeros_like(x)
        s["dgain"] = torch.zeros(Hd, device="cuda") if c["gain_grad"] else None
        nb = wedlm.wedlm_rmsnorm_backward_workspace_size(M, Hd)
        s["ws"] = torch.empty(nb, dtype=torch.uint8, device="cuda")
    return s


def _prepare_qk(c, g):
    M, Hq, Hkv, D = (c[k] for k in ("M", "Hq", "Hkv", "D"))
    s = dict(case=c, qkv=_normal(g, M, (Hq + 2 * Hkv) * D),
             gq=_gain(g, D), gk=_gain(g, D),
             # each stream of each document counts its own positions
             pos=torch.arange(M, dtype=torch.int32, device="cuda") % c["L"]
             if c["L"] <= M else
             torch.randint(0, c["L"], (M,), generator=g, device="cuda",
                           dtype=torch.int32),
             dq=_normal(g, M, Hq, D, scale=0.01),
             dk=_normal(g, M, Hkv, D, scale=0.01),
             dv=_normal(g, M, Hkv, D, scale=0.01))
    if own:
        from paper_2512_22737_amd import wedlm
        s["dqkv"] = torch.zeros_like(s["qkv"])
        s["dgq"] = torch.zeros(D, device="cuda")
        s["dgk"] = torch.zeros(D, device="cuda")
        nb = wedlm.wedlm_qk_norm_rope_backward_workspace_size(M, Hq, Hkv, D)
        s["ws"] = torch.empty(nb, dtype=torch.uint8, device="cuda")
    return s


def _prepare_loss(c, g):
    R, V = c["R"], c["V"]
    x = torch.randn(R, c["stride"], generator=g, device="cuda")
    t = torch.randint(0, V, (R,), generator=g, device="cuda")
    # a part of the positions is predicted well already
    up = torch.rand(R, 1, generator=g, device="cuda") < 0.6
    x.scatter_add_(1, t[:, None], torch.where(up, 10.0, 0.0))
    if c["half"]:
        x = x.to(torch.bfloat16)
    skip = torch.rand(R, generator=g, device="cuda") < c["ignored"]
    # 1 / (share of its block that is masked) over the positions of a batch
    w = 1.0 / (0.1 + 0.9 * torch.rand(R, generator=g, device="cuda")) / R
    s = dict(case=c, x=x, w=w, t=torch.where(skip, -1, t).to(torch.int32))
    if own:
        from paper_2512_22737_amd import wedlm
        s["loss"] = torch.zeros(R, device="cuda")
        s["dx"] = torch.zeros_like(x) if c["grad"] else None
        nb = wedlm.wedlm_token_loss_workspace_size(R, V)
        s["ws"] = torch.empty(nb, dtype=torch.uint8, device="cuda")
    return s


def prepare(case, seed):
    return dict(attn=_prepare_attn, norm=_prepare_norm, qk=_prepare_qk,
                loss=_prepare_loss)[case["kind"]](case, _gen(seed))


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def _run_attn(s):
    c = s["case"]
    q, k, v, dout = s["q"], s["k"], s["v"], s["dout"]
    if own:
        from paper_2512_22737_amd import wedlm
        dq, dk, dv = s["grads"]
        wedlm.wedlm_dual_stream_attn_backward(
            q, k, v, c["block"], s["out"], s["lse"], dout, dq, dk, dv, s["ws"])
        return dict(dq=dq, dk=dk, dv=dv)
    n, L, Hq, Hkv, D = (c[i] for i in ("n_seq", "L", "Hq", "Hkv", "D"))
    G, scale = Hq // Hkv, D ** -0.5
    dq = torch.empty_like(q)
    dk = torch.zeros(n, 2 * L, Hkv, D, device="cuda")
    dv = torch.zeros_like(dk)
    for r in _chunks(c):
        hide = ~_visible(c, r).repeat_interleave(G, 0)
        for b in range(n):
            for h in range(Hkv):
                hh = slice(h * G, (h + 1) * G)
                qq = q[b, r, hh].float().reshape(-1, D)
                do = dout[b, r, hh].float().reshape(-1, D)
                kk, vv = k[b, :, h].float(), v[b, :, h].float()
                p = (qq @ kk.T).mul_(scale).masked_fill_(hide, -math.inf)
                p = torch.exp(p - p.amax(1, keepdim=True))
                p /= p.sum(1, keepdim=True)
                dp = do @ vv.T
                ds = p * (dp - (p * dp).sum(1, keepdim=True))
                dq[b, r, hh] = (ds @ kk).mul_(scale).view(-1, G, D).to(q.dtype)
                dk[b, :, h] += (ds.T @ qq).mul_(scale)
                dv[b, :, h] += p.T @ do
    return dict(dq=dq, dk=dk.to(k.dtype), dv=dv.to(v.dtype))


def _run_norm(s):
    x, gain, dy, dres = s["x"], s["gain"], s["dy"], s["dres"]
    if own:
        from paper_2512_22737_amd import wedlm
        wedlm.wedlm_rmsnorm_backward(x, gain, EPS, dy, s["dx"], s["dgain"],
                                     dres, s["ws"])
        return dict(dx=s["dx"], dgain=s["dgain"])
    r = 1.0 / torch.sqrt((x * x).mean(1, keepdim=True) + EPS)
    xh = x * r
    gy = dy.float()
    dg = (gy * xh).double().sum(0).float() if s["case"]["gain_grad"] else None
    gy = gy * gain.float()
    dx = r * (gy - xh * (gy * xh).mean(1, keepdim=True))
    return dict(dx=dx if dres is None else dres + dx, dgain=dg)


def _run_qk(s):
    c = s["case"]
    M, Hq, Hkv, D = (c[k] for k in ("M", "Hq", "Hkv", "D"))
    if own:
        from paper_2512_22737_amd import wedlm
        wedlm.wedlm_qk_norm_rope_backward(
            s["qkv"], s["gq"], s["gk"], s["pos"], THETA, EPS, s["dq"],
            s["dk"], s["dv"], s["dqkv"], s["dgq"], s["dgk"], s["ws"])
        return dict(dqkv=s["dqkv"], dq_gain=s["dgq"], dk_gain=s["dgk"])
    # far positions: the angles in 64 bits
    i = torch.arange(D // 2, dtype=torch.float64, device="cuda")
    a = s["pos"].double()[:, None] * THETA ** (-2.0 * i / D)
    cos, sin = torch.cos(a).float()[:, None], torch.sin(a).float()[:, None]
    y = s["qkv"].view(M, Hq + 2 * Hkv, D)
    dqkv, grads = torch.empty_like(y), []
    for at, n, gain, d in ((0, Hq, s["gq"], s["dq"]),
                           (Hq, Hkv, s["gk"], s["dk"])):
        lo, hi = d.float().chunk(2, -1)
        dz = torch.cat((lo * cos + hi * sin, hi * cos - lo * sin), -1)
        x = y[:, at:at + n].float()
        r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
        xh = x * r
        grads.append((dz * xh).double().sum((0, 1)).float())
        dz = dz * gain.float()
        dqkv[:, at:at + n] = (r * (dz - xh * (dz * xh).mean(
            -1, keepdim=True))).to(y.dtype)
    dqkv[:, Hq + Hkv:] = s["dv"]
    return dict(dqkv=dqkv.view(M, -1), dq_gain=grads[0], dk_gain=grads[1])


def _run_loss(s):
    c, x, t, w = s["case"], s["x"], s["t"], s["w"]
    V = c["V"]
    if own:
        from paper_2512_22737_amd import wedlm
        wedlm.wedlm_token_loss(x, t, s["loss"], w, s["dx"], s["ws"], V)
        return dict(loss=s["loss"], dlogits=s["dx"][:, :V] if c["grad"]
                    else None)
    z = x[:, :V].float()
    z = z - z.amax(1, keepdim=True)
    e = torch.exp(z)
    total = e.sum(1, keepdim=True)
    live = (t >= 0)[:, None]
    at = t.clamp(min=0).long()[:, None]
    w = torch.where(live, w[:, None], 0.0)
    loss = w * (torch.log(total) - z.gather(1, at))
    d = None
    if c["grad"]:
        e *= w / total
        d = e.scatter_add_(1, at, -w).to(x.dtype)
    return dict(loss=loss[:, 0], dlogits=d)


def run(state):
    return dict(attn=_run_attn, norm=_run_norm, qk=_run_qk,
                loss=_run_loss)[state["case"]["kind"]](state)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(c):
    if c["kind"] == "attn":
        n, L, P, Hq, Hkv, D = (c[k] for k in ("n_seq", "L", "block", "Hq",
                                              "Hkv", "D"))
        # visible (row, key) pairs of one head of one sequence; five products
        K = L // P
        pairs = (L * (L + 1) // 2 + P * P * (K * (K - 1) // 2) +
                 K * (P * (P + 1) // 2))
        rows = n * 2 * L
        return dict(bytes=rows * (4 * Hq * D * 2 + 4 * Hkv * D * 2 + 4 * Hq),
                    flops=5 * 2 * D * pairs * n * Hq)
    if c["kind"] == "norm":
        M, Hd = c["M"], c["Hd"]
        return dict(bytes=M * Hd * (10 + 4 * c["residual"]) + 2 * Hd +
                    4 * Hd * c["gain_grad"], flops=12 * M * Hd)
    if c["kind"] == "qk":
        M, Hq, Hkv, D = (c[k] for k in ("M", "Hq", "Hkv", "D"))
        # the values themselves need not be read for their gradient
        return dict(bytes=2 * M * D * (3 * Hq + 5 * Hkv) + 4 * M + 12 * D,
                    flops=18 * M * (Hq + Hkv) * D)
    R, V = c["R"], c["V"]
    size = 2 if c["half"] else 4
    return dict(bytes=int(R * V * size * (1.0 - c["ignored"] + c["grad"])) +
                12 * R, flops=4 * R * V)


# ---------------------------------------------------------------------------
# 64 bits
# ---------------------------------------------------------------------------

def _leaf(x):
    return x.detach().double().requires_grad_(True)


def _exact_attn(c, s):
    n, Hq, Hkv, D = (c[k] for k in ("n_seq", "Hq", "Hkv", "D"))
    G = Hq // Hkv
    dq = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    dk = torch.zeros(s["k"].shape, dtype=torch.float64, device="cuda")
    dv = torch.zeros_like(dk)
    for r in _chunks(c):
        see = _visible(c, r)[:, None, :]
        for b in range(n):
            for h in range(Hkv):
                hh = slice(h * G, (h + 1) * G)
                q, k, v = (_leaf(s["q"][b, r, hh]), _leaf(s["k"][b, :, h]),
                           _leaf(s["v"][b, :, h]))
                x = (q.reshape(-1, D) @ k.T).view(-1, G, k.shape[0])
                x = torch.where(see, x / math.sqrt(D), -math.inf)
                o = torch.softmax(x, -1).view(-1, k.shape[0]) @ v
                a, e, f = torch.autograd.grad(
                    o, (q, k, v), s["dout"][b, r, hh].double().reshape(-1, D))
                dq[b, r, hh] = a
                dk[b, :, h] += e
                dv[b, :, h] += f
    return dict(dq=dq, dk=dk, dv=dv)


def _exact_norm(c, s):
    x, gain = _leaf(s["x"]), _leaf(s["gain"])
    y = x / torch.sqrt(x.square().mean(1, keepdim=True) + EPS) * gain
    dx, dg = torch.autograd.grad(y, (x, gain), s["dy"].double())
    if s["dres"] is not None:
        dx = dx + s["dres"].double()
    return dict(dx=dx, dgain=dg if c["gain_grad"] else None)


def _exact_qk(c, s):
    M, Hq, Hkv, D = (c[k] for k in ("M", "Hq", "Hkv", "D"))
    y = _leaf(s["qkv"])
    gains = _leaf(s["gq"]), _leaf(s["gk"])
    freq = THETA ** (-torch.arange(0, D, 2, dtype=torch.float64,
                                   device="cuda") / D)
    turn = torch.polar(torch.ones(M, 1, D // 2, dtype=torch.float64,
                                  device="cuda"),
                       (s["pos"].double()[:, None] * freq)[:, None])
    parts = y.view(M, -1, D).split((Hq, Hkv, Hkv), 1)
    outs = []
    for x, gain in zip(parts, gains):
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS) * gain
        z = torch.complex(x[..., :D // 2], x[..., D // 2:]) * turn
        outs.append(torch.cat((z.real, z.imag), -1))
    a, b, e = torch.autograd.grad(
        outs + [parts[2]], (y, *gains),
        [s["dq"].double(), s["dk"].double(), s["dv"].double()])
    return dict(dqkv=a, dq_gain=b, dk_gain=e)


def _exact_loss(c, s):
    loss, grads = [], []
    for i in range(0, c["R"], 256):
        x = _leaf(s["x"][i:i + 256, :c["V"]])
        l = torch.nn.functional.cross_entropy(
            x, s["t"][i:i + 256].long(), ignore_index=-1, reduction="none")
        l = l * s["w"][i:i + 256].double()
        if c["grad"]:
            grads.append(torch.autograd.grad(l.sum(), x)[0])
        loss.append(l.detach())
    return dict(loss=torch.cat(loss),
                dlogits=torch.cat(grads) if c["grad"] else None)


def exact(case, seed):
    return dict(attn=_exact_attn, norm=_exact_norm, qk=_exact_qk,
                loss=_exact_loss)[case["kind"]](case, prepare(case, seed))
