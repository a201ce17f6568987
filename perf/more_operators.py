"""The operators of serving over an 8-bit cache, as cases that can be timed:
rows appended to a cache of e4m3 codes with a scale per page and kv head, the
window's attention over that cache, the fork and the compaction of sequences'
pages, and the sampling of tokens.

listed() are fixed cases over the range of sizes; draw() gives more of the
same ranges.  prepare() builds what a serving program holds before the call,
run() is one pass: the plain form in torch operations, or with `own` the calls
of the binding; exact() is the same in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

PAGE = 16
E4M3 = torch.float8_e4m3fn


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------

def _append(L, B, T, lo, hi, at, Hkv, D):
    return dict(kind="append", L=L, B=B, T=T, lo=lo, hi=hi, at=at, Hkv=Hkv,
                D=D)


def _attn(B, W, Hq, Hkv, D, lo, hi, lse=True):
    return dict(kind="attn", B=B, W=W, Hq=Hq, Hkv=Hkv, D=D, lo=lo, hi=hi,
                lse=lse)


def _fork(L, Hkv, D, parents, children, lo, hi, pool, half=False):
    return dict(kind="fork", L=L, Hkv=Hkv, D=D, parents=parents,
                children=children, lo=lo, hi=hi, pool=pool, half=half)


def _compact(L, Hkv, D, B, pool, used, shared=0.0, half=False):
    return dict(kind="compact", L=L, Hkv=Hkv, D=D, B=B, pool=pool, used=used,
                shared=shared, half=half)


def _sample(B, W, V, half, stride=0, observed=0.0):
    return dict(kind="sample", B=B, W=W, V=V, half=half, stride=stride or V,
                observed=observed)


def listed():
    return [
        # what one decode step commits: a few tokens a sequence, every layer
        dict(_append(36, 16, 32, 0, 4, 1500, 8, 128), name="append_16x4"),
        # prompts of different lengths written at once
        dict(_append(8, 4, 1024, 700, 1024, 0, 8, 128), name="append_4x1024"),
        # a small model's window over a short prefix: latency
        dict(_attn(1, 16, 4, 2, 64, 257, 257), name="attn_1x257"),
        # single tokens of a batch of conversations: the cache is read, no more
        dict(_attn(64, 1, 32, 8, 128, 512, 4096), name="attn_64x4096_w1"),
        # the same batch with a window of 32
        dict(_attn(64, 32, 32, 8, 128, 512, 4096), name="attn_64x4096_w32"),
        # long prefixes, widest window: products
        dict(_attn(8, 64, 32, 8, 128, 32768, 32768), name="attn_8x32768"),
        # eight samples of one prompt
        dict(_fork(36, 8, 128, 1, 8, 2055, 2055, 512), name="fork_8"),
        # a batch of prompts, seven samples each, in the place of others
        dict(_fork(16, 8, 128, 16, 112, 400, 1000, 2048), name="fork_112"),
        # a small pool, bf16 pages of one layer
        dict(_compact(1, 2, 64, 4, 600, 0.5, half=True), name="compact_600"),
        # a pool that many sequences have left, with shared prompts
        dict(_compact(8, 8, 128, 64, 8192, 0.4, 0.2), name="compact_8192"),
        # the next token of one conversation, bf16 logits, padded columns
        dict(_sample(1, 1, 32003, True, 32064), name="sample_1x32003"),
        # every masked row of a batch of windows, full vocabulary
        dict(_sample(64, 32, 151936, False, observed=0.4),
             name="sample_64x32x151936"),
    ]


HEADS = ((4, 2), (8, 2), (4, 4), (32, 8), (32, 8), (28, 4), (16, 8), (16, 2))


def _log(rng, lo, hi):
    """A whole number spread over the logarithm of lo..hi."""
    return max(lo, min(hi, int(round(math.exp(
        rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("append", "attn", "attn", "fork", "compact", "sample",
                       "sample"))
    Hq, Hkv = rng.choice(HEADS)
    D = rng.choice((64, 128))
    if kind == "append":
        L, B = rng.choice((1, 4, 36)), _log(rng, 1, 32)
        T = _log(rng, 1, max(1, 32768 // (L * B)))
        return _append(L, B, T, rng.choice((0, T // 2, T)), T,
                       rng.choice((0, _log(rng, 1, 3000))), Hkv, D)
    if kind == "attn":
        B = _log(rng, 1, 64)
        hi = _log(rng, 16, min(32768, 262144 // B))
        return _attn(B, rng.choice((1, 1, 3, 8, 16, 31, 32, 64)), Hq, Hkv, D,
                     rng.choice((0, hi // 4, hi)), hi, rng.random() < 0.5)
    if kind == "fork":
        parents = _log(rng, 1, 16)
        children = parents * rng.randint(1, 7)
        hi = _log(rng, 1, 1000)
        L = rng.choice((1, 4, 16))
        pool = (parents * (hi // PAGE + 4) + children * (hi // 128 + 4) +
                rng.randint(0, 99))
        return _fork(L, Hkv, D, parents, children, rng.choice((0, hi)), hi,
                     pool, rng.random() < 0.4)
    if kind == "compact":
        L, half = rng.choice((1, 4, 8)), rng.random() < 0.4
        pool = _log(rng, 16, 3900 if half else 7800)
        return _compact(L, Hkv, D, _log(rng, 1, min(64, pool // 4)), pool,
                        rng.choice((0.1, 0.5, 0.9)),
                        rng.choice((0.0, 0.3)), half)
    W = rng.choice((1, 1, 4, 32))
    B = _log(rng, 1, min(64, 1216 // W))
    V = rng.choice((_log(rng, 2, 151936), _log(rng, 500, 151936), 151936))
    return _sample(B, W, V, rng.random() < 0.5,
                   V + rng.choice((0, 0, rng.randint(1, 64))),
                   rng.choice((0.0, 0.5)) if W > 1 else 0.0)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * (seed + 1))
    return g


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda").to(torch.bfloat16)


def _spread(lo, hi, n):
    """n whole numbers over lo..hi, in an order that is not sorted."""
    v = [lo + (hi - lo) * i // max(1, n - 1) for i in range(n)]
    return [v[i * (n // 2 + 1 if math.gcd(n, n // 2 + 1) == 1 else 1) % n]
            for i in range(n)]


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _exponent(a):
    """Smallest exponent e >= 1 with a <= 448 * 2^(e - 127)."""
    m, x = torch.frexp(a)
    e = torch.where(m <= 0.875, x + 118, x + 119)
    return torch.where(a > 0, e, 1).clamp(min=1)


def _codes(x, e):
    """e4m3 codes of x at the scales 2^(e - 127)."""
    return torch.ldexp(x, 127 - e).to(E4M3)


def _values(codes, e):
    return torch.ldexp(codes.float(), e.to(torch.int32) - 127)


def _cache(g, L, P, Hkv, D):
    """Pages of normal keys (some channels larger) and values."""
    k = torch.randn(L, P, Hkv, PAGE, D, generator=g, device="cuda")
    k *= torch.exp(0.7 * torch.randn(D, generator=g, device="cuda"))
    ke = _exponent(k.abs().amax((3, 4)))
    k = _codes(k, ke[..., None, None])
    v = torch.randn(L, P, Hkv, D, PAGE, generator=g, device="cuda")
    ve = _exponent(v.abs().amax((3, 4)))
    v = _codes(v, ve[..., None, None])
    return k, v, ke.to(torch.uint8), ve.to(torch.uint8)


def _prepare_append(c, g):
    L, B, T, Hkv, D = (c[k] for k in ("L", "B", "T", "Hkv", "D"))
    count = _spread(c["lo"], c["hi"], B)
    # sequences stand at different rows of a page
    start = [c["at"] and c["at"] + 5 * b for b in range(B)]
    maxp = max(-(-(s + n) // PAGE) for s, n in zip(start, count)) + 1
    P = B * (-(-max(count) // PAGE) + 2)
    # only the pages that are written are of interest: the table's other
    # entries stay empty
    ids = torch.randperm(P, generator=g, device="cuda").to(torch.int32)
    ids = ids.view(B, -1)
    bt = torch.full((B, maxp), -1, dtype=torch.int32, device="cuda")
    for b in range(B):
        a = start[b] // PAGE
        n = min(ids.shape[1], maxp - a)
        bt[b, a:a + n] = ids[b, :n]
    k8, v8, ke, ve = _cache(g, L, P, Hkv, D)
    return dict(case=c, k=_normal(g, L, B, T, Hkv, D),
                v=_normal(g, L, B, T, Hkv, D), start=_ints(start),
                count=_ints(count), bt=bt, k8=k8, v8=v8, ke=ke, ve=ve,
                status=torch.zeros(B, dtype=torch.int32, device="cuda"))


def _prepare_attn(c, g):
    B, W, Hq, Hkv, D = (c[k] for k in ("B", "W", "Hq", "Hkv", "D"))
    lens = _spread(c["lo"], c["hi"], B)
    need = [-(-n // PAGE) for n in lens]
    maxp, P = max(max(need), 1), max(sum(need), 1)
    ids = torch.randperm(P, generator=g, device="cuda").to(torch.int32)
    bt = torch.full((B, maxp), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        bt[b, :n] = ids[at:at + n]
        at += n
    k8, v8, ke, ve = (x[0] for x in _cache(g, 1, P, Hkv, D))
    return dict(case=c, q=_normal(g, B, W, Hq, D), k=_normal(g, B, W, Hkv, D),
                v=_normal(g, B, W, Hkv, D), k8=k8, v8=v8, ke=ke, ve=ve, bt=bt,
                plen=_ints(lens), mp=max(lens), out=torch.zeros(
                    B, W, Hq, D, dtype=torch.bfloat16, device="cuda"),
                lse=torch.zeros(B, W, Hq, device="cuda") if c["lse"] else None,
                status=torch.zeros(B, dtype=torch.int32, device="cuda"))


def _arrays(c, g):
    """A pool's arrays [L, P, ...] of random bytes: bf16 keys and values, or
    codes with their exponents."""
    L, P, Hkv, D = (c[k] for k in ("L", "pool", "Hkv", "D"))
    n = 2 * D if c["half"] else D
    shapes = [(L, P, Hkv, PAGE, n)] * 2
    if not c["half"]:
        shapes += [(L, P, Hkv)] * 2
    return [torch.randint(0, 256, s, generator=g, device="cuda",
                          dtype=torch.uint8) for s in shapes]


SPAN = 32      # positions that a sequence holds pages for behind its prefix


def _prepare_fork(c, g):
    n, m, P = c["parents"], c["children"], c["pool"]
    lens = _spread(c["lo"], c["hi"], n)
    # the children's rows hold short sequences that have ended
    ended = _spread(c["lo"] // 8, c["hi"] // 8, m)
    need = [-(-(x + SPAN) // PAGE) for x in lens + ended]
    maxp = max(need)
    ids = torch.randperm(P, generator=g, device="cuda").to(torch.int32)
    bt = torch.full((n + m, maxp), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, k in enumerate(need):
        bt[b, :k] = ids[at:at + k]
        at += k
    ref = torch.zeros(P, dtype=torch.int32, device="cuda")
    ref[ids[:at].long()] = 1
    parent = [i % n for i in range(m)]
    return dict(case=c, bt=bt, ref=ref, plen=_ints(lens + ended),
                parent=_ints(parent), child=_ints(range(n, n + m)),
                reserve=_ints([lens[p] + SPAN for p in parent]),
                status=torch.zeros(m, dtype=torch.int32, device="cuda"),
                arrays=_arrays(c, g))


def _prepare_compact(c, g):
    B, P = c["B"], c["pool"]
    used = max(1, int(P * c["used"]))
    # rows of the table share the pages of a prompt and own the others
    common = int(c["shared"] * used)
    each = (used - common) // B
    ids = torch.randperm(P, generator=g, device="cuda").to(torch.int32)
    bt = torch.full((B, common + each + 4), -1, dtype=torch.int32,
                    device="cuda")
    bt[:, :common] = ids[:common]
    bt[:, common:common + each] = ids[common:common + B * each].view(B, each)
    ref = torch.zeros(P, dtype=torch.int32, device="cuda")
    ref[ids[:common].long()] = B
    ref[ids[common:common + B * each].long()] = 1
    return dict(case=c, bt=bt, ref=ref, new_bt=torch.zeros_like(bt),
                new_ref=torch.zeros_like(ref), arrays=_arrays(c, g),
                n_used=torch.zeros(1, dtype=torch.int32, device="cuda"))


def _prepare_sample(c, g):
    B, W, V = c["B"], c["W"], c["V"]
    x = torch.randn(B, W, c["stride"], generator=g, device="cuda").mul_(2.0)
    # most rows have a few likely tokens
    t = torch.randint(0, V, (B, W, 8), generator=g, device="cuda")
    up = torch.rand(B, W, 8, generator=g, device="cuda") * 14.0
    x.scatter_add_(2, t, torch.where(
        torch.rand(B, W, 1, generator=g, device="cuda") < 0.8, up, 0.0))
    if c["half"]:
        x = x.to(torch.bfloat16)
    # requests with settings of their own, some greedy, some without limits
    kinds = dict(temperature=(1.0, 0.7, 1.3, 0.0, 0.2),
                 top_k=(0, 50, 20, 1000), top_p=(0.95, 1.0, 0.8, 0.5, 0.99),
                 min_p=(0.0, 0.05, 0.0))
    pick = {}
    for name, v in kinds.items():
        at = torch.randint(0, len(v), (B,), generator=g, device="cuda")
        pick[name] = torch.tensor(v, device="cuda")[at]
    pick["top_k"] = pick["top_k"].to(torch.int32)
    return dict(case=c, x=x, u=torch.rand(B, W, generator=g, device="cuda"),
                n_obs=_ints(_spread(0, int(2 * c["observed"] * W), B)),
                token=torch.full((B, W), -1, dtype=torch.int32,
                                 device="cuda"),
                logp=torch.zeros(B, W, device="cuda"), **pick)


def prepare(case, seed):
    return dict(append=_prepare_append, attn=_prepare_attn,
                fork=_prepare_fork, compact=_prepare_compact,
                sample=_prepare_sample)[case["kind"]](case, _gen(seed))


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def _append_plain(s, x, codes, e, values):
    """One of the two halves; `values`: pages hold their rows transposed."""
    L, B, T, Hkv, D = x.shape
    P = codes.shape[1]
    start, count = s["start"].long(), s["count"].long()
    j = torch.arange(T, device="cuda")
    b, j = torch.nonzero(j < count[:, None], as_tuple=True)
    page = s["bt"][b, (start[b] + j) // PAGE].long()
    row = (start[b] + j) % PAGE
    new = x[:, b, j].float()                              # [L, n, Hkv, D]
    top = torch.zeros(L, P, Hkv, device="cuda").scatter_reduce_(
        1, page[:, None].expand(L, -1, Hkv), new.abs().amax(3), "amax")
    e0 = e.to(torch.int32)
    need = _exponent(top).to(torch.int32)
    touched = torch.zeros(P, dtype=torch.bool, device="cuda")
    touched[page] = True
    # the page that a sequence's first new row shares with its old ones
    old = torch.nonzero((count > 0) & (start % PAGE > 0))[:, 0]
    op = s["bt"][old, start[old] // PAGE].long()
    e1 = torch.where(touched[:, None], need, e0)
    e1[:, op] = torch.maximum(e0[:, op], need[:, op])
    at = codes[:, op].float()
    again = torch.ldexp(at, (e0 - e1)[:, op][..., None, None]).to(E4M3)
    keep = torch.arange(PAGE, device="cuda") < (start[old] % PAGE)[:, None]
    keep = keep[:, None, None, :] if values else keep[:, None, :, None]
    u8 = codes.view(torch.uint8)
    u8[:, op] = torch.where(keep, again.view(torch.uint8), u8[:, op])
    new = _codes(new, e1[:, page][..., None]).view(torch.uint8)
    new = new.permute(1, 0, 2, 3)
    if values:
        u8[:, page, :, :, row] = new
    else:
        u8[:, page, :, row] = new
    e.copy_(e1)


def _run_append(s):
    if own:
        from paper_2512_22737_amd import wedlm
        wedlm.wedlm_cache8_append(s["k"], s["v"], s["start"], s["count"],
                                  s["k8"], s["v8"], s["ke"], s["ve"], s["bt"],
                                  s["status"])
    else:
        _append_plain(s, s["k"], s["k8"], s["ke"], False)
        _append_plain(s, s["v"], s["v8"], s["ve"], True)
    return dict(k8=s["k8"], v8=s["v8"], k_exp=s["ke"], v_exp=s["ve"],
                status=s["status"])


def _run_attn(s):
    if own:
        from paper_2512_22737_amd import wedlm
        wedlm.wedlm_window_attn_cache8(
            s["q"], s["k"], s["v"], s["k8"], s["v8"], s["ke"], s["ve"],
            s["bt"], s["plen"], s["mp"], s["out"], s["lse"], s["status"])
        return dict(out=s["out"], lse=s["lse"], status=s["status"])
    c = s["case"]
    B, W, Hq, Hkv, D = (c[k] for k in ("B", "W", "Hq", "Hkv", "D"))
    G, n = Hq // Hkv, s["bt"].shape[1] * PAGE
    bt = s["bt"].clamp(min=0).long()
    k = _values(s["k8"][bt], s["ke"][bt][..., None, None])
    k = k.permute(0, 2, 1, 3, 4).reshape(B, Hkv, n, D)
    k = torch.cat((k, s["k"].float().transpose(1, 2)), 2)
    v = _values(s["v8"][bt], s["ve"][bt][..., None, None])
    v = v.permute(0, 2, 1, 4, 3).reshape(B, Hkv, n, D)
    v = torch.cat((v, s["v"].float().transpose(1, 2)), 2)
    q = s["q"].float().view(B, W, Hkv, G, D).permute(0, 2, 1, 3, 4)
    x = q.reshape(B, Hkv, W * G, D) @ k.transpose(2, 3)
    x *= D ** -0.5
    j = torch.arange(n, device="cuda")
    w = torch.arange(W, device="cuda")
    hide = torch.cat((
        (j >= s["plen"][:, None])[:, None].expand(B, W, n),
        (w[None, :] > w[:, None])[None].expand(B, W, W)), 2)
    x.view(B, Hkv, W, G, -1).masked_fill_(hide[:, None, :, None], -math.inf)
    m = x.amax(3, keepdim=True)
    x = x.sub_(m).exp_()
    l = x.sum(3, keepdim=True)
    o = (x @ v) / l
    o = o.view(B, Hkv, W, G, D).permute(0, 2, 1, 3, 4).reshape(B, W, Hq, D)
    z = None
    if c["lse"]:
        z = (m + torch.log(l)).view(B, Hkv, W, G)
        z = z.permute(0, 2, 1, 3).reshape(B, W, Hq)
    return dict(out=o.to(torch.bfloat16), lse=z, status=s["status"])


def _run_fork(s):
    bt, ref, plen = s["bt"], s["ref"], s["plen"]
    if own:
        from paper_2512_22737_amd import wedlm
        wedlm.wedlm_cache_free(s["child"], bt, ref, plen)
        wedlm.wedlm_cache_fork(s["parent"], s["child"], s["reserve"], plen,
                               bt, ref, s["arrays"], s["status"])
        return dict(table=bt, ref=ref, plen=plen, status=s["status"],
                    arrays=s["arrays"])
    parent, child = s["parent"].long(), s["child"].long()
    one = torch.ones((), dtype=torch.int32, device="cuda")
    rows = bt[child]
    ref.index_add_(0, rows.clamp(min=0).view(-1).long(),
                   -(rows >= 0).int().view(-1))
    j = torch.arange(bt.shape[1], device="cuda")
    c = plen[parent].long()
    full, upto = c // PAGE, (torch.maximum(s["reserve"].long(), c) + 15) // PAGE
    rows = bt[parent]
    shares = j < full[:, None]
    fresh = (j >= full[:, None]) & (j < upto[:, None])
    ref.index_add_(0, rows.clamp(min=0).view(-1).long(),
                   shares.int().view(-1))
    free = torch.argsort(ref != 0, stable=True)       # free pages first
    order = (torch.cumsum(fresh.view(-1), 0) - 1).view(fresh.shape)
    given = free[order.clamp(min=0)].int()
    bt[child] = torch.where(shares, rows, torch.where(fresh, given, -1))
    ref[given[fresh].long()] = one
    plen[child] = plen[parent]
    part = torch.nonzero(c % PAGE > 0)[:, 0]
    src = rows[part, full[part]].long()
    dst = given[part, full[part]].long()
    for a in s["arrays"]:
        a[:, dst] = a[:, src]
    return dict(table=bt, ref=ref, plen=plen, status=s["status"],
                arrays=s["arrays"])


def _run_compact(s):
    bt, ref = s["bt"], s["ref"]
    if own:
        from paper_2512_22737_amd import wedlm
        wedlm.wedlm_cache_compact(bt, ref, s["arrays"], s["new_bt"],
                                  s["new_ref"], s["n_used"])
        return dict(table=s["new_bt"], ref=s["new_ref"], n_used=s["n_used"],
                    arrays=s["arrays"])
    P = ref.shape[0]
    ids = torch.arange(P, device="cuda")
    used = ref > 0
    n = used.sum()
    src = torch.nonzero(used & (ids >= n))[:, 0]
    dst = torch.nonzero(~used & (ids < n))[:, 0]
    to = ids.clone()
    to[src] = dst
    new_bt = torch.where(bt >= 0, to[bt.clamp(min=0).long()].int(), -1)
    new_ref = torch.where(used & (ids < n), ref, 0)
    new_ref[dst] = ref[src]
    for a in s["arrays"]:
        a[:, dst] = a[:, src]
    return dict(table=new_bt, ref=new_ref, n_used=n.int().view(1),
                arrays=s["arrays"])


def _run_sample(s):
    c = s["case"]
    token, logp = s["token"], s["logp"]
    if own:
        from paper_2512_22737_amd import wedlm
        wedlm.wedlm_sample(s["x"], s["u"], token, s["temperature"],
                           s["top_k"], s["top_p"], s["min_p"], s["n_obs"],
                           logp, V=c["V"])
        return dict(token=token, logp=logp)
    W, V = c["W"], c["V"]
    b, i = torch.nonzero(torch.arange(W, device="cuda") >=
                         s["n_obs"][:, None], as_tuple=True)
    x, at = torch.sort(s["x"][b, i, :V].float(), dim=1, descending=True,
                       stable=True)
    T = s["temperature"][b].double()[:, None]
    greedy = ~(T > 0)
    k = s["top_k"][b].long()[:, None]
    k = torch.where(greedy, 1, torch.where(k > 0, k, V))
    # values next to a border: 64 bits
    z = (x.double() - x[:, :1].double()) / torch.where(greedy, 1.0, T)
    w = torch.exp(z)
    w = torch.where(torch.arange(V, device="cuda") < k, w, 0.0)
    before = torch.cumsum(w, 1) - w
    p = s["top_p"][b].double()[:, None]
    total = w.sum(1, keepdim=True)
    keep = (p >= 1) | (before < p * total)
    keep[:, 0] = True
    keep &= w >= s["min_p"][b].double()[:, None]
    w = torch.where(keep, w, 0.0)
    total = w.sum(1, keepdim=True)
    w = torch.zeros_like(w).scatter_(1, at, w)        # by token
    sums = torch.cumsum(w, 1)
    u = s["u"][b, i].double()[:, None]
    t = (sums <= u * sums[:, -1:]).sum(1).clamp(max=V - 1)
    token[b, i] = t.int()
    logp[b, i] = torch.log(w.gather(1, t[:, None]) / total)[:, 0].float()
    return dict(token=token, logp=logp)


def run(state):
    return dict(append=_run_append, attn=_run_attn, fork=_run_fork,
                compact=_run_compact, sample=_run_sample)[
                    state["case"]["kind"]](state)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def _page_bytes(c):
    """Bytes of a page over all layers and arrays."""
    rows = c["Hkv"] * PAGE * c["D"] * 2
    return c["L"] * (2 * rows if c["half"] else rows + 2 * c["Hkv"])


def work(c):
    if c["kind"] == "append":
        n = sum(_spread(c["lo"], c["hi"], c["B"])) * c["L"]
        return dict(bytes=n * c["Hkv"] * c["D"] * 2 * 3 + 8 * c["B"],
                    flops=n * c["Hkv"] * c["D"] * 2 * 2)
    if c["kind"] == "attn":
        B, W, Hq, Hkv, D = (c[k] for k in ("B", "W", "Hq", "Hkv", "D"))
        lens = _spread(c["lo"], c["hi"], B)
        pages = sum(-(-n // PAGE) for n in lens)
        return dict(
            bytes=sum(lens) * 2 * Hkv * D + pages * (2 * Hkv + 4) +
            B * W * (2 * D * (2 * Hq + 2 * Hkv) + 4 * Hq * c["lse"]),
            flops=sum(4 * D * Hq * (W * n + W * (W + 1) // 2) for n in lens))
    if c["kind"] == "fork":
        lens = _spread(c["lo"], c["hi"], c["parents"])
        rows = sum(lens[i % c["parents"]] % PAGE for i in range(c["children"]))
        need = sum(-(-(lens[i % c["parents"]] + SPAN) // PAGE)
                   for i in range(c["children"]))
        return dict(bytes=2 * rows * _page_bytes(c) // PAGE + 16 * need +
                    4 * c["pool"], flops=0)
    if c["kind"] == "compact":
        moves = c["pool"] * c["used"] * (1 - c["used"])
        return dict(bytes=int(2 * moves * _page_bytes(c)) + 8 * c["pool"],
                    flops=0)
    B, W, V = c["B"], c["W"], c["V"]
    rows = sum(W - n for n in _spread(0, int(2 * c["observed"] * W), B))
    return dict(bytes=rows * V * (2 if c["half"] else 4) + 12 * rows + 20 * B,
                flops=4 * rows * V)


# ---------------------------------------------------------------------------
# 64 bits
# ---------------------------------------------------------------------------

def _e4m3_table():
    """The magnitudes of e4m3, in rising order of their codes."""
    v = [m * 2.0 ** -9 for m in range(8)]
    v += [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)]
    return torch.tensor(v[:127], dtype=torch.float64, device="cuda")


def _nearest(x, table):
    """The nearest e4m3 value of each x, ties to the even code."""
    a = x.abs().contiguous()
    hi = torch.searchsorted(table, a).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    up, down = table[hi] - a, a - table[lo]
    take = (up < down) | ((up == down) & (hi % 2 == 0))
    return torch.copysign(torch.where(take, table[hi], table[lo]), x)


def _exact_append(c, s):
    table = _e4m3_table()
    start, count = s["start"].tolist(), s["count"].tolist()
    bt = s["bt"].tolist()
    got = dict(k_exp=None, v_exp=None, status=None)
    for name, x, codes, e, values in (("k8", s["k"], s["k8"], s["ke"], False),
                                      ("v8", s["v"], s["v8"], s["ve"], True)):
        out = codes.double()
        if values:
            out = out.transpose(3, 4).contiguous()
        for b in range(c["B"]):
            at, end = start[b], start[b] + count[b]
            while at < end:
                n = min(PAGE - at % PAGE, end - at)
                pg, r = bt[b][at // PAGE], at % PAGE
                y = x[:, b, at - start[b]:at - start[b] + n].double()
                y = y.transpose(1, 2)                     # [L, Hkv, n, D]
                top = y.abs().amax((2, 3)) / 448
                ex = torch.ceil(torch.log2(top.clamp(min=2.0 ** -126)))
                ex = torch.where(2.0 ** (ex - 1) >= top, ex - 1, ex)
                old = e[:, pg].double() - 127
                if r:
                    ex = torch.maximum(ex, old)
                    out[:, pg, :, :r] = _nearest(
                        out[:, pg, :, :r] *
                        (2.0 ** (old - ex))[..., None, None], table)
                out[:, pg, :, r:r + n] = _nearest(
                    y * (2.0 ** -ex)[..., None, None], table)
                at += n
        got[name] = out.transpose(3, 4).contiguous() if values else out
    return got


def _exact_attn(c, s):
    B, W, Hq, Hkv, D = (c[k] for k in ("B", "W", "Hq", "Hkv", "D"))
    G = Hq // Hkv
    out = torch.zeros(B, W, Hq, D, dtype=torch.float64, device="cuda")
    lse = torch.zeros(B, W, Hq, dtype=torch.float64, device="cuda")
    see = torch.ones(W, W, dtype=torch.bool, device="cuda").tril()
    for b, n in enumerate(s["plen"].tolist()):
        pages = s["bt"][b, :-(-n // PAGE)].long()
        for h in range(Hkv):
            scale = 2.0 ** (s["ke"][pages, h].double() - 127)
            k = s["k8"][pages, h].double() * scale[:, None, None]
            scale = 2.0 ** (s["ve"][pages, h].double() - 127)
            v = s["v8"][pages, h].double() * scale[:, None, None]
            k = torch.cat((k.reshape(-1, D)[:n], s["k"][b, :, h].double()))
            v = torch.cat((v.transpose(1, 2).reshape(-1, D)[:n],
                           s["v"][b, :, h].double()))
            q = s["q"][b, :, h * G:(h + 1) * G].double().reshape(-1, D)
            x = (q @ k.T).view(W, G, -1) / math.sqrt(D)
            x[:, :, n:] = torch.where(see[:, None], x[:, :, n:], -math.inf)
            lse[b, :, h * G:(h + 1) * G] = torch.logsumexp(x, 2)
            out[b, :, h * G:(h + 1) * G] = (
                torch.softmax(x, 2).view(W * G, -1) @ v).view(W, G, D)
    return dict(out=out, lse=lse if c["lse"] else None, status=None)


def _exact_sample(c, s):
    V = c["V"]
    token, logp = s["token"].clone(), s["logp"].double()
    n_obs = s["n_obs"].tolist()
    for b in range(c["B"]):
        T, k, p, least = (s[n][b].item() for n in (
            "temperature", "top_k", "top_p", "min_p"))
        for i in range(n_obs[b], c["W"]):
            x = s["x"][b, i, :V].double()
            first = torch.argmax(x)
            if T <= 0:
                token[b, i], logp[b, i] = first, 0.0
                continue
            w = torch.exp((x - x[first]) / T)
            order = torch.argsort(x, descending=True, stable=True)
            order = order[:k] if k > 0 else order
            top = w[order]
            if p < 1:
                share = torch.cumsum(top, 0) / top.sum()
                order = order[:1 + int((share < p).sum())]
            order = order[w[order] >= least]
            order = torch.sort(order)[0]
            sums = torch.cumsum(w[order], 0)
            at = torch.searchsorted(sums, s["u"][b, i].double() * sums[-1],
                                    right=True)
            t = order[at.clamp(max=order.numel() - 1)]
            token[b, i], logp[b, i] = t, torch.log(w[t] / sums[-1])
    return dict(token=token, logp=logp)


def exact(case, seed):
    how = dict(append=_exact_append, attn=_exact_attn, sample=_exact_sample)
    if case["kind"] not in how:
        return None                      # whole numbers and copied bytes
    return how[case["kind"]](case, prepare(case, seed))
