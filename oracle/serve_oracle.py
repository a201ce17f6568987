"""fp64 CPU oracle of the serving operators (include/wedlm_serve.h), written
from their definitions: the 8-bit cache's codes and scales, the attention over
it with the bound of its roundings, sampling, and the pages' bookkeeping.  Test
infrastructure only; shares nothing with the HIP path."""
from __future__ import annotations

import numpy as np

PAGE = 16
CAPACITY, BAD_PAGE, BAD_LEN, BAD_ROW = 1, 2, 4, 8
BF16, F32 = 2.0 ** -8, 2.0 ** -24          # half a step, relative


# ---------------------------------------------------------------------------
# e4m3
# ---------------------------------------------------------------------------

def _magnitudes():
    v = np.zeros(128)
    for c in range(128):
        e, m = c >> 3, c & 7
        v[c] = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
    v[127] = np.nan
    return v


_MAG = _magnitudes()
VALUES = np.concatenate((_MAG, -_MAG))     # of the 256 codes


def encode(x):
    """Nearest e4m3 code of each |x| <= 448, ties to the even code; what is
    not finite becomes NaN (0x7f)."""
    x = np.asarray(x, dtype=np.float64)
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    assert (a <= 448.0).all()
    hi = np.minimum(np.searchsorted(_MAG[:127], a), 126)
    lo = np.maximum(hi - 1, 0)
    up, down = _MAG[hi] - a, a - _MAG[lo]
    c = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    c = c + np.where(np.signbit(x), 128, 0)
    return np.where(np.isfinite(x), c, 127).astype(np.uint8)


def need_exp(x):
    """Smallest exponent >= 1 whose scale holds the largest finite |x|."""
    x = np.abs(np.asarray(x, dtype=np.float64))
    x = x[np.isfinite(x)]
    e = 1
    while x.size and x.max() > 448.0 * 2.0 ** (e - 127):
        e += 1
    return e


def append(k, v, start, count, k8, v8, ke, ve, bt):
    """wedlm_cache8_append on copies; k, v [L, B, T, Hkv, D] fp64.  Returns
    (k8, v8, ke, ve, status)."""
    k8, v8, ke, ve = k8.copy(), v8.copy(), ke.copy(), ve.copy()
    L, B, T, H, D = k.shape
    P = k8.shape[1]
    status = np.zeros(B, np.int32)
    for b in range(B):
        s, n = int(start[b]), int(count[b])
        if s < 0 or n < 0 or n > T:
            status[b] |= BAD_LEN
            continue
        at = s
        while at < s + n:
            r0 = at % PAGE
            m = min(PAGE - r0, s + n - at)
            page = at // PAGE
            j = at - s
            at += m
            if page >= bt.shape[1]:
                status[b] |= CAPACITY
                continue
            p = int(bt[b, page])
            if p < 0 or p >= P:
                status[b] |= BAD_PAGE
                continue
            for l in range(L):
                for h in range(H):
                    for x, codes, ex in ((k, k8, ke), (v, v8, ve)):
                        rows = x[l, b, j:j + m, h]
                        pg = codes[l, p, h]
                        pg = pg if x is k else pg.T          # [16, D] view
                        e = need_exp(rows)
                        if r0:
                            old = int(ex[l, p, h])
                            e = max(e, old)
                            if e > old:
                                pg[:r0] = encode(VALUES[pg[:r0]] *
                                                 2.0 ** (old - e))
                        pg[r0:r0 + m] = encode(rows * 2.0 ** (127 - e))
                        ex[l, p, h] = e
    return k8, v8, ke, ve, status


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------

def gather(k8, v8, ke, ve, bt, b, c):
    """The prefix's keys and values [c, Hkv, D] in fp64."""
    pages = bt[b, :-(-c // PAGE)]
    k = VALUES[k8[pages]] * 2.0 ** (ke[pages].astype(float) - 127)[..., None,
                                                                  None]
    v = VALUES[v8[pages]] * 2.0 ** (ve[pages].astype(float) - 127)[..., None,
                                                                  None]
    k = k.transpose(0, 2, 1, 3).reshape(-1, k8.shape[1], k8.shape[3])[:c]
    v = v.transpose(0, 3, 1, 2).reshape(-1, k8.shape[1], k8.shape[3])[:c]
    return k, v


def attention(q, kw, vw, kp, vp, scale):
    """One sequence: q [W, Hq, D], kw, vw [W, Hkv, D], prefix kp, vp [c, Hkv,
    D] -> out, lse and elementwise bounds of their errors.

    With A = sum p |v|: the weights enter the product in bf16 (half a step of
    A) and the result is rounded to bf16 (another half step of A, |out| <= A).  A score is a sum of D products and carries
    (D + 2) fp32 roundings of S = sum |q k| scale, which move every weight by
    that much relatively and A by twice it; sums over n keys carry n / 16
    roundings (16 are added as a tree per tile) and the exponentials 4."""
    W, Hq, D = q.shape
    Hkv = kw.shape[1]
    G = Hq // Hkv
    c = kp.shape[0]
    out, lse = np.zeros((W, Hq, D)), np.zeros((W, Hq))
    bo, bl = np.zeros((W, Hq, D)), np.zeros((W, Hq))
    for h in range(Hq):
        k = np.concatenate((kp[:, h // G], kw[:, h // G]))
        v = np.concatenate((vp[:, h // G], vw[:, h // G]))
        x = q[:, h] @ k.T * scale
        S = (np.abs(q[:, h]) @ np.abs(k).T * scale).max(1)
        see = np.arange(c + W)[None] <= c + np.arange(W)[:, None]
        x = np.where(see, x, -np.inf)
        m = x.max(1, keepdims=True)
        p = np.exp(x - m)
        l = p.sum(1, keepdims=True)
        p /= l
        out[:, h] = p @ v
        lse[:, h] = (m + np.log(l))[:, 0]
        A = p @ np.abs(v)
        ds = (D + 2) * F32 * S + 4 * F32
        sums = ((c + W) / 16 + 16) * F32
        bo[:, h] = A * (2 * BF16 * (1 + BF16) +
                        (2 * ds + 2 * sums)[:, None] * 1.1)
        bl[:, h] = ds + sums + 4 * F32 * (np.abs(lse[:, h]) + 32)
    return out, lse, bo, bl


# ---------------------------------------------------------------------------
# sampling
# ---------------------------------------------------------------------------

def sample(x, u, T=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One row -> (token, logp)."""
    x = np.where(np.isnan(x), -np.inf, np.asarray(x, np.float64))
    x = np.minimum(x, 3.4028234663852886e38) + 0.0
    V = len(x)
    order = np.lexsort((np.arange(V), -x))
    if not T > 0 or x[order[0]] == -np.inf:
        return int(order[0]), 0.0
    if 0 < top_k < V:
        order = order[:top_k]
    live = x > -np.inf
    w = np.where(live, np.exp((np.where(live, x, x[order[0]]) -
                               x[order[0]]) / T), 0.0)
    if top_p < 1:
        sums = np.cumsum(w[order])
        order = order[:1 + int((sums < max(top_p, 0.0) * sums[-1]).sum())]
    if min_p > 0:
        order = order[w[order] >= min(min_p, 1.0)]
    order = np.sort(order)
    sums = np.cumsum(w[order])
    u = min(max(u, 0.0), 1 - 2.0 ** -24)
    t = order[min(int((sums <= u * sums[-1]).sum()), len(order) - 1)]
    return int(t), float((x[t] - x.max()) / T - np.log(sums[-1]))


# ---------------------------------------------------------------------------
# pages
# ---------------------------------------------------------------------------

def free(rows, bt, ref, plen):
    bt, ref, plen = bt.copy(), ref.copy(), plen.copy()
    for r in dict.fromkeys(int(r) for r in rows):
        if 0 <= r < bt.shape[0]:
            for p in bt[r]:
                if 0 <= p < len(ref) and ref[p] > 0:
                    ref[p] -= 1
            bt[r] = -1
            plen[r] = 0
    return bt, ref, plen


def fork(parent, child, reserve, plen, bt, ref):
    """-> (bt, ref, plen, status, [(from, to) page copies])."""
    B, maxp = bt.shape
    P, n = len(ref), len(parent)
    status = np.zeros(n, np.int32)
    needs = [0] * n
    for i in range(n):
        p, c = int(parent[i]), int(child[i])
        others = [j for j in range(n) if j != i]
        if not 0 <= c < B or not -1 <= p < B:
            status[i] = BAD_ROW
            continue
        length = int(plen[p]) if p >= 0 else 0
        upto = -(-max(length, int(reserve[i]), 0) // PAGE)
        if length < 0 or upto > maxp:
            status[i] = BAD_LEN
        elif any(child[j] == c or parent[j] == c for j in others) or (
                p != c and (bt[c] >= 0).any()):
            status[i] = BAD_ROW
        elif p == c:
            needs[i] = int((bt[c, :upto] < 0).sum())
        elif p >= 0 and not all(0 <= x < P
                                for x in bt[p, :-(-length // PAGE)]):
            status[i] = BAD_PAGE
        else:
            needs[i] = upto - length // PAGE
    ids = [i for i in range(P) if ref[i] <= 0]
    bt, ref, new_len, copies, at = (bt.copy(), ref.copy(), plen.copy(), [], 0)
    for i in range(n):
        at += needs[i]
        if needs[i] and at > len(ids):
            status[i] = CAPACITY
        if status[i]:
            continue
        mine = ids[at - needs[i]:at]
        p, c = int(parent[i]), int(child[i])
        length = int(plen[p]) if p >= 0 else 0
        upto = -(-max(length, int(reserve[i]), 0) // PAGE)
        full = 0 if p == c else length // PAGE
        for j in range(upto):
            if j < full:
                bt[c, j] = bt[p, j]
                ref[bt[p, j]] += 1
            elif p != c or bt[c, j] < 0:
                bt[c, j] = mine.pop(0)
                ref[bt[c, j]] = 1
        if p != c:
            if length % PAGE:
                copies.append((int(bt[p, full]), int(bt[c, full])))
            new_len[c] = length
    return bt, ref, new_len, status, copies


def compact(bt, ref):
    """-> (bt, ref, n_used, [(from, to)])."""
    n = int((ref > 0).sum())
    src = [i for i in range(n, len(ref)) if ref[i] > 0]
    dst = [i for i in range(n) if ref[i] <= 0]
    name = np.arange(len(ref))
    new = np.zeros_like(ref)
    new[:n] = ref[:n]
    for s, d in zip(src, dst):
        name[s] = d
        new[d] = ref[s]
    ok = (bt >= 0) & (bt < len(ref))
    return (np.where(ok, name[np.where(ok, bt, 0)], -1).astype(np.int32), new,
            n, list(zip(src, dst)))
