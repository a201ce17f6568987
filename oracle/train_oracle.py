"""Plain fp64 CPU oracle of the training-time gradients (numpy, test
infrastructure only): the backward passes of the dual-stream attention of
Sec. 4.2, of RMSNorm and of the per-head q/k norm with RoPE, and the masked
tokens' loss.

Each function takes values that are exact in fp64 (bf16 and fp32 inputs
widened) and returns the exact gradients with a bound of how far the HIP
kernels may be off, element by element, from the roundings they make:
half a step of bf16 is 2^-8 relative, of fp32 2^-24."""
from __future__ import annotations

import math

import numpy as np

BF16 = 2.0 ** -8
F32 = 2.0 ** -24


def dual_stream_visible(L, block):
    """[2L, 2L] truth: memory row p sees memory keys 0..p, a prediction row
    the memory before its block and its block's rows up to itself."""
    vis = np.zeros((2 * L, 2 * L), dtype=bool)
    for p in range(L):
        f = p // block * block
        vis[p, :p + 1] = True
        vis[L + p, :f] = True
        vis[L + p, L + f:L + p + 1] = True
    return vis


def attn_forward(q, k, v, vis, scale):
    """q [N, Hq, D], k, v [N, Hkv, D] -> out [N, Hq, D], lse [N, Hq]."""
    Hq, Hkv = q.shape[1], k.shape[1]
    out, lse = np.empty_like(q), np.empty(q.shape[:2])
    for h in range(Hq):
        s = np.where(vis, scale * q[:, h] @ k[:, h * Hkv // Hq].T, -np.inf)
        m = s.max(1, keepdims=True)
        e = np.exp(s - m)
        z = e.sum(1, keepdims=True)
        out[:, h] = e / z @ v[:, h * Hkv // Hq]
        lse[:, h] = (m + np.log(z))[:, 0]
    return out, lse


def attn_backward(q, k, v, dout, vis, scale, out_err=None):
    """-> (dq, dk, dv), (their bounds).

    The kernels round P and dS to bf16 before the products with q, k and dout
    (BF16 of each term), the result once more, and take D = sum dout out from
    a bf16 output: out_err [N, Hq, D] is how far that output may be off (half
    a step of its own by default), and moves dS by P sum |dout| out_err.
    fp32: a sum of n products is off by at most n F32 of the sum of their
    magnitudes, the exponent by F32 of its terms (twice), v_exp_f32 by about
    one step."""
    N, Hq, D = q.shape
    Hkv = k.shape[1]
    dq = np.zeros_like(q)
    dk, dv = np.zeros_like(k), np.zeros_like(v)
    bq, bk, bv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    out, lse = attn_forward(q, k, v, vis, scale)
    if out_err is None:
        out_err = BF16 * np.abs(out)
    for h in range(Hq):
        g = h * Hkv // Hq
        Q, K, V, dO = q[:, h], k[:, g], v[:, g], dout[:, h]
        s = scale * Q @ K.T
        p = np.where(vis, np.exp(np.minimum(s - lse[:, h:h + 1], 0.0)), 0.0)
        dp = dO @ V.T
        delta = (dO * out[:, h]).sum(1, keepdims=True)
        ds = p * (dp - delta)
        dq[:, h] = scale * ds @ K
        dk[:, g] += scale * ds.T @ Q
        dv[:, g] += p.T @ dO
        # relative error of p; absolute errors of dp - delta and of ds
        rel = F32 * ((D + 4) * scale * (np.abs(Q) @ np.abs(K).T) +
                     4 * np.abs(lse[:, h:h + 1]) + 8)
        e_dp = (F32 * (D + 2) * (np.abs(dO) @ np.abs(V).T +
                                 (np.abs(dO) * np.abs(out[:, h])).sum(
                                     1, keepdims=True)) +
                (np.abs(dO) * out_err[:, h]).sum(1, keepdims=True))
        e_p = p * (rel + BF16)
        e_ds = np.abs(ds) * (rel + BF16) + p * (1 + rel + BF16) * e_dp
        n = F32 * 2 * N
        bq[:, h] = scale * (e_ds + n * np.abs(ds)) @ np.abs(K)
        bk[:, g] += scale * (e_ds + n * np.abs(ds)).T @ np.abs(Q)
        bv[:, g] += (e_p + n * p).T @ np.abs(dO)
    # second-order terms, then the result's own rounding
    out = []
    for x, b in ((dq, bq), (dk, bk), (dv, bv)):
        b = 1.01 * b
        out.append(b + BF16 * (np.abs(x) + b))
    return (dq, dk, dv), tuple(out)


def attn_out_error(q, k, v, vis, scale):
    """How far the forward kernel's output may be off: P in bf16, partial
    outputs of the splits in bf16, the output itself."""
    Hq, Hkv = q.shape[1], k.shape[1]
    err = np.empty_like(q)
    out, lse = attn_forward(q, k, v, vis, scale)
    for h in range(Hq):
        K, V = k[:, h * Hkv // Hq], v[:, h * Hkv // Hq]
        p = np.where(vis, np.exp(np.minimum(
            scale * q[:, h] @ K.T - lse[:, h:h + 1], 0.0)), 0.0)
        err[:, h] = 1.02 * (2 * BF16 * p @ np.abs(V) + BF16 * np.abs(out[:, h]))
    return err


def rmsnorm(x, gain, eps):
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gain


def rmsnorm_backward(x, gain, dy, eps, dy_err=None):
    """Norms over the last axis -> (dx, dgain), (their bounds).  dgain is
    summed over all others.  dy_err: how far the kernel's dy may be off.

    fp32: sums of n terms are off by n F32 of their magnitudes' sum (the
    kernels add pairwise, so log2 n would do), r by the sum of squares'
    error and three roundings, each product by one."""
    n, rows = x.shape[-1], x.size // x.shape[-1]
    if dy_err is None:
        dy_err = np.zeros_like(dy)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    xh, u = x * r, dy * gain
    m = (u * xh).mean(-1, keepdims=True)
    dx = r * (u - xh * m)
    other = tuple(range(x.ndim - 1))
    dg = (dy * xh).sum(other)
    rel = F32 * (n / 2 + 6)                       # of r and of xh
    e_u = np.abs(dy_err * gain) + F32 * np.abs(u)
    e_m = ((e_u + (rel + F32 * (n + 3)) * np.abs(u)) * np.abs(xh)).mean(
        -1, keepdims=True)
    b_x = r * (e_u + np.abs(xh) * (e_m + np.abs(m) * (2 * rel + 6 * F32)) +
               (rel + 3 * F32) * (np.abs(u) + np.abs(xh * m)))
    b_g = (np.abs(dy_err * xh) + (rel + F32 * (rows + 3)) *
           np.abs(dy * xh)).sum(other)
    return (dx, dg), (1.01 * b_x, 1.01 * b_g)


def rotate(x, pos, theta, back=False):
    """x [M, heads, D] turned by the angles of pos [M] ("rotate half")."""
    h = x.shape[-1] // 2
    a = pos[:, None, None] * theta ** (-np.arange(h) / h)
    c, s = np.cos(a), np.sin(a) * (-1 if back else 1)
    lo, hi = x[..., :h], x[..., h:]
    return np.concatenate((lo * c - hi * s, hi * c + lo * s), -1)


def qk_norm_rope_backward(x, gain, pos, dy, theta, eps):
    """x, dy [M, heads, D] of the query or the key heads -> (dx, dgain), (their
    bounds), dx with its rounding to bf16.  A cosine or sine is rounded to
    fp32, then two products and a sum: 3 F32 of both terms."""
    h = x.shape[-1] // 2
    dz = rotate(dy, pos.astype(np.float64), theta, back=True)
    lo, hi = np.abs(dy[..., :h]), np.abs(dy[..., h:])
    e = 3 * F32 * (lo + hi)
    (dx, dg), (bx, bg) = rmsnorm_backward(x, gain, dz, eps,
                                          np.concatenate((e, e), -1))
    return (dx, dg), (bx + BF16 * (np.abs(dx) + bx), bg)


def token_loss(logits, target, weight):
    """logits [R, V], target [R], weight [R] -> (loss, dlogits), (their
    bounds).  Rows without loss: target outside the row, or weight 0.

    fp32: an exponent x - m, log2 e and their product are off by 3 F32 of
    its size, v_exp_f32 by a step (2 F32); thread sums and trees by V / 64 +
    16 F32 of the sum of the others at most; logarithms by two steps.  Loss
    and the target's gradient are made from the sum of the others, so that
    their errors are relative to it where the target is the largest."""
    R, V = logits.shape
    loss, d = np.zeros(R), np.zeros((R, V))
    bl, bd = np.zeros(R), np.zeros((R, V))
    for r in range(R):
        t, w = target[r], weight[r]
        if not 0 <= t < V or w == 0:
            continue
        m = logits[r].max()
        if m == -np.inf:
            loss[r] = w * np.inf
            continue
        z = logits[r] - m
        e = np.exp(z)
        a = np.abs(np.where(e > 0, z, 0.0))
        term = 3 * F32 * a + 2 * F32                  # relative, of each e
        rest = e.copy()
        rest[t] = 0.0
        R1, s = rest.sum(), e.sum()
        # absolute errors of the others' sum and of s; v_exp_f32 flushes
        # below 2^-126
        flush = V * 2.0 ** -126
        e_rest = R1 * F32 * (V / 64 + 16) + (rest * term).sum() + flush
        e_s = e_rest + e[t] * term[t] + 2 * F32 * s
        if z[t] == 0:
            loss[r] = w * np.log1p(R1)
            bl[r] = abs(w) * (e_rest + 6 * F32 * np.log1p(R1))
        else:
            loss[r] = w * (np.log(s) - z[t])
            bl[r] = abs(w) * (e_s / s + 6 * F32 * np.log(s) + (
                4 * F32 * abs(z[t]) if z[t] > -np.inf else 0.0))
        p = e / s
        d[r] = w * p
        d[r, t] = -w * R1 / s
        bd[r] = abs(w) * (p * (e_s / s + term + 6 * F32) + 2.0 ** -125)
        bd[r, t] = abs(w) * (R1 / s * (e_s / s + 6 * F32) + e_rest / s +
                             2.0 ** -125)
    return (loss, d), (1.01 * bl, 1.01 * bd)
