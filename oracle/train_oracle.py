"""Plain fp64 CPU oracle of the training-time gradients (numpy, test
infrastructure only): the backward pass of the dual-stream attention of
Sec. 4.2.

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
