"""Softmax attention in 64 bits, query row by query row (numpy): over one sequence's keys, of which a row sees a contiguous range, so that
what it does not see takes no part, whatever stands there.  Gradients from the formulas, and what fp32 kernels that round to a narrower type may be off by.

q [n, H, D] are the queries at positions first .. first + n - 1, k, v [m, Hk, D] all keys of the sequence.
"""
from __future__ import annotations

import numpy as np


def visible(i, m, causal, window):
    """First key and the one behind the last that position i sees."""
    hi = min(i + 1, m) if causal else m
    return (max(0, i - window + 1) if window else 0), hi


def forward(q, k, v, scale, first=0, causal=True, window=0):
    """o [n, H, D] and lse [n, H]; a row that sees no key is zeros, with an lse of -inf."""
    n, H, D = q.shape
    m, Hk, _ = k.shape
    o, lse = np.zeros((n, H, D)), np.full((n, H), -np.inf)
    q4 = q.reshape(n, Hk, H // Hk, D)
    for i in range(n):
        lo, hi = visible(first + i, m, causal, window)
        if hi <= lo:
            continue
        s = scale * np.einsum("hgd,jhd->hgj", q4[i], k[lo:hi])
        top = s.max(-1, keepdims=True)
        p = np.exp(s - top)
        total = p.sum(-1, keepdims=True)
        o[i] = np.einsum("hgj,jhd->hgd", p / total, v[lo:hi]).reshape(H, D)
        lse[i] = (top + np.log(total)).reshape(H)
    return o, lse


def backward(q, k, v, d_o, scale, first=0, causal=True, window=0):
    """dq, dk, dv of sum <d_o, o>."""
    n, H, D = q.shape
    m, Hk, _ = k.shape
    q4, g4 = q.reshape(n, Hk, H // Hk, D), d_o.reshape(n, Hk, H // Hk, D)
    dq, dk, dv = np.zeros_like(q4), np.zeros_like(k), np.zeros_like(v)
    for i in range(n):
        lo, hi = visible(first + i, m, causal, window)
        if hi <= lo:
            continue
        s = scale * np.einsum("hgd,jhd->hgj", q4[i], k[lo:hi])
        p = np.exp(s - s.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        dp = np.einsum("hgd,jhd->hgj", g4[i], v[lo:hi])
        ds = p * (dp - (p * dp).sum(-1, keepdims=True))
        dq[i] = scale * np.einsum("hgj,jhd->hgd", ds, k[lo:hi])
        dk[lo:hi] += scale * np.einsum("hgj,hgd->jhd", ds, q4[i])
        dv[lo:hi] += np.einsum("hgj,hgd->jhd", p, g4[i])
    return dq.reshape(n, H, D), dk, dv


def bounds(q, k, v, scale, u, d_o=None, first=0, causal=True, window=0, rest=False):
    """How far each element may be from the two functions above: o, lse and, with d_o, dq, dk, dv.  u: half a step of the type that outputs, weights and
    their gradients are rounded to.  With e = 2^-24, to first order:
      a score is a sum of D products (D e of the sum of their sizes) times a rounded constant, less a rounded reference: rho of its weight,
          rho = max_j (D e scale |q|.|k_j| + 4 e |s_j|) + 8 e           (the last for the exponential and the reference's product);
      a row's sums over n keys add n e of their terms' sizes, a row's scaling with a new reference 2 e for each of its n / 32 tiles: within 2 n e;
      weights are rounded by u where they meet v, and the quotient by the sum of weights brings rho and 2 n e once more:
          do = u |o| + (u + 2 rho + 4 n e) sum p |v|;     dlse = rho + 2 n e + 4 e (|lse| + 1);
      delta = <d_o, o> takes o with its error; a weight formed again from lse is off by rho + dlse; ds = p (dp - delta) is rounded by u:
          dds = |ds| (u + rho + dlse) + p (D e |d_o|.|v| + <|d_o|, do> + D e |d_o|.|o|);
      rest: o comes with what its rounding left out, rounded in turn: u^2 |o| in the place of u |o| there."""
    n, H, D = q.shape
    m, Hk, _ = k.shape
    G, e = H // Hk, 2.0 ** -24
    q4 = q.reshape(n, Hk, G, D)
    b_o, b_lse = np.zeros((n, Hk, G, D)), np.zeros((n, Hk, G))
    grads = None
    if d_o is not None:
        g4 = d_o.reshape(n, Hk, G, D)
        rows = np.zeros(m)
        b_q, b_k, b_v, s_k, s_v, dk, dv = np.zeros_like(q4), *(np.zeros_like(k) for _ in range(6))
    for i in range(n):
        lo, hi = visible(first + i, m, causal, window)
        if hi <= lo:
            continue
        kk, vv, N = k[lo:hi], v[lo:hi], hi - lo
        s = scale * np.einsum("hgd,jhd->hgj", q4[i], kk)
        p = np.exp(s - s.max(-1, keepdims=True))
        lse = s.max(-1) + np.log(p.sum(-1))
        p /= p.sum(-1, keepdims=True)
        rho = (D * e * scale * np.einsum("hgd,jhd->hgj", abs(q4[i]), abs(kk)) + 4 * e * abs(s)).max(-1) + 8 * e
        o = np.einsum("hgj,jhd->hgd", p, vv)
        b_o[i] = u * abs(o) + (u + 2 * rho + 4 * N * e)[..., None] * np.einsum("hgj,jhd->hgd", p, abs(vv))
        b_lse[i] = rho + 2 * N * e + 4 * e * (abs(lse) + 1)
        if d_o is None:
            continue
        g = g4[i]
        dp = np.einsum("hgd,jhd->hgj", g, vv)
        ds = p * (dp - (p * dp).sum(-1, keepdims=True))
        r = (rho + b_lse[i])[..., None]
        b_delta = (abs(g) * (b_o[i] - (u - u * u) * abs(o) * rest)).sum(-1) + D * e * (abs(g) * abs(o)).sum(-1)
        b_ds = abs(ds) * (u + r) + p * (D * e * np.einsum("hgd,jhd->hgj", abs(g), abs(vv)) + b_delta[..., None])
        dq = scale * np.einsum("hgj,jhd->hgd", ds, kk)
        b_q[i] = (u + e) * abs(dq) + scale * np.einsum("hgj,jhd->hgd", b_ds + 2 * N * e * abs(ds), abs(kk))
        rows[lo:hi] += G
        b_k[lo:hi] += scale * np.einsum("hgj,hgd->jhd", b_ds, abs(q4[i]))
        s_k[lo:hi] += scale * np.einsum("hgj,hgd->jhd", abs(ds), abs(q4[i]))
        b_v[lo:hi] += np.einsum("hgj,hgd->jhd", p * (u + r), abs(g))
        s_v[lo:hi] += np.einsum("hgj,hgd->jhd", p, abs(g))
        dk[lo:hi] += scale * np.einsum("hgj,hgd->jhd", ds, q4[i])
        dv[lo:hi] += np.einsum("hgj,hgd->jhd", p, g)
    if d_o is not None:
        c = 2 * e * rows[:, None, None]
        grads = b_q.reshape(n, H, D), b_k + c * s_k + (u + e) * abs(dk), b_v + c * s_v + (u + e) * abs(dv)
    return (b_o.reshape(n, H, D), b_lse.reshape(n, H)) + (grads or ())
