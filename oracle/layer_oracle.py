"""The operators around the recurrence by their definitions, in 64 bits on the CPU, token by token: short convolution, selective scan, the
two norms.  Gradients are those of these definitions (torch's differentiation in 64 bits; tests/test_layer_oracle.py checks them
against differences).  Nothing here is shared with the library.

Sequences: a list of (first token, token after the last) over the flattened tokens [M, ...].
"""
from __future__ import annotations

import torch


def sequences(N, T, cu=None):
    if cu is None:
        return [(n * T, (n + 1) * T) for n in range(N)]
    cu = [int(c) for c in cu]
    return list(zip(cu[:-1], cu[1:]))


def conv(x, weight, bias, state, seqs, silu):
    """x [M, D], weight [D, W], bias [D] or None, state [n, W-1, D] or None -> y [M, D], last [n, W-1, D]."""
    M, D = x.shape
    W = weight.shape[1]
    ys, lasts = [], []
    for n, (lo, hi) in enumerate(seqs):
        before = x.new_zeros(W - 1, D) if state is None else state[n]
        line = torch.cat([before, x[lo:hi]])
        for t in range(hi - lo):
            p = (line[t:t + W] * weight.t()).sum(0)
            if bias is not None:
                p = p + bias
            ys.append(p * torch.sigmoid(p) if silu else p)
        lasts.append(line[line.shape[0] - (W - 1):])
    y = torch.stack(ys) if ys else x.new_zeros(0, D)
    return y, torch.stack(lasts) if lasts else x.new_zeros(0, W - 1, D)


def ssm(u, delta, A, B, C, skip, z, delta_bias, softplus, h0, seqs):
    """u, delta, z [M, D], A [D, S], B, C [M, G, S], h0 [n, D, S] or None -> y [M, D], hT [n, D, S]."""
    M, D = u.shape
    G, S = B.shape[-2:]
    group = torch.arange(D) // (D // G)
    if delta_bias is not None:
        delta = delta + delta_bias
    if softplus:
        delta = torch.logaddexp(delta, torch.zeros_like(delta))
    ys, last = [], []
    for n, (lo, hi) in enumerate(seqs):
        h = u.new_zeros(D, S) if h0 is None else h0[n]
        for t in range(lo, hi):
            h = torch.exp(delta[t][:, None] * A) * h + (delta[t] * u[t])[:, None] * B[t][group]
            y = (h * C[t][group]).sum(-1)
            if skip is not None:
                y = y + skip * u[t]
            if z is not None:
                y = y * z[t] * torch.sigmoid(z[t])
            ys.append(y)
        last.append(h)
    return torch.stack(ys) if ys else u.new_zeros(0, D), torch.stack(last) if last else u.new_zeros(0, D, S)


def _normed(v, eps):
    return v / torch.sqrt((v * v).sum(-1, keepdim=True) / v.shape[-1] + eps)


def add_norm(x, weight, residual, scale, eps):
    r = x if scale is None else scale * x
    if residual is not None:
        r = residual + r
    return weight * _normed(r, eps), r


def gated_norm(x, gate, weight, eps, activation, gate_first):
    g = torch.sigmoid(gate)
    if activation == "silu":
        g = g * gate
    return weight * _normed(x * g, eps) if gate_first else weight * _normed(x, eps) * g


def gradients(f, inputs, d_outs):
    """Outputs of f(**inputs) and the gradients of sum <d_out, out> with respect to every tensor among the inputs."""
    leaves = {k: v.detach().double().cpu().requires_grad_(True) for k, v in inputs.items() if v is not None}
    outs = f(**{k: leaves.get(k) for k in inputs})
    outs = outs if isinstance(outs, tuple) else (outs,)
    total = sum((o * d.detach().double().cpu()).sum() for o, d in zip(outs, d_outs) if d is not None)
    grads = torch.autograd.grad(total, list(leaves.values()), allow_unused=True)
    return [o.detach() for o in outs], {k: torch.zeros_like(v) if g is None else g for (k, v), g in zip(leaves.items(), grads)}
