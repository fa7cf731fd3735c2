"""Two layers of a hybrid model out of this package's operators, trained for some steps and then served token by token.

    python examples/hybrid_layers.py

Each layer is: residual stream + scaled output of the layer before and its norm (kla_add_norm), projections, short convolution
(kla_conv), a recurrence - the Kaczmarz delta rule (kla_chunk) in the first layer, the selective scan (kla_ssm) in the second -,
norm of its heads times the gate (kla_gated_norm), output projection.  Serving keeps, per layer, the inputs of the last tokens for the
convolution and the state of the recurrence (kla_conv_step, kla_decode_step, kla_ssm_step).
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2605_08587_amd as kla  # noqa: E402

WIDTH, HEADS, DK, DV, TAPS, STATES = 256, 4, 64, 64, 4, 16
INNER, EPS = HEADS * DV, 1e-6


def parameters(seed=0, device="cuda"):
    g = torch.Generator(device=device).manual_seed(seed)

    def r(*shape, std):
        return torch.randn(shape, generator=g, device=device) * std
    p = {}
    for layer in ("delta", "scan"):
        columns = (2 * HEADS * DK + INNER if layer == "delta" else INNER) + INNER + (2 * HEADS if layer == "delta" else INNER + 2 * STATES)
        conv = 2 * HEADS * DK + INNER if layer == "delta" else INNER
        p[layer] = dict(norm=torch.ones(WIDTH, device=device), scale=torch.ones(WIDTH, device=device), proj=r(WIDTH, columns, std=WIDTH ** -0.5),
                        taps=r(conv, TAPS, std=TAPS ** -0.5), bias=torch.zeros(conv, device=device),
                        head_norm=torch.ones(DV, device=device), out=r(INNER, WIDTH, std=INNER ** -0.5))
    p["scan"]["A"] = -torch.arange(1.0, STATES + 1, device=device).repeat(INNER, 1)
    p["scan"]["skip"] = torch.ones(INNER, device=device)
    step = torch.exp(torch.rand(INNER, generator=g, device=device) * math.log(100.0) + math.log(1e-3))
    p["scan"]["step_bias"] = torch.log(torch.expm1(step))
    p["final_norm"] = torch.ones(WIDTH, device=device)
    for t in leaves(p):
        t.requires_grad_(True)
    return p


def leaves(p):
    for v in p.values():
        if isinstance(v, dict):
            yield from leaves(v)
        else:
            yield v


def _gates(a, b):
    """Log decay and write gate of the delta rule, fp32, from their two projections."""
    return -torch.nn.functional.softplus(a.float()) * 0.1, torch.sigmoid(b.float())


def delta_layer(p, x, residual, cache=None, cu=None, cu_host=None):
    """x: output of the layer before [N, T, WIDTH]; one token [N, WIDTH] with a cache.  Returns (output, residual stream)."""
    one = x.dim() == 2
    n, residual = kla.kla_add_norm(x, p["norm"], residual, scale=p["scale"], eps=EPS, residual_dtype=torch.float32)
    qkv, gate, a, b = (n @ p["proj"].to(n.dtype)).split([2 * HEADS * DK + INNER, INNER, HEADS, HEADS], dim=-1)
    if one:
        qkv = kla.kla_conv_step(qkv, p["taps"], cache["conv"], p["bias"])
    else:
        qkv, last = kla.kla_conv(qkv, p["taps"], p["bias"], cu_seqlens=cu, cu_seqlens_host=cu_host, want_state=cache is not None)
    q, k, v = (t.unflatten(-1, (HEADS, -1)).contiguous() for t in qkv.split([HEADS * DK, HEADS * DK, INNER], dim=-1))
    log_alpha, eta = _gates(a, b)
    if one:
        o = kla.kla_decode_step(q, k, v, log_alpha, eta, EPS, cache["state"], normalize_q=True)
    else:
        o, state = kla.kla_chunk(q, k, v, log_alpha, eta, EPS, cu_seqlens=cu, cu_seqlens_host=cu_host, normalize_q=True)
        if cache is not None:
            cache.update(conv=last, state=state)
    y = kla.kla_gated_norm(o, gate.unflatten(-1, (HEADS, DV)), p["head_norm"], eps=EPS)
    return y.flatten(-2) @ p["out"].to(y.dtype), residual


def scan_layer(p, x, residual, cache=None, cu=None, cu_host=None):
    one = x.dim() == 2
    n, residual = kla.kla_add_norm(x, p["norm"], residual, scale=p["scale"], eps=EPS)
    u, gate, step, B, C = (n @ p["proj"].to(n.dtype)).split([INNER, INNER, INNER, STATES, STATES], dim=-1)
    B, C = B.unsqueeze(-2), C.unsqueeze(-2)                      # one group
    kw = dict(skip=p["skip"], delta_bias=p["step_bias"])
    if one:
        u = kla.kla_conv_step(u, p["taps"], cache["conv"], p["bias"])
        y = kla.kla_ssm_step(u, step, p["A"], B, C, cache["state"], **kw)
    else:
        u, last = kla.kla_conv(u, p["taps"], p["bias"], cu_seqlens=cu, cu_seqlens_host=cu_host, want_state=cache is not None)
        y, state = kla.kla_ssm(u, step, p["A"], B, C, cu_seqlens=cu, cu_seqlens_host=cu_host, **kw)
        if cache is not None:
            cache.update(conv=last, state=state)
    y = kla.kla_gated_norm(y.unflatten(-1, (HEADS, DV)), gate.unflatten(-1, (HEADS, DV)), p["head_norm"], eps=EPS, gate_first=True)
    return y.flatten(-2) @ p["out"].to(y.dtype), residual


def model(p, x, caches=None, cu=None, cu_host=None):
    c = caches or {"delta": None, "scan": None}
    y, r = delta_layer(p["delta"], x, None, c["delta"], cu, cu_host)
    y, r = scan_layer(p["scan"], y, r, c["scan"], cu, cu_host)
    return kla.kla_add_norm(y, p["final_norm"], r, eps=EPS)[0]


def train(p, steps=150, N=4, T=256, seed=1):
    """Predict each token's input of four tokens ago: what the layers have to remember.  Returns the losses."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    opt = torch.optim.Adam(list(leaves(p)), lr=3e-3)
    losses = []
    for _ in range(steps):
        x = torch.randn(N, T, WIDTH, generator=g, device="cuda").bfloat16()
        loss = (model(p, x)[:, 4:].float() - x[:, :-4].float()).square().mean()
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(loss.item())
    return losses


@torch.no_grad()
def serve(p, prompt, tokens):
    """prompt [N, T, WIDTH], then the tokens [N, M, WIDTH] one at a time; returns the outputs of all of them."""
    caches = {"delta": {}, "scan": {}}
    out = [model(p, prompt, caches)]
    for t in range(tokens.shape[1]):
        out.append(model(p, tokens[:, t].contiguous(), caches)[:, None])
    return torch.cat(out, 1)


def main():
    p = parameters()
    losses = train(p)
    print("loss over %d steps: %.3f -> %.3f" % (len(losses), losses[0], losses[-1]), flush=True)
    x = torch.randn(3, 200, WIDTH, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").bfloat16()
    with torch.no_grad():
        whole = model(p, x)
        lens = [50, 150, 1]
        cu_host = torch.tensor([0, 50, 200, 201], dtype=torch.int32)
        packed = model(p, torch.cat([x[i, :n] for i, n in enumerate(lens)])[None], cu=cu_host.cuda(), cu_host=cu_host)[0]
    served = serve(p, x[:, :180].contiguous(), x[:, 180:])
    off = ((served - whole).float().norm() / whole.float().norm()).item()
    apart = max(((packed[a:b] - whole[i, :b - a]).float().norm() / whole[i, :b - a].float().norm()).item()
                for i, (a, b) in enumerate(zip(cu_host[:-1].tolist(), cu_host[1:].tolist())))
    print("prompt and single tokens against the whole at once: %.2e; packed against apart: %.2e" % (off, apart), flush=True)
    return losses, off, apart


if __name__ == "__main__":
    main()
