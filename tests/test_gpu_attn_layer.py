"""Attention as the mixing layer of a hybrid block, with the operators that stand around it: norm, projection into queries, keys, values and gate, short
convolution, attention, gated norm of the heads, output projection.  Gradients of everything against 64 bits; served from a paged cache in pieces and
token by token it gives what it computes as a whole."""
import math

import pytest
import torch

from layer_cases import offsets

pytestmark = pytest.mark.gpu
WIDTH, H, HK, D, TAPS, WINDOW, EPS = 128, 4, 2, 64, 4, 40, 1e-6
CONV = (H + 2 * HK) * D


@pytest.fixture(scope="module")
def kla():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2605_08587_amd as m
    m.lib()
    return m


def _parameters(dtype=torch.float32):
    g = torch.Generator().manual_seed(1)
    r = lambda *s, std=1.0: torch.randn(s, generator=g) * std
    p = dict(norm=1 + 0.1 * r(WIDTH), proj=r(WIDTH, CONV + H * D, std=WIDTH ** -0.5), taps=r(CONV, TAPS, std=0.5), bias=0.1 * r(CONV), head_norm=1 + 0.1 * r(D),
             out=r(H * D, WIDTH, std=(H * D) ** -0.5))
    return {k: v.cuda() for k, v in p.items()}


def _split(t):
    return t.split([H * D, HK * D, HK * D], dim=-1)


def _layer(kla, p, x, residual, mix, conv):
    n, residual = kla.kla_add_norm(x, p["norm"], residual, eps=EPS, residual_dtype=torch.float32)
    qkv, gate = (n @ p["proj"].to(n.dtype)).split([CONV, H * D], dim=-1)
    qkv = conv(qkv)
    q, k, v = (t.unflatten(-1, (-1, D)) for t in _split(qkv))        # column ranges of the convolution's output
    o = mix(q, k, v)
    y = kla.kla_gated_norm(o, gate.unflatten(-1, (H, D)), p["head_norm"], eps=EPS)
    return y.flatten(-2) @ p["out"].to(y.dtype), residual


def _reference(p, x, residual):
    """One sequence [T, WIDTH] in doubles, elementary operations only."""
    r = residual + x
    n = p["norm"] * r / torch.sqrt((r * r).mean(-1, keepdim=True) + EPS)
    a = n @ p["proj"]
    qkv, gate = a[:, :CONV], a[:, CONV:].view(-1, H, D)
    padded = torch.cat([qkv.new_zeros(TAPS - 1, CONV), qkv])
    c = sum(padded[j:j + len(x)] * p["taps"][:, j] for j in range(TAPS)) + p["bias"]
    c = c / (1 + torch.exp(-c))
    q, k, v = (t.reshape(len(x), t.shape[-1] // D, D) for t in _split(c))
    i = torch.arange(len(x))
    seen = (i[:, None] >= i) & (i[:, None] - i < WINDOW)
    o = []
    for h in range(H):
        s = torch.where(seen, q[:, h] @ k[:, h // 2].t() / math.sqrt(D), -math.inf)
        o.append(torch.softmax(s, -1) @ v[:, h // 2])
    o = torch.stack(o, 1)
    u = o / torch.sqrt((o * o).mean(-1, keepdim=True) + EPS) * p["head_norm"] * gate / (1 + torch.exp(-gate))
    return u.flatten(1) @ p["out"], r


def test_gradients_through_a_packed_layer(kla):
    lengths, cu = [70, 1, 0, 129], offsets([70, 1, 0, 129])
    kw = dict(cu_seqlens=cu.cuda(), cu_seqlens_host=cu)
    p = {k: v.requires_grad_() for k, v in _parameters().items()}
    g = torch.Generator().manual_seed(2)
    x, res, dy, dr = (torch.randn(1, 200, WIDTH, generator=g) for _ in range(4))
    xs, rs = x.cuda().requires_grad_(), res.cuda().requires_grad_()
    y, r = _layer(kla, p, xs, rs, lambda q, k, v: kla.kla_attn(q, k, v, window=WINDOW, **kw), lambda t: kla.kla_conv(t, p["taps"], p["bias"], **kw)[0])
    got = torch.autograd.grad((y, r), [xs, rs, *p.values()], (dy.cuda(), dr.cuda()))
    p64 = {k: v.detach().cpu().double().requires_grad_() for k, v in p.items()}
    x64, r64 = x[0].double().requires_grad_(), res[0].double().requires_grad_()
    outs, at = [], 0
    for n in lengths:
        outs.append(_reference(p64, x64[at:at + n], r64[at:at + n]))
        at += n
    y64, s64 = torch.cat([o[0] for o in outs]), torch.cat([o[1] for o in outs])
    want = torch.autograd.grad((y64, s64), [x64, r64, *p64.values()], (dy[0].double(), dr[0].double()))
    # fp32 all the way: a dozen operators, sums of up to 512 terms of 2^-24 each, and the products before and behind in torch's fp32
    for name, a, b in zip(["y", "x", "res", *p], (y, *got), (y64, *want)):
        e = float((a.detach().double().cpu().view_as(b) - b).abs().max() / b.abs().max())
        assert e <= 1e-4, (name, e)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@torch.no_grad()
def test_served_as_a_whole_in_pieces_and_by_tokens(kla, dtype):
    p = _parameters()
    N, T, page = 3, 150, 16
    x = torch.randn(N, T, WIDTH, generator=torch.Generator().manual_seed(3)).cuda().to(dtype)
    whole, _ = _layer(kla, p, x, None, lambda q, k, v: kla.kla_attn(q, k, v, window=WINDOW), lambda t: kla.kla_conv(t, p["taps"], p["bias"])[0])
    kc, vc = (torch.full((N * -(-T // page), HK, page, D), float("nan"), device="cuda", dtype=dtype) for _ in range(2))
    table = torch.arange(len(kc), dtype=torch.int32, device="cuda").view(N, -1).flip(0).contiguous()
    cached, state, out, at = torch.zeros(N, dtype=torch.int32, device="cuda"), torch.zeros(N, TAPS - 1, CONV, device="cuda", dtype=dtype), [], 0
    for n in (64, 37):
        def conv(t):
            y, last = kla.kla_conv(t, p["taps"], p["bias"], state, want_state=True)
            state.copy_(last)
            return y
        out.append(_layer(kla, p, x[:, at:at + n].contiguous(), None,
                          lambda q, k, v: kla.kla_attn_extend(q, k, v, kc, vc, table, cached, window=WINDOW), conv)[0])
        cached += n
        at += n
    for t in range(at, T):
        out.append(_layer(kla, p, x[:, t].contiguous(), None, lambda q, k, v: kla.kla_attn_step(q, k, v, kc, vc, table, cached, window=WINDOW),
                          lambda u: kla.kla_conv_step(u, p["taps"], state, p["bias"]))[0][:, None])
        cached += 1
    off = ((torch.cat(out, 1) - whole).float().norm() / whole.float().norm()).item()
    # bf16: the products of torch and of attention round differently for other shapes, about ten roundings of 2^-9 in a row
    assert off <= (2e-2 if dtype == torch.bfloat16 else 1e-5)
