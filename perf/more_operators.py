"""Softmax attention beside the recurrence in hybrid stacks, through the package's public entry points or in plain form.

  attn    attention over whole sequences, grouped heads, fixed-length and packed batches: "attn_fwd" forward alone (prefill, evaluation),
          "attn_train" forward and the gradients of queries, keys and values
  extend  a chunk of new tokens for each of several sequences over a paged cache, their keys and values stored in it
  step    the same for one token of each sequence

Heads of 64 or 128, 8 or 16 of them, as in the tests and benchmark, sharing 2 to 16 key heads; the training context of 4K tokens, prompts
up to 16K, caches up to 32K.
"""
from __future__ import annotations

import math
import random

import torch

own = False
MOST = 2 ** 27                                            # scores that the plain forms hold at once


def _case(name, kind, dtype="bf16", N=1, T=1, H=16, Hk=4, D=128, n_seq=0, lo=0, hi=0, causal=True, window=0, wide=False, page=64,
          cached_lo=0, cached_hi=0):
    """N sequences of T tokens, or n_seq > 0 packed ones of lo..hi tokens (new ones: extend, step).  H query heads of D share Hk key
    heads; window: how many keys a query sees at most (0: all); wide: q, k, v are column ranges of one projection's output; the cache
    holds cached_lo..cached_hi tokens of a sequence in pages of `page`."""
    c = dict(kind=kind, dtype=dtype, N=N, T=T, H=H, Hk=Hk, D=D, n_seq=n_seq, lo=lo, hi=hi, causal=causal, window=window, wide=wide,
             page=page, cached_lo=cached_lo, cached_hi=cached_hi)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one prompt of no round length: mostly latency
        _case("attn_prompt_t200", "attn_fwd", T=200, H=8, Hk=8),
        # a packed batch of unequal prompts, q, k and v cut out of one projection
        _case("attn_packed", "attn_fwd", n_seq=16, lo=512, hi=4096, wide=True),
        # one long prompt
        _case("attn_prefill_t16384", "attn_fwd", T=16384),
        # an encoder's batch: every token sees all of its sequence
        _case("attn_both_ways", "attn_fwd", N=4, T=1500, H=8, Hk=8, D=64, causal=False),
        # training at the benchmark's shape, 8 sequences of 4K tokens, a key head for every query head
        _case("attn_train_4k", "attn_train", N=8, T=4096, H=8, Hk=8),
        # packed training with a sliding window, four query heads to a key head
        _case("attn_train_window", "attn_train", n_seq=6, lo=1000, hi=5000, D=64, window=1024, wide=True),
        # single precision, odd lengths: reference runs
        _case("attn_train_fp32", "attn_train", dtype="fp32", N=2, T=777, H=8, Hk=2, D=64),
        # the next pieces of four long prompts that are taken in by chunks
        _case("extend_chunk", "extend", n_seq=4, lo=100, hi=600, cached_lo=1000, cached_hi=16000),
        # five drafted tokens to be verified for each of 16 users, small pages
        _case("extend_draft", "extend", N=16, T=5, page=16, cached_lo=2000, cached_hi=8000),
        # single precision, short caches, some of them empty
        _case("extend_fp32", "extend", dtype="fp32", n_seq=3, lo=1, hi=200, H=8, Hk=2, D=64, page=32, cached_lo=0, cached_hi=1500),
        # one user's next token in a context of 4K
        _case("step_b1", "step", N=1, cached_lo=4095, cached_hi=4095),
        # a serving batch of 32 users with long contexts: bound by the cache
        _case("step_b32", "step", N=32, cached_lo=4000, cached_hi=32000),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the same kinds.  Sizes over their logarithm, lengths odd; smaller until it costs no more than the largest listed."""
    kind = rng.choice(["attn_fwd", "attn_fwd", "attn_train", "attn_train", "extend", "extend", "step", "step"])
    dtype = "fp32" if rng.random() < 0.2 else "bf16"
    H, Hk = rng.choice([(8, 8), (8, 2), (16, 4), (16, 4), (16, 16), (16, 2), (12, 4), (6, 2)])
    kw = dict(dtype=dtype, H=H, Hk=Hk, D=rng.choice([64, 128, 128]), window=rng.choice([0, 0, 0, _log_int(rng, 16, 4000)]))
    if kind in ("extend", "step"):
        kw["page"] = rng.choice([16, 32, 64, 64, 128, 256])
        hi = _log_int(rng, 16, 32000)
        kw.update(cached_hi=hi, cached_lo=rng.choice([0, hi // 8, hi // 2, hi]))
        if kind == "step":
            c = _case(None, kind, N=_log_int(rng, 1, 128), **kw)
        elif rng.random() < 0.5:
            c = _case(None, kind, N=_log_int(rng, 1, 32), T=_log_int(rng, 1, 64), **kw)
        else:
            most = _log_int(rng, 8, 2000)
            c = _case(None, kind, n_seq=rng.randint(2, 12), lo=max(1, most // 8), hi=most, **kw)
    else:
        kw.update(causal=rng.random() < 0.8 or kw["window"] > 0, wide=rng.random() < 0.4)
        if rng.random() < 0.4:
            most = _log_int(rng, 32, 8000)
            c = _case(None, kind, n_seq=rng.randint(2, 24), lo=max(1, most // rng.choice([2, 8, 64])), hi=most, **kw)
        else:
            c = _case(None, kind, N=rng.choice([1, 1, 2, 3, 8]), T=_log_int(rng, 16, 16000) | 1, **kw)
    while _costs_too_much(c):
        for k in ("N", "n_seq", "T", "hi", "lo", "cached_hi", "cached_lo"):
            floor = 2 if k == "n_seq" and c[k] else (1 if c[k] and not k.startswith("cached") else 0)
            c[k] = max(floor, int(c[k] * 0.8)) if c[k] else c[k]
    return c


def _costs_too_much(c):
    """The flops and bytes of the largest listed cases; fp32 a tenth of the flops."""
    w = work(c)
    return w["flops"] > (1e11 if c["dtype"] == "fp32" else 1e12) or w["bytes"] > 1.2e9


def _lengths(c):
    """New tokens of every sequence.  They and the cached ones follow from the case, so that its work does."""
    if not c["n_seq"]:
        return [c["T"]] * c["N"]
    r = random.Random(c["n_seq"] * 1_000_003 + c["lo"] * 1_009 + c["hi"])
    return [r.randint(c["lo"], c["hi"]) for _ in range(c["n_seq"])]


def _cached(c):
    r = random.Random(c["cached_lo"] * 1_009 + c["cached_hi"])
    return [r.randint(c["cached_lo"], c["cached_hi"]) if c["kind"] in ("extend", "step") else 0 for _ in _lengths(c)]


def prepare(case, seed):
    c = case
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(int(seed))
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    H, Hk, D = c["H"], c["Hk"], c["D"]

    def randn(*shape):
        return torch.randn(shape, generator=gen, device=dev, dtype=torch.float32)

    s = dict(case=c, cu=None, cu_host=None, lengths=_lengths(c))
    if c["n_seq"]:
        offs = [0]
        for n in s["lengths"]:
            offs.append(offs[-1] + n)
        s["cu_host"] = torch.tensor(offs, dtype=torch.int32)      # a data loader has the offsets on the host
        s["cu"] = s["cu_host"].to(dev)
        lead = (1, offs[-1])
    else:
        lead = (c["N"],) if c["kind"] == "step" else (c["N"], c["T"])
    # some heads look at many keys, others at few
    sharp = torch.linspace(1, 4, H, device=dev)[:, None]
    if c["wide"]:
        p = randn(*lead, (2 * H + 2 * Hk) * D)                    # the last H D columns: a gate that nobody takes here
        p[..., :H * D].view(*lead, H, D).mul_(sharp)
        q, k, v, _ = p.to(dt).split([H * D, Hk * D, Hk * D, H * D], dim=-1)
    else:
        q, k, v = (randn(*lead, H, D) * sharp).to(dt), randn(*lead, Hk, D).to(dt), randn(*lead, Hk, D).to(dt)
    s.update(q=q.view(*lead, H, D), k=k.view(*lead, Hk, D), v=v.view(*lead, Hk, D))
    if c["kind"] == "attn_train":
        s["q"], s["k"], s["v"] = (s[x].detach().requires_grad_() for x in "qkv")
        s["d_o"] = randn(*lead, H, D).to(dt)
    if c["kind"] in ("extend", "step"):
        page, cached = c["page"], _cached(c)
        pages = [-(-(n + m) // page) for n, m in zip(s["lengths"], cached)]
        total = sum(pages) + 1
        s["k_cache"], s["v_cache"] = randn(total, Hk, page, D).to(dt), randn(total, Hk, page, D).to(dt)
        order = torch.randperm(total, generator=gen, device=dev).to(torch.int32)
        table = torch.zeros(len(pages), max(pages), dtype=torch.int32, device=dev)
        at = 0
        for i, n in enumerate(pages):
            table[i, :n] = order[at:at + n]
            at += n
        s["table"], s["cached"], s["cached_host"] = table, torch.tensor(cached, dtype=torch.int32, device=dev), cached
    return s


def _own(s):
    import paper_2605_08587_amd as kla
    c = s["case"]
    if c["kind"] == "step":
        o = kla.kla_attn_step(s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"], s["cached"], window=c["window"])
        return o, s["k_cache"], s["v_cache"]
    if c["kind"] == "extend":
        o = kla.kla_attn_extend(s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"], s["cached"], window=c["window"],
                                cu_seqlens=s["cu"], cu_seqlens_host=s["cu_host"])
        return o, s["k_cache"], s["v_cache"]
    kw = dict(causal=c["causal"], window=c["window"], cu_seqlens=s["cu"], cu_seqlens_host=s["cu_host"])
    if c["kind"] == "attn_fwd":
        return kla.kla_attn_fwd(s["q"], s["k"], s["v"], **kw)
    o = kla.kla_attn(s["q"], s["k"], s["v"], **kw)
    return (o, *torch.autograd.grad(o, (s["q"], s["k"], s["v"]), s["d_o"]))


# ---- plain form: products, exponentials and sums over whole score matrices, in 32 bits ------------------------------------------------


def _hidden(c, first, n, device, m):
    """True where key 0..m-1 is not for the query at position first..first+n-1."""
    i = torch.arange(first, first + n, device=device)[:, None]
    j = torch.arange(m, device=device)[None, :]
    no = torch.zeros(n, m, dtype=torch.bool, device=device)
    if c["causal"]:
        no = j > i
    if c["window"]:
        no = no | (j <= i - c["window"])
    return no


def _plain_one(c, q, k, v, first, d_o=None):
    """q [n, H, D] at positions first.., k, v [m, Hk, D]: o [n, H, D], lse [n, H], and, with d_o, dq, dk, dv; all fp32."""
    n, H, D = q.shape
    m, Hk, _ = k.shape
    G = H // Hk
    scale = 1 / math.sqrt(D)
    kt = k.float().permute(1, 2, 0).contiguous()                                   # [Hk, D, m]
    kh, vh = (t.float().transpose(0, 1).contiguous() for t in (k, v))              # [Hk, m, D]
    vt = vh.transpose(1, 2).contiguous()

    def rows(t, a, b):                                                             # [b - a, H, D] as [Hk, (b - a) G, D]
        return t[a:b].float().view(b - a, Hk, G, D).transpose(0, 1).reshape(Hk, (b - a) * G, D)

    def back(t, a, b):
        return t.view(Hk, b - a, G, -1).transpose(0, 1).reshape(b - a, H, -1)
    o, lse = q.new_empty((n, H, D), dtype=torch.float32), q.new_empty((n, H), dtype=torch.float32)
    if d_o is not None:
        dq, dk, dv = torch.empty_like(o), torch.zeros_like(kh), torch.zeros_like(vh)
    step = max(1, MOST // max(1, H * m))
    for a in range(0, n, step):
        b = min(n, a + step)
        qr = rows(q, a, b)
        p = torch.matmul(qr, kt).mul_(scale)
        hidden = _hidden(c, first + a, b - a, q.device, m)
        p.view(Hk, b - a, G, m).masked_fill_(hidden[None, :, None, :], -math.inf)
        top = p.amax(-1, keepdim=True)
        p = p.sub_(top).exp_()
        total = p.sum(-1, keepdim=True)
        p = p.div_(total)
        out = torch.matmul(p, vh)
        o[a:b], lse[a:b] = back(out, a, b), back(top + torch.log(total), a, b)[..., 0]
        if d_o is not None:
            g = rows(d_o, a, b)
            dv += torch.matmul(p.transpose(1, 2).contiguous(), g)
            ds = torch.matmul(g, vt)
            ds = ds.sub_((g * out).sum(-1, keepdim=True)).mul_(p).mul_(scale)
            dq[a:b] = back(torch.matmul(ds, kh), a, b)
            dk += torch.matmul(ds.transpose(1, 2).contiguous(), qr)
    if d_o is None:
        return o, lse
    return o, lse, dq, dk.transpose(0, 1), dv.transpose(0, 1)


def _paged(s, store):
    """Every sequence's keys and values, cached and new ones; store: the new ones are written into their pages first."""
    c = s["case"]
    page, Hk, D = c["page"], c["Hk"], c["D"]
    k, v = s["k"].reshape(-1, Hk, D), s["v"].reshape(-1, Hk, D)
    at, got = 0, []
    for i, (n, m) in enumerate(zip(s["lengths"], s["cached_host"])):
        if store:
            where = torch.arange(m, m + n, device=k.device)
            pages, slots = s["table"][i, where // page].long(), where % page
            s["k_cache"][pages, :, slots] = k[at:at + n]
            s["v_cache"][pages, :, slots] = v[at:at + n]
        pages = s["table"][i, :-(-(n + m) // page)].long()
        got.append(tuple(t[pages].transpose(1, 2).reshape(-1, Hk, D)[:n + m] for t in (s["k_cache"], s["v_cache"])))
        at += n
    return got


def run(s):
    if own:
        return _own(s)
    c = s["case"]
    H, Hk, D = c["H"], c["Hk"], c["D"]
    q, k, v = (s[x].detach().reshape(-1, h, D) for x, h in (("q", H), ("k", Hk), ("v", Hk)))
    dt, shape = q.dtype, s["q"].shape
    outs, at = [], 0
    if c["kind"] in ("extend", "step"):
        for (kk, vv), n, m in zip(_paged(s, True), s["lengths"], s["cached_host"]):
            outs.append(_plain_one(c, q[at:at + n], kk, vv, m)[0].to(dt))
            at += n
        return torch.cat(outs).view(shape), s["k_cache"], s["v_cache"]
    d_o = s["d_o"].reshape(-1, H, D) if "d_o" in s else None
    for n in s["lengths"]:
        here = slice(at, at + n)
        outs.append(_plain_one(c, q[here], k[here], v[here], 0, None if d_o is None else d_o[here]))
        at += n
    whole = [torch.cat(ts) for ts in zip(*outs)]
    if d_o is None:
        return whole[0].to(dt).view(shape), whole[1].view(shape[:-1])
    return (whole[0].to(dt).view(shape), *(t.to(dt).view(s[x].shape) for t, x in zip(whole[2:], "qkv")))


# ---- the definitions in 64 bits, query head by query head -----------------------------------------------------------------------------


def _exact_head(c, q, k, v, first, g):
    """One query head [n, D] over one key head [m, D] in doubles: o, lse and, with the gradient g of o, dq, dk, dv."""
    n, m = len(q), len(k)
    o, lse = torch.empty_like(q), q.new_empty(n)
    dq, dk, dv = torch.empty_like(q), torch.zeros_like(k), torch.zeros_like(v)
    step = max(1, 2 ** 26 // max(1, m))
    for a in range(0, n, step):
        b = min(n, a + step)
        pos = torch.arange(first + a, first + b, device=q.device).unsqueeze(1)
        key = torch.arange(m, device=q.device).unsqueeze(0)
        seen = key <= pos if c["causal"] else torch.ones_like(key <= pos)
        if c["window"]:
            seen &= pos - key < c["window"]
        score = torch.where(seen, q[a:b] @ k.t() / D_ROOT[q.shape[1]], -math.inf)
        lse[a:b] = torch.logsumexp(score, 1)
        weight = torch.exp(score - lse[a:b, None])
        o[a:b] = weight @ v
        if g is not None:
            along = g[a:b] @ v.t()
            ds = weight * (along - (weight * along).sum(1, keepdim=True)) / D_ROOT[q.shape[1]]
            dq[a:b] = ds @ k
            dk += ds.t() @ q[a:b]
            dv += weight.t() @ g[a:b]
    return o, lse, dq, dk, dv


D_ROOT = {64: 8.0, 128: math.sqrt(128.0)}


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    H, Hk, D = c["H"], c["Hk"], c["D"]
    q, k, v = (s[x].detach().reshape(-1, h, D) for x, h in (("q", H), ("k", Hk), ("v", Hk)))
    paged = c["kind"] in ("extend", "step")
    train = c["kind"] == "attn_train"
    keys = _paged(s, True) if paged else None
    o = torch.empty(q.shape, dtype=torch.float64, device=q.device)
    lse = o.new_empty(o.shape[:2])
    dq, dk, dv = (torch.zeros(t.shape, dtype=torch.float64, device=q.device) for t in (q, k, v)) if train else (None,) * 3
    at = 0
    for i, n in enumerate(s["lengths"]):
        here = slice(at, at + n)
        for h in range(H):
            j = h // (H // Hk)
            kk, vv = (keys[i][0][:, j], keys[i][1][:, j]) if paged else (k[here, j], v[here, j])
            g = s["d_o"].reshape(-1, H, D)[here, h].double() if train else None
            r = _exact_head(c, q[here, h].double(), kk.double(), vv.double(), s["cached_host"][i] if paged else 0, g)
            o[here, h], lse[here, h] = r[:2]
            if train:
                dq[here, h] = r[2]
                dk[here, j] += r[3]
                dv[here, j] += r[4]
        at += n
    shape = s["q"].shape
    if paged:
        return o.view(shape), s["k_cache"], s["v_cache"]              # (what is stored is not computed)
    if not train:
        return o.view(shape), lse.view(shape[:-1])
    return o.view(shape), dq.view(shape), dk.view(s["k"].shape), dv.view(s["v"].shape)


def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    H, Hk, D, w = c["H"], c["Hk"], c["D"], c["window"]
    pairs = new = read = 0
    for n, m in zip(_lengths(c), _cached(c)):
        new += n
        if not c["causal"]:
            pairs += n * n
        elif not w:
            pairs += n * m + n * (n + 1) // 2
        else:
            full = max(0, n + m - max(m, w - 1))                      # queries that see a whole window
            rest = n - full
            pairs += full * w + rest * m + rest * (rest + 1) // 2
        read += min(m, w - 1) if w else m
    rows = new * D * e                                                # one head of the new tokens
    if c["kind"] == "attn_fwd":
        return {"bytes": rows * (2 * H + 2 * Hk) + new * H * 4, "flops": 4 * D * H * pairs}
    if c["kind"] == "attn_train":
        return {"bytes": rows * (5 * H + 6 * Hk), "flops": 14 * D * H * pairs}
    return {"bytes": rows * (2 * H + 4 * Hk) + read * D * e * 2 * Hk, "flops": 4 * D * H * pairs}
