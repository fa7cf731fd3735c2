"""The operators of a recurrent layer around the Kaczmarz recurrence, through the package's public entry points or in plain form.

  conv        short causal convolution of every channel with its SiLU: the step between the projections and the recurrence
  ssm         selective state space scan: the other recurrence of hybrid layers, one decay per channel and state
  add_norm    the residual stream plus the scaled output of a block, and its RMS norm for the next one
  gated_norm  RMS norm of the recurrence's heads times the activated gate, ahead of the output projection

Kinds: "*_step" one token for a batch of sequences (states updated in place), "*_fwd" forward alone (prefill, evaluation),
"*_train" forward and the gradients of everything that has one.  Model width 1024 and 8 or 16 heads of 128 or 256 as in the
tests and benchmark; inner width 1024 to 4096, four taps, 16 states.
"""
from __future__ import annotations

import math
import random

import torch

own = False
EPS = 1e-6


def _case(name, kind, dtype="bf16", N=1, T=1, D=2048, W=4, S=16, G=1, H=1, n_seq=0, lo=0, hi=0, carry=False, bias=True, act=True,
          gate=True, wide=False, res="fp32", scale=True, first=False):
    """N sequences of T tokens, or n_seq > 0 packed ones of lo..hi tokens.  D channels (of a head: gated_norm, with H heads),
    W taps, S states, G groups of B and C; carry: states of earlier tokens come in; bias, act, gate: the optional parts;
    wide: inputs are column ranges of one wider projection; res: type of the residual stream; first: gate before the norm."""
    c = dict(kind=kind, dtype=dtype, N=N, T=T, D=D, W=W, S=S, G=G, H=H, n_seq=n_seq, lo=lo, hi=hi, carry=carry, bias=bias, act=act,
             gate=gate, wide=wide, res=res, scale=scale, first=first)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one user's next token: all latency
        _case("conv_step_b1", "conv_step"),
        # a packed batch of unequal prompts that continue from earlier states, channels cut out of a wider projection
        _case("conv_packed", "conv_fwd", D=4096, n_seq=16, lo=512, hi=4096, carry=True, wide=True),
        # training at the benchmark's shape, 8 sequences of 4K tokens
        _case("conv_train_4k", "conv_train", N=8, T=4096),
        # a serving batch of 64 sequences: bound by the states
        _case("ssm_step_b64", "ssm_step", N=64),
        # the long evaluation context, one sequence, half the inner width
        _case("ssm_prefill_t65536", "ssm_fwd", T=65536, D=1024),
        # single precision, packed, odd lengths, continued: reference runs
        _case("ssm_fp32_packed", "ssm_fwd", dtype="fp32", D=1000, n_seq=5, lo=100, hi=900, carry=True),
        # training of one layer, 4 sequences of 2K tokens
        _case("ssm_train_2k", "ssm_train", N=4, T=2048),
        # a serving batch of 64 next tokens: the step between two blocks
        _case("add_norm_b64", "add_norm_fwd", T=64, D=1024),
        # the same for training at the benchmark's shape, the stream in single precision, a learned scale
        _case("add_norm_train_4k", "add_norm_train", N=8, T=4096, D=1024),
        # one prompt of no round length, gate cut out of a wider projection
        _case("gated_norm_t200", "gated_norm_fwd", T=200, D=128, H=8, wide=True),
        # training at the benchmark's shape with value expansion 2
        _case("gated_norm_train_4k", "gated_norm_train", N=8, T=4096, D=256, H=8),
        # one norm over the whole inner width behind the gate, single precision, odd width and length
        _case("gated_norm_train_fp32", "gated_norm_train", dtype="fp32", N=3, T=333, D=2002, first=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the same kinds.  Sizes over their logarithm, lengths odd."""
    kind = rng.choice(["conv_step", "conv_fwd", "conv_train", "ssm_step", "ssm_fwd", "ssm_fwd", "ssm_train", "ssm_train",
                       "add_norm_fwd", "add_norm_train", "gated_norm_fwd", "gated_norm_train"])
    op = kind.rsplit("_", 1)[0]
    dtype = "fp32" if rng.random() < 0.25 else "bf16"
    kw = dict(dtype=dtype, bias=rng.random() < 0.7, act=rng.random() < 0.8, carry=rng.random() < 0.4, wide=rng.random() < 0.4,
              gate=rng.random() < 0.7)
    D = rng.choice([1024, 2048, 2048, 4096, _log_int(rng, 64, 3000)])
    if kind.endswith("_step"):
        return _case(None, kind, N=_log_int(rng, 1, 512), D=D, W=rng.choice([3, 4, 4]), S=rng.choice([8, 16, 16, 32]), **kw)
    if op in ("add_norm", "gated_norm"):
        most = 2 ** 25 if kind.endswith("_train") else 2 ** 26          # elements of one call
        H, d = (1, D) if op == "add_norm" or rng.random() < 0.3 else (rng.choice([4, 8, 16]), rng.choice([64, 128, 128, 256]))
        rows = max(1, _log_int(rng, 64, most // (H * d)) // (2 if dtype == "fp32" else 1))
        return _case(None, kind, T=rows | 1, D=d, H=H, res=rng.choice([dtype, "fp32"]), scale=rng.random() < 0.6,
                     first=rng.random() < 0.3, **kw)
    if op == "ssm":
        S = rng.choice([8, 16, 16, 16, 32])
        G = rng.choice([1, 1, 2]) if D % 2 == 0 else 1
        most = (2 ** 27 if kind == "ssm_train" else 2 ** 29) // S      # channels times tokens of one call
        kw.update(S=S, G=G)
    else:
        most = 2 ** 26
        kw.update(W=rng.choice([2, 3, 4, 4]))
    tokens = max(8, _log_int(rng, 64, max(128, most // D)) // (2 if dtype == "fp32" else 1))
    if rng.random() < 0.35 and tokens >= 64:
        n_seq = rng.randint(2, 12)
        hi = max(2, 2 * tokens // n_seq)
        return _case(None, kind, D=D, n_seq=n_seq, lo=max(1, hi // rng.choice([4, 8, 16])), hi=hi, **kw)
    N = rng.choice([1, 1, 2, 3, 8])
    T = max(1, tokens // N)
    return _case(None, kind, N=N, T=T | 1, D=D, **kw)


def _lengths(c):
    """The lengths of a packed batch follow from the case, so that its work does."""
    if not c["n_seq"]:
        return [c["T"]] * c["N"]
    r = random.Random(c["n_seq"] * 1_000_003 + c["lo"] * 1_009 + c["hi"])
    return [r.randint(c["lo"], c["hi"]) for _ in range(c["n_seq"])]


def prepare(case, seed):
    c = case
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(int(seed))
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    op, how = c["kind"].rsplit("_", 1)
    D, W, S, G, H = c["D"], c["W"], c["S"], c["G"], c["H"]

    def randn(*shape):
        return torch.randn(shape, generator=gen, device=dev, dtype=torch.float32)

    s = dict(case=c, cu=None, cu_host=None)
    if c["n_seq"]:
        offs = [0]
        for n in _lengths(c):
            offs.append(offs[-1] + n)
        s["cu_host"] = torch.tensor(offs, dtype=torch.int32)      # a data loader has the offsets on the host
        s["cu"] = s["cu_host"].to(dev)
        lead, n_states = (1, offs[-1]), c["n_seq"]
    else:
        lead, n_states = ((c["N"],) if how == "step" else (c["N"], c["T"])), c["N"]

    def columns(*widths):
        """Inputs of these widths, apart or as column ranges of one projection's output."""
        if c["wide"]:
            return [t for t in randn(*lead, sum(widths)).to(dt).split(list(widths), dim=-1)]
        return [randn(*lead, w).to(dt) for w in widths]

    # (the 8 columns that nobody takes: what else such a projection gives)
    if op == "conv":
        s["x"], _ = columns(D, 8)
        s["weight"] = randn(D, W) * W ** -0.5
        s["bias"] = randn(D) * 0.1 if c["bias"] else None
        s["state"] = randn(n_states, W - 1, D).to(dt) if c["carry"] or how == "step" else None
        wrt = ["x", "weight", "bias", "state"]
        out = [("d_y", (*lead, D), dt)]
    elif op == "ssm":
        s["u"], s["z"] = columns(D, D)
        s["z"] = s["z"] if c["gate"] else None
        s["delta"], s["B"], s["C"] = columns(D, G * S, G * S)
        s["B"], s["C"] = (t.unflatten(-1, (G, S)) for t in (s["B"], s["C"]))
        # steps of 0.001 to 0.1 before the projection's part, decays of 1 to S per unit of step: what such layers start from
        step = torch.exp(torch.rand(D, generator=gen, device=dev) * math.log(100.0) + math.log(1e-3))
        s["delta"].mul_(0.5)
        s["delta_bias"] = torch.log(torch.expm1(step))
        s["A"] = -torch.arange(1, S + 1, device=dev, dtype=torch.float32) * torch.exp(0.1 * randn(D, S))
        s["skip"] = 1 + 0.1 * randn(D) if c["bias"] else None
        s["h0"] = randn(n_states, D, S) * 0.1 if c["carry"] or how == "step" else None
        wrt = ["u", "delta", "A", "B", "C", "skip", "z", "delta_bias", "h0"]
        out = [("d_y", (*lead, D), dt)]
    elif op == "add_norm":
        s["x"], _ = columns(D, 8)
        s["weight"] = 1 + 0.1 * randn(D)
        s["residual"] = (3 * randn(*lead, D)).to(torch.float32 if c["res"] == "fp32" else dt)
        s["scale"] = 0.5 + 0.1 * randn(D) if c["scale"] else None
        wrt = ["x", "weight", "residual", "scale"]
        out = [("d_y", (*lead, D), dt), ("d_r", (*lead, D), s["residual"].dtype)]
    else:
        s["gate"], _ = columns(H * D, 8)
        s["gate"] = s["gate"].unflatten(-1, (H, D))
        # heads of unequal size, as a recurrence leaves them
        s["x"] = (randn(*lead, H, D) * torch.exp(randn(*lead, H, 1))).to(dt)
        s["weight"] = 1 + 0.1 * randn(D)
        wrt = ["x", "gate", "weight"]
        out = [("d_y", (*lead, H, D), dt)]
    if how == "train":
        s["wrt"] = [n for n in wrt if s.get(n) is not None]
        for n in s["wrt"]:
            s[n] = s[n].detach().requires_grad_(True)
        for n, shape, t in out:
            s[n] = randn(*shape).to(t)
    return s


# ---- the framework's operators --------------------------------------------------------------------------------------------------


def _own(s):
    import paper_2605_08587_amd as kla
    c = s["case"]
    op, how = c["kind"].rsplit("_", 1)
    packed = dict(cu_seqlens=s["cu"], cu_seqlens_host=s["cu_host"])
    if op == "conv":
        if how == "step":
            return kla.kla_conv_step(s["x"], s["weight"], s["state"], bias=s["bias"], silu=c["act"]), s["state"]
        f = kla.kla_conv if how == "train" else kla.kla_conv_fwd
        r = f(s["x"], s["weight"], bias=s["bias"], state=s["state"], silu=c["act"], want_state=how != "train", **packed)
    elif op == "ssm":
        x = (s["u"], s["delta"], s["A"], s["B"], s["C"])
        kw = dict(skip=s["skip"], z=s["z"], delta_bias=s["delta_bias"], softplus=True)
        if how == "step":
            return kla.kla_ssm_step(*x, s["h0"], **kw), s["h0"]
        f = kla.kla_ssm if how == "train" else kla.kla_ssm_fwd
        r = f(*x, h0=s["h0"], **kw, **packed)
    elif op == "add_norm":
        f = kla.kla_add_norm if how == "train" else kla.kla_add_norm_fwd
        r = f(s["x"], s["weight"], s["residual"], scale=s["scale"], eps=EPS)
    else:
        f = kla.kla_gated_norm if how == "train" else kla.kla_gated_norm_fwd
        r = (f(s["x"], s["gate"], s["weight"], eps=EPS, activation="silu" if c["act"] else "sigmoid", gate_first=c["first"]),)
    if how != "train":
        return r
    outs, grads = (r, (s["d_y"], s["d_r"])) if op == "add_norm" else (r[:1], (s["d_y"],))
    g = torch.autograd.grad(outs, [s[n] for n in s["wrt"]], grads)
    return tuple(t.detach() for t in outs), g


# ---- their plain forms: elementary operations in 32 bits ------------------------------------------------------------------------


def _sequences(s, tokens, device):
    """Per token of the flattened batch: its sequence, its place there; per sequence: first token and length."""
    c = s["case"]
    if s["cu"] is not None:
        first, after = s["cu"][:-1].long(), s["cu"][1:].long()
    else:
        first = torch.arange(c["N"], device=device) * c["T"]
        after = first + c["T"]
    tok = torch.arange(tokens, device=device)
    seq = (tok[:, None] >= after[None, :]).sum(1)
    return tok, seq, tok - first[seq], first, after - first


def _silu_and_slope(x):
    p = 1 / (1 + torch.exp(-x))
    return x * p, p * (1 + x * (1 - p))


def _softplus(x):
    return torch.clamp(x, min=0) + torch.log1p(torch.exp(-x.abs()))


def _plain_conv(s, train):
    c, x = s["case"], s["x"].detach()
    D, W, dt, lead = c["D"], c["W"], x.dtype, x.shape[:-1]
    w = s["weight"].detach()
    bias = None if s["bias"] is None else s["bias"].detach()
    st = None if s["state"] is None else s["state"].detach().float()
    if c["kind"].endswith("_step"):
        line = torch.cat([st, x.float()[:, None]], 1)
        pre = (line * w.t()).sum(1) + (0 if bias is None else bias)
        s["state"].copy_(line[:, 1:])
        return (_silu_and_slope(pre)[0] if c["act"] else pre).to(dt), s["state"]
    x = x.float().reshape(-1, D)
    tok, seq, pos, first, length = _sequences(s, x.shape[0], x.device)
    if st is None:
        st = x.new_zeros(len(first), W - 1, D)

    def tap(j):
        back = W - 1 - j
        inside = (pos >= back)[:, None]
        return torch.where(inside, x[(tok - back).clamp(min=0)], st[seq, (W - 1 + pos - back).clamp(max=W - 2)])
    line = [tap(j) for j in range(W)]
    pre = sum(line[j] * w[:, j] for j in range(W)) + (0 if bias is None else bias)
    y, slope = _silu_and_slope(pre) if c["act"] else (pre, torch.ones_like(pre))
    place = length[:, None] - (W - 1) + torch.arange(W - 1, device=x.device)
    if not train:
        last = torch.where((place >= 0)[..., None], x[(first[:, None] + place).clamp(min=0)],
                           st.gather(1, (W - 1 + place).clamp(max=W - 2)[..., None].expand_as(st)))
        return y.view(*lead, D).to(dt), last.to(dt)
    d_pre = s["d_y"].float().reshape(-1, D) * slope
    n = len(tok)

    def ahead(back):
        inside = (pos + back < length[seq])[:, None]
        return torch.where(inside, d_pre[(tok + back).clamp(max=n - 1)], 0.0)
    grads = dict(x=sum(ahead(W - 1 - j) * w[:, j] for j in range(W)).view(*lead, D).to(dt),
                 weight=torch.stack([(d_pre * line[j]).sum(0) for j in range(W)], 1), bias=d_pre.sum(0))
    if s["state"] is not None:
        # entry i of the state is i - (W - 1) tokens from the sequence's first: tap j meets it at token i - j
        at = [[(first + i - j).clamp(max=n - 1) for j in range(i + 1)] for i in range(W - 1)]
        grads["state"] = torch.stack([sum(torch.where((i - j < length)[:, None], d_pre[at[i][j]], 0.0) * w[:, j] for j in range(i + 1))
                                      for i in range(W - 1)], 1).to(dt)
    return (y.view(*lead, D).to(dt),), tuple(grads[k] for k in s["wrt"])


def _linear_scan(a, b, most):
    """h_t = a_t h_{t-1} + b_t along the first axis, by doubling; a_t = 0 begins anew."""
    step = 1
    while step < most:
        head = b[:step]
        b = torch.cat([head, torch.addcmul(b[step:], a[step:], b[:-step])])
        a = torch.cat([a[:step], a[step:] * a[:-step]])
        step *= 2
    return b


def _plain_ssm(s, train):
    c = s["case"]
    D, S, G = c["D"], c["S"], c["G"]
    u_, dt, lead = s["u"].detach(), s["u"].dtype, s["u"].shape[:-1]
    u, raw = u_.float().reshape(-1, D), s["delta"].detach().float().reshape(-1, D) + s["delta_bias"].detach()
    A = s["A"].detach()
    per = D // G
    B, C = (s[n].detach().float().reshape(-1, G, S).repeat_interleave(per, 1) for n in ("B", "C"))
    z = None if s["z"] is None else s["z"].detach().float().reshape(-1, D)
    skip = None if s["skip"] is None else s["skip"].detach()
    delta = _softplus(raw)
    a = torch.exp(delta[..., None] * A)
    b = (delta * u)[..., None] * B
    if c["kind"].endswith("_step"):
        h = a * s["h0"] + b
        y = (h * C).sum(-1) + (0 if skip is None else skip * u)
        s["h0"].copy_(h)
        return (y if z is None else y * _silu_and_slope(z)[0]).to(dt), s["h0"]
    tok, seq, pos, first, length = _sequences(s, u.shape[0], u.device)
    most = max(_lengths(c))
    starts = tok[pos == 0]
    h0 = None if s["h0"] is None else s["h0"].detach()
    if h0 is not None:
        b[starts] += a[starts] * h0
    kept = a.clone() if train else None
    a[starts] = 0
    h = _linear_scan(a, b, most)
    del a, b
    core = (h * C).sum(-1) + (0 if skip is None else skip * u)
    gate, slope = (1.0, None) if z is None else _silu_and_slope(z)
    y = (core * gate).view(*lead, D).to(dt)
    ends = first + length - 1
    if not train:
        return y, h[ends]
    a = kept
    d_y = s["d_y"].float().reshape(-1, D)
    d_core = d_y * gate
    after = torch.cat([a[1:], torch.zeros_like(a[:1])])
    after[ends] = 0
    g = _linear_scan(after.flip(0), (d_core[..., None] * C).flip(0), most).flip(0)
    before = torch.cat([torch.zeros_like(h[:1]), h[:-1]])
    before[starts] = 0.0 if h0 is None else h0
    via = g * a * before                                  # gradient of the exponent
    through = (g * B).sum(-1)
    d_delta = (via * A).sum(-1) + u * through
    d_raw = d_delta / (1 + torch.exp(-raw))
    d_u = delta * through + (0 if skip is None else skip * d_core)

    def groups(t):
        return t.view(-1, G, per, S).sum(2).view(*lead, G, S).to(dt)
    grads = dict(u=d_u.view(*lead, D).to(dt), delta=d_raw.view(*lead, D).to(dt), A=(via * delta[..., None]).sum(0),
                 B=groups(g * (delta * u)[..., None]), C=groups(h * d_core[..., None]), skip=(d_core * u).sum(0),
                 z=None if z is None else (d_y * core * slope).view(*lead, D).to(dt), delta_bias=d_raw.sum(0), h0=a[starts] * g[starts])
    return (y,), tuple(grads[k] for k in s["wrt"])


def _rms(v):
    return 1 / torch.sqrt((v * v).mean(-1, keepdim=True) + EPS)


def _plain_add_norm(s, train):
    x, r, w = s["x"].detach().float(), s["residual"].detach().float(), s["weight"].detach()
    scale = 1.0 if s["scale"] is None else s["scale"].detach()
    dt, rt = s["x"].dtype, s["residual"].dtype
    total = r + scale * x
    f = _rms(total)
    outs = ((total * f * w).to(dt), total.to(rt))
    if not train:
        return outs
    d_y, d_r = s["d_y"].float(), s["d_r"].float()
    unit = total * f
    d_unit = d_y * w
    d = d_r + f * (d_unit - unit * (d_unit * unit).mean(-1, keepdim=True))
    D = x.shape[-1]
    grads = dict(x=(scale * d).to(dt), weight=(d_y * unit).view(-1, D).sum(0), residual=d.to(rt), scale=(d * x).view(-1, D).sum(0))
    return outs, tuple(grads[k] for k in s["wrt"])


def _plain_gated_norm(s, train):
    c = s["case"]
    x, t, w, dt = s["x"].detach().float(), s["gate"].detach().float(), s["weight"].detach(), s["x"].dtype
    if c["act"]:
        gate, slope = _silu_and_slope(t)
    else:
        gate = 1 / (1 + torch.exp(-t))
        slope = gate * (1 - gate)
    v = x * gate if c["first"] else x
    f = _rms(v)
    unit = v * f
    y = unit * w if c["first"] else unit * w * gate
    if not train:
        return (y.to(dt),)
    d_y = s["d_y"].float()
    d_out = d_y if c["first"] else d_y * gate
    d_unit = d_out * w
    d_v = f * (d_unit - unit * (d_unit * unit).mean(-1, keepdim=True))
    d_gate = d_v * x if c["first"] else d_y * unit * w
    grads = dict(x=(d_v * gate if c["first"] else d_v).to(dt), gate=(d_gate * slope).to(dt), weight=(d_out * unit).view(-1, c["D"]).sum(0))
    return (y.to(dt),), tuple(grads[k] for k in s["wrt"])


def run(s):
    if own:
        return _own(s)
    op, how = s["case"]["kind"].rsplit("_", 1)
    return {"conv": _plain_conv, "ssm": _plain_ssm, "add_norm": _plain_add_norm, "gated_norm": _plain_gated_norm}[op](s, how == "train")


# ---- the definitions in 64 bits, token by token ---------------------------------------------------------------------------------


def _f64(t):
    return None if t is None else t.detach().double()


def _batches(s, c):
    """(index, first token, token after the last) of every sequence in the flattened batch."""
    offs = [0]
    for n in _lengths(c):
        offs.append(offs[-1] + n)
    return list(zip(range(len(offs) - 1), offs, offs[1:]))


def _exact_conv(s, c, train):
    D, W = c["D"], c["W"]
    x = _f64(s["x"])
    w, bias, st = _f64(s["weight"]), _f64(s["bias"]), _f64(s["state"])
    lead, x = x.shape[:-1], x.reshape(-1, D)
    if c["kind"].endswith("_step"):
        pieces = [(i, i, i + 1) for i in range(c["N"])]
    else:
        pieces = _batches(s, c)
    ys, lasts, dxs, dsts = [], [], [], []
    dw, db = torch.zeros_like(w), torch.zeros(D, dtype=torch.float64, device=x.device)
    for i, lo, hi in pieces:
        line = torch.cat([x.new_zeros(W - 1, D) if st is None else st[i], x[lo:hi]])
        pre = line.unfold(0, W, 1).mul(w).sum(-1) + (0 if bias is None else bias)     # [tokens, D, W] windows
        ys.append(pre * torch.sigmoid(pre) if c["act"] else pre)
        lasts.append(line[-(W - 1):])
        if train:
            d = _f64(s["d_y"]).reshape(-1, D)[lo:hi]
            if c["act"]:
                p = torch.sigmoid(pre)
                d = d * (p + pre * p * (1 - p))
            back = torch.zeros_like(line)
            for j in range(W):
                back[j:j + hi - lo] += d * w[:, j]
                dw[:, j] += (d * line[j:j + hi - lo]).sum(0)
            db += d.sum(0)
            dsts.append(back[:W - 1])
            dxs.append(back[W - 1:])
    y = torch.cat(ys).view(*lead, D)
    if not train:
        return y, torch.stack(lasts)
    grads = dict(x=torch.cat(dxs).view(*lead, D), weight=dw, bias=db, state=torch.stack(dsts))
    return (y,), tuple(grads[k] for k in s["wrt"])


def _exact_ssm(s, c, train):
    D, S, G = c["D"], c["S"], c["G"]
    lead = s["u"].shape[:-1]
    u, raw = _f64(s["u"]).reshape(-1, D), _f64(s["delta"]).reshape(-1, D) + _f64(s["delta_bias"])
    A, z = _f64(s["A"]), _f64(s["z"])
    B, C = (_f64(s[n]).reshape(-1, G, S) for n in ("B", "C"))
    group = torch.arange(D, device=u.device) // (D // G)
    delta = torch.log1p(torch.exp(-raw.abs())) + raw.clamp(min=0)
    skip = 0 if s["skip"] is None else _f64(s["skip"])
    gate = 1.0
    if z is not None:
        z = z.reshape(-1, D)
        gate = z * torch.sigmoid(z)
    if c["kind"].endswith("_step"):
        rows = torch.arange(c["N"], device=u.device)[:, None]             # all sequences side by side, one token each
    elif c["n_seq"]:
        rows = None
    else:
        rows = torch.arange(c["N"], device=u.device)[:, None] * c["T"] + torch.arange(c["T"], device=u.device)
    pieces = [(slice(None), rows)] if rows is not None else [
        (slice(i, i + 1), torch.arange(lo, hi, device=u.device)[None]) for i, lo, hi in _batches(s, c)]
    core, last = torch.empty_like(u), []
    if train:
        d_y = _f64(s["d_y"]).reshape(-1, D)
        d_core = d_y * gate
        g_u, g_delta = torch.empty_like(u), torch.empty_like(u)
        g_A, g_B, g_C, first = torch.zeros_like(A), torch.zeros_like(B), torch.zeros_like(C), []
    for which, at in pieces:
        n, T = at.shape
        h = u.new_zeros(n, D, S) if s["h0"] is None else _f64(s["h0"][which]).clone()
        was = []
        for t in range(T):
            i = at[:, t]
            was.append(h if train else None)
            h = torch.exp(delta[i][..., None] * A) * h + (delta[i] * u[i])[..., None] * B[i][:, group]
            core[i] = (h * C[i][:, group]).sum(-1)
        last.append(h)
        if not train:
            continue
        g = torch.zeros_like(h)
        for t in reversed(range(T)):
            i = at[:, t]
            a, b = torch.exp(delta[i][..., None] * A), B[i][:, group]
            now = was[t + 1] if t + 1 < T else h
            g = g + d_core[i][..., None] * C[i][:, group]
            g_C[i] = (now * d_core[i][..., None]).view(n, G, D // G, S).sum(2)
            g_B[i] = (g * (delta[i] * u[i])[..., None]).view(n, G, D // G, S).sum(2)
            e = g * a * was[t]
            g_A += (e * delta[i][..., None]).sum(0)
            gb = (g * b).sum(-1)
            g_delta[i] = (e * A).sum(-1) + gb * u[i]
            g_u[i] = gb * delta[i]
            g = g * a
        first.append(g)
    core = core + skip * u
    y = (core * gate).view(*lead, D)
    if not train:
        return y, torch.cat(last)
    g_raw = g_delta * torch.sigmoid(raw)
    grads = dict(u=(g_u + skip * d_core).view(*lead, D), delta=g_raw.view(*lead, D), A=g_A, B=g_B.view(*lead, G, S), C=g_C.view(*lead, G, S),
                 skip=(d_core * u).sum(0), delta_bias=g_raw.sum(0), h0=torch.cat(first))
    if z is not None:
        p = torch.sigmoid(z)
        grads["z"] = (d_y * core * (p + z * p * (1 - p))).view(*lead, D)
    return (y,), tuple(grads[k] for k in s["wrt"])


def _exact_norm(s, c, train):
    """Both norms by their definition; the gradients by torch's own differentiation of it."""
    names = [n for n in ("x", "weight", "residual", "scale", "gate") if s.get(n) is not None]
    v = {n: _f64(s[n]).requires_grad_(train) for n in names}

    def normed(t):
        return t / (t.square().sum(-1, keepdim=True) / t.shape[-1] + EPS) ** 0.5
    if "gate" in v:
        g = torch.sigmoid(v["gate"]) * (v["gate"] if c["act"] else 1)
        outs = (normed(v["x"] * g) * v["weight"] if c["first"] else normed(v["x"]) * v["weight"] * g,)
    else:
        total = v["residual"] + v["x"] * v.get("scale", 1.0)
        outs = (normed(total) * v["weight"], total)
    if not train:
        return outs
    d = (_f64(s["d_y"]),) + ((_f64(s["d_r"]),) if len(outs) > 1 else ())
    return tuple(t.detach() for t in outs), torch.autograd.grad(outs, [v[n] for n in s["wrt"]], d)


def exact(case, seed):
    c = case
    op, how = c["kind"].rsplit("_", 1)
    tokens = sum(_lengths(c)) if how != "step" else 1
    steps = tokens if c["n_seq"] else c["T"]
    if op == "ssm" and (steps > 70_000 or how == "train" and steps > 20_000):
        return None                                       # token by token this takes too long
    s = prepare(c, seed)
    return {"conv": _exact_conv, "ssm": _exact_ssm, "add_norm": _exact_norm, "gated_norm": _exact_norm}[op](s, c, how == "train")


def work(case):
    c = case
    op, how = c["kind"].rsplit("_", 1)
    e = 2 if c["dtype"] == "bf16" else 4
    D, W, S, G, H = c["D"], c["W"], c["S"], c["G"], c["H"]
    train = how == "train"
    tokens = c["N"] if how == "step" else sum(_lengths(c))
    states = c["n_seq"] or c["N"]
    n = tokens * D * H
    if op == "conv":
        # x in, y out; backward d_y (and x) in, d_x out; the taps; states in and out
        state = states * (W - 1) * D * e
        bytes_ = 2 * n * e + 4 * D * (W + c["bias"]) + state * ((c["carry"] or how == "step") + (not train))
        flops = n * (2 * W + 5 * c["act"])
        if train:
            bytes_ += 2 * n * e + 4 * D * (W + c["bias"]) + state * c["carry"]
            flops += n * (4 * W + 8 * c["act"])
        return {"bytes": bytes_, "flops": flops}
    if op == "ssm":
        # u, delta (z) in, y out, B and C in; per state exp, two products, two products with sums
        state = states * D * S * 4
        bytes_ = n * e * (3 + c["gate"]) + tokens * 2 * G * S * e + 4 * D * (S + 1 + c["bias"]) + state * ((c["carry"] or how == "step") + (not train))
        flops = n * (7 * S + 12)
        if train:
            bytes_ += n * e * (3 + 2 * c["gate"]) + tokens * 2 * G * S * e + 4 * D * (S + 1 + c["bias"]) + state * c["carry"]
            flops += n * (16 * S + 20)
        return {"bytes": bytes_, "flops": flops}
    if op == "add_norm":
        r = 4 if c["res"] == "fp32" else e
        bytes_, flops = n * (2 * e + 2 * r) + 8 * D, n * 6
        if train:
            # d_y, d_r in, d_x, d_residual out
            bytes_ += n * (2 * e + 2 * r) + 8 * D
            flops += n * 14
        return {"bytes": bytes_, "flops": flops}
    bytes_, flops = n * 3 * e + 4 * D, n * 9
    if train:
        bytes_ += n * 3 * e + 4 * D
        flops += n * 20
    return {"bytes": bytes_, "flops": flops}
