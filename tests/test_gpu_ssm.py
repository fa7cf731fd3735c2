"""Selective state space scan against its definition in 64 bits: forward, backward, single tokens, at the lengths, widths, groups, strides
and values where it can go wrong."""
import pytest
import torch

from layer_cases import SCAN, bits, close, columns, offsets, randn, to_gpu
from oracle import layer_oracle as lo

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kla():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2605_08587_amd as m
    m.lib()
    return m


def _inputs(dtype, lead, n, D, G, S, opt, wide, seed):
    g = torch.Generator().manual_seed(seed)
    cols = columns(g, lead, [D, D, D, G * S, G * S], dtype, wide)
    dev_cols = to_gpu(cols)
    if not isinstance(cols, list):
        whole, at = cols
        cols = [whole[..., a:a + w] for a, w in at]
    d, dev = {}, {}
    for i, k in enumerate(("u", "delta", "z")):
        d[k], dev[k] = cols[i], dev_cols[i]
    for i, k in enumerate(("B", "C")):
        d[k], dev[k] = cols[3 + i].unflatten(-1, (G, S)), dev_cols[3 + i].unflatten(-1, (G, S))
    more = dict(A=-torch.arange(1, S + 1) * torch.exp(0.2 * randn(g, D, S)), skip=randn(g, D), delta_bias=randn(g, D) - 1, h0=randn(g, n, D, S))
    for k, v in more.items():
        d[k], dev[k] = v, v.cuda()
    for k in ("skip", "z", "delta_bias", "h0"):
        if k not in opt:
            d[k] = dev[k] = None
    return g, d, dev


ALL = ("skip", "z", "delta_bias", "h0")
CASES = [
    # dtype, N, T, D, G, S, lens, what is given, softplus, wide
    (torch.bfloat16, 1, 1, 64, 1, 16, None, ALL, True, False),
    (torch.bfloat16, 2, 2, 16, 1, 8, None, ALL, True, False),
    (torch.bfloat16, 2, 75, 200, 1, 16, None, ALL, True, True),
    (torch.bfloat16, 1, 130, 132, 2, 16, None, ("z",), True, "odd"),
    (torch.bfloat16, 3, 33, 70, 1, 32, None, ("skip", "delta_bias"), True, False),
    (torch.bfloat16, 1, 21, 48, 3, 64, None, ALL, True, True),
    (torch.bfloat16, 1, 0, 130, 1, 16, [0, 1, 16, 17, 0, 100, 2], ALL, True, "odd"),
    (torch.bfloat16, 1, 0, 64, 2, 8, [31, 33, 64, 1, 0], ("z", "h0"), True, False),
    (torch.float32, 1, 3, 5, 1, 16, None, ALL, True, False),
    (torch.float32, 2, 100, 66, 2, 16, None, ALL, True, "odd"),
    (torch.float32, 2, 40, 64, 1, 8, None, (), True, False),
    (torch.float32, 1, 0, 96, 1, 32, [8, 7, 9, 50, 0], ("h0", "skip"), True, True),
    (torch.float32, 1, 18, 32, 1, 64, None, ("delta_bias", "z"), True, False),
    (torch.float32, 1, 50, 64, 1, 16, None, ("delta_bias",), "positive", False),
    (torch.bfloat16, 1, 600, 64, 1, 16, None, ALL, True, False),
]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_against_definition(kla, case):
    dtype, N, T, D, G, S, lens, opt, softplus, wide = CASES[case]
    print("ssm", CASES[case], flush=True)
    lead, n = ((1, sum(lens)), len(lens)) if lens else ((N, T), N)
    g, d, dev = _inputs(dtype, lead, n, D, G, S, opt, wide, 200 + case)
    if softplus == "positive":          # steps given as they are
        softplus = False
        d["delta"] = d["delta"].abs() + 2
        d["delta_bias"] = d["delta_bias"].abs()
        dev["delta"], dev["delta_bias"] = d["delta"].cuda(), d["delta_bias"].cuda()
    cu = offsets(lens) if lens else None
    dy, dh = randn(g, *lead, D, dtype=dtype), randn(g, n, D, S)
    seqs = lo.sequences(N, T, cu)
    flat = {k: v if v is None or k in ("A", "skip", "delta_bias", "h0") else v.flatten(0, 1) for k, v in d.items()}
    f = lambda **k: lo.ssm(**k, softplus=softplus, seqs=seqs)  # noqa: E731
    (y_ref, h_ref), g_ref = lo.gradients(f, flat, (dy.flatten(0, 1), dh))
    packed = {} if cu is None else dict(cu_seqlens=cu.cuda(), cu_seqlens_host=cu)
    y, hT = kla.kla_ssm_fwd(**dev, softplus=softplus, **packed)
    torch.cuda.synchronize()
    close("y", y.flatten(0, 1), y_ref, SCAN)
    close("hT", hT, h_ref, SCAN)
    gr = kla.kla_ssm_bwd(**dev, d_y=dy.cuda(), d_hT=dh.cuda(), softplus=softplus, **packed)
    torch.cuda.synchronize()
    for k in g_ref:
        close("d" + k, gr["d" + k].reshape(g_ref[k].shape), g_ref[k], SCAN)
    for k in ("skip", "z", "delta_bias", "h0"):
        assert (gr["d" + k] is None) == (d[k] is None)

    # through autograd, with the checkpoints of the forward and without: the same bits
    leaves = {k: None if v is None else v.detach().requires_grad_(True) for k, v in dev.items()}
    wrt = [v for v in leaves.values() if v is not None]
    got = []
    for save in (True, False):
        y2, h2 = kla.kla_ssm(**leaves, softplus=softplus, save=save, **packed)
        assert torch.equal(bits(y2.detach()), bits(y)) and torch.equal(bits(h2.detach()), bits(hT))
        got.append(torch.autograd.grad((y2, h2), wrt, (dy.cuda(), dh.cuda())))
    for k, p, q in zip((k for k, v in leaves.items() if v is not None), *got):
        assert torch.equal(bits(p), bits(gr["d" + k])) and torch.equal(bits(q), bits(gr["d" + k])), k
    y2, _ = kla.kla_ssm(**leaves, softplus=softplus, **packed)
    a = torch.autograd.grad(y2, wrt, dy.cuda())
    _, g_ref = lo.gradients(lambda **k: f(**k)[0], flat, (dy.flatten(0, 1),))
    for (k, _), p in zip(((k, v) for k, v in leaves.items() if v is not None), a):
        close("autograd " + k, p.reshape(g_ref[k].shape), g_ref[k], SCAN)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("S", [8, 16, 32, 64])
@pytest.mark.parametrize("wide", [False, "odd"])
def test_step_by_step_is_the_whole(kla, dtype, S, wide):
    N, T, D, G = 3, 7, 90, 2
    g, d, dev = _inputs(dtype, (N, T), N, D, G, S, ALL, wide, S)
    print("ssm step", dtype, S, wide, flush=True)
    y, hT = kla.kla_ssm_fwd(**dev)
    h = dev["h0"].clone()
    ys = []
    for t in range(T):
        x = {k: v[:, t] for k, v in dev.items() if k in ("u", "delta", "z", "B", "C")}
        ys.append(kla.kla_ssm_step(**x, A=dev["A"], skip=dev["skip"], delta_bias=dev["delta_bias"], h=h))
    torch.cuda.synchronize()
    close("y", torch.stack(ys, 1), y, SCAN)
    close("h", h, hT, SCAN)
    # the state may come back in the place of the one that went in
    again = dev["h0"].clone()
    y2, h2 = kla.kla_ssm_fwd(**dict(dev, h0=again), hT=again)
    assert h2 is again and torch.equal(bits(again), bits(hT)) and torch.equal(bits(y2), bits(y))


def test_extreme_steps(kla):
    """Steps from nothing to a hundred and gates of any size: what is forgotten is forgotten, and softplus keeps its digits where it is small."""
    D, S, T = 64, 16, 40
    g, d, dev = _inputs(torch.float32, (1, T), 1, D, 1, S, ("z", "h0"), False, 77)
    d["delta"] = torch.linspace(-30, 100, T)[None, :, None].expand(1, T, D).contiguous()
    d["z"] = 40 * d["z"]
    dev.update(delta=d["delta"].cuda(), z=d["z"].cuda())
    flat = {k: v if v is None or k in ("A", "h0") else v.flatten(0, 1) for k, v in d.items()}
    dy = randn(g, 1, T, D)
    (y_ref, h_ref), g_ref = lo.gradients(lambda **k: lo.ssm(**k, softplus=True, seqs=[(0, T)]), flat, (dy[0], None))
    y, hT = kla.kla_ssm_fwd(**dev)
    gr = kla.kla_ssm_bwd(**dev, d_y=dy.cuda())
    # row by row: the rows differ by thirteen orders of magnitude
    for t in range(T):
        close("y %d" % t, y[0, t], y_ref[t], SCAN)
        close("du %d" % t, gr["du"][0, t], g_ref["u"][t], SCAN)
        close("ddelta %d" % t, gr["ddelta"][0, t], g_ref["delta"][t], 10 * SCAN)     # differences of terms ten times its size
    close("hT", hT, h_ref, SCAN)


def test_states_that_forget_at_once(kla):
    """A = -inf in some places: such a state is its last token's alone, also behind the end of a sequence that ends inside a tile."""
    D, S, T = 40, 16, 21
    g, d, dev = _inputs(torch.float32, (1, T), 1, D, 1, S, ALL, False, 78)
    flat = {k: v if k in ("A", "skip", "delta_bias", "h0") else v.flatten(0, 1) for k, v in d.items()}
    flat["A"] = d["A"].clone()
    flat["A"][::3, 5:] = -1e30                           # (the same in 64 bits, and with gradients that exist)
    dev["A"] = flat["A"].clamp(min=-1e29).cuda()
    dev["A"][dev["A"] < -1e28] = float("-inf")
    dy, dh = randn(g, 1, T, D), randn(g, 1, D, S)
    (y_ref, h_ref), g_ref = lo.gradients(lambda **k: lo.ssm(**k, softplus=True, seqs=[(0, T)]), flat, (dy[0], dh))
    y, hT = kla.kla_ssm_fwd(**dev)
    gr = kla.kla_ssm_bwd(**dev, d_y=dy.cuda(), d_hT=dh.cuda())
    close("y", y[0], y_ref, SCAN)
    close("hT", hT, h_ref, SCAN)
    for k in g_ref:
        close("d" + k, gr["d" + k].reshape(g_ref[k].shape), g_ref[k], SCAN)


def test_other_sequences_do_not_reach_in(kla):
    lens, D = [17, 40, 3, 64], 80
    cu = offsets(lens)
    g, d, dev = _inputs(torch.bfloat16, (1, sum(lens)), 4, D, 1, 16, ("z", "skip"), False, 8)
    dy = randn(g, 1, sum(lens), D, dtype=torch.bfloat16).cuda()
    bad = {k: None if v is None else v.clone() for k, v in dev.items()}
    for k in ("u", "delta", "z", "B", "C"):
        bad[k][:, 17:57] = float("nan")
        bad[k][:, 57:60] = float("inf")
    out = []
    for x in (dev, bad):
        y, h = kla.kla_ssm_fwd(**x, cu_seqlens=cu.cuda(), cu_seqlens_host=cu)
        gr = kla.kla_ssm_bwd(**x, d_y=dy, cu_seqlens=cu.cuda(), cu_seqlens_host=cu)
        out.append((y, gr["du"], gr["ddelta"], gr["dz"], gr["dB"], gr["dC"], h))
    torch.cuda.synchronize()
    for p, q in zip(out[0][:-1], out[1]):
        for a, b in ((0, 17), (60, 124)):
            assert torch.equal(bits(p[:, a:b]), bits(q[:, a:b]))
    assert torch.equal(bits(out[0][-1][[0, 3]]), bits(out[1][-1][[0, 3]]))


def test_no_tokens(kla):
    for N, T in ((0, 4), (2, 0)):
        g, d, dev = _inputs(torch.bfloat16, (N, T), N, 40, 1, 16, ALL, False, 3)
        y, hT = kla.kla_ssm_fwd(**dev)
        assert y.shape == (N, T, 40) and torch.equal(bits(hT), bits(dev["h0"]))
        dh = torch.randn(N, 40, 16, device="cuda")
        gr = kla.kla_ssm_bwd(**dev, d_y=y, d_hT=dh)
        assert not gr["dA"].any() and not gr["dskip"].any() and not gr["ddelta_bias"].any() and torch.equal(bits(gr["dh0"]), bits(dh))


def _close_runs(name, p, q):
    """Two orders of the same sums, each within the bar of the definition."""
    close(name, p, q, 2 * SCAN + (2.0 ** -8 if p.dtype == torch.bfloat16 else 0))


@pytest.mark.parametrize("packed", [False, True])
def test_long_few_channels(kla, packed):
    """Few channels and many tokens, and the same tokens in pieces with the states handed on: the forward's, the backward's."""
    D, S, T = 128, 16, 6000
    g, d, dev = _inputs(torch.float32, (1, T), 1, D, 1, S, ALL, False, 31)
    dev["delta_bias"] -= 3                               # states that remember hundreds of tokens
    dy = randn(g, 1, T, D).cuda()
    lens = [1000, 5000]
    if packed:
        cu = offsets(lens)
        dev["h0"] = torch.cat([dev["h0"], randn(g, 1, D, S).cuda()])
        kw = dict(cu_seqlens=cu.cuda(), cu_seqlens_host=cu)
    else:
        kw = {}
    print("ssm long", packed, flush=True)
    y, hT = kla.kla_ssm_fwd(**dev, **kw)
    gr = kla.kla_ssm_bwd(**dev, d_y=dy, **kw)

    def piece(lo_, hi, h0, dh):
        x = {k: v[:, lo_:hi].contiguous() if k in ("u", "delta", "z", "B", "C") else v for k, v in dev.items()}
        x["h0"] = h0
        return kla.kla_ssm_fwd(**x)[1], lambda dh: kla.kla_ssm_bwd(**x, d_y=dy[:, lo_:hi].contiguous(), d_hT=dh), kla.kla_ssm_fwd(**x)[0]
    edges = [0, 1000, 1640, 2600, 4111, 6000]
    h, back, ys = dev["h0"][:1].contiguous(), [], []
    for a, b in zip(edges, edges[1:]):
        if packed and a == 1000:
            h = dev["h0"][1:].contiguous()
        h, f, yy = piece(a, b, h, None)
        back.append((a, b, f))
        ys.append(yy)
    _close_runs("y", y, torch.cat(ys, 1))
    _close_runs("hT", hT[-1:], h)
    dh, dA = None, 0
    for a, b, f in reversed(back):
        gp = f(dh)
        dh = gp["dh0"]
        if packed and a == 1000:
            _close_runs("dh0 of the second", gr["dh0"][1:], dh)
            dh = None
        dA = dA + gp["dA"]
        for k in ("du", "ddelta", "dz", "dB", "dC"):
            _close_runs(k, gr[k][:, a:b], gp[k])
    _close_runs("dh0", gr["dh0"][:1], dh)
    _close_runs("dA", gr["dA"], dA)


def test_offsets_beyond_32_bits(kla):
    """The last tokens of a batch of more than 2^31 elements: as those tokens alone from the state before them."""
    D, S, T = 4096, 16, 2 ** 19 + 1003
    print("ssm", T, D, flush=True)
    u = torch.empty(1, T, D, dtype=torch.bfloat16, device="cuda").normal_()
    B, C = (torch.empty(1, T, 1, S, dtype=torch.bfloat16, device="cuda").normal_() for _ in range(2))
    A = -torch.arange(1.0, S + 1, device="cuda").repeat(D, 1)
    cut = T - 100
    y, hT = kla.kla_ssm_fwd(u, u, A, B, C, z=u)
    part = [t[:, cut:].contiguous() for t in (u, B, C)]
    _, mid = kla.kla_ssm_fwd(u[:, :cut], u[:, :cut], A, B[:, :cut], C[:, :cut], z=u[:, :cut])
    tail, end = kla.kla_ssm_fwd(part[0], part[0], A, part[1], part[2], z=part[0], h0=mid)
    _close_runs("y", y[:, cut:], tail)
    _close_runs("hT", hT, end)
    g = kla.kla_ssm_bwd(u, u, A, B, C, y, z=u)
    t = kla.kla_ssm_bwd(part[0], part[0], A, part[1], part[2], y[:, cut:].contiguous(), z=part[0], h0=mid)
    for k in ("du", "ddelta", "dz", "dB", "dC"):
        _close_runs(k, g[k][:, cut:], t[k])


@pytest.mark.parametrize("packed", [False, True])
def test_steps_of_zero_where_states_forget_at_once(kla, packed):
    """A = -inf in some places and steps of 0, in whole segments too: a step of 0 leaves every state as it is, in segments, in one piece and
    token by token."""
    D, S, T = 72, 16, 640
    g, d, dev = _inputs(torch.float32, (1, T), 2 if packed else 1, D, 1, S, ("skip", "h0"), False, 79)
    d["delta"] = d["delta"].abs()
    d["delta"][:, 100:420] = 0                           # (segments of 64 tokens: the third to the sixth have no other step)
    d["delta"][:, 500:] = 0
    flat = {k: v if v is None or k in ("A", "skip", "h0") else v.flatten(0, 1) for k, v in d.items()}
    flat["A"] = d["A"].clone()
    flat["A"][::3, 5:] = -1e30                           # (the same in 64 bits, and with gradients that exist)
    dev["A"] = flat["A"].clamp(min=-1e29).cuda()
    dev["A"][dev["A"] < -1e28] = float("-inf")
    dev["delta"] = d["delta"].cuda()
    cu = offsets([300, 340]) if packed else None
    kw = dict(softplus=False, **(dict(cu_seqlens=cu.cuda(), cu_seqlens_host=cu) if packed else {}))
    seqs = lo.sequences(1, T, cu)
    dy, dh = randn(g, 1, T, D), randn(g, len(seqs), D, S)
    (y_ref, h_ref), g_ref = lo.gradients(lambda **k: lo.ssm(**k, softplus=False, seqs=seqs), flat, (dy[0], dh))
    assert kla.lib().kla_ssm_fwd_workspace_bytes(1, T, D, 1, S, None if cu is None else cu.data_ptr(), 2 if packed else 0) > 0      # in segments
    y, hT = kla.kla_ssm_fwd(**dev, **kw)
    gr = kla.kla_ssm_bwd(**dev, d_y=dy.cuda(), d_hT=dh.cuda(), **kw)
    close("y", y[0], y_ref, SCAN)
    close("hT", hT, h_ref, SCAN)
    for k in g_ref:
        got, ref = gr["d" + k].reshape(g_ref[k].shape).cpu(), g_ref[k]
        if k == "delta":                                 # exp(step A) has no derivative at a step of 0 where A = -inf
            none = (d["delta"][0] == 0) & torch.isinf(dev["A"].cpu()).any(1)
            got, ref = got.masked_fill(none, 0), ref.masked_fill(none, 0)
        close("d" + k, got, ref, SCAN)
    h = dev["h0"][:1].clone()
    for t in (0, 1, 100, 101, 500):
        if t == 100:                                     # (the states of the tokens between)
            x = {k: v[:, 2:100].contiguous() if k in ("u", "delta", "B", "C") else v for k, v in dev.items()}
            h = kla.kla_ssm_fwd(**dict(x, h0=h), softplus=False)[1]
        if t == 500:
            x = {k: v[:, 102:500].contiguous() if k in ("u", "delta", "B", "C") else v for k, v in dev.items()}
            h = kla.kla_ssm_fwd(**dict(x, h0=h), softplus=False)[1]
        x = {k: v[:, t] for k, v in dev.items() if k in ("u", "delta", "B", "C")}
        ys = kla.kla_ssm_step(**x, A=dev["A"], skip=dev["skip"], h=h, softplus=False)
        if t < 300 or not packed:
            close("step %d" % t, ys[0], y_ref[t], SCAN)


@pytest.mark.parametrize("T", [21, 333])
@pytest.mark.parametrize("what", ["B", "C", "u"])
def test_infinities_in_the_last_token(kla, T, what):
    """An infinity in the last token of a sequence that ends inside a tile is that token's: what is read in the place of the tokens that are not there makes
    no NaN of it, in the states, the outputs or what its gradient does not reach."""
    D, S, at = 40, 16, 3
    g, d, dev = _inputs(torch.float32, (1, T), 1, D, 1, S, ALL, False, 80)
    d["u"] = d["u"].abs() + 0.1
    if what == "u":
        d["u"][0, -1, at] = float("inf")
        d["B"][0, -1, 0] = d["B"][0, -1, 0].abs() + 0.1
        d["C"][0, -1, 0] = d["C"][0, -1, 0].abs() + 0.1
    else:
        d[what][0, -1, 0, at] = float("inf")
    dev.update({k: d[k].cuda() for k in ("u", "B", "C")})
    flat = {k: v if v is None or k in ("A", "skip", "delta_bias", "h0") else v.flatten(0, 1) for k, v in d.items()}
    dy, dh = randn(g, 1, T, D), randn(g, 1, D, S)
    (y_ref, h_ref), g_ref = lo.gradients(lambda **k: lo.ssm(**k, softplus=True, seqs=[(0, T)]), flat, (dy[0], dh))
    y, hT = kla.kla_ssm_fwd(**dev)
    gr = kla.kla_ssm_bwd(**dev, d_y=dy.cuda(), d_hT=dh.cuda())

    def same(name, p, ref):
        p, ref = p.cpu().reshape(ref.shape), ref
        wild = ~torch.isfinite(ref)
        assert torch.equal(p[wild].double().nan_to_num(7, 1, -1), ref[wild].nan_to_num(7, 1, -1)), name
        close(name, p.masked_fill(wild, 0), ref.masked_fill(wild, 0), SCAN)
    same("y", y, y_ref)
    same("hT", hT, h_ref)
    same("dskip", gr["dskip"], g_ref["skip"])
    if what != "C":                                      # the infinity is not part of the states before it, nor of their gradients
        same("dA", gr["dA"], g_ref["A"])
        same("dh0", gr["dh0"], g_ref["h0"])
    elif T < 100:                                        # (over more tokens the decays of such a state leave fp32's range: 0 times infinity)
        same("dh0", gr["dh0"], g_ref["h0"])


def test_steps_to_the_last_digits(kla):
    """softplus of the steps in fp32, seen through one token with maps of ones (y is S times the step): relative to the step itself, from e^-85 to 100, and
    at the values that are none.  Bar: units of 2^-23 of two hardware functions, eight roundings of 2^-24, and the fp32 constant of 2.8e-9 |x|."""
    D, S = 4096, 8
    raw = torch.linspace(-85, 100, D - 8)
    raw = torch.cat([raw, torch.tensor([float("inf"), float("-inf"), float("nan"), 3.4e38, -3.4e38, 0.0, -0.0, 1e-30])])
    one, A = torch.ones(1, 1, 1, S, device="cuda"), -torch.ones(D, S, device="cuda")
    u, d = torch.ones(1, 1, D, device="cuda"), raw.cuda()[None, None]
    y, _ = kla.kla_ssm_fwd(u, d, A, one, one)
    z = kla.kla_ssm_step(u[0], d[0], A, one[0], one[0], torch.zeros(1, D, S, device="cuda"))
    ref = torch.logaddexp(raw.double(), torch.zeros(D, dtype=torch.float64))
    bar = 2 * 2.0 ** -23 + 8 * 2.0 ** -24 + 2.8e-9 * raw.double().abs()
    for t in (y[0, 0], z[0]):
        t = t.cpu().double() / S
        ok = (S * ref < 3.4e38) & (ref > 0)              # (what y holds: 8 times 3.4e38 is infinite)
        off = ((t - ref).abs() / ref)[ok]
        worst = int((off / bar[ok]).argmax())
        assert (off <= bar[ok]).all(), (float(raw[ok][worst]), float(off[worst]))
        assert t[-8] == t[-5] == float("inf") and t[-7] == t[-4] == 0 and torch.isnan(t[-6])


def test_step_of_rows_far_apart(kla):
    """A token out of [N, T, D] whose rows are more than 2^24 elements apart: the bits of the same token by itself."""
    N, D, G, S, row = 3, 72, 2, 16, 2 ** 24 + 72
    g = torch.Generator(device="cuda").manual_seed(6)
    whole = torch.empty(N, row, dtype=torch.bfloat16, device="cuda")
    at, part = 0, {}
    for k, w in (("u", D), ("delta", D), ("z", D), ("B", G * S), ("C", G * S)):
        part[k] = whole[:, at:at + w]
        part[k].copy_(torch.randn(N, w, generator=g, device="cuda"))
        at += w
    part["B"], part["C"] = part["B"].unflatten(-1, (G, S)), part["C"].unflatten(-1, (G, S))
    A, h = -torch.rand(D, S, generator=g, device="cuda"), torch.randn(N, D, S, generator=g, device="cuda")
    print("ssm step", row, flush=True)
    h2 = h.clone()
    y = kla.kla_ssm_step(**part, A=A, h=h)
    y2 = kla.kla_ssm_step(**{k: v.contiguous() for k, v in part.items()}, A=A, h=h2)
    assert torch.equal(bits(y), bits(y2)) and torch.equal(bits(h), bits(h2))
