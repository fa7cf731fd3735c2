"""Softmax attention over whole sequences on the GPU, both directions, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from attn_cases import check, f64, offsets, randn
from layer_cases import bits
from oracle import attn_oracle as ao

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]


@pytest.fixture(scope="module")
def kla():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2605_08587_amd as m
    m.lib()
    return m


def _inputs(seed, dtype, lead, H, Hk, D, wide=False, sharp=2.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda h, s=1.0: randn(g, *lead, h, D, dtype=dtype, wide=wide, sharp=s)
    return r(H, sharp), r(Hk), r(Hk), randn(g, *lead, H, D, dtype=dtype)


def _run(kla, dtype, lead, H, Hk, D, causal=True, window=0, lengths=None, wide=False, scale=None, seed=0):
    q, k, v, d_o = _inputs(seed, dtype, lead, H, Hk, D, wide)
    cu = None if lengths is None else offsets(lengths)
    kw = dict(scale=scale, causal=causal, window=window)
    if cu is not None:
        kw.update(cu_seqlens=cu.cuda(), cu_seqlens_host=cu)
    flat = lambda t: t.flatten(0, 1)
    for rest in (None,) + ((torch.full_like(d_o, float("nan")),) if dtype == torch.bfloat16 else ()):
        o, lse = kla.kla_attn_fwd(q, k, v, rest=rest, **kw)
        g = kla.kla_attn_bwd(q, k, v, o, lse, d_o, rest=rest, **kw)
        torch.cuda.synchronize()
        check([lead[1]] * lead[0] if lengths is None else lengths, flat(q), flat(k), flat(v), flat(o), flat(lse), D ** -0.5 if scale is None else scale,
              causal, window, flat(d_o), [flat(g[x]) for x in ("dq", "dk", "dv")], rest=rest is not None)
        if rest is not None and rest.numel():                # half a step of o at most, and no less than what was left out
            assert (rest.double().abs() <= 2.0 ** -8 * o.double().abs() + 1e-30).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("N,T,H,Hk", [(1, 1, 1, 1), (2, 1, 4, 2), (1, 2, 3, 1), (1, 31, 2, 2), (1, 32, 4, 2), (2, 33, 6, 2), (1, 63, 2, 1), (1, 65, 4, 1), (3, 127, 7, 1),
                                      (1, 129, 10, 2), (1, 300, 4, 4)])
def test_lengths_and_heads(kla, dtype, D, N, T, H, Hk):
    _run(kla, dtype, (N, T), H, Hk, D, seed=T)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,H,Hk,D,window", [(70, 2, 2, 64, 1), (200, 4, 2, 128, 2), (200, 3, 1, 64, 33), (333, 8, 2, 128, 64), (333, 5, 5, 64, 100), (150, 4, 1, 128, 149),
                                             (150, 4, 1, 128, 150), (150, 2, 1, 64, 2 ** 31 - 1)])
def test_windows(kla, dtype, T, H, Hk, D, window):
    _run(kla, dtype, (1, T), H, Hk, D, window=window, seed=window % 1000)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,T,H,Hk,D", [(2, 1, 2, 1, 64), (1, 100, 4, 2, 128), (2, 257, 3, 3, 64)])
def test_both_ways(kla, dtype, N, T, H, Hk, D):
    _run(kla, dtype, (N, T), H, Hk, D, causal=False, seed=T)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lengths,H,Hk,D,kw", [
    ([5, 0, 1, 130, 0, 64], 4, 2, 64, {}), ([0, 0], 2, 1, 128, {}), ([33, 200, 1], 6, 2, 128, dict(window=40)), ([100, 60], 3, 3, 64, dict(causal=False)),
    ([3, 1, 0, 2, 9, 17] * 25, 2, 1, 64, {}), ([1] * 130, 4, 4, 128, {})])
def test_packed(kla, dtype, lengths, H, Hk, D, kw):
    _run(kla, dtype, (1, sum(lengths)), H, Hk, D, lengths=lengths, wide=True, seed=len(lengths), **kw)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,H,Hk,window", [(70, 32, 2, 0), (41, 32, 1, 0), (90, 64, 1, 20), (21, 48, 1, 0), (17, 128, 1, 0), (19, 80, 1, 7)])
def test_wide_groups(kla, dtype, D, T, H, Hk, window):
    """Heads of a group that fill a tile, divide it, or go over several."""
    _run(kla, dtype, (1, T), H, Hk, D, window=window, wide=True, seed=T)


def test_thousands_of_sequences(kla):
    """More than 64 x 64 sequences, most of them empty: a tile's sequence is looked for in three steps."""
    lengths = [0, 1, 0, 0, 2, 0, 0, 0, 0, 1] * 600
    _run(kla, torch.float32, (1, sum(lengths)), 2, 1, 64, lengths=lengths, seed=19)


def test_the_largest_strides(kla):
    """Tokens 2^24 elements apart, which a tile counts from its first in 32 bits."""
    g = torch.Generator(device="cuda").manual_seed(21)
    w = torch.empty(1, 70, 1 << 24, device="cuda")
    q, k, v = (randn(g, 1, 70, h, 64) for h in (2, 1, 1))
    far = [w[..., a:a + t.shape[2] * 64].unflatten(-1, (-1, 64)) for a, t in ((0, q), (512, k), ((1 << 24) - 64, v))]
    for f, t in zip(far, (q, k, v)):
        f.copy_(t)
    for lead in (slice(None), slice(0, 1)):                  # (the second: rows of one token each, whose stride says nothing)
        near, apart = [[t[:, lead] for t in ts] for ts in ((q, k, v), far)]
        o, lse = kla.kla_attn_fwd(*(t.contiguous() for t in near))
        o2, lse2 = kla.kla_attn_fwd(*apart)
        assert torch.equal(bits(o), bits(o2)) and torch.equal(bits(lse), bits(lse2))
        a, b = (kla.kla_attn_bwd(*ts, o, lse, o) for ts in ([t.contiguous() for t in near], apart))
        assert all(torch.equal(bits(a[x]), bits(b[x])) for x in a)


@pytest.mark.parametrize("dtype", DTYPES)
def test_many_workgroups(kla, dtype):
    """Enough rows for the form in which four waves share tiles of keys; a window keeps the oracle quick."""
    _run(kla, dtype, (6, 700), 16, 8, 64 if dtype == torch.float32 else 128, window=90, seed=5)
    _run(kla, dtype, (1, 500), 66, 66, 64, seed=6, wide=True)
    _run(kla, dtype, (4, 610), 16, 16, 128, window=40, seed=22)
    _run(kla, dtype, (1, 320 * 20), 4, 4, 128, lengths=[320, 321, 319] * 6 + [640], window=70, seed=7, wide=True)


@pytest.mark.parametrize("scale", [1e-3, 1.0])
def test_scale(kla, scale):
    _run(kla, torch.float32, (1, 90), 2, 1, 64, scale=scale, seed=8)
    _run(kla, torch.bfloat16, (1, 90), 2, 1, 128, scale=scale, seed=9)


def test_scores_far_apart(kla):
    """Scores of some hundreds: weights underflow, the running reference jumps."""
    q, k, v, _ = _inputs(10, torch.float32, (1, 400), 2, 1, 64, sharp=40.0)
    k = k * torch.linspace(0.01, 2, 400, device="cuda")[None, :, None, None]
    o, lse = kla.kla_attn_fwd(q, k, v)
    check([400], q[0], k[0], v[0], o[0], lse[0], 0.125, True, 0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("H,D", [(2, 64), (2, 128), (150, 64), (130, 128)])
def test_rows_are_not_scaled_for_others(kla, dtype, H, D):
    """Rows whose largest score comes first keep their reference, and their bits, whatever the rows beside them do: even tokens' scores fall along the
    keys; odd ones' rise in one call, so that their tile is scaled again and again, and fall in the other."""
    T = 390
    _q, _k, v, _ = _inputs(24, dtype, (1, T), H, H, D)
    q, k = torch.zeros_like(v), torch.zeros_like(v)
    k[..., 0] = -torch.arange(T, device="cuda").to(dtype)[:, None]
    q[..., 0] = torch.linspace(0.5, 1.7, H, device="cuda").to(dtype)
    rising = q.clone()
    rising[:, 1::2] *= -1
    (o, lse), (o2, lse2) = (kla.kla_attn_fwd(x, k, v, scale=0.3, causal=False) for x in (q, rising))
    assert torch.equal(bits(o[:, ::2]), bits(o2[:, ::2])) and torch.equal(bits(lse[:, ::2]), bits(lse2[:, ::2]))
    assert (lse2[:, 1::2] > lse[:, 1::2] + 40).all()


def test_remainder(kla):
    """o and rest together are o before its rounding: what the other rounding of the way, of the weights, leaves is within its own bound."""
    q, k, v, _ = _inputs(20, torch.bfloat16, (1, 150), 4, 2, 64)
    rest = torch.empty_like(q)
    o, _lse = kla.kla_attn_fwd(q, k, v, rest=rest)
    a = [f64(t[0]) for t in (q, k, v)]
    ref, bound = ao.forward(*a, 0.125)[0], ao.bounds(*a, 0.125, 2.0 ** -8)[0]
    both = f64(o[0]) + f64(rest[0])
    assert (abs(both - ref) <= bound - (2.0 ** -8 - 2.0 ** -16) * abs(ref)).all()
    assert np.linalg.norm(both - ref) < 0.85 * np.linalg.norm(f64(o[0]) - ref)
    with pytest.raises(kla.KlaError, match="DTYPE"):
        kla.kla_attn_fwd(q.float(), k.float(), v.float(), rest=rest)
    with pytest.raises(TypeError, match="rest"):
        kla.kla_attn_fwd(q, k, v, rest=rest.float())


NAN, INF = float("nan"), float("inf")


def _expected(kind, q, k, v, d_o, scale, causal, window):
    with np.errstate(all="ignore"):
        o = ao.forward(f64(q), f64(k), f64(v), scale, causal=causal, window=window)
        g = ao.backward(f64(q), f64(k), f64(v), f64(d_o), scale, causal=causal, window=window)
    return (*o, *g)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,H,Hk,causal,window", [(150, 4, 2, True, 0), (150, 4, 2, True, 37), (90, 2, 2, False, 0), (300, 66, 66, True, 50), (650, 90, 90, True, 50), (650, 90, 90, False, 0)])
@pytest.mark.parametrize("where,value", [("v", INF), ("v", NAN), ("v", -INF), ("k", NAN), ("q", NAN), ("d_o", INF), ("d_o", NAN), ("q", INF)])
def test_what_is_not_finite_stays_where_it_is_seen(kla, dtype, T, H, Hk, causal, window, where, value):
    """One token's row holds an infinity or a NaN: rows and keys that do not meet it are as if it were not there, and those that do are infinite or NaN
    where the formulas are."""
    D, at = 64, 70
    t = dict(zip(("q", "k", "v", "d_o"), _inputs(11, dtype, (1, T), H, Hk, D, sharp=1.0)))
    clean = {n: x.clone() for n, x in t.items()}
    t[where][0, at, 0, 5] = value
    if where == "v":
        t["v"][0, at + 3, Hk - 1, 9] = -value
    kw = dict(causal=causal, window=window)
    out = []
    for x in (t, clean):
        o, lse = kla.kla_attn_fwd(x["q"], x["k"], x["v"], **kw)
        out.append((o, lse, *kla.kla_attn_bwd(x["q"], x["k"], x["v"], o, lse, x["d_o"], **kw).values()))
    h = min(2, Hk)                                          # (the heads in question, and no more for the oracle's sake)
    G = H // Hk
    pick = lambda x: (x["q"][0, :, :h * G], x["k"][0, :, :h], x["v"][0, :, :h], x["d_o"][0, :, :h * G])
    if Hk > h:
        t["v"][0, at + 3, Hk - 1, 9] = 0
    for name, got, was, ref in zip(("o", "lse", "dq", "dk", "dv"), out[0], out[1], _expected(where, *pick(t), D ** -0.5, causal, window)):
        heads = h if name in ("dk", "dv") else h * G
        x, w = f64(got[0, :, :heads]), f64(was[0, :, :heads])
        bad = ~np.isfinite(ref)
        # exactly those rows that meet it (a row is one token's head) are not finite ..
        rows = lambda m: m.any(-1) if m.ndim == 3 else m
        assert (rows(~np.isfinite(x)) == rows(bad)).all(), name
        # .. and the infinities of the forward are infinities
        if name in ("o", "lse"):
            assert np.array_equal(x[bad], ref[bad], equal_nan=True), name
        # where nothing of it is met the result is the one without it
        clean_rows = ~rows(bad)
        if name in ("o", "lse"):
            same = clean_rows
        else:                                               # a gradient's row can change and stay finite: those that meet nothing of the token at all
            tok = np.arange(T)
            sees = (tok[:, None] >= tok[None, :]) if causal else np.ones((T, T), bool)
            if window:
                sees &= tok[:, None] - tok[None, :] < window
            apart = ~sees[:, at] & ~sees[at, :] & ~sees[:, at + 3] if where == "v" else ~sees[:, at] & ~sees[at, :]
            same = clean_rows & (apart & ~(sees.T @ sees[:, at]))[:, None]
        tol = 2.0 ** -7 * abs(w).max() if dtype == torch.bfloat16 else 1e-5 * abs(w).max()
        assert same.any() or not causal or name in ("dq", "dk", "dv")
        assert (abs(x[same] - w[same]) <= tol).all(), name


def test_rows_whose_scores_are_all_minus_infinity_are_nan(kla):
    q, k, v, _ = _inputs(12, torch.float32, (1, 80), 2, 2, 64)
    k[0, :40, :, 0] = -INF
    q[..., 0] = 1.0
    o, lse = kla.kla_attn_fwd(q, k, v)
    assert torch.isnan(o[0, :40]).all() and torch.isfinite(o[0, 40:]).all()
    assert (lse[0, :40] == -INF).all() or torch.isnan(lse[0, :40]).all()
    ref = ao.forward(f64(q[0, 40:]), f64(k[0, 40:]), f64(v[0, 40:]), 0.125)[0]       # weights of zero take nothing from their values
    assert abs(f64(o[0, 40:]) - ref).max() < 1e-5


def test_same_bits_twice_and_in_place_of_what_was_there(kla):
    q, k, v, d_o = _inputs(13, torch.bfloat16, (2, 500), 8, 2, 128)
    o, lse = kla.kla_attn_fwd(q, k, v)
    g = kla.kla_attn_bwd(q, k, v, o, lse, d_o)
    out, l2 = torch.full_like(o, NAN), torch.full_like(lse, NAN)
    before = out._version
    r = kla.kla_attn_fwd(q, k, v, out=out, lse=l2)
    assert r[0] is out or r[0].data_ptr() == out.data_ptr()
    assert torch.equal(bits(out), bits(o)) and torch.equal(bits(l2), bits(lse)) and out._version > before
    assert kla.kla_attn_fwd(q, k, v, want_lse=False)[1] is None
    h = kla.kla_attn_bwd(q, k, v, o, lse, d_o, workspace=torch.full((1 << 26,), 255, dtype=torch.uint8, device="cuda"))
    assert all(torch.equal(bits(g[x]), bits(h[x])) for x in g)


@pytest.mark.parametrize("native", [True, False])
def test_autograd(kla, monkeypatch, native):
    if not native:
        monkeypatch.setattr(kla, "_native", kla._StepByStep)
    q, k, v, d_o = _inputs(14, torch.bfloat16, (1, 260), 8, 2, 64, wide=True)
    cu = offsets([100, 0, 160])
    kw = dict(window=50, scale=0.2, cu_seqlens=cu.cuda(), cu_seqlens_host=cu)
    rest = torch.empty_like(d_o)
    o, lse = kla.kla_attn_fwd(q, k, v, rest=rest, **kw)
    g = kla.kla_attn_bwd(q, k, v, o, lse, d_o, rest=rest, **kw)
    leaves = [t.detach().requires_grad_(True) for t in (q, k, v)]
    y = kla.kla_attn(*leaves, **kw)
    assert torch.equal(bits(y.detach()), bits(o))
    for a, b in zip(torch.autograd.grad(y, leaves, d_o), g.values()):
        assert torch.equal(bits(a), bits(b))
    only = kla.kla_attn(q, leaves[1], v, **kw)               # one of the three
    assert torch.equal(bits(torch.autograd.grad(only, leaves[1], d_o)[0]), bits(g["dk"]))
    scattered = d_o.transpose(1, 2).contiguous().transpose(1, 2)
    assert torch.equal(bits(torch.autograd.grad(kla.kla_attn(*leaves, **kw), leaves, scattered)[0]), bits(g["dq"]))
    with torch.no_grad():
        assert not kla.kla_attn(*leaves, **kw).requires_grad
    with pytest.raises(RuntimeError, match="create_graph"):
        torch.autograd.grad(kla.kla_attn(*leaves, **kw).sum(), leaves, create_graph=True)
    y = kla.kla_attn(*leaves, **kw)
    kw["cu_seqlens"].add_(0)
    with pytest.raises(RuntimeError, match="cu_seqlens"):
        torch.autograd.grad(y, leaves, d_o)
    y = kla.kla_attn(*leaves, **kw)
    with torch.no_grad():
        leaves[0].mul_(1)
    with pytest.raises(RuntimeError, match="modified"):
        torch.autograd.grad(y, leaves, d_o)


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("before", [1, 3, 8])
def test_gradients_at_any_address(kla, monkeypatch, native, dtype, before):
    """Autograd hands over a piece of a larger gradient, wherever it begins."""
    if not native:
        monkeypatch.setattr(kla, "_native", kla._StepByStep)
    q, k, v, d_o = _inputs(23, dtype, (2, 70), 4, 2, 64)
    o, lse = kla.kla_attn_fwd(q, k, v)
    leaves = [t.detach().requires_grad_(True) for t in (q, k, v)]
    want = torch.autograd.grad(kla.kla_attn(*leaves), leaves, d_o)
    seen = []
    y = kla.kla_attn(*leaves)
    y.register_hook(lambda g: seen.append(g.data_ptr() % 16))
    together = torch.cat([torch.zeros(before, device="cuda", dtype=dtype), y.flatten()])
    have = torch.autograd.grad(together, leaves, torch.cat([torch.ones(before, device="cuda", dtype=dtype), d_o.flatten()]))
    assert seen == [before * q.element_size() % 16]          # (or this tests nothing)
    assert all(torch.equal(bits(a), bits(b)) for a, b in zip(have, want))


@pytest.mark.parametrize("dtype", DTYPES)
def test_gradients_by_differences(kla, dtype):
    """<d, gradient> against the forward's own differences, in steps large enough for its rounding."""
    q, k, v, d_o = _inputs(15, torch.float32, (1, 130), 4, 2, 64, sharp=1.0)
    leaves = [t.detach().requires_grad_(True) for t in (q, k, v)]
    y = kla.kla_attn(*leaves, window=60)
    grads = torch.autograd.grad(y, leaves, d_o)
    f = lambda *x: (d_o.double() * kla.kla_attn_fwd(*x, window=60)[0].double()).sum().item()
    gen = torch.Generator(device="cuda").manual_seed(16)
    for i, g in enumerate(grads):
        d = torch.randn(g.shape, generator=gen, device="cuda")
        d /= d.norm()
        step = 2.0 ** -4
        up, down = [list((q, k, v)) for _ in range(2)]
        up[i], down[i] = up[i] + step * d, down[i] - step * d
        want = (f(*up) - f(*down)) / (2 * step)
        have = (g.double() * d.double()).sum().item()
        # the forward's rounding, 2e-7 of values whose weighted sum has a norm below |d_o|, over the step; the third difference over 6
        noise = 4e-7 * d_o.norm().item() / step + step ** 2 * g.norm().item()
        assert abs(want - have) <= noise, (i, want, have, noise)


def test_misaligned_rows_are_refused(kla):
    q, k, v, _ = _inputs(17, torch.bfloat16, (1, 20), 4, 2, 64)
    w = torch.zeros(1, 20, 4 * 64 + 4, device="cuda", dtype=torch.bfloat16)
    with pytest.raises(kla.KlaError, match="ALIGN"):
        kla.kla_attn_fwd(w[..., 4:].unflatten(-1, (4, 64)), k, v)
    with pytest.raises(ValueError, match="overlap"):
        kla.kla_attn_fwd(q, k[:, :1].expand(1, 20, 2, 64), v)
    with pytest.raises(ValueError, match="contiguous"):
        kla.kla_attn_fwd(q.transpose(1, 2).contiguous().transpose(1, 2), k, v)
    with pytest.raises(kla.KlaError, match="SHAPE"):
        kla.kla_attn_fwd(q, k, v, causal=False, window=4)


def test_offsets_beyond_32_bits(kla):
    """2^31 elements and more in q, o and the gradients: the last tokens are as right as the first."""
    T, H, D = 1 << 17, 130, 128
    g = torch.Generator(device="cuda").manual_seed(18)
    q = torch.randn(1, T, H, D, generator=g, device="cuda", dtype=torch.bfloat16)
    k, v = (torch.randn(1, T, 65, D, generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    assert q.numel() > 2 ** 31
    o, lse = kla.kla_attn_fwd(q, k, v, window=20)
    grads = kla.kla_attn_bwd(q, k, v, o, lse, q, window=20)
    for a in (0, T // 2, T - 100):
        w = slice(max(0, a - 60), a + 100)
        part = [f64(t[0, w, 128:130]) for t in (q,)] + [f64(t[0, w, 64:]) for t in (k, v)]
        ro, _ = ao.forward(*part, D ** -0.5, window=20)
        rg = ao.backward(*part, part[0], D ** -0.5, window=20)
        b = ao.bounds(*part, D ** -0.5, 2.0 ** -8, d_o=part[0], window=20)
        inner = slice(a - w.start + (20 if a else 0), a - w.start + (100 if a == T - 100 else 60))
        for x, r, bb in ((o[0, w, 128:130], ro, b[0]), (grads["dq"][0, w, 128:130], rg[0], b[2]), (grads["dk"][0, w, 64:], rg[1], b[3]),
                         (grads["dv"][0, w, 64:], rg[2], b[4])):
            assert (abs(f64(x) - r)[inner] <= bb[inner]).all()
