"""The operators around the recurrence through the native half of the binding and step by step in Python: the same bits, the same refusals."""
import pytest
import torch

from layer_cases import bits, offsets

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kla():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2605_08587_amd as m
    m.lib()
    return m


def _inputs(dtype, wide, packed):
    g = torch.Generator(device="cuda").manual_seed(4)

    def r(*s, dt=dtype):
        return torch.randn(s, generator=g, device="cuda").to(dt)
    N, T, D, S, G = (1, 90, 40, 16, 2) if packed else (2, 45, 40, 16, 2)
    f = torch.float32
    whole = r(N, T, 4 * D + 2 * G * S + 5)
    x, u, delta, z, B, C = (t if wide else t.contiguous() for t in whole[..., 5:].split([D] * 4 + [G * S] * 2, -1))
    n = 3 if packed else N
    d = dict(x=x, u=u, delta=delta, z=z, B=B.unflatten(-1, (G, S)), C=C.unflatten(-1, (G, S)), w=r(D, 4, dt=f), b=r(D, dt=f), st=r(n, 3, D),
             A=-r(D, S, dt=f).abs(), skip=r(D, dt=f), bias=r(D, dt=f), h0=r(n, D, S, dt=f), dy=r(N, T, D), dst=r(n, 3, D), dh=r(n, D, S, dt=f),
             res=r(N, T, D, dt=f), dres=r(N, T, D, dt=f), w5=r(D // 5, dt=f))
    cu = offsets([40, 0, 50])
    kw = dict(cu_seqlens=cu.cuda(), cu_seqlens_host=cu) if packed else {}
    return d, kw


def _all(kla, d, kw):
    """Every entry point, forward and through autograd; what it returns."""
    out = {}
    d = dict(d)

    def heads(t):
        return t.unflatten(-1, (5, -1))
    names = ("x", "u", "delta", "z", "B", "C", "w", "b", "st", "A", "skip", "bias", "h0", "res", "w5")
    out["conv_fwd"] = kla.kla_conv_fwd(d["x"], d["w"], d["b"], d["st"], **kw)
    out["ssm_fwd"] = kla.kla_ssm_fwd(d["u"], d["delta"], d["A"], d["B"], d["C"], d["skip"], d["z"], d["bias"], h0=d["h0"], **kw)
    out["add_fwd"] = kla.kla_add_norm_fwd(d["x"], d["b"], d["res"], d["skip"])
    out["add_first"] = kla.kla_add_norm_fwd(d["x"], d["b"], residual_dtype=torch.float32)
    out["gated_fwd"] = (kla.kla_gated_norm_fwd(heads(d["x"]), heads(d["z"]), d["w5"], gate_first=True),)
    if not kw:
        st, h = d["st"].clone(), d["h0"].clone()
        y = kla.kla_conv_step(d["x"][:, 3], d["w"], st, d["b"])
        out["steps"] = (y, st, kla.kla_ssm_step(d["u"][:, 3], d["delta"][:, 3], d["A"], d["B"][:, 3], d["C"][:, 3], h, z=d["z"][:, 3]), h)
    for n in names:
        d[n] = d[n].detach().requires_grad_(True)
    y, last = kla.kla_conv(d["x"], d["w"], d["b"], d["st"], want_state=True, **kw)
    out["conv"] = (y, last, *torch.autograd.grad((y, last), [d[n] for n in ("x", "w", "b", "st")], (d["dy"], d["dst"])))
    y, h = kla.kla_ssm(d["u"], d["delta"], d["A"], d["B"], d["C"], d["skip"], d["z"], d["bias"], h0=d["h0"], **kw)
    out["ssm"] = (y, h, *torch.autograd.grad((y, h), [d[n] for n in ("u", "delta", "A", "B", "C", "skip", "z", "bias", "h0")], (d["dy"], d["dh"])))
    y, h = kla.kla_ssm(d["u"], d["delta"], d["A"], d["B"], d["C"], softplus=False, **kw)
    out["ssm, only the states"] = torch.autograd.grad(h, [d["u"], d["A"]], d["dh"])
    y, r = kla.kla_add_norm(d["x"], d["b"], d["res"], d["skip"])
    out["add"] = (y, r, *torch.autograd.grad((y, r), [d[n] for n in ("x", "b", "res", "skip")], (d["dy"], d["dres"])))
    out["add, only the stream"] = torch.autograd.grad(kla.kla_add_norm(d["x"], d["b"], d["res"])[1], [d["x"], d["b"]], d["dres"])
    y = kla.kla_gated_norm(heads(d["x"]), heads(d["z"]), d["w5"], activation="sigmoid")
    out["gated"] = (y, *torch.autograd.grad(y, [d["x"], d["z"], d["w5"]], heads(d["dy"])))
    with torch.no_grad():
        out["no grad"] = kla.kla_conv(d["x"], d["w"], **kw)[:1] + kla.kla_ssm(d["u"], d["delta"], d["A"], d["B"], d["C"], **kw)
    assert not any(t.requires_grad for t in out["no grad"])
    return out


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("packed", [False, True])
def test_same_bits(kla, monkeypatch, dtype, wide, packed):
    d, kw = _inputs(dtype, wide, packed)
    assert kla._binding().__name__ == "kla_binding"
    native = _all(kla, d, kw)
    monkeypatch.setattr(kla, "_native", kla._StepByStep)
    steps = _all(kla, d, kw)
    for k in native:
        assert len(native[k]) == len(steps[k])
        for p, q in zip(native[k], steps[k]):
            assert p.dtype == q.dtype and p.shape == q.shape and torch.equal(bits(p.detach()), bits(q.detach())), k


def test_native_takes_ordinary_calls(kla, monkeypatch):
    """What tests and benchmarks time is the native half: with Python's checks out of reach every ordinary call still works."""
    d, kw = _inputs(torch.bfloat16, True, True)
    for f in ("_conv_check", "_ssm_check", "_add_norm_check", "_gated_norm_check"):
        monkeypatch.setattr(kla.layer, f, None)
    _all(kla, d, kw)


@pytest.mark.parametrize("native", [True, False])
def test_refusals(kla, monkeypatch, native):
    if not native:
        monkeypatch.setattr(kla, "_native", kla._StepByStep)
    d, _ = _inputs(torch.bfloat16, False, False)
    x, w, A, B, C = d["x"], d["w"], d["A"], d["B"], d["C"]
    with pytest.raises(ValueError, match="contiguous"):
        kla.kla_conv_fwd(x.transpose(1, 2).contiguous().transpose(1, 2), w)
    with pytest.raises(ValueError, match="evenly"):
        kla.kla_conv_fwd(torch.zeros(2, 50, 40, device="cuda", dtype=x.dtype)[:, :45], w)
    with pytest.raises(ValueError, match="overlap"):
        kla.kla_conv_fwd(x[:1, :1].expand(2, 45, 40), w)
    with pytest.raises(TypeError):
        kla.kla_conv_fwd(x.half(), w)
    with pytest.raises(kla.KlaError, match="SHAPE"):
        kla.kla_conv_fwd(x, torch.zeros(40, 5, device="cuda"))
    with pytest.raises(kla.KlaError, match="SHAPE"):
        kla.kla_ssm_fwd(x, x, A[:, :12].contiguous(), B[..., :12].contiguous(), C[..., :12].contiguous())
    with pytest.raises(kla.KlaError, match="SHAPE"):
        kla.kla_gated_norm_fwd(torch.zeros(2, 1, 8200, device="cuda"), torch.zeros(2, 1, 8200, device="cuda"), torch.zeros(8200, device="cuda"))
    with pytest.raises(kla.KlaError, match="SEQLENS"):
        kla.kla_conv_fwd(x[:1], w, cu_seqlens=torch.tensor([0, 44], dtype=torch.int32, device="cuda"))
    with pytest.raises(TypeError, match="residual"):
        kla.kla_add_norm_fwd(x.float(), d["b"], x)
    with pytest.raises(RuntimeError, match="GPU"):
        kla.kla_conv_step(x[:, 0], w.cpu(), d["st"])

    # gradients of gradients, offsets changed before the backward
    xs = x.detach().requires_grad_(True)
    for y in (kla.kla_conv(xs, w)[0], kla.kla_ssm(xs, x, A, B, C)[0], kla.kla_add_norm(xs, d["b"])[0],
              kla.kla_gated_norm(xs[..., None, :], x[..., None, :], d["b"])):
        with pytest.raises(RuntimeError, match="create_graph"):
            torch.autograd.grad(y.sum(), xs, create_graph=True)
    cu = torch.tensor([0, 20, 45], dtype=torch.int32)
    for f in (lambda c: kla.kla_conv(xs[:1], w, cu_seqlens=c, cu_seqlens_host=cu)[0],
              lambda c: kla.kla_ssm(xs[:1], x[:1], A, B[:1], C[:1], cu_seqlens=c, cu_seqlens_host=cu)[0]):
        c = cu.cuda()
        y = f(c)
        c[1] = 21
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.sum().backward()


def test_inputs_changed_before_the_backward(kla):
    d, _ = _inputs(torch.float32, False, False)
    xs = d["x"].clone().requires_grad_(True)
    z = xs * 1
    y, _ = kla.kla_conv(z, d["w"])
    z.mul_(2)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


@pytest.mark.parametrize("native", [True, False])
def test_what_a_call_writes_counts_as_changed(kla, monkeypatch, native):
    """A tensor that a differentiable call saved and another call then writes in place: the backward refuses, as after torch's own."""
    if not native:
        monkeypatch.setattr(kla, "_native", kla._StepByStep)
    d, _ = _inputs(torch.float32, False, False)
    x, A, B, C, w, b = d["x"], d["A"], d["B"], d["C"], d["w"], d["b"]
    xs, ws = x.detach().requires_grad_(True), w.detach().clone().requires_grad_(True)
    heads = lambda t: t.unflatten(-1, (5, -1))  # noqa: E731

    def conv(**kw):
        return lambda t: kla.kla_conv(xs, w, b, t, **kw)[0]

    def ssm(**kw):
        return lambda t: kla.kla_ssm(xs, x, A, B, C, h0=t, **kw)[0]
    like = lambda t: lambda: t.clone()  # noqa: E731
    cases = {
        "conv_step state": (like(d["st"]), conv(), lambda t: kla.kla_conv_step(x[:, 0], w, t, b)),
        "conv_fwd state_out": (like(d["st"]), conv(), lambda t: kla.kla_conv_fwd(x, w, b, state_out=t)),
        "conv_fwd out": (like(x), lambda t: kla.kla_conv(t, ws)[0],
                         lambda t: kla.kla_conv_fwd(x, w, out=t)),
        "conv_step out": (like(x[:, 0]), lambda t: kla.kla_conv(t[:, None], ws)[0],
                          lambda t: kla.kla_conv_step(x[:, 0], w, d["st"].clone(), out=t)),
        "ssm_step h": (like(d["h0"]), ssm(), lambda t: kla.kla_ssm_step(x[:, 0], x[:, 1], A, B[:, 0], C[:, 0], t)),
        "ssm_fwd hT": (like(d["h0"]), ssm(save=False), lambda t: kla.kla_ssm_fwd(x, x, A, B, C, h0=t, hT=t)),
        "ssm_fwd out": (like(x), lambda t: kla.kla_ssm(xs, t, A, B, C)[0], lambda t: kla.kla_ssm_fwd(x, x, A, B, C, out=t)),
        "ssm_step out": (like(x[:, 0]), lambda t: kla.kla_ssm(xs[:, :1], t[:, None], A, B[:, :1], C[:, :1])[0],
                         lambda t: kla.kla_ssm_step(x[:, 0], x[:, 1], A, B[:, 0], C[:, 0], d["h0"].clone(), out=t)),
        "add_norm_fwd residual_out": (like(d["res"]), lambda t: kla.kla_add_norm(xs, b, t)[0], lambda t: kla.kla_add_norm_fwd(x, b, t, residual_out=t)),
        "add_norm_fwd out": (like(x), lambda t: kla.kla_add_norm(t, b, xs)[0], lambda t: kla.kla_add_norm_fwd(x, b, out=t)),
        "gated_norm_fwd out": (like(heads(x).contiguous()), lambda t: kla.kla_gated_norm(heads(xs), t, d["w5"]),
                               lambda t: kla.kla_gated_norm_fwd(heads(x), heads(x), d["w5"], out=t)),
    }
    for name, (make, use, write) in cases.items():
        t = make()
        y = use(t)
        y.sum().backward()                               # (nothing has changed yet)
        y = use(t)
        before = t._version
        write(t)
        assert t._version > before, name
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.sum().backward()
    # a tensor that counts nothing, and one that nobody saved, are written as before
    with torch.inference_mode():
        st, h = d["st"].clone(), d["h0"].clone()
    kla.kla_conv_step(x[:, 0], w, st, b)
    kla.kla_ssm_step(x[:, 0], x[:, 1], A, B[:, 0], C[:, 0], h)
    with torch.inference_mode():
        kla.kla_conv_step(x[:, 0], w, st, b)
        kla.kla_conv_step(x[:, 0], w, d["st"], b)
