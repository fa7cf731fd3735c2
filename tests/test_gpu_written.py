"""The recurrence's calls that write a tensor of the caller's count as changes of it: a differentiable call that saved it refuses its backward."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("native", [True, False])
def test_what_a_call_writes_counts_as_changed(monkeypatch, native):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2605_08587_amd as kla
    kla.lib()
    if not native:
        monkeypatch.setattr(kla, "_native", kla._StepByStep)
    g = torch.Generator(device="cuda").manual_seed(1)
    N, T, H, D, eps = 2, 70, 2, 64, 1e-6
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    q, k, v, la, eta, S = r(N, T, H, D), r(N, T, H, D), r(N, T, H, D), -r(N, T, H).abs(), r(N, T, H).sigmoid(), r(N, H, D, D)
    lad, ld = -r(N, T, H, D).abs(), -r(N, H, D).abs()
    ks = k.clone().requires_grad_(True)
    one = [t[:, 0].contiguous() for t in (q, k, v, la, eta)]

    def state(**kw):
        return lambda t: kla.kla_chunk(q, ks, v, la, eta, eps, h0=t, **kw)[0]

    def value(t):
        return kla.kla_chunk(q, ks, t, la, eta, eps)[0]
    cases = {
        "decode S": (S, state(), lambda t: kla.kla_decode_step(*one, eps, t)),
        "decode diag S": (S, state(save=False), lambda t: kla.kla_decode_step_diag(*one[:3], ld, one[4], eps, t)),
        "decode out": (v[:, :1].clone(), lambda t: kla.kla_chunk(q[:, :1].contiguous(), ks[:, :1].contiguous(), t, la[:, :1].contiguous(),
                                                                 eta[:, :1].contiguous(), eps)[0],
                       lambda t: kla.kla_decode_step(*one, eps, S.clone(), out=t[:, 0])),
        "fwd out": (v, value, lambda t: kla.kla_chunk_fwd(q, k, v, la, eta, eps, out=t)),
        "fwd hT": (S, state(), lambda t: kla.kla_chunk_fwd(q, k, v, la, eta, eps, h0=t, hT=t)),
        "static": (v, value, lambda t: kla.kla_chunk_fwd_static(q, k, v, la, eta, eps, t)),
        "static hT": (S, state(), lambda t: kla.kla_chunk_fwd_static(q, k, v, la, eta, eps, torch.empty_like(v), hT=t)),
        "diag": (v, value, lambda t: kla.kla_chunk_fwd_diag(q, k, v, lad, eta, eps, out=t)),
        "diag hT": (S, state(), lambda t: kla.kla_chunk_fwd_diag(q, k, v, lad, eta, eps, hT=t)),
        "bwd": (v, value, lambda t: kla.kla_chunk_bwd(q, k, v, la, eta, eps, v, out=dict(dv=t))),
        "beta": (eta, lambda t: kla.kla_chunk(q, ks, v, la, t, eps)[0], lambda t: kla.kla_beta(k, eta, eps, out=t)),
    }
    for name, (like, use, write) in cases.items():
        t = like.clone()
        use(t).sum().backward()                          # (nothing has changed yet)
        y = use(t)
        before = t._version
        write(t)
        assert t._version > before, name
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.sum().backward()
    with torch.inference_mode():
        t = S.clone()
        kla.kla_decode_step(*one, eps, t)
        kla.kla_decode_step(*one, eps, S)
    kla.kla_decode_step(*one, eps, t)
