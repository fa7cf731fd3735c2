"""The differentiable calls under torch.inference_mode, packed, with tensors made outside of it and inside (which count no changes): they are
forwards like any other, natively and step by step."""
import pytest
import torch

from layer_cases import bits, offsets

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("inside", [True, False])
def test_packed_forwards(monkeypatch, native, inside):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2605_08587_amd as kla
    kla.lib()
    if not native:
        monkeypatch.setattr(kla, "_native", kla._StepByStep)
    g = torch.Generator(device="cuda").manual_seed(1)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    T, D, S, H = 90, 128, 16, 2
    d = dict(x=r(1, T, D), w=r(D, 4), A=-r(D, S).abs(), B=r(1, T, 1, S), q=r(1, T, H, 64), la=-r(1, T, H).abs(), eta=r(1, T, H).sigmoid())
    host = offsets([40, 0, 50])
    dev = host.cuda()

    def calls(x, w, A, B, q, la, eta, dev, host):
        kw = dict(cu_seqlens=dev, cu_seqlens_host=host)
        return (kla.kla_conv(x, w, **kw)[0], *kla.kla_ssm(x, x, A, B, B, **kw), *kla.kla_chunk(q, q, q, la, eta, 1e-6, **kw),
                kla.kla_conv(x, w, cu_seqlens=dev)[0])
    ref = calls(**d, dev=dev, host=host)
    with torch.inference_mode():
        if inside:
            d, dev, host = {k: v.clone() for k, v in d.items()}, dev.clone(), host.clone()
            assert dev.is_inference()
        out = calls(**d, dev=dev, host=host)
    assert all(torch.equal(bits(a), bits(b)) for a, b in zip(ref, out))
