"""The 64-bit definitions of the operators around the recurrence (oracle/layer_oracle.py): gradients against differences, and identities
that pin them without the library."""
import pytest
import torch

from oracle import layer_oracle as lo

H = 1e-5        # step of the differences: their own error is about H^2 = 1e-10 of third derivatives of order 1..100


def _check_gradients(f, inputs, n_outs, gen):
    outs = f(**inputs)
    outs = outs if isinstance(outs, tuple) else (outs,)
    ds = [torch.randn(o.shape, generator=gen, dtype=torch.float64) for o in outs[:n_outs]]
    _, grads = lo.gradients(f, inputs, ds)

    def total(k, v):
        r = f(**{**inputs, k: v})
        r = r if isinstance(r, tuple) else (r,)
        return float(sum((o * d).sum() for o, d in zip(r, ds)))
    for k, v in inputs.items():
        if v is None:
            continue
        way = torch.randn(v.shape, generator=gen, dtype=torch.float64)
        diff = (total(k, v + H * way) - total(k, v - H * way)) / (2 * H)
        got = float((grads[k] * way).sum())
        assert abs(diff - got) <= 1e-6 * max(1.0, abs(got)), (k, diff, got)


def _gen(seed):
    g = torch.Generator().manual_seed(seed)
    return g, lambda *s: torch.randn(s, generator=g, dtype=torch.float64)


@pytest.mark.parametrize("silu", [False, True])
@pytest.mark.parametrize("W", [2, 3, 4])
def test_conv_gradients(W, silu):
    g, r = _gen(W)
    seqs = lo.sequences(1, 0, [0, 5, 5, 6, 8])
    _check_gradients(lambda **k: lo.conv(**k, seqs=seqs, silu=silu),
                     dict(x=r(8, 3), weight=r(3, W), bias=r(3), state=r(4, W - 1, 3)), 2, g)


@pytest.mark.parametrize("softplus", [False, True])
def test_ssm_gradients(softplus):
    g, r = _gen(7)
    seqs = lo.sequences(1, 0, [0, 4, 4, 9])
    _check_gradients(lambda **k: lo.ssm(**k, softplus=softplus, seqs=seqs),
                     dict(u=r(9, 4), delta=0.3 * r(9, 4), A=-r(4, 8).abs(), B=r(9, 2, 8), C=r(9, 2, 8), skip=r(4), z=r(9, 4),
                          delta_bias=0.1 * r(4), h0=r(3, 4, 8)), 2, g)


def test_norm_gradients():
    g, r = _gen(9)
    _check_gradients(lambda **k: lo.add_norm(**k, eps=0.1), dict(x=r(5, 6), weight=r(6), residual=r(5, 6), scale=r(6)), 2, g)
    for act in ("silu", "sigmoid"):
        for first in (False, True):
            _check_gradients(lambda **k: lo.gated_norm(**k, eps=0.1, activation=act, gate_first=first),
                             dict(x=r(5, 2, 6), gate=r(5, 2, 6), weight=r(6)), 1, g)


def test_conv_is_a_padded_correlation():
    _, r = _gen(11)
    x, w, b = r(20, 5), r(5, 4), r(5)
    y, last = lo.conv(x, w, b, None, [(0, 20)], False)
    ref = torch.nn.functional.conv1d(torch.nn.functional.pad(x.t()[None], (3, 0)), w[:, None], b, groups=5)[0].t()
    assert torch.allclose(y, ref, atol=1e-12) and torch.equal(last[0], x[-3:])


def test_ssm_without_decay_is_a_running_sum():
    """A = 0, delta = 1: h is the sum of u B so far; and one token's answer is that of the whole with the state handed on."""
    _, r = _gen(13)
    u, B, C = r(12, 3), r(12, 1, 8), r(12, 1, 8)
    zero = torch.zeros(3, 8, dtype=torch.float64)
    y, hT = lo.ssm(u, torch.ones(12, 3, dtype=torch.float64), zero, B, C, None, None, None, False, None, [(0, 12)])
    h = torch.cumsum(u[:, :, None] * B, 0)
    assert torch.allclose(y, (h * C).sum(-1), atol=1e-12) and torch.allclose(hT[0], h[-1], atol=1e-12)
    A, d = -r(3, 8).abs(), r(12, 3)
    whole, end = lo.ssm(u, d, A, B, C, None, None, None, True, None, [(0, 12)])
    _, h5 = lo.ssm(u[:5], d[:5], A, B[:5], C[:5], None, None, None, True, None, [(0, 5)])
    rest, end2 = lo.ssm(u[5:], d[5:], A, B[5:], C[5:], None, None, None, True, h5, [(0, 7)])
    assert torch.allclose(whole[5:], rest, atol=1e-12) and torch.allclose(end, end2, atol=1e-12)
