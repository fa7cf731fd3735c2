"""The oracle of softmax attention (oracle/attn_oracle.py): closed forms, and its gradients against differences of its forward."""
import numpy as np
import pytest

from oracle import attn_oracle as ao

RNG = np.random.default_rng(0)


def _case(n, m, H, Hk, D):
    return RNG.standard_normal((n, H, D)), RNG.standard_normal((m, Hk, D)), RNG.standard_normal((m, Hk, D))


def test_closed_forms():
    q, k, v = _case(5, 5, 4, 2, 8)
    o, lse = ao.forward(q, k, v, 0.3)
    for h in range(4):                                      # the first token sees itself alone
        assert np.allclose(o[0, h], v[0, h // 2]) and np.isclose(lse[0, h], 0.3 * q[0, h] @ k[0, h // 2])
    o, lse = ao.forward(np.zeros_like(q), k, v, 0.3)        # equal scores: the mean
    for i in range(5):
        assert np.allclose(o[i, 3], v[:i + 1, 1].mean(0)) and np.isclose(lse[i, 3], np.log(i + 1))
    o, _ = ao.forward(q, k, v, 0.3, window=1)
    assert np.allclose(o, v.repeat(2, 1))
    o, _ = ao.forward(q, k, v, 0.3, causal=False)
    perm = RNG.permutation(5)                               # no order among the keys
    assert np.allclose(o, ao.forward(q, k[perm], v[perm], 0.3, causal=False)[0])
    o2, _ = ao.forward(q, k + 1.0, v, 0.3, causal=False)    # a shift of all scores of a row changes nothing
    assert np.allclose(o, o2)


def test_positions_and_hidden_keys():
    q, k, v = _case(6, 6, 2, 1, 8)
    whole = ao.forward(q, k, v, 0.5, window=3)
    for at in range(1, 6):                                  # the rest of a sequence over what came before
        part = ao.forward(q[at:], k, v, 0.5, first=at, window=3)
        assert np.array_equal(part[0], whole[0][at:]) and np.array_equal(part[1], whole[1][at:])
    k2, v2 = k.copy(), v.copy()
    k2[4:], v2[4:] = np.nan, np.inf
    assert np.array_equal(ao.forward(q[:4], k2, v2, 0.5)[0], ao.forward(q[:4], k, v, 0.5)[0])
    none = ao.forward(q[:2], k[:0], v[:0], 0.5)
    assert not none[0].any() and (none[1] == -np.inf).all()


@pytest.mark.parametrize("causal,window", [(True, 0), (True, 3), (False, 0)])
def test_gradients_by_differences(causal, window):
    q, k, v = _case(7, 7, 4, 2, 6)
    g = RNG.standard_normal(q.shape)
    f = lambda *x: (g * ao.forward(*x, 0.4, causal=causal, window=window)[0]).sum()
    grads = ao.backward(q, k, v, g, 0.4, causal=causal, window=window)
    for which, grad in enumerate(grads):
        for _ in range(12):
            d = RNG.standard_normal(grad.shape)
            x = [q, k, v]
            up, down = list(x), list(x)
            up[which], down[which] = x[which] + 1e-5 * d, x[which] - 1e-5 * d
            assert np.isclose((f(*up) - f(*down)) / 2e-5, (grad * d).sum(), rtol=1e-6, atol=1e-7)


def test_bounds_hold_for_a_rounded_computation():
    """An fp32 computation in numpy, with outputs rounded to 2^-8, stays within the bounds, and is not far below them (they would catch a mistake)."""
    q, k, v = (x.astype(np.float32) for x in _case(20, 20, 4, 2, 64))
    r = lambda x: (np.ascontiguousarray(x, dtype=np.float32).view(np.uint32) + 0x8000 & 0xffff0000).astype(np.uint32).view(np.float32)
    q, k, v = r(q), r(k), r(v)
    o, lse = ao.forward(*(x.astype(np.float64) for x in (q, k, v)), 0.125)
    b_o, b_lse = ao.bounds(*(x.astype(np.float64) for x in (q, k, v)), 0.125, 2.0 ** -8)
    for h in range(4):
        s = np.where(np.tri(20, dtype=bool), np.float32(0.125) * (q[:, h] @ k[:, h // 2].T), -np.inf).astype(np.float32)
        p = np.exp(s - s.max(1, keepdims=True))
        got = r((r(p) @ v[:, h // 2]) / p.sum(1, keepdims=True))
        assert (abs(got - o[:, h]) <= b_o[:, h]).all()
        assert (abs(s.max(1) + np.log(p.sum(1)) - lse[:, h]) <= b_lse[:, h]).all()
    assert (b_o < 0.02 * abs(v).max()).all()
