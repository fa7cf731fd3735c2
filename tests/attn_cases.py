"""Inputs and comparisons of the tests of softmax attention: against oracle/attn_oracle.py, element by element, within its bounds."""
import numpy as np
import torch

from oracle import attn_oracle as ao

U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def f64(t):
    return t.detach().double().cpu().numpy()


def randn(gen, *shape, dtype=torch.float32, wide=False, sharp=1.0):
    """A GPU tensor; wide: the first columns of a wider one whose others are NaN."""
    x = (torch.randn(shape, generator=gen, device="cuda") * sharp).to(dtype)
    if not wide:
        return x
    w = torch.full((*shape[:-2], shape[-2] * shape[-1] + 24), float("nan"), device="cuda", dtype=dtype)
    w[..., 8:8 + shape[-2] * shape[-1]] = x.flatten(-2)
    return w[..., 8:8 + shape[-2] * shape[-1]].unflatten(-1, shape[-2:])


def offsets(lengths):
    return torch.tensor(np.concatenate([[0], np.cumsum(lengths)]), dtype=torch.int32)


def within(name, x, ref, bound):
    x = f64(x)
    assert x.shape == ref.shape, (name, x.shape, ref.shape)
    assert np.isfinite(x).all(), name
    over = abs(x - ref) - bound
    assert x.size == 0 or over.max() <= 0, "%s: off by %.3g at %s, at most %.3g" % (
        name, abs(x - ref).flat[over.argmax()], np.unravel_index(over.argmax(), x.shape), bound.flat[over.argmax()])


def check(lengths, q, k, v, o, lse, scale, causal, window, d_o=None, grads=None, tag="", rest=False):
    """Flattened tokens [M, heads, D] of sequences of these lengths, against the oracle."""
    u, at = U[q.dtype], 0
    for n in lengths:
        here = slice(at, at + n)
        a = [f64(t[here]) for t in (q, k, v)]
        kw = dict(causal=causal, window=window)
        ro, rl = ao.forward(*a, scale, **kw)
        g = None if d_o is None else f64(d_o[here])
        b = ao.bounds(*a, scale, u, d_o=g, rest=rest, **kw)
        within(tag + " o", o[here], ro, b[0])
        within(tag + " lse", lse[here], rl, b[1])
        if g is not None:
            for name, x, r, bb in zip(("dq", "dk", "dv"), grads, ao.backward(*a, g, scale, **kw), b[2:]):
                within(tag + " " + name, x[here], r, bb)
        at += n


# Batches that come to at least 512 tiles of 128 query rows: lengths, packed or not, query heads of a key head, key heads, causal, window
MANY_TILES = {
    "one head each": ([140], False, 1, 260, True, 0),
    "groups of three": ([200], False, 3, 104, True, 0),
    "packed, groups of four, window": ([130, 1, 257, 60], True, 4, 31, True, 70),
    "packed, window, one head each": ([200, 0, 129, 300], True, 1, 75, True, 33),
    "both ways": ([150, 150], False, 1, 130, False, 0),
    "packed, both ways, groups of four": ([129, 64], True, 4, 74, False, 0),
}


def many_tiles(name):
    lengths, _packed, G, Hk, _causal, _window = MANY_TILES[name]
    return sum(-(-n * G // 128) for n in lengths) * Hk
