"""Inputs and comparisons of the tests of the operators around the recurrence."""
import torch

# max |x - ref| / max |ref|.  bf16 results are rounded once: half a unit in the last of 8 bits is 2^-8 of a value at most, and
# what is in fp32 before it adds at most the fp32 bar.  fp32: convolution and norms are sums of a few terms or pairwise sums over a row, about
# 20 roundings of 2^-24 and functions of 2 units each: 4e-6.  The scan carries its state: every step rounds the exponent and the state,
# which stay in it for as many tokens as it remembers, up to a few hundred here: 2e-5.
BF16, SUMS, SCAN = 2.0 ** -8, 4e-6, 2e-5


def bar(dtype, base):
    return base + (BF16 if dtype == torch.bfloat16 else 0.0)


def off(x, ref):
    x, ref = x.detach().double().cpu(), ref.detach().double().cpu()
    assert x.shape == ref.shape, (x.shape, ref.shape)
    assert torch.isfinite(x).all()
    if not x.numel():
        return 0.0
    top = float(ref.abs().max())
    return float((x - ref).abs().max()) / (top if top else 1.0)


def close(name, x, ref, base):
    e, b = off(x, ref), bar(x.dtype, base)
    assert e <= b, "%s: %.3g, at most %.3g" % (name, e, b)


def bits(t):
    return t.contiguous().view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)


def randn(gen, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=gen).to(dtype)


def columns(gen, lead, widths, dtype, wide):
    """CPU tensors [*lead, w], apart or as ranges of one wider tensor whose other columns are NaN."""
    if not wide:
        return [randn(gen, *lead, w, dtype=dtype) for w in widths]
    pad = 3 if wide == "odd" else 8
    whole = torch.full((*lead, sum(widths) + pad * (len(widths) + 1)), float("nan"), dtype=dtype)
    out, at = [], pad
    for w in widths:
        whole[..., at:at + w] = randn(gen, *lead, w, dtype=dtype)
        out.append((at, w))
        at += w + pad
    return whole, out


def to_gpu(cols):
    if isinstance(cols, list):
        return [t.cuda() for t in cols]
    whole, at = cols
    whole = whole.cuda()
    return [whole[..., a:a + w] for a, w in at]


def offsets(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return torch.tensor(cu, dtype=torch.int32)
