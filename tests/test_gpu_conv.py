"""Short causal convolution against its definition in 64 bits: forward, backward, single tokens, at the lengths, widths, strides and
values where it can go wrong."""
import pytest
import torch

from layer_cases import SUMS, bits, close, columns, offsets, randn, to_gpu
from oracle import layer_oracle as lo

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kla():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2605_08587_amd as m
    m.lib()
    return m


def _inputs(dtype, N, T, D, W, lens, bias, state, wide, seed):
    g = torch.Generator().manual_seed(seed)
    lead = (1, sum(lens)) if lens else (N, T)
    n = len(lens) if lens else N
    cols = columns(g, lead, [D], dtype, wide)
    x = cols[0] if isinstance(cols, list) else to_cpu(cols)[0]
    d = dict(x=x, weight=randn(g, D, W), bias=randn(g, D) if bias else None, state=randn(g, n, W - 1, D, dtype=dtype) if state else None)
    dev = {k: None if v is None else v.cuda() for k, v in d.items()}
    dev["x"] = to_gpu(cols)[0]
    dy, ds = randn(g, *lead, D, dtype=dtype), randn(g, n, W - 1, D, dtype=dtype)
    return d, dev, dy, ds, (None if not lens else offsets(lens))


def to_cpu(cols):
    whole, at = cols
    return [whole[..., a:a + w] for a, w in at]


CASES = [
    # dtype, N, T, D, W, lens, bias, state, silu, wide
    (torch.bfloat16, 1, 1, 8, 4, None, True, True, True, False),
    (torch.bfloat16, 2, 3, 64, 4, None, True, False, True, False),
    (torch.bfloat16, 3, 131, 1000, 4, None, False, True, True, True),
    (torch.bfloat16, 2, 70, 33, 3, None, True, True, True, "odd"),
    (torch.bfloat16, 1, 0, 1032, 4, [1, 2, 3, 0, 200, 4, 0, 65], True, True, True, False),
    (torch.bfloat16, 1, 0, 512, 2, [0, 0, 5, 0], False, True, False, True),
    (torch.bfloat16, 1, 0, 40, 4, [2, 1, 0, 1, 2, 33, 31, 32], True, False, True, "odd"),
    (torch.float32, 1, 2, 5, 4, None, True, True, True, False),
    (torch.float32, 2, 97, 260, 4, None, True, True, True, True),
    (torch.float32, 1, 257, 7, 3, None, False, False, False, "odd"),
    (torch.float32, 1, 0, 128, 4, [16, 15, 1, 17, 128, 3], True, True, True, False),
    (torch.float32, 4, 20, 2, 2, None, True, True, True, False),
]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_against_definition(kla, case):
    dtype, N, T, D, W, lens, bias, state, silu, wide = CASES[case]
    print("conv", CASES[case], flush=True)
    d, dev, dy, ds, cu = _inputs(dtype, N, T, D, W, lens, bias, state, wide, 100 + case)
    seqs = lo.sequences(N, T, cu)
    flat = dict(d, x=d["x"].reshape(-1, D))
    (y_ref, last_ref), g_ref = lo.gradients(lambda **k: lo.conv(**k, seqs=seqs, silu=silu), flat, (dy.reshape(-1, D), ds))
    packed = {} if cu is None else dict(cu_seqlens=cu.cuda(), cu_seqlens_host=cu)
    y, last = kla.kla_conv_fwd(**dev, silu=silu, **packed)
    torch.cuda.synchronize()
    close("y", y.reshape(-1, D), y_ref, SUMS)
    assert torch.equal(last.cpu().double(), last_ref)
    g = kla.kla_conv_bwd(dev["x"], dev["weight"], dy.cuda(), dev["bias"], dev["state"], ds.cuda(), silu=silu, **packed)
    torch.cuda.synchronize()
    close("dx", g["dx"].reshape(-1, D), g_ref["x"], SUMS)
    close("dweight", g["dweight"], g_ref["weight"], SUMS)
    for n, r in (("dbias", "bias"), ("dstate", "state")):
        assert (g[n] is None) == (d[r] is None)
        if g[n] is not None:
            close(n, g[n], g_ref[r], SUMS)
    # without a gradient of the states, through autograd, the same call twice
    leaves = {k: None if v is None else v.detach().requires_grad_(True) for k, v in dev.items()}
    y2, none = kla.kla_conv(**leaves, silu=silu, **packed)
    assert none is None and torch.equal(bits(y2.detach()), bits(y))
    wrt = [v for v in leaves.values() if v is not None]
    a = torch.autograd.grad(y2, wrt, dy.cuda(), retain_graph=True)
    b = torch.autograd.grad(y2, wrt, dy.cuda())
    assert all(torch.equal(bits(p), bits(q)) for p, q in zip(a, b))
    _, g_ref = lo.gradients(lambda **k: lo.conv(**k, seqs=seqs, silu=silu)[0], flat, (dy.reshape(-1, D),))
    for (k, v), p in zip(((k, v) for k, v in leaves.items() if v is not None), a):
        close("autograd " + k, p.reshape(g_ref[k].shape), g_ref[k], SUMS)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("W", [2, 3, 4])
@pytest.mark.parametrize("wide", [False, True, "odd"])
def test_step_by_step_is_the_whole(kla, dtype, W, wide):
    """Token by token from a state, the whole at once and the whole in two halves agree to the bit: the same sums in the same order."""
    g = torch.Generator().manual_seed(W)
    B, T, D = 3, 9, 40
    x = to_gpu(columns(g, (B, T), [D], dtype, wide))[0]
    w, b, st = randn(g, D, W).cuda(), randn(g, D).cuda(), randn(g, B, W - 1, D, dtype=dtype).cuda()
    print("conv step", dtype, W, wide, flush=True)
    y, last = kla.kla_conv_fwd(x, w, b, st)
    one = st.clone()
    ys = [kla.kla_conv_step(x[:, t], w, one, b) for t in range(T)]
    h1, mid = kla.kla_conv_fwd(x[:, :4].contiguous(), w, b, st)
    h2, end = kla.kla_conv_fwd(x[:, 4:].contiguous(), w, b, mid)
    torch.cuda.synchronize()
    assert torch.equal(bits(torch.stack(ys, 1)), bits(y)) and torch.equal(bits(one), bits(last))
    assert torch.equal(bits(torch.cat([h1, h2], 1)), bits(y)) and torch.equal(bits(end), bits(last))


def test_other_sequences_do_not_reach_in(kla):
    """NaN and infinities in one packed sequence leave the others' outputs and gradients as they are, to the bit."""
    g = torch.Generator().manual_seed(5)
    lens, D = [7, 33, 2, 90], 96
    cu = offsets(lens)
    x, dy = randn(g, 1, sum(lens), D, dtype=torch.bfloat16).cuda(), randn(g, 1, sum(lens), D, dtype=torch.bfloat16).cuda()
    w = randn(g, D, 4).cuda()
    bad = x.clone()
    bad[:, 7:40] = float("nan")
    bad[:, 40:42] = float("inf")
    out = []
    for t in (x, bad):
        y, _ = kla.kla_conv_fwd(t, w, cu_seqlens=cu.cuda(), cu_seqlens_host=cu)
        gr = kla.kla_conv_bwd(t, w, dy, cu_seqlens=cu.cuda(), cu_seqlens_host=cu)
        out.append((y, gr["dx"]))
    torch.cuda.synchronize()
    for p, q in zip(*out):
        for lo_, hi in ((0, 7), (42, 132)):
            assert torch.equal(bits(p[:, lo_:hi]), bits(q[:, lo_:hi]))


def test_no_tokens(kla):
    w, b = torch.randn(24, 4).cuda(), torch.randn(24).cuda()
    for shape in ((0, 5, 24), (3, 0, 24)):
        x = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
        st = torch.randn(shape[0], 3, 24, device="cuda").to(torch.bfloat16)
        y, last = kla.kla_conv_fwd(x, w, b, st)
        assert y.shape == x.shape and torch.equal(bits(last), bits(st))
        ds = torch.randn(shape[0], 3, 24, device="cuda").to(torch.bfloat16)
        g = kla.kla_conv_bwd(x, w, x, b, st, ds)
        assert not g["dweight"].any() and not g["dbias"].any() and torch.equal(bits(g["dstate"]), bits(ds))
    assert kla.kla_conv_step(torch.empty(0, 24, device="cuda"), w, torch.empty(0, 3, 24, device="cuda")).shape == (0, 24)


def test_offsets_beyond_32_bits(kla):
    """The last tokens of a batch of more than 2^31 elements: as those tokens alone from the state before them."""
    D, T = 4096, 2 ** 19 + 4099
    print("conv", T, D, flush=True)
    x = torch.empty(1, T, D, dtype=torch.bfloat16, device="cuda").normal_()
    w = torch.randn(D, 4).cuda()
    y, last = kla.kla_conv_fwd(x, w)
    tail, end = kla.kla_conv_fwd(x[:, -40:].contiguous(), w, state=x[:, -43:-40].contiguous())
    assert torch.equal(bits(y[:, -40:]), bits(tail)) and torch.equal(bits(last), bits(end))
    del y
    g = kla.kla_conv_bwd(x, w, x)
    t = kla.kla_conv_bwd(x[:, -40:].contiguous(), w, x[:, -40:].contiguous(), state=x[:, -43:-40].contiguous())
    assert torch.equal(bits(g["dx"][:, -40:]), bits(t["dx"]))


@pytest.mark.parametrize("D", [1, 3, 4, 5, 8, 9, 13, 255, 517, 1027])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_widths_around_vectors(kla, D, dtype):
    """Rows whose last vector begins within the one before it, or that have none: alike, every value written twice included."""
    g = torch.Generator().manual_seed(D)
    lens = [3, 0, 70, 1, 40]
    cu, M = offsets(lens), sum(lens)
    x, w, b = randn(g, 1, M, D, dtype=dtype), randn(g, D, 4), randn(g, D)
    st, dy, ds = randn(g, 5, 3, D, dtype=dtype), randn(g, 1, M, D, dtype=dtype), randn(g, 5, 3, D, dtype=dtype)
    print("conv", D, dtype, flush=True)
    seqs = lo.sequences(1, M, cu)
    (y_ref, last_ref), ref = lo.gradients(lambda **k: lo.conv(**k, seqs=seqs, silu=True), dict(x=x[0], weight=w, bias=b, state=st), (dy[0], ds))
    packed = dict(cu_seqlens=cu.cuda(), cu_seqlens_host=cu)
    y, last = kla.kla_conv_fwd(x.cuda(), w.cuda(), b.cuda(), st.cuda(), **packed)
    got = kla.kla_conv_bwd(x.cuda(), w.cuda(), dy.cuda(), b.cuda(), st.cuda(), ds.cuda(), **packed)
    close("y", y[0], y_ref, SUMS)
    assert torch.equal(last.cpu().double(), last_ref)
    for k, v in (("x", got["dx"][0]), ("weight", got["dweight"]), ("bias", got["dbias"]), ("state", got["dstate"])):
        close("d" + k, v, ref[k], SUMS)


def _whole(x, weight, bias, state, seqs, silu):
    """The definition a sequence and a tap at a time, for lengths at which token by token takes too long."""
    ys, lasts, W = [], [], weight.shape[1]
    for n, (lo_, hi) in enumerate(seqs):
        line = torch.cat([x.new_zeros(W - 1, x.shape[1]) if state is None else state[n], x[lo_:hi]])
        p = sum(line[j:j + hi - lo_] * weight[:, j] for j in range(W)) + bias
        ys.append(p * torch.sigmoid(p) if silu else p)
        lasts.append(line[hi - lo_:])
    return torch.cat(ys), torch.stack(lasts)


@pytest.mark.parametrize("dtype,W,silu,state,wide", [(torch.bfloat16, 4, True, True, "odd"), (torch.float32, 3, False, True, False),
                                                     (torch.float32, 4, True, False, True), (torch.bfloat16, 2, False, True, False)])
def test_long_strips_of_packed_batches(kla, dtype, W, silu, state, wide):
    """As many tokens and channels as are taken in strips of 32 forward and 64 backward, whose sequences begin and end within them: every output and
    gradient, those of the states from both sides among them."""
    lens, D = [1, 0, 70, 5000, 63, 64, 65, 2, 9500, 3], 2051
    print("conv strips", dtype, W, silu, state, wide, flush=True)
    d, dev, dy, ds, cu = _inputs(dtype, 0, 0, D, W, lens, True, state, wide, 300 + W)
    M = sum(lens)
    assert M // 64 * ((D + 255) // 256) > 2048           # (the rule's side that the other tests are not on)
    seqs = lo.sequences(0, 0, cu)
    flat = dict(d, x=d["x"].reshape(-1, D))
    (y_ref, last_ref), ref = lo.gradients(lambda **k: _whole(**k, seqs=seqs, silu=silu), flat, (dy.reshape(-1, D), ds))
    short = {k: v if v is None else v[..., :5].double() if k in ("x", "state") else v[:5].double() for k, v in flat.items()}
    short["x"], few = short["x"][:71], seqs[:3]          # (the same definition)
    for p, q in zip(lo.conv(**short, seqs=few, silu=silu), _whole(**short, seqs=few, silu=silu)):
        assert torch.allclose(p, q, rtol=0, atol=1e-12)
    packed = dict(cu_seqlens=cu.cuda(), cu_seqlens_host=cu)
    y, last = kla.kla_conv_fwd(**dev, silu=silu, **packed)
    got = kla.kla_conv_bwd(dev["x"], dev["weight"], dy.cuda(), dev["bias"], dev["state"], ds.cuda(), silu=silu, **packed)
    close("y", y.reshape(-1, D), y_ref, SUMS)
    assert torch.equal(last.cpu().double(), last_ref)
    for k, v in (("x", got["dx"].reshape(-1, D)), ("weight", got["dweight"]), ("bias", got["dbias"]), ("state", got["dstate"])):
        if v is not None:
            close("d" + k, v, ref[k], SUMS)
