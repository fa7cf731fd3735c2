"""The norms before and after a block against their definitions in 64 bits: forward and backward, at the widths, strides and values where
they can go wrong."""
import pytest
import torch

from layer_cases import SUMS, bits, close, columns, randn, to_gpu
from oracle import layer_oracle as lo

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture(scope="module")
def kla():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2605_08587_amd as m
    m.lib()
    return m


def _pair(cols):
    if isinstance(cols, list):
        return cols, to_gpu(cols)
    whole, at = cols
    return [whole[..., a:a + w] for a, w in at], to_gpu(cols)


b16, f32 = torch.bfloat16, torch.float32
# every row width's kernel: 1..8192 columns, in rows of 16 bytes and not, and rows from none to more than the workgroups
WIDTHS = [1, 7, 64, 128, 200, 256, 333, 512, 520, 1000, 1024, 2002, 2048, 4096, 4100, 8192]


@pytest.mark.parametrize("D", WIDTHS)
@pytest.mark.parametrize("dtype,res", [(b16, b16), (b16, f32), (f32, f32)])
def test_add_norm(kla, D, dtype, res):
    g = torch.Generator().manual_seed(D)
    wide = (False, True, "odd")[D % 3]
    (x,), (xd,) = _pair(columns(g, (3, 11), [D], dtype, wide))
    for has_res, has_scale in ((True, True), (False, True), (True, False), (False, False)):
        print("add_norm", D, dtype, res, wide, has_res, has_scale, flush=True)
        d = dict(x=x, weight=randn(g, D), residual=2 * randn(g, 3, 11, D).to(res) if has_res else None, scale=randn(g, D) if has_scale else None)
        dy, dr = randn(g, 3, 11, D, dtype=dtype), randn(g, 3, 11, D, dtype=res)
        dev = {k: None if v is None else v.cuda().requires_grad_(True) for k, v in dict(d, x=None).items()}
        dev["x"] = xd.detach().requires_grad_(True)
        y, r = kla.kla_add_norm(**dev, eps=EPS, residual_dtype=res)
        wrt = [k for k in dev if dev[k] is not None]
        both = torch.autograd.grad((y, r), [dev[k] for k in wrt], (dy.cuda(), dr.cuda()), retain_graph=True)
        alone = torch.autograd.grad(y, [dev[k] for k in wrt], dy.cuda())
        for outs, got in (((dy, dr), both), ((dy, None), alone)):
            (y_ref, r_ref), ref = lo.gradients(lambda **k: lo.add_norm(**k, eps=EPS), d, outs)
            # where a row is one element its norm hardly depends on it: the gradient is what is left of terms that cancel
            for k, p in zip(wrt, got):
                if D > 7 or k == "weight":
                    close("d" + k, p, ref[k], SUMS)
        close("y", y, y_ref, SUMS)
        close("r", r, r_ref, SUMS)
        assert r.dtype == (res if has_res or res != dtype else dtype)


@pytest.mark.parametrize("D", WIDTHS)
@pytest.mark.parametrize("dtype", [b16, f32])
def test_gated_norm(kla, D, dtype):
    g = torch.Generator().manual_seed(1000 + D)
    H = 1 if D > 512 else 3
    wide = (False, True, "odd")[D % 3]
    cols, dev_cols = _pair(columns(g, (2, 9), [H * D, H * D], dtype, wide))
    x, gate = (t.unflatten(-1, (H, D)) for t in cols)
    w, dy = randn(g, D), randn(g, 2, 9, H, D, dtype=dtype)
    for act in ("silu", "sigmoid"):
        for first in (False, True):
            print("gated_norm", D, dtype, wide, act, first, flush=True)
            dev = [t.unflatten(-1, (H, D)).detach().requires_grad_(True) for t in dev_cols] + [w.cuda().requires_grad_(True)]
            y = kla.kla_gated_norm(*dev, eps=EPS, activation=act, gate_first=first)
            got = torch.autograd.grad(y, dev, dy.cuda())
            (y_ref,), ref = lo.gradients(lambda **k: lo.gated_norm(**k, eps=EPS, activation=act, gate_first=first), dict(x=x, gate=gate, weight=w),
                                         (dy,))
            close("y", y, y_ref, SUMS)
            for k, p in zip(("x", "gate", "weight"), got):
                if D > 7 or k == "weight" or (k == "gate" and not first):
                    close("d" + k, p, ref[k], SUMS)


def test_many_rows(kla):
    """More rows than one pass of the backward's workgroups takes: the parameters' gradients are sums over all of them."""
    g = torch.Generator(device="cuda").manual_seed(1)
    for M, D in ((40000, 128), (9001, 1000), (5000, 2048), (1500, 8192)):
        x, dy = (torch.randn(M, D, device="cuda", generator=g) for _ in range(2))
        w = torch.randn(D, device="cuda", generator=g)
        n = x.double() / torch.sqrt((x.double() ** 2).mean(-1, keepdim=True) + EPS)
        gr = kla.kla_add_norm_bwd(x, w, dy, eps=EPS)
        close("dweight", gr["dweight"], (dy.double() * n).sum(0), SUMS)
        gate = torch.randn(M, D, device="cuda", generator=g)
        gr = kla.kla_gated_norm_bwd(x[:, None], gate[:, None], w, dy[:, None], eps=EPS, activation="sigmoid")
        close("dweight", gr["dweight"], (dy.double() * n * torch.sigmoid(gate.double())).sum(0), SUMS)


def test_rows_of_zeros_and_what_is_not_finite(kla):
    """A row of zeros gives zeros, with eps = 0 too; a row that is not finite is its own affair."""
    g = torch.Generator().manual_seed(2)
    for D in (100, 1024, 3000):
        x = randn(g, 6, D, dtype=b16).cuda()
        w = randn(g, D).cuda()
        x[2] = 0
        y, r = kla.kla_add_norm_fwd(x, w, eps=0.0)
        assert not y[2].any() and torch.isfinite(y).all() and torch.equal(bits(r), bits(x))
        gr = kla.kla_add_norm_bwd(x, w, x, eps=0.0)
        assert torch.isfinite(gr["dx"]).all() and torch.isfinite(gr["dweight"]).all()
        bad = x.clone()
        bad[1, 5], bad[4, -1] = float("inf"), float("nan")
        y2, _ = kla.kla_add_norm_fwd(bad, w, eps=0.0)
        z = kla.kla_gated_norm_fwd(bad[:, None], x[:, None], w)
        z0 = kla.kla_gated_norm_fwd(x[:, None], x[:, None], w)
        for i in (0, 2, 3, 5):
            assert torch.equal(bits(y2[i]), bits(y[i])) and torch.equal(bits(z[i]), bits(z0[i]))
        assert torch.isnan(y2[4]).all()


def test_no_rows_and_large_gates(kla):
    for shape in ((0, 64), (0, 3, 64)):
        x = torch.empty(shape, device="cuda", dtype=b16)
        w = torch.ones(64, device="cuda")
        y, r = kla.kla_add_norm_fwd(x, w)
        assert y.shape == x.shape == r.shape and not kla.kla_add_norm_bwd(x, w, x)["dweight"].any()
        x = x.reshape(0, 1, 64)
        assert kla.kla_gated_norm_fwd(x, x, w).shape == x.shape and not kla.kla_gated_norm_bwd(x, x, w, x)["dweight"].any()
    x, w = torch.randn(4, 1, 64, device="cuda"), torch.ones(64, device="cuda")
    big = torch.full_like(x, 3e38)
    big[::2] *= -1
    y = kla.kla_gated_norm_fwd(x, big, w, activation="sigmoid")
    ref = lo.gated_norm(x.double().cpu(), big.double().cpu(), w.double().cpu(), 1e-6, "sigmoid", False)
    close("y", y, ref, SUMS)
    assert not kla.kla_gated_norm_fwd(x, big, w)[::2].any()


def test_the_stream_may_be_updated_in_place(kla):
    g = torch.Generator().manual_seed(3)
    x, w, r = randn(g, 50, 1024, dtype=b16).cuda(), randn(g, 1024).cuda(), randn(g, 50, 1024).cuda()
    y, r2 = kla.kla_add_norm_fwd(x, w, r)
    same = r.clone()
    y3, r3 = kla.kla_add_norm_fwd(x, w, same, residual_out=same)
    assert r3 is same and torch.equal(bits(r2), bits(r3)) and torch.equal(bits(y), bits(y3))


def test_offsets_beyond_32_bits(kla):
    M, D = 2 ** 20 + 7, 2048
    print("norms", M, D, flush=True)
    x = torch.empty(M, D, dtype=b16, device="cuda").normal_()
    w = torch.randn(D, device="cuda")
    y, r = kla.kla_add_norm_fwd(x, w, x)
    t, _ = kla.kla_add_norm_fwd(x[-9:], w, x[-9:].contiguous())
    assert torch.equal(bits(y[-9:]), bits(t))
    g = kla.kla_add_norm_bwd(x, w, y, x, d_residual_out=x)
    s = kla.kla_add_norm_bwd(x[-9:], w, t, x[-9:].contiguous(), d_residual_out=x[-9:].contiguous())
    assert torch.equal(bits(g["dx"][-9:]), bits(s["dx"])) and torch.equal(bits(g["dresidual"][-9:]), bits(s["dresidual"]))
    del r, g
    z = kla.kla_gated_norm_fwd(x.view(M, 16, 128), y.view(M, 16, 128), w[:128].contiguous())
    u = kla.kla_gated_norm_fwd(x[-9:].reshape(9, 16, 128), y[-9:].reshape(9, 16, 128), w[:128].contiguous())
    assert torch.equal(bits(z[-9:]), bits(u))


@pytest.mark.parametrize("D", [3, 4, 5, 8, 9, 15, 127, 129, 1025, 2047, 4099, 8191])
def test_widths_around_vectors(kla, D):
    """Rows whose last vector is short, or that have none."""
    for dtype, res in ((b16, f32), (f32, f32)):
        test_add_norm(kla, D, dtype, res)
        test_gated_norm(kla, D, dtype)


def test_in_place_where_waves_share_columns(kla):
    """The stream updated in place at widths whose last vector begins within one of another wave's: the bits of the call with a stream of
    its own, in many rows at once."""
    for dtype, res, widths in ((b16, b16, (1025, 1031, 1537, 2047, 2049, 4097, 8185)), (b16, f32, (1025, 1031, 1537, 2047, 2049, 8185)),
                               (f32, f32, (513, 1025, 1027, 2047, 2049, 4097, 8189))):
        for D in widths:
            print("add_norm in place", dtype, res, D, flush=True)
            g = torch.Generator().manual_seed(D)
            x, w, s = randn(g, 700, D, dtype=dtype).cuda(), randn(g, D).cuda(), randn(g, D).cuda()
            r, dy, dr = randn(g, 700, D).to(res).cuda(), randn(g, 700, D, dtype=dtype).cuda(), randn(g, 700, D).to(res).cuda()
            y, r2 = kla.kla_add_norm_fwd(x, w, r, s, eps=EPS)
            same = r.clone()
            y3, r3 = kla.kla_add_norm_fwd(x, w, same, s, eps=EPS, residual_out=same)
            assert r3 is same and torch.equal(bits(r2), bits(r3)) and torch.equal(bits(y), bits(y3))
            close("r", r3, r.double() + s.double() * x.double(), SUMS)
            # and the gradient of the stream in the place of the one that comes in, which the C ABI permits
            own = kla.kla_add_norm_bwd(x, w, dy, r, s, EPS, dr)
            ws = torch.empty(kla.lib().kla_add_norm_bwd_workspace_bytes(700, D, 1 if dtype == b16 else 0), dtype=torch.uint8, device="cuda")
            dx, dw, ds = torch.empty_like(x), torch.empty_like(w), torch.empty_like(s)
            rc = kla.lib().kla_add_norm_bwd(*(v.data_ptr() if torch.is_tensor(v) else v for v in (
                x, D, r, s, w, EPS, dy, dr, dx, dr, ds, dw, 700, D, 1 if dtype == b16 else 0, 1 if res == b16 else 0, ws, ws.numel(),
                torch.cuda.current_stream().cuda_stream)))
            assert rc == 0
            for k, t in (("dx", dx), ("dresidual", dr), ("dscale", ds), ("dweight", dw)):
                assert torch.equal(bits(own[k]), bits(t)), k


@pytest.mark.parametrize("D", [5, 64, 1000, 2048])
def test_rows_whose_squares_are_denormal(kla, D):
    """eps = 0 and rows so small that the mean of their squares has no leading 1 in fp32: normalised like any other.  Squares that fp32 cannot hold at all
    make a row of zeros."""
    g = torch.Generator().manual_seed(D)
    x, w, gate = randn(g, 7, D), randn(g, D), randn(g, 7, D)
    size = torch.tensor([1.0, 1e-18, 3e-20, 1e-20, 3e-21, 1e-21, 1e-26])[:, None]
    x = (x.sign() * (0.5 + x.abs())) * size
    print("norms", D, flush=True)
    y, _ = kla.kla_add_norm_fwd(x.cuda(), w.cuda(), eps=0.0)
    z = kla.kla_gated_norm_fwd(x[:, None].cuda(), gate[:, None].cuda(), w.cuda(), eps=0.0, activation="sigmoid")
    ref = lo.add_norm(x.double(), w.double(), None, None, 0.0)[0]
    ref_z = lo.gated_norm(x.double(), gate.double(), w.double(), 0.0, "sigmoid", False)
    for i in range(6):
        # an element's square rounds to a multiple of 2^-149, by half of one at most: against a mean square of at least size^2 / 4
        b = SUMS + 0.5 * 2.0 ** -149 / (float(size[i]) ** 2 / 4)
        close("y %d" % i, y[i], ref[i], b)
        close("gated %d" % i, z[i, 0], ref_z[i], b)
    assert not y[6].any() and not z[6].any()
    dx = kla.kla_add_norm_bwd(x[:4].cuda(), w.cuda(), (gate[:4] * size[:4]).cuda(), eps=0.0)["dx"]
    _, ref = lo.gradients(lambda x: lo.add_norm(x, w.double(), None, None, 0.0)[0], dict(x=x[:4]), ((gate * size)[:4],))
    for i in range(4):
        if D > 7:                                        # (narrow rows: what is left of terms that cancel)
            close("dx %d" % i, dx[i], ref["x"][i], 4 * (SUMS + 0.5 * 2.0 ** -149 / (float(size[i]) ** 2 / 4)))


@pytest.mark.parametrize("D", [9, 100, 333, 1001, 2047, 8191])
@pytest.mark.parametrize("dtype", [b16, f32])
def test_infinities_where_vectors_overlap(kla, D, dtype):
    """An infinity in a column that two vectors of a row share counts once: the row's other elements are 0 and its own a NaN, as by the definition, wherever it
    stands; and so do infinities in the gradient."""
    g = torch.Generator().manual_seed(D)
    w = randn(g, D)
    cols = sorted({0, 3, D - 1, D - 2, D - 3, D - 4, D - 5, D - 6, D - 7, D - 8, D - 9} & set(range(D)))
    x, gate, dy = (randn(g, len(cols), D, dtype=dtype) for _ in range(3))
    bad = x.clone()
    bad[torch.arange(len(cols)), cols] = float("inf")
    print("norms", D, dtype, flush=True)
    y, _ = kla.kla_add_norm_fwd(bad.cuda(), w.cuda(), eps=EPS)
    z = kla.kla_gated_norm_fwd(bad[:, None].cuda(), gate[:, None].cuda(), w.cuda(), eps=EPS)[:, 0]
    for t in (y, z):
        t = t.cpu()
        for r, c in enumerate(cols):
            assert torch.isnan(t[r, c]) and not t[r, :c].any() and not t[r, c + 1:].any(), (r, c)
    # an infinite gradient at one element: the definition's infinities everywhere, with their signs
    wild = dy.clone()
    wild[torch.arange(len(cols)), cols] = float("inf")
    for f, at in ((lambda t: kla.kla_add_norm_bwd(x.cuda(), w.cuda(), t.cuda(), eps=EPS)["dx"], None),
                  (lambda t: kla.kla_gated_norm_bwd(x[:, None].cuda(), gate[:, None].cuda(), w.cuda(), t[:, None].cuda(), eps=EPS)["dx"][:, 0], gate)):
        dx = f(wild).cpu().double()
        e = wild.double() * w.double() * (1 if at is None else at.double() * torch.sigmoid(at.double()))
        n = lo._normed(x.double(), EPS)
        ref = e - n * (e * n).mean(-1, keepdim=True)
        assert torch.equal(torch.isnan(dx), torch.isnan(ref))
        assert torch.equal(dx[~torch.isnan(ref)], ref[~torch.isnan(ref)])
