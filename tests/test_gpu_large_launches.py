"""Calls whose work is more than the 2^32 - 1 threads that one launch can have: the tokens, rows and sequences at the far end come out as they do by
themselves."""
import pytest
import torch

from layer_cases import SCAN, SUMS, bits, close

pytestmark = pytest.mark.gpu
b16 = torch.bfloat16
MOST = 0xffffffff // 256                                # workgroups of 256 threads


@pytest.fixture(scope="module")
def kla():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2605_08587_amd as m
    m.lib()
    torch.cuda.empty_cache()
    yield m
    torch.cuda.empty_cache()


def _randn(*shape, dtype=b16):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_()


def test_conv_step(kla):
    B, D = MOST + 6, 8
    print("conv step", B, D, flush=True)
    x, w, st = _randn(B, D), _randn(D, 2, dtype=torch.float32), _randn(B, 1, D)
    part = [slice(0, 5), slice(MOST - 3, MOST + 6)]
    ref = [(kla.kla_conv_step(x[p], w, s, silu=False), s) for p, s in ((p, st[p].clone()) for p in part)]
    y = kla.kla_conv_step(x, w, st, silu=False)
    for p, (a, s) in zip(part, ref):
        assert torch.equal(bits(y[p]), bits(a)) and torch.equal(bits(st[p]), bits(s))


def test_ssm_step(kla):
    N, D, S = MOST + 6, 1, 8
    print("ssm step", N, D, flush=True)
    u, z, B, C = _randn(N, D), _randn(N, D), _randn(N, 1, S), _randn(N, 1, S)
    A, h = -torch.ones(D, S, device="cuda"), _randn(N, D, S, dtype=torch.float32)
    part = [slice(0, 5), slice(MOST - 3, MOST + 6)]
    ref = [(kla.kla_ssm_step(u[p], u[p], A, B[p], C[p], s, z=z[p]), s) for p, s in ((p, h[p].clone()) for p in part)]
    y = kla.kla_ssm_step(u, u, A, B, C, h, z=z)
    for p, (a, s) in zip(part, ref):
        assert torch.equal(bits(y[p]), bits(a)) and torch.equal(bits(h[p]), bits(s))


def test_norms(kla):
    M, D = 16 * MOST + 9, 2
    print("norms", M, D, flush=True)
    x, w = _randn(M, D), torch.tensor([0.5, 2.0], device="cuda")
    part = [slice(0, 5), slice(16 * MOST - 3, 16 * MOST + 9)]
    y, r = kla.kla_add_norm_fwd(x, w, x)
    for p in part:
        a, b = kla.kla_add_norm_fwd(x[p], w, x[p].contiguous())
        assert torch.equal(bits(y[p]), bits(a)) and torch.equal(bits(r[p]), bits(b))
    del r
    z = kla.kla_gated_norm_fwd(x.view(M // 3, 3, D), y.view(M // 3, 3, D), w)
    for p in (slice(0, 5), slice(M // 3 - 9, M // 3)):
        a = kla.kla_gated_norm_fwd(x.view(M // 3, 3, D)[p].contiguous(), y.view(M // 3, 3, D)[p].contiguous(), w)
        assert torch.equal(bits(z[p]), bits(a))


def test_gradients_of_many_parameters(kla):
    """The sums over workgroups: a column for every tap and bias."""
    D, W = (0xffffffff // 1024 * 64) // 3 + 100, 2
    print("conv", D, flush=True)
    x, w, b, dy = _randn(1, 2, D), _randn(D, W, dtype=torch.float32), _randn(D, dtype=torch.float32), _randn(1, 2, D)
    g = kla.kla_conv_bwd(x, w, dy, b)
    for p in (slice(0, 200), slice(D - 200, D)):
        a = kla.kla_conv_bwd(x[..., p].contiguous(), w[p].contiguous(), dy[..., p].contiguous(), b[p].contiguous())
        assert torch.equal(bits(g["dx"][..., p]), bits(a["dx"]))
        close("dweight", g["dweight"][p], a["dweight"], SUMS)
        close("dbias", g["dbias"][p], a["dbias"], SUMS)


def test_scan_of_many_sequences_and_groups(kla):
    """A group of its own for every channel and 4100 sequences of one token: 2^32 threads of the scan, most of which have no channel."""
    N, D, S = 4100, 4096, 8
    assert N * D > MOST
    print("ssm", N, D, flush=True)
    f = torch.float32
    u, z, dy, B, C = _randn(N, 1, D), _randn(N, 1, D), _randn(N, 1, D), _randn(N, 1, D, S), _randn(N, 1, D, S)
    A, h0, dh = -torch.rand(D, S, device="cuda"), _randn(N, D, S, dtype=f), _randn(N, D, S, dtype=f)
    y, hT = kla.kla_ssm_fwd(u, u, A, B, C, z=z, h0=h0)
    g = kla.kla_ssm_bwd(u, u, A, B, C, dy, z=z, h0=h0, d_hT=dh)
    for p in (slice(0, 3), slice(N - 60, N)):
        x = dict(u=u[p], delta=u[p], A=A, B=B[p], C=C[p], z=z[p], h0=h0[p])
        a, b = kla.kla_ssm_fwd(**x)
        assert torch.equal(bits(y[p]), bits(a)) and torch.equal(bits(hT[p]), bits(b))
        q = kla.kla_ssm_bwd(**x, d_y=dy[p], d_hT=dh[p])
        for k in ("du", "ddelta", "dz", "dB", "dC", "dh0"):
            assert torch.equal(bits(g[k][p]), bits(q[k])), k
    dA = torch.zeros(D, S, dtype=torch.float64, device="cuda")
    for p in range(0, N, 300):
        d = torch.nn.functional.softplus(u[p:p + 300, 0].double())[..., None]
        zd = z[p:p + 300, 0].double()
        gh = (dy[p:p + 300, 0].double() * zd * torch.sigmoid(zd))[..., None] * C[p:p + 300, 0].double() + dh[p:p + 300].double()
        dA += (gh * torch.exp(d * A.double()) * h0[p:p + 300].double() * d).sum(0)
    close("dA", g["dA"], dA, SCAN)


def test_scan_of_many_tokens(kla):
    """The gradients of B and C of more than 2^28 tokens."""
    N, T, D, S = 64, 2 ** 22 + 16, 1, 8
    print("ssm", N, T, flush=True)
    u, B, C, dy = _randn(N, T, D), _randn(N, T, 1, S), _randn(N, T, 1, S), _randn(N, T, D)
    A = -torch.arange(1.0, S + 1, device="cuda").repeat(D, 1)
    assert N * T * 2 * S > 256 * MOST
    g = kla.kla_ssm_bwd(u, u, A, B, C, dy)
    for n in (0, N - 1):
        p = slice(n, n + 1)
        q = kla.kla_ssm_bwd(u[p], u[p], A, B[p], C[p], dy[p])
        for k in ("dB", "dC"):
            # (cut into other segments: two orders of the same sums, each rounded once)
            close(k, g[k][p], q[k], 2 * SCAN + 2.0 ** -8)


def test_beta(kla):
    """The recurrence's write coefficients of more than 2^29 tokens and heads."""
    n, dk = 32 * MOST + 9, 64
    print("beta", n, flush=True)
    k, eta = torch.empty(n, dk, dtype=b16, device="cuda").fill_(0.5), torch.rand(n, device="cuda")
    k[-9:] = _randn(9, dk)
    beta = kla.kla_beta(k, eta, 1e-6)
    for p in (slice(0, 7), slice(n - 40, n)):
        assert torch.equal(bits(beta[p]), bits(kla.kla_beta(k[p], eta[p].clone(), 1e-6)))
