"""Host-side checks of the operators around the recurrence that need no GPU: every refusal comes before anything is launched (the pointers
are fakes), the workspace queries, and what the Python functions refuse."""
import os

import numpy as np
import pytest
import torch

import paper_2605_08587_amd as kla

pytestmark = pytest.mark.skipif(not os.path.exists(kla.LIB_PATH), reason="libkla.so not built (python -m paper_2605_08587_amd.build)")

OK, E_NULL, E_SHAPE, E_DTYPE, E_ALIGN, E_WS, E_SEQ = 0, -1, -2, -3, -4, -5, -6
BF16, F32 = kla.KLA_BF16, kla.KLA_F32
CU = np.array([0, 30, 64], dtype=np.int32)
WS = dict(ws=0x100000, ws_bytes=1 << 30)


def _call(name, defaults, over):
    a = dict(defaults)
    assert set(over) <= set(a), over
    a.update(over)
    return getattr(kla.lib(), name)(*a.values())


SEQS = dict(cu_dev=None, cu_host=None, n_seq=0)
CONV = dict(x=0x1000, ld=64, w=0x2000, b=None, st=None)


def conv_fwd(**o):
    return _call("kla_conv_fwd", dict(**CONV, y=0x3000, last=None, **SEQS, N=1, T=64, D=64, W=4, dt=BF16, stream=None, opts=1), o)


def conv_bwd(**o):
    return _call("kla_conv_bwd", dict(**CONV, dy=0x3000, dlast=None, dx=0x4000, dw=0x5000, db=None, dst=None, **SEQS, N=1, T=64, D=64, W=4,
                                      dt=BF16, **WS, stream=None, opts=1), o)


def conv_step(**o):
    return _call("kla_conv_step", dict(x=0x1000, ld=64, w=0x2000, b=None, st=0x3000, y=0x4000, B=1, D=64, W=4, dt=BF16, stream=None, opts=1), o)


SSM = dict(u=0x1000, ld_u=64, delta=0x2000, ld_d=64, A=0x3000, B=0x4000, ld_B=16, C=0x5000, ld_C=16, skip=None, z=None, ld_z=0, bias=None)
SIZES = dict(N=1, T=64, D=64, G=1, S=16, dt=BF16)


def ssm_fwd(**o):
    return _call("kla_ssm_fwd", dict(**SSM, h0=None, y=0x6000, hT=None, saved=None, saved_bytes=0, **SEQS, **SIZES, **WS, stream=None, opts=2), o)


def ssm_bwd(**o):
    return _call("kla_ssm_bwd", dict(**SSM, h0=None, dy=0x6000, dhT=None, saved=None, saved_bytes=0, du=0x7000, dd=0x8000, dA=0x9000, dB=0xa000,
                                     dC=0xb000, dskip=None, dz=None, dbias=None, dh0=None, **SEQS, **SIZES, **WS, stream=None, opts=2), o)


def ssm_step(**o):
    return _call("kla_ssm_step", dict(**SSM, h=0x6000, y=0x7000, N=1, D=64, G=1, S=16, dt=BF16, stream=None, opts=2), o)


ADD = dict(x=0x1000, ld=64, r=0x2000, s=None, w=0x3000, eps=1e-6)


def add_fwd(**o):
    return _call("kla_add_norm_fwd", dict(**ADD, y=0x4000, r2=0x5000, M=8, D=64, dt=BF16, rdt=F32, stream=None), o)


def add_bwd(**o):
    return _call("kla_add_norm_bwd", dict(**ADD, dy=0x4000, dr2=None, dx=0x5000, dr=0x6000, ds=None, dw=0x7000, M=8, D=64, dt=BF16, rdt=F32, **WS,
                                          stream=None), o)


GATED = dict(x=0x1000, ld=128, g=0x2000, ld_g=128, w=0x3000, eps=1e-6)


def gated_fwd(**o):
    return _call("kla_gated_norm_fwd", dict(**GATED, y=0x4000, M=8, H=2, D=64, dt=BF16, stream=None, opts=0), o)


def gated_bwd(**o):
    return _call("kla_gated_norm_bwd", dict(**GATED, dy=0x4000, dx=0x5000, dg=0x6000, dw=0x7000, M=8, H=2, D=64, dt=BF16, **WS, stream=None, opts=0), o)


@pytest.mark.parametrize("f,required,parameters", [
    (conv_fwd, "x w y", "w"), (conv_bwd, "x w dy dx dw", "w dw"), (conv_step, "x w st y", "w"), (ssm_fwd, "u delta A B C y", "A"),
    (ssm_bwd, "u delta A B C dy du dd dA dB dC", "A dA"), (ssm_step, "u delta A B C h y", "A h"), (add_fwd, "x w y", "w"),
    (add_bwd, "x w dy dx dw", "w dw"), (gated_fwd, "x g w y", "w"), (gated_bwd, "x g w dy dx dg dw", "w dw")])
def test_pointers(f, required, parameters):
    for p in required.split():
        assert f(**{p: None}) == E_NULL, p
        assert f(**{p: 0x1001}) == E_ALIGN, p
    for p in parameters.split():
        assert f(**{p: 0x1002}) == E_ALIGN, p
    assert f(dt=7) == E_DTYPE
    assert f(dt=F32, **{required.split()[0]: 0x1002}) == E_ALIGN


def test_shapes():
    for f in (conv_fwd, conv_bwd, conv_step):
        for bad in (dict(W=1), dict(W=5), dict(D=0), dict(D=-1), dict(ld=63), dict(opts=2), dict(opts=1 << 30)):
            assert f(**bad) == E_SHAPE, bad
    for f in (ssm_fwd, ssm_bwd, ssm_step):
        for bad in (dict(S=15), dict(S=0), dict(S=128), dict(D=0), dict(G=0), dict(G=3), dict(ld_u=63), dict(ld_d=63), dict(ld_B=15), dict(ld_C=15),
                    dict(z=0x8000, ld_z=63), dict(opts=1), dict(G=2), dict(N=-1)):
            assert f(**bad) == E_SHAPE, bad
    assert ssm_bwd(z=0x8000, ld_z=64) == E_NULL           # a gate has a gradient
    for f in (add_fwd, add_bwd):
        for bad in (dict(D=0), dict(D=8193), dict(M=-1), dict(eps=-1.0), dict(eps=float("nan")), dict(ld=63)):
            assert f(**bad) == E_SHAPE, bad
        assert f(rdt=7) == E_DTYPE and f(dt=F32, rdt=BF16) == E_DTYPE
    for f in (gated_fwd, gated_bwd):
        for bad in (dict(D=0), dict(D=8193), dict(H=0), dict(M=-1), dict(eps=-1.0), dict(eps=float("nan")), dict(ld=127), dict(ld_g=127), dict(opts=1)):
            assert f(**bad) == E_SHAPE, bad


@pytest.mark.parametrize("f", [conv_fwd, conv_bwd, ssm_fwd, ssm_bwd])
def test_offsets(f):
    dev, host = 0xc000, CU.ctypes.data
    assert f(N=-1) == E_SHAPE and f(T=-1) == E_SHAPE and f(n_seq=-1) == E_SHAPE
    assert f(N=2, cu_dev=dev, cu_host=host, n_seq=2) == E_SHAPE
    assert f(cu_dev=None, cu_host=host, n_seq=2) == E_NULL and f(cu_dev=dev, cu_host=None, n_seq=2) == E_NULL
    assert f(cu_dev=dev, cu_host=host, n_seq=2, T=65) == E_SEQ
    assert f(cu_dev=dev, cu_host=host, n_seq=0) == E_SEQ
    for wrong in ([1, 30, 64], [0, 70, 64], [0, 30, 63]):
        w = np.array(wrong, dtype=np.int32)
        assert f(cu_dev=dev, cu_host=w.ctypes.data, n_seq=2) == E_SEQ, wrong


def test_limits():
    many = np.zeros(65537, dtype=np.int32)
    many[-1] = 64
    for f in (ssm_fwd, ssm_bwd):
        assert f(cu_dev=0xc000, cu_host=many.ctypes.data, n_seq=65536) == E_SHAPE
        assert f(N=65536, T=0) == E_SHAPE
        for ld in ("ld_u", "ld_d", "ld_B", "ld_C"):
            assert f(**{ld: (1 << 24) + 1}) == E_SHAPE
    assert conv_fwd(st=0x4000, last=0x4000) == E_SHAPE          # read and written at once


@pytest.mark.parametrize("f", [conv_bwd, ssm_bwd, add_bwd, gated_bwd])
def test_workspace(f):
    assert f(ws=None) == E_WS and f(ws=0x100010) == E_WS and f(ws_bytes=100) == E_WS


def test_queries():
    lib = kla.lib()
    assert lib.kla_conv_bwd_workspace_bytes(8, 4096, 1024, 4) >= 1024 * 5 * 4
    assert lib.kla_conv_bwd_workspace_bytes(0, 4096, 1024, 4) == 0
    for bad in ((-1, 1, 8, 4), (1, 1, 0, 4), (1, 1, 8, 5), (1, 1, 8, 1)):
        assert lib.kla_conv_bwd_workspace_bytes(*bad) == 0
    # one checkpoint of [D, S] fp32 per 16 tokens (8 from S = 32 on)
    assert lib.kla_ssm_saved_bytes(2, 64, 128, 1, 32, None, 0) == 2 * 8 * 128 * 32 * 4
    assert lib.kla_ssm_saved_bytes(2, 64, 128, 1, 16, None, 0) == 2 * 4 * 128 * 16 * 4
    assert lib.kla_ssm_saved_bytes(2, 65, 128, 1, 16, None, 0) == 2 * 5 * 128 * 16 * 4
    cu = np.array([0, 30, 30, 100], dtype=np.int32).ctypes
    assert lib.kla_ssm_saved_bytes(1, 100, 128, 1, 16, cu.data, 3) >= (2 + 5) * 128 * 16 * 4
    assert ssm_fwd(saved=0x10000, saved_bytes=4 * 64 * 16 * 4 - 4) == E_WS and ssm_bwd(saved=0x10000, saved_bytes=100) == E_WS
    wrong = np.array([0, 30, 99], dtype=np.int32).ctypes
    for q, more in ((lib.kla_ssm_saved_bytes, ()), (lib.kla_ssm_fwd_workspace_bytes, ()), (lib.kla_ssm_bwd_workspace_bytes, (1,))):
        for bad in ((-1, 1, 64, 1, 16, None, 0), (1, 1, 64, 1, 15, None, 0), (1, 1, 64, 3, 16, None, 0), (2, 100, 64, 1, 16, cu.data, 3),
                    (1, 100, 64, 1, 16, None, 3), (1, 100, 64, 1, 16, wrong.data, 2)):
            assert q(*bad, *more) == 0
    assert lib.kla_ssm_bwd_workspace_bytes(1, 64, 64, 1, 16, None, 0, 0) - lib.kla_ssm_bwd_workspace_bytes(1, 64, 64, 1, 16, None, 0, 1) == \
        lib.kla_ssm_saved_bytes(1, 64, 64, 1, 16, None, 0)
    # few channels and many tokens are taken in segments, with states for each of them; so are a packed batch's where one is long
    f = lib.kla_ssm_fwd_workspace_bytes
    assert f(1, 255, 2048, 1, 16, None, 0) == 0 and f(1, 4096, 2048, 1, 16, None, 0) > 8 * 2048 * 16 * 4 and f(8, 4096, 2048, 1, 16, None, 0) == 0
    even, odd = np.arange(0, 4097, 512, dtype=np.int32), np.array([0, 10, 20, 30, 40, 50, 60, 70, 4096], dtype=np.int32)
    assert f(1, 4096, 2048, 1, 16, even.ctypes.data, 8) == 0 and f(1, 4096, 2048, 1, 16, odd.ctypes.data, 8) > 0
    assert lib.kla_add_norm_bwd_workspace_bytes(8, 64, BF16) > 0 and lib.kla_add_norm_bwd_workspace_bytes(8, 8193, BF16) == 0
    assert lib.kla_gated_norm_bwd_workspace_bytes(8, 2, 64, BF16) > 0 and lib.kla_gated_norm_bwd_workspace_bytes(8, 0, 64, BF16) == 0
    assert lib.kla_add_norm_bwd_workspace_bytes(0, 64, BF16) == 0


def test_options_match_the_header():
    hdr = open(kla.HEADER_PATH).read()
    for n in ("SILU", "SOFTPLUS", "SIGMOID", "GATE_FIRST"):
        assert "KLA_LAYER_%s = %d" % (n, getattr(kla, "KLA_LAYER_" + n)) in hdr


def test_python_refusals():
    """Wrong extents, types and places are refused before the library is called: CPU tensors suffice."""
    x, w = torch.zeros(2, 5, 8), torch.zeros(8, 4)
    with pytest.raises(RuntimeError, match="GPU"):
        kla.kla_conv_fwd(x, w)
    with pytest.raises(ValueError, match="weight"):
        kla.kla_conv_fwd(x, torch.zeros(7, 4))
    with pytest.raises(TypeError, match="weight"):
        kla.kla_conv_fwd(x, w.double())
    with pytest.raises(TypeError):
        kla.kla_conv_fwd(x.half(), w)
    with pytest.raises(ValueError, match="state"):
        kla.kla_conv_fwd(x, w, state=torch.zeros(2, 4, 8))
    with pytest.raises(ValueError):
        kla.kla_conv_fwd(x[0], w)
    with pytest.raises(TypeError, match="cu_seqlens"):
        kla.kla_conv_fwd(x[:1], w, cu_seqlens=torch.tensor([0, 5]))
    with pytest.raises(ValueError, match="without cu_seqlens"):
        kla.kla_conv_fwd(x[:1], w, cu_seqlens_host=torch.tensor([0, 5], dtype=torch.int32))
    with pytest.raises(ValueError, match="state"):
        kla.kla_conv_step(x[0], w, torch.zeros(5, 2, 8))
    u, A, B = torch.zeros(2, 5, 8), torch.zeros(8, 16), torch.zeros(2, 5, 1, 16)
    with pytest.raises(RuntimeError, match="GPU"):
        kla.kla_ssm_fwd(u, u, A, B, B)
    with pytest.raises(ValueError, match="delta"):
        kla.kla_ssm_fwd(u, u[:1], A, B, B)
    with pytest.raises(ValueError, match="A must"):
        kla.kla_ssm_fwd(u, u, A[:, :8], B, B)
    with pytest.raises(TypeError, match="C must"):
        kla.kla_ssm_fwd(u, u, A, B, B.bfloat16())
    with pytest.raises(ValueError):
        kla.kla_ssm_fwd(u, u, A, B[:, :, 0], B)
    with pytest.raises(ValueError, match="z must"):
        kla.kla_ssm_step(u[:, 0], u[:, 0], A, B[:, 0], B[:, 0], torch.zeros(2, 8, 16), z=u)
    with pytest.raises(RuntimeError, match="GPU"):
        kla.kla_add_norm_fwd(x, torch.zeros(8))
    with pytest.raises(TypeError, match="residual stream"):
        kla.kla_add_norm_fwd(x, torch.zeros(8), x.bfloat16())
    with pytest.raises(ValueError, match="scale"):
        kla.kla_add_norm_fwd(x, torch.zeros(8), x, scale=torch.zeros(1))
    with pytest.raises(ValueError, match="activation"):
        kla.kla_gated_norm_fwd(x, x, torch.zeros(8), activation="tanh")
    with pytest.raises(ValueError, match="gate"):
        kla.kla_gated_norm_fwd(x, x[:1], torch.zeros(8))


@pytest.mark.parametrize("t,inner,ld", [
    (lambda: torch.zeros(3, 4, 8), 1, 8), (lambda: torch.zeros(3, 4, 20)[..., 4:12], 1, 20), (lambda: torch.zeros(3, 1, 20)[..., 4:12], 1, 20),
    (lambda: torch.zeros(1, 1, 20)[..., 4:12], 1, 8), (lambda: torch.zeros(3, 4, 20)[..., :16].unflatten(-1, (2, 8)), 2, 20),
    (lambda: torch.zeros(3, 0, 8), 1, 8), (lambda: torch.zeros(4, 6, 8)[:, 2], 1, 48)])
def test_row_strides(t, inner, ld):
    assert kla.layer._rows("x", t(), inner) == ld


@pytest.mark.parametrize("t,inner", [
    (lambda: torch.zeros(3, 8, 4).transpose(1, 2), 1), (lambda: torch.zeros(3, 6, 8)[:, :4], 1), (lambda: torch.zeros(3, 1, 8).expand(3, 4, 8), 1),
    (lambda: torch.zeros(1, 1, 8).expand(3, 4, 8), 1), (lambda: torch.zeros(3, 4, 2, 20)[..., :8], 2), (lambda: torch.zeros(3, 4, 16)[..., ::2], 1)])
def test_rows_that_are_none(t, inner):
    with pytest.raises(ValueError):
        kla.layer._rows("x", t(), inner)


def test_a_step_takes_rows_any_distance_apart():
    """One token out of [N, T, D] with long T: its rows are T D apart.  (N = 0: nothing is launched.)"""
    far = (1 << 24) + 1
    for ld in ("ld_u", "ld_d", "ld_B", "ld_C", "ld_z"):
        assert ssm_step(N=0, z=0x8000, **{"ld_z": 64, ld: far}) == OK, ld
    for f in (ssm_fwd, ssm_bwd):
        assert f(z=0x8000, ld_z=far, **({"dz": 0xf000} if f is ssm_bwd else {})) == E_SHAPE
        assert f(ld_z=far, T=0, N=0, **(dict(dA=None) if f is ssm_bwd else dict(A=None))) == E_NULL      # (without a gate its stride means nothing)


def test_widths_that_round_beyond_an_int():
    """A row of nearly 2^31 channels, rounded up to whole vectors and workgroups, is no int any more: refused, not wrapped around."""
    for D in ((1 << 30) + 1, (1 << 31) - 1):
        for f in (conv_fwd, conv_bwd, conv_step):
            assert f(D=D, ld=D, **({} if f is conv_step else dict(T=0))) == E_SHAPE
        assert kla.lib().kla_conv_bwd_workspace_bytes(1, 1, D, 4) == 0
    assert conv_step(D=1 << 30, ld=1 << 30, B=0) == OK


def test_convolution_in_place():
    """A convolution cannot write where it reads: other threads still need what is there."""
    assert conv_fwd(y=0x1000) == E_SHAPE
    assert conv_bwd(dx=0x1000) == E_SHAPE and conv_bwd(dx=0x3000) == E_SHAPE
    assert conv_bwd(st=0x6000, dst=0x6000) == E_SHAPE and conv_bwd(st=0x6000, dlast=0x7000, dst=0x7000) == E_SHAPE
