"""Selective scan against its definition in 64 bits in every form its plans take: segments for all numbers of states, groups, with and without
a gate, packed and not; workgroups of 64 channels, in segments and whole."""
import pytest
import torch

from layer_cases import SCAN, bits, close, offsets, randn
from oracle import layer_oracle as lo
from test_gpu_ssm import ALL, _inputs

pytestmark = pytest.mark.gpu
b16, f32 = torch.bfloat16, torch.float32
NO_GATE = ("skip", "delta_bias", "h0")


@pytest.fixture(scope="module")
def kla():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2605_08587_amd as m
    m.lib()
    return m


def _hold(kla, dtype, N, T, D, G, S, lens, opt, wide, seed, segments):
    print("ssm plan", dtype, N, T, D, G, S, lens, opt, wide, flush=True)
    lead, n = ((1, sum(lens)), len(lens)) if lens else ((N, T), N)
    g, d, dev = _inputs(dtype, lead, n, D, G, S, opt, wide, seed)
    cu = offsets(lens) if lens else None
    cut = kla.lib().kla_ssm_fwd_workspace_bytes(*lead, D, G, S, None if cu is None else cu.data_ptr(), len(lens) if lens else 0) > 0
    assert cut == segments
    dy, dh = randn(g, *lead, D, dtype=dtype), randn(g, n, D, S)
    seqs = lo.sequences(N, T, cu)
    flat = {k: v if v is None or k in ("A", "skip", "delta_bias", "h0") else v.flatten(0, 1) for k, v in d.items()}
    (y_ref, h_ref), g_ref = lo.gradients(lambda **k: lo.ssm(**k, softplus=True, seqs=seqs), flat, (dy.flatten(0, 1), dh))
    packed = {} if cu is None else dict(cu_seqlens=cu.cuda(), cu_seqlens_host=cu)
    leaves = {k: None if v is None else v.detach().requires_grad_(True) for k, v in dev.items()}
    wrt = {k: v for k, v in leaves.items() if v is not None}
    got = []
    for save in (True, False):                           # checkpoints left by the forward, and formed again
        y, hT = kla.kla_ssm(**leaves, save=save, **packed)
        got.append((y.detach(), hT.detach(), *torch.autograd.grad((y, hT), list(wrt.values()), (dy.cuda(), dh.cuda()))))
    assert all(torch.equal(bits(p), bits(q)) for p, q in zip(*got))
    close("y", got[0][0].flatten(0, 1), y_ref, SCAN)
    close("hT", got[0][1], h_ref, SCAN)
    for k, p in zip(wrt, got[0][2:]):
        close("d" + k, p.reshape(g_ref[k].shape), g_ref[k], SCAN)


@pytest.mark.parametrize("dtype", [b16, f32])
@pytest.mark.parametrize("S", [8, 16, 32, 64])
@pytest.mark.parametrize("opt,G,lens,T", [(ALL, 1, None, 300), (NO_GATE, 2, None, 257), (ALL, 2, [3, 260, 0, 301], 0), (NO_GATE, 1, [33, 0, 400], 0)])
def test_segments(kla, dtype, S, opt, G, lens, T):
    _hold(kla, dtype, 2, T, 76, G, S, lens, opt, ("odd" if G == 2 else False), S + G, True)


@pytest.mark.parametrize("dtype", [b16, f32])
@pytest.mark.parametrize("S", [8, 16, 32])
def test_workgroups_of_64_channels_in_segments(kla, dtype, S):
    """Two groups of 865 channels in 14 workgroups each, five segments: 140 workgroups of 64 channels are one round over the CUs, those of 32 two."""
    _hold(kla, dtype, 1, 320, 1730, 2, S, None, ALL if S != 16 else NO_GATE, False, 40 + S, True)


@pytest.mark.parametrize("dtype", [b16, f32])
@pytest.mark.parametrize("S", [8, 16, 32])
@pytest.mark.parametrize("opt", [ALL, NO_GATE])
def test_workgroups_of_64_channels(kla, dtype, S, opt):
    """140 sequences, one workgroup of 64 channels each; and packed ones of unequal lengths."""
    _hold(kla, dtype, 140, 9, 64, 1, S, None, opt, True, 50 + S, False)
    _hold(kla, dtype, 1, 0, 61, 1, S, [i % 20 for i in range(150)], opt, "odd", 60 + S, False)
