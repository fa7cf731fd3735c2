"""The operators around the recurrence under graph capture and on a stream of the caller's: no call allocates behind the caller's back,
synchronises or copies from the host, and results are the same to the bit (fixed order of every sum)."""
import pytest
import torch

from layer_cases import bits, offsets

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kla():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2605_08587_amd as m
    m.lib()
    return m


def _calls(kla):
    g = torch.Generator(device="cuda").manual_seed(1)

    def r(*s, dt=torch.bfloat16):
        return torch.randn(s, generator=g, device="cuda").to(dt)
    f = torch.float32
    cu = offsets([100, 3, 0, 197])
    packed = dict(cu_seqlens=cu.cuda(), cu_seqlens_host=cu)
    N, T, D, S = 2, 150, 256, 16
    x, w, b, dy = r(N, T, D), r(D, 4, dt=f), r(D, dt=f), r(N, T, D)
    xp, dyp = r(1, 300, D), r(1, 300, D)
    A, skip = -r(D, S, dt=f).abs(), r(D, dt=f)
    B, C, Bp, Cp = r(N, T, 1, S), r(N, T, 1, S), r(1, 300, 1, S), r(1, 300, 1, S)
    long = [r(1, 9000, 64), r(1, 9000, 64), -r(64, S, dt=f).abs(), r(1, 9000, 1, S), r(1, 9000, 1, S)]
    st, h = r(N, 3, D), r(N, D, S, dt=f)

    def step():
        s, hh = st.clone(), h.clone()
        y = kla.kla_conv_step(x[:, 0], w, s, b)
        return y, s, kla.kla_ssm_step(y, x[:, 1], A, B[:, 0], C[:, 0], hh, z=x[:, 2]), hh
    return {
        "conv": lambda: kla.kla_conv_fwd(x, w, b),
        "conv packed": lambda: kla.kla_conv_fwd(xp, w, b, **packed),
        "conv bwd": lambda: tuple(v for v in kla.kla_conv_bwd(xp, w, dyp, b, **packed).values() if v is not None),
        "ssm": lambda: kla.kla_ssm_fwd(x, dy, A, B, C, skip, x, h0=h),
        "ssm packed": lambda: kla.kla_ssm_fwd(xp, dyp, A, Bp, Cp, skip, xp, **packed),
        "ssm long": lambda: kla.kla_ssm_fwd(*long),
        "ssm bwd": lambda: tuple(v for v in kla.kla_ssm_bwd(xp, dyp, A, Bp, Cp, dyp, skip, xp, **packed).values() if v is not None),
        "ssm bwd long": lambda: tuple(v for v in kla.kla_ssm_bwd(*long, long[0]).values() if v is not None),
        "step": step,
        "norms": lambda: (*kla.kla_add_norm_fwd(x, b, dy, skip), kla.kla_gated_norm_fwd(x.view(N, T, 2, 128), dy.view(N, T, 2, 128), b[:128].contiguous())),
        "norms bwd": lambda: (*kla.kla_add_norm_bwd(x, b, dy, x, skip).values(),
                              *kla.kla_gated_norm_bwd(x.view(N, T, 2, 128), dy.view(N, T, 2, 128), b[:128].contiguous(), x.view(N, T, 2, 128)).values()),
    }


NAMES = ["conv", "conv packed", "conv bwd", "ssm", "ssm packed", "ssm long", "ssm bwd", "ssm bwd long", "step", "norms", "norms bwd"]


@pytest.mark.parametrize("name", NAMES)
def test_graph_replays(kla, name):
    f = _calls(kla)[name]
    ref = [t.clone() for t in f()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        f()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = f()
    for _ in range(3):
        for t in out:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(bits(p), bits(q)) for p, q in zip(out, ref))
        assert all(torch.equal(bits(p), bits(q)) for p, q in zip(f(), ref))      # eager work between the replays
        torch.cuda.synchronize()


@pytest.mark.parametrize("name", NAMES)
def test_on_another_stream(kla, name):
    """Behind work of the same stream that makes the inputs late: the results are those of the inputs as they are then."""
    calls = _calls(kla)
    ref = [t.clone() for t in calls[name]()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        a = torch.randn(2048, 2048, device="cuda")
        for _ in range(20):
            a = torch.tanh(a @ a)
        late = _calls(kla)[name]
        out = late()
    side.synchronize()
    assert all(torch.equal(bits(p), bits(q)) for p, q in zip(out, ref))
