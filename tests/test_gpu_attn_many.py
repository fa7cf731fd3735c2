"""Attention over whole sequences with enough rows for every kernel of its own: the forward whose four waves share tiles of keys, and dk, dv and dq as launches
apart.  Three key heads of different inputs are held to the definition in 64 bits; all others repeat one of the three, and have to come out like it bit by bit."""
import pytest
import torch

from attn_cases import MANY_TILES, check, many_tiles, offsets, randn
from layer_cases import bits

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]


@pytest.fixture(scope="module")
def kla():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2605_08587_amd as m
    m.lib()
    return m


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("name", sorted(MANY_TILES))
def test_every_form_of_many_tiles(kla, dtype, D, name):
    lengths, packed, G, Hk, causal, window = MANY_TILES[name]
    assert many_tiles(name) >= 512
    lead = (1, sum(lengths)) if packed else (len(lengths), lengths[0])
    gen = torch.Generator(device="cuda").manual_seed(len(name))
    of = torch.arange(Hk, device="cuda") % 3                 # the inputs of each key head
    def heads(per, sharp=1.0):
        x = randn(gen, *lead, 3 * per, D, dtype=dtype, sharp=sharp).unflatten(2, (3, per))
        return x[:, :, of].flatten(2, 3).contiguous()
    q, k, v, d_o = heads(G, 2.0), heads(1), heads(1), heads(G)
    kw = dict(causal=causal, window=window)
    if packed:
        cu = offsets(lengths)
        kw.update(cu_seqlens=cu.cuda(), cu_seqlens_host=cu)
    for rest in (None,) + ((torch.empty_like(q),) if dtype == torch.bfloat16 else ()):
        o, lse = kla.kla_attn_fwd(q, k, v, rest=rest, **kw)
        g = kla.kla_attn_bwd(q, k, v, o, lse, d_o, rest=rest, **kw)
        three = lambda t, per: t.flatten(0, 1)[:, :3 * per]
        check(lengths, three(q, G), three(k, 1), three(v, 1), three(o, G), three(lse, G), D ** -0.5, causal, window, three(d_o, G),
              [three(g["dq"], G), three(g["dk"], 1), three(g["dv"], 1)], tag=name, rest=rest is not None)
        for what, t, per in (("o", o, G), ("lse", lse, G), ("dq", g["dq"], G), ("dk", g["dk"], 1), ("dv", g["dv"], 1)):
            t = bits(t).unflatten(2, (Hk, per))
            assert torch.equal(t, t[:, :, of]), what
