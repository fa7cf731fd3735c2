"""New tokens over a paged cache on the GPU: what they see, what is stored, and that nothing else of the cache is touched or taken."""
import numpy as np
import pytest
import torch

from attn_cases import U, f64, offsets, randn, within
from layer_cases import bits
from oracle import attn_oracle as ao

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]


@pytest.fixture(scope="module")
def kla():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2605_08587_amd as m
    m.lib()
    return m


class Case:
    """A cache whose used pages are scattered over it; everything that holds no token is NaN."""

    def __init__(self, seed, dtype, H, Hk, D, page, cached, new, room=3, sharp=2.0, wide=False):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.cached_host, self.new, self.page = list(cached), list(new), page
        need = [-(-(c + n) // page) for c, n in zip(cached, new)]
        P = sum(need) + room
        self.kc, self.vc = (torch.full((P, Hk, page, D), float("nan"), device="cuda", dtype=dtype) for _ in range(2))
        order = torch.randperm(P, generator=torch.Generator().manual_seed(seed)).int()
        self.table = torch.full((len(new), max(need + [1]) + 1), -1, dtype=torch.int32)
        at = 0
        for i, n in enumerate(need):
            self.table[i, :n] = order[at:at + n]
            at += n
        M = sum(new)
        r = lambda m, h, s=1.0: randn(g, 1, m, h, D, dtype=dtype, wide=wide, sharp=s)
        self.q, self.k, self.v = r(M, H, sharp), r(M, Hk), r(M, Hk)
        self.old = []
        for i, c in enumerate(cached):
            k, v = (torch.randn(c, Hk, D, generator=g, device="cuda").to(dtype) for _ in range(2))
            self.old.append((k, v))
            self.put(self.kc, self.vc, i, 0, k, v)
        self.table, self.cached = self.table.cuda(), torch.tensor(list(cached), dtype=torch.int32, device="cuda")
        self.cu = offsets(new)

    def put(self, kc, vc, i, pos, k, v):
        where = torch.arange(pos, pos + len(k))
        pages, slots = self.table.cpu()[i, where // self.page].long(), where % self.page
        kc[pages.cuda(), :, slots.cuda()] = k
        vc[pages.cuda(), :, slots.cuda()] = v

    def check(self, o, lse, scale, window, kc, vc):
        at = 0
        want_k, want_v = self.kc.clone(), self.vc.clone()
        for i, (c, n) in enumerate(zip(self.cached_host, self.new)):
            here = slice(at, at + n)
            q, k, v = self.q[0, here], torch.cat([self.old[i][0], self.k[0, here]]), torch.cat([self.old[i][1], self.v[0, here]])
            a = [f64(t) for t in (q, k, v)]
            ro, rl = ao.forward(*a, scale, first=c, window=window)
            b = ao.bounds(*a, scale, U[self.q.dtype], first=c, window=window)
            within("o of sequence %d" % i, o[here], ro, b[0])
            if lse is not None:
                within("lse of sequence %d" % i, lse[here], rl, b[1])
            self.put(want_k, want_v, i, c, self.k[0, here], self.v[0, here])
            at += n
        assert torch.equal(bits(kc), bits(want_k)) and torch.equal(bits(vc), bits(want_v))


def _extend(kla, c, scale=None, window=0, max_len=None, fixed=False, **kw):
    kc, vc = c.kc.clone(), c.vc.clone()
    if fixed:
        n, t = len(c.new), c.new[0]
        q, k, v = (x.view(n, t, *x.shape[2:]) if x.is_contiguous() else x[0].unflatten(0, (n, t)) for x in (c.q, c.k, c.v))
        o, lse = kla.kla_attn_extend(q, k, v, kc, vc, c.table, c.cached, scale=scale, window=window, max_len=max_len, want_lse=True, **kw)
        o, lse = o.flatten(0, 1), lse.flatten(0, 1)
    else:
        o, lse = kla.kla_attn_extend(c.q, c.k, c.v, kc, vc, c.table, c.cached, scale=scale, window=window, cu_seqlens=c.cu.cuda(), cu_seqlens_host=c.cu,
                                     max_len=max_len, want_lse=True, **kw)
        o, lse = o[0], lse[0]
    c.check(o, lse, c.q.shape[-1] ** -0.5 if scale is None else scale, window, kc, vc)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("H,Hk,D,page,cached,new,window", [
    (4, 2, 64, 16, [0], [1], 0), (4, 2, 128, 16, [15, 16, 17], [1, 1, 1], 0), (2, 2, 64, 32, [0, 31, 100], [2, 5, 40], 0), (8, 1, 128, 64, [63, 500], [4, 3], 0),
    (6, 2, 64, 16, [200, 0, 7], [0, 33, 1], 0), (3, 1, 128, 128, [300, 1000], [50, 70], 0), (4, 4, 128, 16, [77, 300], [130, 1], 40),
    (4, 2, 64, 1024, [900, 1500], [200, 7], 1), (16, 2, 128, 16, [333, 1200], [9, 2], 100), (5, 5, 64, 64, [2000], [300], 0)])
def test_new_tokens(kla, dtype, H, Hk, D, page, cached, new, window):
    c = Case(len(cached) + page, dtype, H, Hk, D, page, cached, new)
    _extend(kla, c, window=window)
    _extend(kla, c, window=window, max_len=2 ** 31 - 1)      # (rows beyond 32: four waves that share tiles)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,t,H,Hk,D", [(3, 5, 8, 2, 64), (2, 40, 4, 4, 128), (70, 1, 4, 1, 64)])
def test_fixed_lengths_in_a_wider_tensor(kla, dtype, n, t, H, Hk, D):
    c = Case(n, dtype, H, Hk, D, 32, [(37 * i) % 150 for i in range(n)], [t] * n, wide=True)
    _extend(kla, c, fixed=True, scale=0.3)
    _extend(kla, c, scale=0.3)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("max_len", [0, 1, 700, 2 ** 31 - 1])
def test_the_bound_only_cuts_the_work(kla, dtype, max_len):
    _extend(kla, Case(1, dtype, 8, 2, 128, 16, [10, 0, 1500], [3, 4, 2]), max_len=max_len)
    _extend(kla, Case(2, dtype, 8, 2, 64, 16, [10, 900], [30, 40]), max_len=max_len, window=200)


def _step(kla, c, **kw):
    kc, vc = c.kc.clone(), c.vc.clone()
    o = kla.kla_attn_step(c.q[0], c.k[0], c.v[0], kc, vc, c.table, c.cached, **kw)
    c.check(o, None, c.q.shape[-1] ** -0.5, kw.get("window", 0), kc, vc)
    return o


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("H,Hk,D,page,cached,window", [
    (1, 1, 64, 16, [0], 0), (8, 2, 128, 64, [4095], 0), (16, 2, 64, 16, [0, 1, 15, 16, 100, 3000], 0), (40, 1, 128, 32, [70, 600], 0), (4, 4, 64, 256, [511, 512, 513], 0),
    (8, 2, 128, 16, [5000, 3], 17), (2, 1, 64, 16, list(range(130)), 0), (64, 1, 64, 64, [900, 20], 0)])
@pytest.mark.parametrize("wide", [False, True])
def test_single_tokens(kla, dtype, H, Hk, D, page, cached, window, wide):
    _step(kla, Case(sum(cached) % 97, dtype, H, Hk, D, page, cached, [1] * len(cached), wide=wide), window=window)


def test_no_sequences(kla):
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, device="cuda", dtype=dt)
    c, t, n = z(4, 2, 16, 64), z(0, 3, dt=torch.int32), z(0, dt=torch.int32)
    assert kla.kla_attn_step(z(0, 4, 64), z(0, 2, 64), z(0, 2, 64), c, c.clone(), t, n).shape == (0, 4, 64)
    assert kla.kla_attn_extend(z(2, 0, 4, 64), z(2, 0, 2, 64), z(2, 0, 2, 64), c, c.clone(), z(2, 3, dt=torch.int32), z(2, dt=torch.int32)).shape == (2, 0, 4, 64)


@pytest.mark.parametrize("H", [2, 66])
def test_entries_that_are_no_pages(kla, H):
    """They read as the nearest page and take nothing in; lengths below 0 and beyond the table are cut; every other page stays as it was."""
    c = Case(3, torch.float32, H, 2, 64, 16, [40, 40, 40], [3, 3, 3], room=0)
    P, W = len(c.kc), c.table.shape[1]
    kc, vc = torch.randn_like(c.kc), torch.randn_like(c.vc)
    table = torch.tensor([[-5, 1, P - 1, 0], [2, P + 7, 2 ** 31 - 1, 0], [3, 4, 5, 6]], dtype=torch.int32, device="cuda")[:, :W]
    assert W == 4
    cached = torch.tensor([40, -3, 1 << 30], dtype=torch.int32, device="cuda")
    k2, v2 = kc.clone(), vc.clone()
    o = kla.kla_attn_extend(c.q.view(3, 3, H, 64), c.k.view(3, 3, 2, 64), c.v.view(3, 3, 2, 64), k2, v2, table, cached, max_len=64)
    want_k, want_v = kc.clone(), vc.clone()
    for i, (n, pages) in enumerate(((40, [0, 1, P - 1]), (0, []), (64, [3, 4, 5, 6]))):
        k, v = (torch.cat([t[p].transpose(0, 1) for p in pages] + [t[0, 0, :0].new_empty(0, 2, 64)])[:n] for t in (kc, vc))
        a = [f64(t) for t in (c.q[0, 3 * i:3 * i + 3], torch.cat([k, c.k[0, 3 * i:3 * i + 3]]), torch.cat([v, c.v[0, 3 * i:3 * i + 3]]))]
        within("o", o[i], ao.forward(*a, 0.125, first=n)[0], ao.bounds(*a, 0.125, 2.0 ** -24, first=n)[0])
    for t in range(3):
        want_k[P - 1, :, 8 + t], want_v[P - 1, :, 8 + t] = c.k[0, t], c.v[0, t]          # sequence 0: positions 40 .. 42
        want_k[2, :, t], want_v[2, :, t] = c.k[0, 3 + t], c.v[0, 3 + t]                  # sequence 1: 0 .. 2
    assert torch.equal(bits(k2), bits(want_k)) and torch.equal(bits(v2), bits(want_v))
    # a new token whose entry is no page is seen all the same, and stored nowhere
    table[0, 2], table[1, 0] = P, -1
    k2, v2 = kc.clone(), vc.clone()
    kla.kla_attn_extend(c.q.view(3, 3, H, 64), c.k.view(3, 3, 2, 64), c.v.view(3, 3, 2, 64), k2, v2, table, cached, max_len=64)
    assert torch.equal(bits(k2), bits(kc)) and torch.equal(bits(v2), bits(vc))


def test_sequences_that_share_pages(kla):
    """A common beginning in the same pages of two sequences: only read."""
    c = Case(4, torch.bfloat16, 8, 2, 64, 16, [64, 70], [2, 5])
    c.table[1, :4] = c.table[0, :4]
    c.old[1] = tuple(torch.cat([a[:64], b[64:]]) for a, b in zip(c.old[0], c.old[1]))
    _extend(kla, c)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("cached,max_len", [(50, None), (50, 2 ** 31 - 1), (3000, None), (3000, 2 ** 31 - 1)])
def test_later_tokens_that_are_not_finite(kla, dtype, value, D, cached, max_len):
    """A new token's values are seen from it on only, whatever they are."""
    c = Case(5, dtype, 4, 2, D, 16, [cached], [40])
    c.v[0, 20, 1, 3] = value
    kc, vc = c.kc.clone(), c.vc.clone()
    o = kla.kla_attn_extend(c.q, c.k, c.v, kc, vc, c.table, c.cached, max_len=max_len)[0]
    assert torch.isfinite(o[:20]).all() and torch.isfinite(o[:, :2]).all() and torch.isfinite(o[..., 4:]).all()
    x = o[20:, 2:, 3].float()
    assert (torch.isnan(x) if value != value else x == value).all()
    assert not torch.isfinite(vc).all()                     # and stored as they are


def test_caches_beyond_32_bits(kla):
    """Pages whose elements lie beyond 2^32 of the cache."""
    P, Hk, page, D = 2200, 8, 2 * 1024 // 2, 128
    kc = torch.zeros(P, Hk, page, D, dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    c = Case(6, torch.bfloat16, 8, 8, D, page, [1500, 900], [1, 1], room=0)
    table = c.table.clone()
    far = torch.tensor([P - 1, 3, P - 2, 5], device="cuda", dtype=torch.int32)
    for i in range(len(c.kc)):
        kc[far[i].item()], vc[far[i].item()] = c.kc[i].nan_to_num(0), c.vc[i].nan_to_num(0)
    table = torch.where(table >= 0, far[table.clamp(min=0).long()], table)
    o = kla.kla_attn_step(c.q[0], c.k[0], c.v[0], kc, vc, table, c.cached)
    k2, v2 = c.kc.clone(), c.vc.clone()
    want = kla.kla_attn_step(c.q[0], c.k[0], c.v[0], k2, v2, c.table, c.cached)
    assert kc.numel() > 2 ** 31 and torch.equal(bits(o), bits(want))
    for i in range(len(k2)):
        assert torch.equal(bits(kc[far[i].item()]), bits(k2[i].nan_to_num(0))) and torch.equal(bits(vc[far[i].item()]), bits(v2[i].nan_to_num(0)))


def test_caches_of_more_than_2_to_32_elements(kla):
    """Pages whose elements, not only their bytes, lie beyond 2^32 of the cache, for single tokens and for chunks."""
    P, Hk, page, D = 4200, 8, 1024, 128
    c = Case(13, torch.bfloat16, 8, Hk, D, page, [1500, 900, 1000], [1, 1, 70], room=0)
    kc, vc = (torch.empty(P, Hk, page, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    far = [P - 1 - i for i in range(len(c.kc))]
    assert min(far) * Hk * page * D > 2 ** 32
    table = torch.where(c.table >= 0, torch.tensor(far, device="cuda", dtype=torch.int32)[c.table.clamp(min=0).long()], c.table)

    def calls(kc, vc, table):
        a = kla.kla_attn_step(c.q[0, :2], c.k[0, :2], c.v[0, :2], kc, vc, table[:2], c.cached[:2])
        b = [kla.kla_attn_extend(*(t[:, 2:].contiguous() for t in (c.q, c.k, c.v)), kc, vc, table[2:], c.cached[2:], max_len=m) for m in (None, 2 ** 31 - 1)]
        return (a, *b)
    for i, p in enumerate(far):
        kc[p], vc[p] = c.kc[i], c.vc[i]
    near_k, near_v = c.kc.clone(), c.vc.clone()
    for x, y in zip(calls(kc, vc, table), calls(near_k, near_v, c.table)):
        assert torch.isfinite(x).all() and torch.equal(bits(x), bits(y))
    for i, p in enumerate(far):
        assert torch.equal(bits(kc[p]), bits(near_k[i])) and torch.equal(bits(vc[p]), bits(near_v[i]))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("native", [True, False])
def test_single_tokens_far_apart(kla, monkeypatch, native, dtype):
    """The t-th token of each sequence of a long batch: more than 2^24 elements from one to the next."""
    if not native:
        monkeypatch.setattr(kla, "_native", kla._StepByStep)
    c = Case(14, dtype, 8, 2, 128, 16, [70, 0], [1, 1])
    T = (1 << 24) // (2 * 128) + 8
    far = []
    for x in (c.q, c.k, c.v):
        w = torch.empty(2, T if x is not c.q else T // 4 + 2, *x.shape[2:], dtype=dtype, device="cuda")
        w[:, 7] = x[0]
        assert w.stride(0) > 1 << 24
        far.append(w[:, 7:8])
    for q, k, v in (far, (far[0], c.k.view(2, 1, 2, 128), far[2])):
        kc, vc = c.kc.clone(), c.vc.clone()
        c.check(kla.kla_attn_step(q[:, 0], k[:, 0], v[:, 0], kc, vc, c.table, c.cached), None, 128 ** -0.5, 0, kc, vc)
        kc, vc = c.kc.clone(), c.vc.clone()
        o, lse = kla.kla_attn_extend(q, k, v, kc, vc, c.table, c.cached, want_lse=True)
        c.check(o[:, 0], lse[:, 0], 128 ** -0.5, 0, kc, vc)
    with pytest.raises(ValueError, match="2\\^24"):
        kla.kla_attn_fwd(*far)
    with pytest.raises(ValueError, match="2\\^24"):
        kla.kla_attn(*far)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cached,new,max_len", [(3000, 1, None), (3000, 40, 2 ** 31 - 1), (60, 1, None)])
def test_scores_that_are_minus_infinity_or_nan(kla, dtype, cached, new, max_len):
    """Keys in several parts: a NaN among scores of -inf is a NaN in o and lse, as the formulas have it, in whichever part it stands."""
    for at in (None, 5, cached // 2, cached - 1):
        c = Case(15, dtype, 4, 2, 64, 16, [cached], [new])
        c.q[..., 0] = 1.0
        c.k[..., 0] = -float("inf")
        c.kc[..., 0] = -float("inf")                         # (the whole cache: every old key, and what holds none)
        if at is not None:
            page = c.table[0, at // 16].item()
            c.kc[page, :, at % 16, 1] = float("nan")
        o, lse = kla.kla_attn_extend(c.q, c.k, c.v, c.kc, c.vc, c.table, c.cached, want_lse=True, max_len=max_len)
        assert torch.isnan(o).all(), at
        assert (lse == -float("inf")).all() if at is None else torch.isnan(lse).all(), at


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_prompt_whole_by_chunks_and_by_tokens(kla, dtype):
    """One prompt: at once without a cache, in chunks over one, and its last tokens one at a time in a captured graph whose lengths advance on the device."""
    H, Hk, D, T, page, window = 8, 2, 64, 150, 16, 60
    g = torch.Generator(device="cuda").manual_seed(7)
    q, k, v = (randn(g, 2, T, h, D, dtype=dtype) for h in (H, Hk, Hk))
    whole, _ = kla.kla_attn_fwd(q, k, v, window=window)
    pages = -(-T // page)
    kc, vc = (torch.full((2 * pages, Hk, page, D), float("nan"), dtype=dtype, device="cuda") for _ in range(2))
    table = torch.randperm(2 * pages, generator=torch.Generator().manual_seed(8)).int().view(2, pages).cuda()
    cached = torch.zeros(2, dtype=torch.int32, device="cuda")
    got, at = [], 0
    for n in (1, 40, 64, 25):
        got.append(kla.kla_attn_extend(*(t[:, at:at + n].contiguous() for t in (q, k, v)), kc, vc, table, cached, window=window))
        cached += n
        at += n
    sq, sk, sv = (t[:, at].clone() for t in (q, k, v))
    out = torch.empty(2, H, D, dtype=dtype, device="cuda")
    kla.kla_attn_step(sq, sk, sv, kc, vc, table, cached, window=window, out=out)      # (the same token is stored again by the first replay)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kla.kla_attn_step(sq, sk, sv, kc, vc, table, cached, window=window, out=out)
        cached += 1
    for t in range(at, T):
        for s, x in ((sq, q), (sk, k), (sv, v)):
            s.copy_(x[:, t])
        graph.replay()
        got.append(out.clone()[:, None])
        if t % 7 == 0:
            torch.cuda.synchronize()
    got = torch.cat(got, 1)
    assert cached.tolist() == [T, T]
    for i in range(2):
        a = [f64(t[i]) for t in (q, k, v)]
        ref, b = ao.forward(*a, D ** -0.5, window=window)[0], ao.bounds(*a, D ** -0.5, U[dtype], window=window)[0]
        within("whole", whole[i], ref, b)
        within("piece by piece", got[i], ref, b)


@pytest.mark.parametrize("native", [True, False])
def test_what_is_written_counts_as_changed(kla, monkeypatch, native):
    if not native:
        monkeypatch.setattr(kla, "_native", kla._StepByStep)
    c = Case(9, torch.bfloat16, 4, 2, 64, 16, [20, 30], [1, 1])
    versions = [t._version for t in (c.kc, c.vc)]
    _step(kla, c)
    kla.kla_attn_step(c.q[0], c.k[0], c.v[0], c.kc, c.vc, c.table, c.cached)
    kla.kla_attn_extend(c.q, c.k, c.v, c.kc, c.vc, c.table, c.cached, cu_seqlens=c.cu.cuda(), cu_seqlens_host=c.cu)
    assert all(t._version >= n + 2 for t, n in zip((c.kc, c.vc), versions))


def test_two_halves_of_the_binding_same_bits(kla, monkeypatch):
    c = Case(10, torch.bfloat16, 8, 2, 128, 32, [500, 33, 0], [4, 1, 9])

    def calls():
        kw = dict(cu_seqlens=c.cu.cuda(), cu_seqlens_host=c.cu)
        kc, vc = c.kc.clone(), c.vc.clone()
        a = kla.kla_attn_extend(c.q, c.k, c.v, kc, vc, c.table, c.cached, want_lse=True, max_len=600, **kw)
        b = kla.kla_attn_step(c.q[0, :3], c.k[0, :3], c.v[0, :3], kc, vc, c.table, c.cached, window=70, scale=0.1)
        return (*a, b, kc, vc, *kla.kla_attn_fwd(c.q, c.k, c.v, causal=False, **kw))
    assert kla._binding().__name__ == "kla_binding"
    native = calls()
    monkeypatch.setattr(kla.attention, "_heads", None)       # (Python's half is out of reach: the native half took every call)
    calls()
    monkeypatch.undo()
    monkeypatch.setattr(kla, "_native", kla._StepByStep)
    for x, y in zip(native, calls()):
        assert torch.equal(bits(x), bits(y))


def test_streams_and_graphs(kla):
    """On a stream of the caller's, and captured: whole sequences in both directions and a chunk over the cache, replayed between eager calls; two
    graphs with workspaces of their own."""
    g = torch.Generator(device="cuda").manual_seed(11)
    q, k, v, d_o = (randn(g, 2, 300, h, 64, dtype=torch.bfloat16) for h in (8, 2, 2, 8))
    c = Case(12, torch.bfloat16, 8, 2, 64, 16, [700, 90], [6, 3])
    cu = c.cu.cuda()

    def calls():
        o, lse = kla.kla_attn_fwd(q, k, v)
        kc, vc = c.kc.clone(), c.vc.clone()
        x = kla.kla_attn_extend(c.q, c.k, c.v, kc, vc, c.table, c.cached, cu_seqlens=cu, cu_seqlens_host=c.cu)
        return (o, lse, *kla.kla_attn_bwd(q, k, v, o, lse, d_o).values(), x, kc, vc)
    eager = calls()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = calls()
    torch.cuda.synchronize()
    assert all(torch.equal(bits(a), bits(b)) for a, b in zip(eager, other))
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            r = calls()
        graphs.append((graph, r))
    for i in range(6):
        graph, r = graphs[i % 2]
        graph.replay()
        if i % 3:
            calls()
            torch.cuda.synchronize()
        assert all(torch.equal(bits(a), bits(b)) for a, b in zip(eager, r))
