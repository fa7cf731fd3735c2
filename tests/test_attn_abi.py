"""Host-side checks of softmax attention that need no GPU: every refusal comes before anything is launched (the pointers are fakes), the workspace queries,
and what the Python functions refuse."""
import os
import re

import numpy as np
import pytest
import torch

import paper_2605_08587_amd as kla
from attn_cases import MANY_TILES, many_tiles

pytestmark = pytest.mark.skipif(not os.path.exists(kla.LIB_PATH), reason="libkla.so not built (python -m paper_2605_08587_amd.build)")

OK, E_NULL, E_SHAPE, E_DTYPE, E_ALIGN, E_WS, E_SEQ = 0, -1, -2, -3, -4, -5, -6
BF16, F32 = kla.KLA_BF16, kla.KLA_F32
CU = np.array([0, 30, 64], dtype=np.int32)


def _call(name, defaults, over):
    a = dict(defaults)
    assert set(over) <= set(a), over
    a.update(over)
    return getattr(kla.lib(), name)(*a.values())


IN = dict(q=0x1000, ld_q=512, k=0x2000, ld_k=256, v=0x3000, ld_v=256)
SEQS = dict(cu_dev=None, cu_host=None, n_seq=0)
SIZES = dict(N=1, T=64, H=8, Hk=4, D=64)
CACHE = dict(kc=0x10000, vc=0x20000, table=0x30000, ld_table=8, cached=0x40000)
WS = dict(ws=0x100000, ws_bytes=1 << 40)


def fwd(**o):
    return _call("kla_attn_fwd", dict(**IN, o=0x4000, lse=None, rest=None, scale=0.125, window=0, **SEQS, **SIZES, dt=BF16, stream=None, opts=1), o)


def bwd(**o):
    return _call("kla_attn_bwd", dict(**IN, o=0x4000, lse=0x5000, rest=None, do=0x6000, dq=0x7000, dk=0x8000, dv=0x9000, scale=0.125, window=0, **SEQS, **SIZES, dt=BF16,
                                      **WS, stream=None, opts=1), o)


PAGES = dict(n_pages=100, page=16, max_pages=8, max_len=128)


def extend(**o):
    return _call("kla_attn_extend", dict(**IN, **CACHE, o=0x4000, lse=None, scale=0.125, window=0, **SEQS, **SIZES, **PAGES, dt=BF16, **WS, stream=None), o)


def step(**o):
    return _call("kla_attn_step", dict(**IN, **CACHE, o=0x4000, scale=0.125, window=0, B=4, H=8, Hk=4, D=64, **PAGES, dt=BF16, **WS, stream=None), o)


@pytest.mark.parametrize("f,required,vectors", [
    (fwd, "q k v o", "q k v o"), (bwd, "q k v o lse do dq dk dv", "q k v o do dq dk dv"), (extend, "q k v kc vc table cached o", "q k v kc vc o"),
    (step, "q k v kc vc table cached o", "q k v kc vc o")])
def test_pointers(f, required, vectors):
    for p in required.split():
        assert f(**{p: None}) == E_NULL, p
        assert f(**{p: 0xa0001}) == E_ALIGN, p
    for p in vectors.split():                              # rows are taken 16 bytes at a time
        assert f(**{p: 0xa0008}) == E_ALIGN, p
    for ld in ("ld_q", "ld_k", "ld_v"):
        assert f(**{ld: 516}) == E_ALIGN, ld               # 8 bytes in bf16
        assert f(**{ld: 518, "dt": F32}) == E_ALIGN, ld
    for dt in (-1, 2, 7):
        assert f(dt=dt) == E_DTYPE


@pytest.mark.parametrize("f", [fwd, bwd, extend, step])
def test_shapes(f):
    nan, inf = float("nan"), float("inf")
    for bad in (dict(H=0), dict(Hk=0), dict(H=7), dict(H=-8), dict(Hk=-4), dict(Hk=16), dict(D=32), dict(D=96), dict(D=256), dict(D=0), dict(D=-64), dict(ld_q=504),
                dict(ld_k=248), dict(ld_v=248), dict(ld_q=(1 << 24) + 8), dict(ld_k=(1 << 24) + 8), dict(ld_v=(1 << 24) + 8), dict(scale=0.0), dict(scale=-1.0),
                dict(scale=nan), dict(scale=inf), dict(window=-1)):
        assert f(**bad) == E_SHAPE, bad
    assert f(H=1 << 20, Hk=1 << 10, ld_q=1 << 26) == E_SHAPE     # H D beyond 2^24
    if f is step:
        assert f(B=-1) == E_SHAPE
        return
    for bad in (dict(N=-1), dict(T=-1), dict(T=(1 << 30) // 2 + 1)):
        assert f(**bad) == E_SHAPE, bad
    if f is not extend:
        for bad in (dict(opts=2), dict(opts=1 << 30), dict(opts=0, window=5)):
            assert f(**bad) == E_SHAPE, bad


@pytest.mark.parametrize("f", [extend, step])
def test_pages(f):
    for bad in (dict(page=0), dict(page=8), dict(page=24), dict(page=2048), dict(page=-16), dict(n_pages=0), dict(n_pages=-1), dict(max_pages=0), dict(max_pages=-1),
                dict(ld_table=7), dict(max_pages=(1 << 26) + 1, ld_table=1 << 27), dict(max_len=-1)):
        assert f(**bad) == E_SHAPE, bad


@pytest.mark.parametrize("f", [fwd, bwd, extend])
def test_offsets(f):
    dev, host = 0xc000, CU.ctypes.data
    assert f(n_seq=-1) == E_SHAPE
    assert f(N=2, cu_dev=dev, cu_host=host, n_seq=2) == E_SHAPE
    assert f(cu_dev=None, cu_host=host, n_seq=2) == E_NULL and f(cu_dev=dev, cu_host=None, n_seq=2) == E_NULL
    assert f(cu_dev=dev, cu_host=host, n_seq=2, T=65) == E_SEQ
    assert f(cu_dev=dev, cu_host=host, n_seq=0) == E_SEQ
    for wrong in ([1, 30, 64], [0, 70, 64], [0, 30, 63]):
        w = np.array(wrong, dtype=np.int32)
        assert f(cu_dev=dev, cu_host=w.ctypes.data, n_seq=2) == E_SEQ, wrong


def test_outputs_apart_from_inputs():
    for f in (fwd, extend, step):
        for p in ("q", "k", "v"):
            assert f(o=IN[p]) == E_SHAPE, p
    for out in ("dq", "dk", "dv"):
        for p in ("q", "k", "v"):
            assert bwd(**{out: IN[p]}) == E_SHAPE
        assert bwd(**{out: 0x4000}) == E_SHAPE and bwd(**{out: 0x6000}) == E_SHAPE
    assert bwd(dq=0x8000) == E_SHAPE and bwd(dv=0x8000) == E_SHAPE and bwd(dv=0x7000) == E_SHAPE
    for f in (extend, step):
        assert f(vc=0x10000) == E_SHAPE
        for c in ("kc", "vc"):
            for p in (0x1000, 0x2000, 0x3000, 0x4000):
                assert f(**{c: p}) == E_SHAPE


def test_remainder():
    for f in (fwd, bwd):
        assert f(rest=0xb000, dt=F32) == E_DTYPE and f(rest=0xb008) == E_ALIGN
    for p in (0x1000, 0x2000, 0x3000, 0x4000):
        assert fwd(rest=p) == E_SHAPE
    for out in ("dq", "dk", "dv"):
        assert bwd(rest=0xb000, **{out: 0xb000}) == E_SHAPE


def test_workspace():
    for f in (bwd, lambda **o: extend(max_len=4096, **o), lambda **o: step(max_len=4096, **o)):
        assert f(ws=None) == E_WS and f(ws=0x100010) == E_WS and f(ws_bytes=100) == E_WS


def test_queries():
    lib = kla.lib()
    rows = 8 * 4096 * 8
    assert lib.kla_attn_bwd_workspace_bytes(8, 4096, 8, 8, 128, None, 0, BF16) == 2 * 4 * rows      # a float or two for each row
    assert lib.kla_attn_bwd_workspace_bytes(1, 512, 8, 2, 128, None, 0, BF16) > 2 * 4 * 512 * 8     # and parts of dk, dv where workgroups are few
    wrong = np.array([0, 30, 63], dtype=np.int32)
    for q, more in ((lib.kla_attn_bwd_workspace_bytes, (BF16,)), (lib.kla_attn_extend_workspace_bytes, (0, 4096, BF16))):
        assert q(1, 64, 8, 4, 64, CU.ctypes.data, 2, *more) > 0
        for bad in ((-1, 64, 8, 4, 64, None, 0), (1, -1, 8, 4, 64, None, 0), (1, 64, 8, 3, 64, None, 0), (1, 64, 8, 4, 65, None, 0), (1, 64, 0, 4, 64, None, 0),
                    (1, 64, 8, 4, 64, None, 2), (2, 64, 8, 4, 64, CU.ctypes.data, 2), (1, 64, 8, 4, 64, wrong.ctypes.data, 2)):
            assert q(*bad, *more) == 0, bad
        assert q(1, 64, 8, 4, 64, None, 0, *more[:-1], 7) == 0
    e = lib.kla_attn_extend_workspace_bytes
    assert e(4, 1, 8, 4, 64, None, 0, 0, 16, BF16) == 0                       # short caches: one part, no workspace
    assert e(4, 1, 8, 4, 64, None, 0, 0, -1, BF16) == 0 and e(4, 1, 8, 4, 64, None, 0, -1, 4096, BF16) == 0
    assert e(1, 1, 8, 4, 64, None, 0, 0, 4096, BF16) >= 2 * 8 * 65 * 4


def test_nothing_to_do():
    """No tokens: accepted before any pointer is looked at, nothing launched."""
    none = dict(q=None, k=None, v=None, o=None)
    for shape in (dict(N=0), dict(T=0)):
        assert fwd(**none, **shape) == OK
        assert bwd(**none, lse=None, do=None, dq=None, dk=None, dv=None, **shape) == OK
        assert extend(**none, kc=None, vc=None, table=None, cached=None, **shape) == OK
    assert step(**none, kc=None, vc=None, table=None, cached=None, B=0) == OK
    zeros = np.zeros(4, dtype=np.int32)
    assert fwd(**none, cu_dev=0xc000, cu_host=zeros.ctypes.data, n_seq=3, T=0) == OK


def test_options_match_the_header():
    assert "KLA_ATTN_CAUSAL = %d" % kla.KLA_ATTN_CAUSAL in open(kla.HEADER_PATH).read()


def test_python_refusals():
    q, k = torch.zeros(2, 5, 8, 64), torch.zeros(2, 5, 4, 64)
    with pytest.raises(RuntimeError, match="GPU"):
        kla.kla_attn_fwd(q, k, k)
    with pytest.raises(RuntimeError, match="GPU"):
        kla.kla_attn(q, k, k)
    with pytest.raises(ValueError, match="v must"):
        kla.kla_attn_fwd(q, k, k[:, :4])
    with pytest.raises(ValueError, match="k must"):
        kla.kla_attn_fwd(q, k[..., :32], k[..., :32])
    with pytest.raises(ValueError, match="share"):
        kla.kla_attn_fwd(q, torch.zeros(2, 5, 3, 64), torch.zeros(2, 5, 3, 64))
    with pytest.raises(TypeError, match="k must"):
        kla.kla_attn_fwd(q, k.bfloat16(), k)
    with pytest.raises(TypeError):
        kla.kla_attn_fwd(q.half(), k.half(), k.half())
    with pytest.raises(ValueError, match=r"q must"):
        kla.kla_attn_fwd(q[0], k, k)
    with pytest.raises(TypeError, match="cu_seqlens"):
        kla.kla_attn_fwd(q[:1], k[:1], k[:1], cu_seqlens=torch.tensor([0, 5]))
    with pytest.raises(ValueError, match="without cu_seqlens"):
        kla.kla_attn_fwd(q[:1], k[:1], k[:1], cu_seqlens_host=torch.tensor([0, 5], dtype=torch.int32))
    with pytest.raises(ValueError, match="size"):
        kla.kla_attn_fwd(q, k, k, window=2 ** 31)
    with pytest.raises(ValueError, match="required"):
        kla.kla_attn_bwd(q, k, k, q, None, q)
    c, table, cached = torch.zeros(10, 4, 16, 64), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    for f, lead in ((kla.kla_attn_extend, slice(None)), (kla.kla_attn_step, 0)):
        a = (q[:, lead], k[:, lead], k[:, lead])
        with pytest.raises(RuntimeError, match="GPU"):
            f(*a, c, c, table, cached)
    a = (q[:, 0], k[:, 0], k[:, 0])
    with pytest.raises(ValueError, match="q must"):
        kla.kla_attn_step(q, k, k, c, c, table, cached)
    for bad, what in ((dict(k_cache=c[:, :3]), "k_cache"), (dict(v_cache=c[:9]), "v_cache"), (dict(k_cache=c.bfloat16()), "k_cache"),
                      (dict(page_table=table[:1]), "page_table"), (dict(page_table=table.long()), "page_table"), (dict(cached=cached[:1]), "cached"),
                      (dict(cached=cached.float()), "cached"), (dict(out=torch.zeros(2, 8, 32)), "out"), (dict(page_table=table[0]), "page_table"),
                      (dict(max_len=2 ** 31), "size")):
        d = dict(dict(k_cache=c, v_cache=c, page_table=table, cached=cached), **bad)
        with pytest.raises((ValueError, TypeError), match=what):
            kla.kla_attn_step(*a, **d)
        if "out" not in bad:
            with pytest.raises((ValueError, TypeError), match=what):
                kla.kla_attn_extend(q, k, k, **d)


def test_python_refuses_tokens_too_far_apart():
    """By the name of the tensor and the limit; single tokens over a cache are not refused for it."""
    q = torch.empty_strided((1, 2, 8, 64), (1 << 26, (1 << 24) + 4, 64, 1))
    k = torch.zeros(1, 2, 4, 64)
    c, table, cached = torch.zeros(10, 4, 16, 64), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    lse = torch.zeros(1, 2, 8)
    for f in (lambda a, b, v: kla.kla_attn_fwd(a, b, v), lambda a, b, v: kla.kla_attn(a, b, v), lambda a, b, v: kla.kla_attn_bwd(a, b, v, k, lse, k),
              lambda a, b, v: kla.kla_attn_extend(a, b, v, c, c, table[:1], cached[:1])):
        with pytest.raises(ValueError, match=r"q: the tokens .* 2\^24"):
            f(q, k, k)
        with pytest.raises(ValueError, match=r"v: the tokens .* 2\^24"):
            f(k.repeat(1, 1, 2, 1), k, q[:, :, :4])
    with pytest.raises(RuntimeError, match="GPU"):
        kla.kla_attn_step(q[0], k[0], k[0], c, c, table, cached)
    with pytest.raises(RuntimeError, match="GPU"):
        kla.kla_attn_extend(q.transpose(0, 1), k.transpose(0, 1), k.transpose(0, 1), c, c, table, cached)


@pytest.mark.parametrize("f", [fwd, bwd, extend, step])
def test_groups_beyond_the_limit(f):
    assert f(H=(1 << 16) + 1, Hk=1, ld_q=1 << 23) == E_SHAPE


def test_cases_of_many_tiles_reach_their_kernels():
    """The batches of MANY_TILES come to as many tiles as the library asks for before it takes the kernels that they are there for."""
    src = open(os.path.join(os.path.dirname(kla.__file__), "csrc", "kla_attn_api.hip")).read()
    apart = int(re.search(r"constexpr long kAttnBeside = (\d+);", src).group(1))
    share = [int(x) for x in re.search(r"units >= \(D == 64 \? (\d+) : (\d+)\) \? 128 : 32", src).groups()]
    assert min(many_tiles(n) for n in MANY_TILES) >= max(apart, *share)
