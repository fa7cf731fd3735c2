"""Softmax attention beside the recurrences of a hybrid stack (include/kla.h): over whole sequences, and for new tokens over a paged cache.
Argument marshalling only, as in the package itself: every step runs in the HIP kernels.

kla_attn_fwd / kla_attn_bwd are the two directions and kla_attn the differentiable call; kla_attn_extend takes new tokens of several sequences over
their cached ones, kla_attn_step one token of each.  q [..., H, D] and k, v [..., Hk, D] may be column ranges of a wider tensor: the heads
of a token are contiguous, the tokens evenly spaced and at most 2^24 elements apart, and a row starts at a multiple of 16 bytes.  (Single tokens over
a cache that are further apart, like q[:, t] of a long batch, are copied first.)
"""
from __future__ import annotations

import ctypes

import torch

from . import _check, _dev, _dt, _ptr, _stream, _written, _ws_bytes, lib
from .layer import _Offsets, _batch, _call, _eager, _host, _native, _no_second, _on_gpu, _rows, _sizes, _workspace

KLA_ATTN_CAUSAL = 1
MAX_STRIDE = 2 ** 24                                     # elements from one token to the next

_vp, _i, _l, _f, _z, _u = ctypes.c_void_p, ctypes.c_int, ctypes.c_long, ctypes.c_float, ctypes.c_size_t, ctypes.c_uint
_SEQS = [_vp, _vp, _i]
_IN = [_vp, _l] * 3
_CACHE = [_vp, _vp, _vp, _l, _vp]
SIGNATURES = {
    "kla_attn_fwd": (_i, [*_IN, _vp, _vp, _vp, _f, _i, *_SEQS, *[_i] * 6, _vp, _u]),
    "kla_attn_bwd_workspace_bytes": (_z, [*[_i] * 5, _vp, _i, _i]),
    "kla_attn_bwd": (_i, [*_IN, *[_vp] * 7, _f, _i, *_SEQS, *[_i] * 6, _vp, _z, _vp, _u]),
    "kla_attn_extend_workspace_bytes": (_z, [*[_i] * 5, _vp, *[_i] * 4]),
    "kla_attn_extend": (_i, [*_IN, *_CACHE, _vp, _vp, _f, _i, *_SEQS, *[_i] * 10, _vp, _z, _vp]),
    "kla_attn_step": (_i, [*_IN, *_CACHE, _vp, _f, _i, *[_i] * 9, _vp, _z, _vp]),
}
# what kla_binding.so calls, in the order of its bind_attn
NATIVE = ("kla_attn_fwd", "kla_attn_bwd_workspace_bytes", "kla_attn_bwd", "kla_attn_extend_workspace_bytes", "kla_attn_extend", "kla_attn_step")


def _scale(scale, q):
    return q.shape[-1] ** -0.5 if scale is None and q.dim() and q.shape[-1] else float(scale or 0.0)


def _heads(q, k, v, lead):
    """lead: number of leading dimensions; returns H, Hk, D, the type and the token strides of q, k, v."""
    if q.dim() != lead + 2 or k.dim() != lead + 2:
        raise ValueError("q must be [%s, H, D] and k, v [%s, Hk, D]" % (("N, T",) * 2 if lead == 2 else ("B",) * 2))
    at, (H, D), Hk = tuple(q.shape[:lead]), q.shape[-2:], k.shape[-2]
    dt = _dt(q)
    _sizes(*q.shape, Hk)
    _check("k", k, (*at, Hk, D), q.dtype)
    _check("v", v, (*at, Hk, D), q.dtype)
    if Hk == 0 or H % Hk:
        raise ValueError("%d query heads cannot share %d key heads evenly" % (H, Hk))
    ld = _rows("q", q, 2), _rows("k", k, 2), _rows("v", v, 2)
    for name, n in zip("qkv", ld):
        if n > MAX_STRIDE:
            raise ValueError("%s: the tokens are %d elements apart, more than 2^24" % (name, n))
    return H, Hk, D, dt, ld


def _near(*ts):
    """Single tokens, one of each sequence: a copy of those that are too far apart, like a position of all sequences of a long batch."""
    return [t.contiguous() if t.dim() > 2 and _rows(name, t, 2) > MAX_STRIDE else t for name, t in zip("qkv", ts)]


def kla_attn_fwd(q, k, v, scale=None, causal=True, window=0, cu_seqlens=None, cu_seqlens_host=None, want_lse=True, out=None, lse=None, rest=None):
    """Softmax attention of q [N,T,H,D] over k, v [N,T,Hk,D] of the same sequence (D 64 or 128, H a multiple of Hk): returns (o, lse), lse [N,T,H]
    fp32 the logarithms of the rows' sums (None unless want_lse).  causal: a token sees those up to itself, and with window > 0 only the last
    `window` of them; scale: of the scores, D ** -0.5 by default.  Packed batches by cu_seqlens as in kla_chunk_fwd.  rest: a bfloat16 tensor like o that
    receives what o's rounding leaves out, for kla_attn_bwd."""
    host = _host(cu_seqlens, cu_seqlens_host)
    r = _native("attn_fwd", "kla_attn_fwd", q, k, v, _scale(scale, q), bool(causal), window, cu_seqlens, host, bool(want_lse), out, lse, rest)
    if r is not None:
        return r
    H, Hk, D, dt, ld = _heads(q, k, v, 2)
    N, T = q.shape[:2]
    _, cu_hp, n_seq, _n = _batch(q, cu_seqlens, host)
    _sizes(window)
    _check("out", out, (N, T, H, D), q.dtype)
    _check("lse", lse, (N, T, H), torch.float32)
    _check("rest", rest, (N, T, H, D), torch.bfloat16)
    _on_gpu(q, k, v, cu_seqlens, out, lse, rest)
    _dev(cu_seqlens, out, lse, rest)
    given = out, lse, rest
    if out is None:
        out = torch.empty((N, T, H, D), dtype=q.dtype, device=q.device)
    if lse is None and want_lse:
        lse = torch.empty((N, T, H), dtype=torch.float32, device=q.device)
    _call("kla_attn_fwd", _ptr(q), ld[0], _ptr(k), ld[1], _ptr(v), ld[2], _ptr(out), _ptr(lse), _ptr(rest), _scale(scale, q), int(window), _ptr(cu_seqlens),
          cu_hp, n_seq, N, T, H, Hk, D, dt, _stream(), KLA_ATTN_CAUSAL if causal else 0)
    _written(*given)
    return out, lse


def kla_attn_bwd(q, k, v, o, lse, d_o, scale=None, causal=True, window=0, cu_seqlens=None, cu_seqlens_host=None, workspace=None, rest=None):
    """Backward of kla_attn_fwd, from what it returned (and left in rest): a dict of dq, dk, dv."""
    for name, t in (("o", o), ("lse", lse), ("d_o", d_o)):
        if t is None:
            raise ValueError("%s is required" % name)
    H, Hk, D, dt, ld = _heads(q, k, v, 2)
    N, T = q.shape[:2]
    _, cu_hp, n_seq, _n = _batch(q, cu_seqlens, cu_seqlens_host)
    _sizes(window)
    _check("o", o, (N, T, H, D), q.dtype)
    _check("d_o", d_o, (N, T, H, D), q.dtype)
    _check("lse", lse, (N, T, H), torch.float32)
    _check("rest", rest, (N, T, H, D), torch.bfloat16)
    _on_gpu(q, k, v, o, lse, d_o, cu_seqlens, workspace, rest)
    _dev(o, lse, d_o, cu_seqlens, workspace, rest)
    if workspace is None:
        workspace = _workspace(int(lib().kla_attn_bwd_workspace_bytes(N, T, H, Hk, D, cu_hp, n_seq, dt)), q)
    g = {name: torch.empty(t.shape, dtype=t.dtype, device=t.device) for name, t in (("dq", q), ("dk", k), ("dv", v))}
    _call("kla_attn_bwd", _ptr(q), ld[0], _ptr(k), ld[1], _ptr(v), ld[2], _ptr(o), _ptr(lse), _ptr(rest), _ptr(d_o), *(_ptr(t) for t in g.values()),
          _scale(scale, q), int(window), _ptr(cu_seqlens), cu_hp, n_seq, N, T, H, Hk, D, dt, _ptr(workspace), _ws_bytes(workspace), _stream(),
          KLA_ATTN_CAUSAL if causal else 0)
    return g


def _at_16_bytes(t):
    """Contiguous and at a multiple of 16 bytes: a gradient can be a piece of a larger tensor, wherever it begins."""
    t = t.contiguous()
    return t if t.data_ptr() % 16 == 0 else t.clone()


class _Attn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, scale, causal, window, cu_seqlens, cu_seqlens_host):
        ctx.offsets = _Offsets(cu_seqlens, cu_seqlens_host)
        wanted = any(ctx.needs_input_grad)
        rest = torch.empty(q.shape, dtype=q.dtype, device=q.device) if wanted and q.dtype == torch.bfloat16 else None
        o, lse = kla_attn_fwd(q, k, v, scale, causal, window, cu_seqlens, cu_seqlens_host, want_lse=wanted, rest=rest)
        ctx.save_for_backward(q, k, v, o, lse, rest)
        ctx.misc = (scale, causal, window)
        return o

    @staticmethod
    def backward(ctx, d_o):
        _no_second("kla_attn")
        *saved, rest = ctx.saved_tensors
        g = kla_attn_bwd(*saved, _at_16_bytes(d_o), *ctx.misc, rest=rest, **ctx.offsets.check())
        return (*g.values(), None, None, None, None, None)


def kla_attn(q, k, v, scale=None, causal=True, window=0, cu_seqlens=None, cu_seqlens_host=None):
    """Differentiable kla_attn_fwd: o, gradients with respect to q, k and v.  The graph holds q, k, v, o, the rows' lse and, in bfloat16, what o's
    rounding leaves out."""
    host = _host(cu_seqlens, cu_seqlens_host)
    if _eager():
        r = _native("attn_train", "kla_attn_fwd", q, k, v, _scale(scale, q), bool(causal), window, cu_seqlens, host)
        if r is not None:
            return r
    return _Attn.apply(q, k, v, scale, bool(causal), int(window), cu_seqlens, host)


def _cache_check(q, k_cache, v_cache, page_table, cached, Hk, D, n):
    if k_cache.dim() != 4 or page_table.dim() != 2:
        raise ValueError("k_cache, v_cache must be [pages, Hk, page, D] and page_table [sequences, max_pages]")
    n_pages, page, max_pages = k_cache.shape[0], k_cache.shape[2], page_table.shape[1]
    _check("k_cache", k_cache, (n_pages, Hk, page, D), q.dtype)
    _check("v_cache", v_cache, (n_pages, Hk, page, D), q.dtype)
    _check("page_table", page_table, (n, max_pages), torch.int32)
    _check("cached", cached, (n,), torch.int32)
    _sizes(n_pages, page, max_pages, max_pages * page)
    return n_pages, page, max_pages, _rows("page_table", page_table)


def kla_attn_extend(q, k, v, k_cache, v_cache, page_table, cached, scale=None, window=0, cu_seqlens=None, cu_seqlens_host=None, max_len=None,
                    want_lse=False, out=None, lse=None, workspace=None):
    """New tokens of several sequences over a paged cache: q [N,T,H,D], k, v [N,T,Hk,D] (packed batches by cu_seqlens) stand behind cached [sequences]
    (int32) earlier tokens each and see those and the new ones up to themselves (the last `window` of them, if it is not 0).  The keys and
    values of position p of sequence s stand in k_cache, v_cache [pages,Hk,page,D] at [page_table[s, p // page], :, p % page] (page_table
    int32, page a power of two from 16 to 1024); those of the new tokens are stored there.  cached is not advanced.  Returns o, with want_lse
    (o, lse).  max_len: a bound of cached + new tokens, if the caller knows a closer one than the table's width (only how the work
    is cut depends on it: a chunk over short caches in a wide table can be slower without)."""
    host = _host(cu_seqlens, cu_seqlens_host)
    if workspace is None:
        r = _native("attn_extend", "kla_attn_extend", q, k, v, k_cache, v_cache, page_table, cached, _scale(scale, q), window, cu_seqlens, host, max_len,
                    bool(want_lse), out, lse)
        if r is not None:
            return r if r[1] is not None else r[0]
    if cu_seqlens is None and q.dim() == 4 and q.shape[1] == 1:
        q, k, v = _near(q, k, v)
    H, Hk, D, dt, ld = _heads(q, k, v, 2)
    N, T = q.shape[:2]
    _, cu_hp, n_seq, n = _batch(q, cu_seqlens, host)
    _sizes(window)
    n_pages, page, max_pages, ld_table = _cache_check(q, k_cache, v_cache, page_table, cached, Hk, D, n)
    max_len = max_pages * page if max_len is None else int(max_len)
    _sizes(max_len)
    _check("out", out, (N, T, H, D), q.dtype)
    _check("lse", lse, (N, T, H), torch.float32)
    _on_gpu(q, k, v, k_cache, v_cache, page_table, cached, cu_seqlens, out, lse, workspace)
    _dev(k_cache, v_cache, cached, cu_seqlens, out, lse, workspace)
    if workspace is None:
        workspace = _workspace(int(lib().kla_attn_extend_workspace_bytes(N, T, H, Hk, D, cu_hp, n_seq, int(window), max_len, dt)), q)
    given = out, lse
    if out is None:
        out = torch.empty((N, T, H, D), dtype=q.dtype, device=q.device)
    if lse is None and want_lse:
        lse = torch.empty((N, T, H), dtype=torch.float32, device=q.device)
    _call("kla_attn_extend", _ptr(q), ld[0], _ptr(k), ld[1], _ptr(v), ld[2], _ptr(k_cache), _ptr(v_cache), _ptr(page_table), ld_table, _ptr(cached),
          _ptr(out), _ptr(lse), _scale(scale, q), int(window), _ptr(cu_seqlens), cu_hp, n_seq, N, T, H, Hk, D, n_pages, page, max_pages, max_len, dt,
          _ptr(workspace), _ws_bytes(workspace), _stream())
    _written(k_cache, v_cache, *given)
    return (out, lse) if lse is not None else out


def kla_attn_step(q, k, v, k_cache, v_cache, page_table, cached, scale=None, window=0, max_len=None, out=None, workspace=None):
    """One new token of B sequences: q [B,H,D], k, v [B,Hk,D]; otherwise as kla_attn_extend.  Returns o [B,H,D]."""
    if workspace is None:
        r = _native("attn_step", "kla_attn_step", q, k, v, k_cache, v_cache, page_table, cached, _scale(scale, q), window, max_len, out)
        if r is not None:
            return r
    q, k, v = _near(q, k, v)
    H, Hk, D, dt, ld = _heads(q, k, v, 1)
    B = q.shape[0]
    _sizes(window)
    n_pages, page, max_pages, ld_table = _cache_check(q, k_cache, v_cache, page_table, cached, Hk, D, B)
    max_len = max_pages * page if max_len is None else int(max_len)
    _sizes(max_len)
    _check("out", out, (B, H, D), q.dtype)
    _on_gpu(q, k, v, k_cache, v_cache, page_table, cached, out, workspace)
    _dev(k_cache, v_cache, cached, out, workspace)
    if workspace is None:
        workspace = _workspace(int(lib().kla_attn_extend_workspace_bytes(B, 1, H, Hk, D, None, 0, int(window), max_len, dt)), q)
    given = out
    if out is None:
        out = torch.empty((B, H, D), dtype=q.dtype, device=q.device)
    _call("kla_attn_step", _ptr(q), ld[0], _ptr(k), ld[1], _ptr(v), ld[2], _ptr(k_cache), _ptr(v_cache), _ptr(page_table), ld_table, _ptr(cached),
          _ptr(out), _scale(scale, q), int(window), B, H, Hk, D, n_pages, page, max_pages, max_len, dt, _ptr(workspace), _ws_bytes(workspace), _stream())
    _written(k_cache, v_cache, given)
    return out
