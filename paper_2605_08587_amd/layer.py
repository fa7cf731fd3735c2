"""The operators around the recurrence in a layer (second half of include/kla.h): short convolution, selective scan, the norms before
and after a block.  Argument marshalling only, as in the package itself: every step runs in the HIP kernels.

*_fwd / *_bwd are the two directions, *_step the form for single tokens, and the plain names (kla_conv, kla_ssm, kla_add_norm,
kla_gated_norm) one differentiable call each.  Inputs [..., D] may be column ranges of a wider tensor (x, z = proj.split(...)): a row has
to be contiguous and the rows evenly spaced.  Parameters are fp32; activations bfloat16 or float32, all of one type.
"""
from __future__ import annotations

import ctypes

import torch

from . import KlaError, _binding, _check, _counting, _dev, _dt, _host_cu, _ptr, _stream, _written, _ws_bytes, lib

KLA_LAYER_SILU, KLA_LAYER_SOFTPLUS, KLA_LAYER_SIGMOID, KLA_LAYER_GATE_FIRST = 1, 2, 4, 8

_vp, _i, _l, _f, _z, _u = ctypes.c_void_p, ctypes.c_int, ctypes.c_long, ctypes.c_float, ctypes.c_size_t, ctypes.c_uint
_SEQS = [_vp, _vp, _i]
_SSM_IN = [_vp, _l, _vp, _l, _vp, _vp, _l, _vp, _l, _vp, _vp, _l, _vp]     # u .. delta_bias
SIGNATURES = {
    "kla_conv_fwd": (_i, [_vp, _l, _vp, _vp, _vp, _vp, _vp, *_SEQS, _i, _i, _i, _i, _i, _vp, _u]),
    "kla_conv_bwd_workspace_bytes": (_z, [_i] * 4),
    "kla_conv_bwd": (_i, [_vp, _l, *[_vp] * 9, *_SEQS, *[_i] * 5, _vp, _z, _vp, _u]),
    "kla_conv_step": (_i, [_vp, _l, _vp, _vp, _vp, _vp, *[_i] * 4, _vp, _u]),
    "kla_ssm_fwd_workspace_bytes": (_z, [*[_i] * 5, _vp, _i]),
    "kla_ssm_saved_bytes": (_z, [*[_i] * 5, _vp, _i]),
    "kla_ssm_bwd_workspace_bytes": (_z, [*[_i] * 5, _vp, _i, _i]),
    "kla_ssm_fwd": (_i, [*_SSM_IN, _vp, _vp, _vp, _vp, _z, *_SEQS, *[_i] * 6, _vp, _z, _vp, _u]),
    "kla_ssm_bwd": (_i, [*_SSM_IN, *[_vp] * 4, _z, *[_vp] * 9, *_SEQS, *[_i] * 6, _vp, _z, _vp, _u]),
    "kla_ssm_step": (_i, [*_SSM_IN, _vp, _vp, *[_i] * 5, _vp, _u]),
    "kla_add_norm_fwd": (_i, [_vp, _l, _vp, _vp, _vp, _f, _vp, _vp, _l, _i, _i, _i, _vp]),
    "kla_add_norm_bwd_workspace_bytes": (_z, [_l, _i, _i]),
    "kla_add_norm_bwd": (_i, [_vp, _l, _vp, _vp, _vp, _f, *[_vp] * 6, _l, _i, _i, _i, _vp, _z, _vp]),
    "kla_gated_norm_fwd": (_i, [_vp, _l, _vp, _l, _vp, _f, _vp, _l, _i, _i, _i, _vp, _u]),
    "kla_gated_norm_bwd_workspace_bytes": (_z, [_l, _i, _i, _i]),
    "kla_gated_norm_bwd": (_i, [_vp, _l, _vp, _l, _vp, _f, *[_vp] * 4, _l, _i, _i, _i, _vp, _z, _vp, _u]),
}
# what kla_binding.so calls, in the order of its bind_layer
NATIVE = ("kla_conv_fwd", "kla_conv_bwd_workspace_bytes", "kla_conv_bwd", "kla_conv_step", "kla_ssm_fwd_workspace_bytes", "kla_ssm_saved_bytes",
          "kla_ssm_fwd", "kla_ssm_bwd_workspace_bytes", "kla_ssm_bwd", "kla_ssm_step", "kla_add_norm_fwd", "kla_add_norm_bwd_workspace_bytes",
          "kla_add_norm_bwd", "kla_gated_norm_fwd", "kla_gated_norm_bwd_workspace_bytes", "kla_gated_norm_bwd")


def _native(entry, name, *args):
    """The call through the native half of the binding, or None if it does not take it."""
    f = getattr(_binding(), entry, None)
    r = None if f is None else f(*args)
    if type(r) is int:
        raise KlaError(r, name)
    return r


def _host(cu_seqlens, cu_seqlens_host):
    return _host_cu(cu_seqlens)[0] if cu_seqlens is not None and cu_seqlens_host is None else cu_seqlens_host


def _eager():
    """Tracing, function transforms and forward-mode differentiation are for the Python functions to take or to refuse."""
    return torch._C._get_tracing_state() is None and not torch._C._are_functorch_transforms_active() and torch.autograd.forward_ad._current_level < 0


def _no_second(name):
    if torch.is_grad_enabled():
        raise RuntimeError("%s: the gradients have no gradients of their own (create_graph)" % name)


def _rows(name, t, inner=1):
    """Elements from one row (the last `inner` dimensions) to the next."""
    if t is None:
        return 0
    row = 1
    for size, stride in zip(reversed(t.shape[-inner:]), reversed(t.stride()[-inner:])):
        if size != 1 and stride != row and t.numel():
            raise ValueError("%s: the last %s must be contiguous" % (name, "dimension" if inner == 1 else "%d dimensions" % inner))
        row *= size
    ld, count = None, 1
    for size, stride in zip(reversed(t.shape[:-inner]), reversed(t.stride()[:-inner])):
        if size != 1:
            if ld is not None and stride != ld * count and t.numel():
                raise ValueError("%s: the rows must be evenly spaced" % name)
            ld = stride if ld is None else ld
        count *= size
    ld = row if ld is None else ld
    if ld < row and t.numel():
        raise ValueError("%s: the rows must not overlap" % name)
    return max(ld, row)


def _on_gpu(*ts):
    """GPU tensors, whatever their strides, on the current device."""
    for t in ts:
        if t is not None:
            if not t.is_cuda:
                raise RuntimeError("KLA kernels need GPU tensors (no CPU fallback)")
            if t.device.index != torch.cuda.current_device():
                raise RuntimeError("tensors must be on the current device")


def _call(name, *args):
    rc = getattr(lib(), name)(*args)
    if rc != 0:
        raise KlaError(rc, name)


def _sizes(*ns):
    if max(ns) >= 2 ** 31:
        raise ValueError("a size of %d" % max(ns))


def _workspace(need, like):
    return torch.empty(need, dtype=torch.uint8, device=like.device) if need else None


def _batch(x, cu_seqlens, cu_seqlens_host):
    cu_host, cu_hp, n_seq = _host_cu(cu_seqlens, cu_seqlens_host)
    if cu_seqlens is None and cu_seqlens_host is not None:
        raise ValueError("cu_seqlens_host without cu_seqlens")
    return cu_host, cu_hp, n_seq, (n_seq if n_seq > 0 else x.shape[0])


class _Offsets:
    """The offsets of a packed batch between a forward and its backward: a host copy of its own, and the device's unchanged."""

    def __init__(self, cu, host):
        self.cu = self.host = None
        if cu is not None:
            self.host = _host_cu(cu, host)[0].clone()
            self.cu = _counting(cu)
            self.version = self.cu._version

    def check(self):
        if self.cu is not None and self.cu._version != self.version:
            raise RuntimeError("one of the variables needed for gradient computation has been modified by an inplace operation: cu_seqlens")
        return dict(cu_seqlens=self.cu, cu_seqlens_host=self.host)


# ---- short convolution ---------------------------------------------------------------------------------------------------------------


def _conv_check(x, weight, bias, state, cu_seqlens, cu_seqlens_host, **more):
    if x.dim() != 3 or weight.dim() != 2:
        raise ValueError("x must be [N, T, D] and weight [D, W]")
    N, T, D = x.shape
    W = weight.shape[1]
    dt = _dt(x)
    _, cu_hp, n_seq, n_states = host = _batch(x, cu_seqlens, cu_seqlens_host)
    _sizes(N, T, D, W)
    _check("weight", weight, (D, W), torch.float32)
    _check("bias", bias, (D,), torch.float32)
    st = (n_states, W - 1, D)
    _check("state", state, st, x.dtype)
    for name, (t, shape, dtype) in more.items():
        _check(name, t, {"y": (N, T, D), "state": st, "w": (D, W), "b": (D,)}[shape], x.dtype if dtype is None else dtype)
    _on_gpu(x)
    _dev(weight, bias, state, cu_seqlens, *(t for t, _, _ in more.values()))
    _on_gpu(weight, bias, state, cu_seqlens)
    return N, T, D, W, dt, st, host


def kla_conv_fwd(x, weight, bias=None, state=None, cu_seqlens=None, cu_seqlens_host=None, silu=True, want_state=True, out=None,
                 state_out=None):
    """Short causal convolution of every channel of x [N,T,D] (weight [D,W] fp32, W = 2..4, bias [D] fp32) with SiLU; returns
    (y, state_out): state_out [n_states,W-1,D] are the last W-1 inputs of every sequence (None unless want_state), what `state` of
    the call for the tokens that follow takes.  Packed batches by cu_seqlens as in kla_chunk_fwd."""
    host = _host(cu_seqlens, cu_seqlens_host)
    r = _native("conv_fwd", "kla_conv_fwd", x, weight, bias, state, cu_seqlens, host, bool(silu), bool(want_state), out, state_out)
    if r is not None:
        return r
    N, T, D, W, dt, st, (_, cu_hp, n_seq, _n) = _conv_check(x, weight, bias, state, cu_seqlens, host, out=(out, "y", None),
                                                         state_out=(state_out, "state", None))
    ld = _rows("x", x)
    given = out, state_out
    if out is None:
        out = torch.empty((N, T, D), dtype=x.dtype, device=x.device)
    if state_out is None and want_state:
        state_out = torch.empty(st, dtype=x.dtype, device=x.device)
    _call("kla_conv_fwd", _ptr(x), ld, _ptr(weight), _ptr(bias), _ptr(state), _ptr(out), _ptr(state_out), _ptr(cu_seqlens), cu_hp, n_seq,
          N, T, D, W, dt, _stream(), KLA_LAYER_SILU if silu else 0)
    _written(*given)
    return out, state_out


def kla_conv_bwd(x, weight, d_y, bias=None, state=None, d_state_out=None, cu_seqlens=None, cu_seqlens_host=None, silu=True,
                 want_dstate=True):
    """Backward of kla_conv_fwd: a dict of dx, dweight, dbias and dstate (None without bias; without a state, or unwanted)."""
    N, T, D, W, dt, st, (_, cu_hp, n_seq, _n) = _conv_check(x, weight, bias, state, cu_seqlens, cu_seqlens_host, d_y=(d_y, "y", None),
                                                         d_state_out=(d_state_out, "state", None))
    if d_y is None:
        raise ValueError("d_y is required")
    ld = _rows("x", x)
    ws = _workspace(int(lib().kla_conv_bwd_workspace_bytes(N, T, D, W)), x)
    g = dict(dx=torch.empty((N, T, D), dtype=x.dtype, device=x.device), dweight=torch.empty_like(weight),
             dbias=None if bias is None else torch.empty_like(bias),
             dstate=torch.empty_like(state) if state is not None and want_dstate else None)
    _call("kla_conv_bwd", _ptr(x), ld, _ptr(weight), _ptr(bias), _ptr(state), _ptr(d_y), _ptr(d_state_out), _ptr(g["dx"]), _ptr(g["dweight"]),
          _ptr(g["dbias"]), _ptr(g["dstate"]), _ptr(cu_seqlens), cu_hp, n_seq, N, T, D, W, dt, _ptr(ws), _ws_bytes(ws), _stream(),
          KLA_LAYER_SILU if silu else 0)
    return g


def kla_conv_step(x, weight, state, bias=None, silu=True, out=None):
    """One token of B sequences: x [B,D]; state [B,W-1,D] is updated in place; returns y [B,D]."""
    r = _native("conv_step", "kla_conv_step", x, weight, state, bias, bool(silu), out)
    if r is not None:
        return r
    if x.dim() != 2 or weight.dim() != 2:
        raise ValueError("x must be [B, D] and weight [D, W]")
    (B, D), W, dt = x.shape, weight.shape[1], _dt(x)
    _sizes(B, D, W)
    _check("weight", weight, (D, W), torch.float32)
    _check("bias", bias, (D,), torch.float32)
    _check("state", state, (B, W - 1, D), x.dtype)
    _check("out", out, (B, D), x.dtype)
    _on_gpu(x, weight, bias, state, out)
    _dev(weight, bias, state, out)
    ld = _rows("x", x)
    given = out
    if out is None:
        out = torch.empty((B, D), dtype=x.dtype, device=x.device)
    _call("kla_conv_step", _ptr(x), ld, _ptr(weight), _ptr(bias), _ptr(state), _ptr(out), B, D, W, dt, _stream(), KLA_LAYER_SILU if silu else 0)
    _written(state, given)
    return out


class _Conv(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, state, cu_seqlens, cu_seqlens_host, silu, want_state):
        ctx.offsets = _Offsets(cu_seqlens, cu_seqlens_host)
        y, last = kla_conv_fwd(x, weight, bias, state, cu_seqlens, cu_seqlens_host, silu, want_state)
        ctx.save_for_backward(x, weight, bias, state)
        ctx.set_materialize_grads(False)
        ctx.silu = silu
        return y, last

    @staticmethod
    def backward(ctx, d_y, d_last):
        _no_second("kla_conv")
        x, weight, bias, state = ctx.saved_tensors
        d_y = x.new_zeros(x.shape) if d_y is None else d_y.contiguous()
        g = kla_conv_bwd(x, weight, d_y, bias, state, None if d_last is None else d_last.contiguous(), silu=ctx.silu,
                         want_dstate=ctx.needs_input_grad[3], **ctx.offsets.check())
        return g["dx"], g["dweight"], g["dbias"], g["dstate"], None, None, None, None


def kla_conv(x, weight, bias=None, state=None, cu_seqlens=None, cu_seqlens_host=None, silu=True, want_state=False):
    """Differentiable kla_conv_fwd: (y, state_out), gradients with respect to x, weight, bias and state."""
    host = _host(cu_seqlens, cu_seqlens_host)
    if _eager():
        r = _native("conv_train", "kla_conv_fwd", x, weight, bias, state, cu_seqlens, host, bool(silu), bool(want_state))
        if r is not None:
            return r
    return _Conv.apply(x, weight, bias, state, cu_seqlens, host, bool(silu), bool(want_state))


# ---- selective scan ------------------------------------------------------------------------------------------------------------------


def _ssm_check(u, delta, A, B, C, skip, z, delta_bias, lead):
    """lead: number of leading dimensions; returns D, G, S, the type and the row strides of u, delta, B, C, z."""
    if u.dim() != lead + 1 or A.dim() != 2 or B.dim() != lead + 2:
        raise ValueError("u, delta, z must be [%s, D], B, C [%s, G, S] and A [D, S]" % (("N, T",) * 2 if lead == 2 else ("N",) * 2))
    at, D = tuple(u.shape[:lead]), u.shape[-1]
    G, S = B.shape[-2:]
    dt = _dt(u)
    _sizes(*u.shape, *B.shape)
    _check("delta", delta, u.shape, u.dtype)
    _check("z", z, u.shape, u.dtype)
    _check("A", A, (D, S), torch.float32)
    _check("B", B, (*at, G, S), u.dtype)
    _check("C", C, (*at, G, S), u.dtype)
    _check("skip", skip, (D,), torch.float32)
    _check("delta_bias", delta_bias, (D,), torch.float32)
    _on_gpu(u, delta, A, B, C, skip, z, delta_bias)
    _dev(A, skip, delta_bias)
    return D, G, S, dt, (_rows("u", u), _rows("delta", delta), _rows("B", B, 2), _rows("C", C, 2), _rows("z", z))


def _ssm_in(u, delta, A, B, C, skip, z, delta_bias, ld):
    return (_ptr(u), ld[0], _ptr(delta), ld[1], _ptr(A), _ptr(B), ld[2], _ptr(C), ld[3], _ptr(skip), _ptr(z), ld[4], _ptr(delta_bias))


def kla_ssm_fwd(u, delta, A, B, C, skip=None, z=None, delta_bias=None, softplus=True, h0=None, cu_seqlens=None, cu_seqlens_host=None,
                want_hT=True, out=None, hT=None, workspace=None, _saved=None):
    """Selective state space scan of u [N,T,D] with steps softplus(delta + delta_bias), decay rates A [D,S] (fp32), input and output maps
    B, C [N,T,G,S] (G groups of D/G channels), skip [D] and gate z [N,T,D]; returns (y, hT), hT [n_states,D,S] fp32 the states after the
    last tokens, which h0 of the call for the tokens that follow takes.  Packed batches by cu_seqlens as in kla_chunk_fwd."""
    host = _host(cu_seqlens, cu_seqlens_host)
    if workspace is None and _saved is None:
        r = _native("ssm_fwd", "kla_ssm_fwd", u, delta, A, B, C, skip, z, delta_bias, bool(softplus), h0, cu_seqlens, host, bool(want_hT), out, hT)
        if r is not None:
            return r
    D, G, S, dt, ld = _ssm_check(u, delta, A, B, C, skip, z, delta_bias, 2)
    N, T = u.shape[:2]
    _, cu_hp, n_seq, n_states = _batch(u, cu_seqlens, host)
    _check("h0", h0, (n_states, D, S), torch.float32)
    _check("out", out, (N, T, D), u.dtype)
    _check("hT", hT, (n_states, D, S), torch.float32)
    _on_gpu(h0, cu_seqlens, out, hT, workspace)
    _dev(h0, cu_seqlens, out, hT, workspace)
    if workspace is None:
        workspace = _workspace(int(lib().kla_ssm_fwd_workspace_bytes(N, T, D, G, S, cu_hp, n_seq)), u)
    given = out, hT
    if out is None:
        out = torch.empty((N, T, D), dtype=u.dtype, device=u.device)
    if hT is None and want_hT:
        hT = torch.empty((n_states, D, S), dtype=torch.float32, device=u.device)
    _call("kla_ssm_fwd", *_ssm_in(u, delta, A, B, C, skip, z, delta_bias, ld), _ptr(h0), _ptr(out), _ptr(hT), _ptr(_saved), _ws_bytes(_saved),
          _ptr(cu_seqlens), cu_hp, n_seq, N, T, D, G, S, dt, _ptr(workspace), _ws_bytes(workspace), _stream(),
          KLA_LAYER_SOFTPLUS if softplus else 0)
    _written(*given)
    return out, hT


def kla_ssm_bwd(u, delta, A, B, C, d_y, skip=None, z=None, delta_bias=None, softplus=True, h0=None, d_hT=None, cu_seqlens=None,
                cu_seqlens_host=None, want_dh0=True, workspace=None, _saved=None):
    """Backward of kla_ssm_fwd: a dict of du, ddelta, dA, dB, dC, dskip, dz, ddelta_bias, dh0 (None where the input is; dh0 also where
    unwanted).  _saved: what kla_ssm's forward left behind for these inputs."""
    D, G, S, dt, ld = _ssm_check(u, delta, A, B, C, skip, z, delta_bias, 2)
    N, T = u.shape[:2]
    _, cu_hp, n_seq, n_states = _batch(u, cu_seqlens, cu_seqlens_host)
    _check("h0", h0, (n_states, D, S), torch.float32)
    _check("d_y", d_y, (N, T, D), u.dtype)
    _check("d_hT", d_hT, (n_states, D, S), torch.float32)
    if d_y is None:
        raise ValueError("d_y is required")
    _on_gpu(h0, cu_seqlens, d_y, d_hT, workspace, _saved)
    _dev(h0, cu_seqlens, d_y, d_hT, workspace, _saved)
    if workspace is None:
        workspace = _workspace(int(lib().kla_ssm_bwd_workspace_bytes(N, T, D, G, S, cu_hp, n_seq, _saved is not None)), u)

    def new(t, wanted=True):
        return torch.empty(t.shape, dtype=t.dtype, device=t.device) if t is not None and wanted else None
    g = dict(du=new(u), ddelta=new(u), dA=new(A), dB=new(B), dC=new(C), dskip=new(skip), dz=new(z), ddelta_bias=new(delta_bias),
             dh0=new(h0, want_dh0))
    _call("kla_ssm_bwd", *_ssm_in(u, delta, A, B, C, skip, z, delta_bias, ld), _ptr(h0), _ptr(d_y), _ptr(d_hT), _ptr(_saved), _ws_bytes(_saved),
          *(_ptr(t) for t in g.values()), _ptr(cu_seqlens), cu_hp, n_seq, N, T, D, G, S, dt, _ptr(workspace), _ws_bytes(workspace),
          _stream(), KLA_LAYER_SOFTPLUS if softplus else 0)
    return g


def kla_ssm_step(u, delta, A, B, C, h, skip=None, z=None, delta_bias=None, softplus=True, out=None):
    """One token of N sequences: u, delta, z [N,D], B, C [N,G,S]; h [N,D,S] fp32 is updated in place; returns y [N,D]."""
    r = _native("ssm_step", "kla_ssm_step", u, delta, A, B, C, h, skip, z, delta_bias, bool(softplus), out)
    if r is not None:
        return r
    D, G, S, dt, ld = _ssm_check(u, delta, A, B, C, skip, z, delta_bias, 1)
    N = u.shape[0]
    _check("h", h, (N, D, S), torch.float32)
    _check("out", out, (N, D), u.dtype)
    _on_gpu(h, out)
    _dev(h, out)
    given = out
    if out is None:
        out = torch.empty((N, D), dtype=u.dtype, device=u.device)
    _call("kla_ssm_step", *_ssm_in(u, delta, A, B, C, skip, z, delta_bias, ld), _ptr(h), _ptr(out), N, D, G, S, dt, _stream(),
          KLA_LAYER_SOFTPLUS if softplus else 0)
    _written(h, given)
    return out


class _Ssm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, u, delta, A, B, C, skip, z, delta_bias, h0, softplus, cu_seqlens, cu_seqlens_host, save):
        ctx.offsets = _Offsets(cu_seqlens, cu_seqlens_host)
        saved = None
        if save and any(ctx.needs_input_grad) and u.is_cuda and u.dim() == 3 and B.dim() == 4 and max(u.shape) < 2 ** 31:
            _, cu_hp, n_seq = _host_cu(ctx.offsets.cu, ctx.offsets.host)
            keep = int(lib().kla_ssm_saved_bytes(*u.shape, *B.shape[-2:], cu_hp, n_seq))
            try:
                saved = _workspace(keep, u)
            except torch.OutOfMemoryError:               # the backward forms them again
                saved = None
        y, hT = kla_ssm_fwd(u, delta, A, B, C, skip, z, delta_bias, softplus, h0, cu_seqlens, cu_seqlens_host, _saved=saved)
        ctx.save_for_backward(u, delta, A, B, C, skip, z, delta_bias, h0, saved)
        ctx.set_materialize_grads(False)
        ctx.softplus = softplus
        return y, hT

    @staticmethod
    def backward(ctx, d_y, d_hT):
        _no_second("kla_ssm")
        u, delta, A, B, C, skip, z, delta_bias, h0, saved = ctx.saved_tensors
        d_y = u.new_zeros(u.shape) if d_y is None else d_y.contiguous()
        g = kla_ssm_bwd(u, delta, A, B, C, d_y, skip, z, delta_bias, ctx.softplus, h0, None if d_hT is None else d_hT.contiguous(),
                        want_dh0=ctx.needs_input_grad[8], _saved=saved, **ctx.offsets.check())
        return (*g.values(), None, None, None, None)


def kla_ssm(u, delta, A, B, C, skip=None, z=None, delta_bias=None, softplus=True, h0=None, cu_seqlens=None, cu_seqlens_host=None, save=True):
    """Differentiable kla_ssm_fwd: (y, hT), gradients with respect to every tensor argument.  Where a gradient is wanted the forward leaves
    the states at every 16th token (every 8th from S = 32 on) behind for the backward, 4 bytes per token and channel at S = 16; save=False: the
    backward forms them again.  Same results either way."""
    host = _host(cu_seqlens, cu_seqlens_host)
    if _eager():
        r = _native("ssm_train", "kla_ssm_fwd", u, delta, A, B, C, skip, z, delta_bias, bool(softplus), h0, cu_seqlens, host, bool(save))
        if r is not None:
            return r
    return _Ssm.apply(u, delta, A, B, C, skip, z, delta_bias, h0, bool(softplus), cu_seqlens, host,
                      bool(save) and torch.is_grad_enabled())


# ---- norms ---------------------------------------------------------------------------------------------------------------------------


def _add_norm_check(x, weight, residual, scale, residual_dtype, **more):
    if x.dim() < 1:
        raise ValueError("x must be [..., D]")
    D, dt = x.shape[-1], _dt(x)
    res_type = residual.dtype if residual is not None else residual_dtype or x.dtype
    if res_type not in (x.dtype, torch.float32):
        raise TypeError("the residual stream must be float32 or %s, got %s" % (x.dtype, res_type))
    _check("weight", weight, (D,), torch.float32)
    _check("scale", scale, (D,), torch.float32)
    _check("residual", residual, x.shape, res_type)
    for name, (t, dtype) in more.items():
        _check(name, t, x.shape, x.dtype if dtype is None else res_type)
    _sizes(D)
    _on_gpu(x, weight, residual, scale, *(t for t, _ in more.values()))
    _dev(weight, residual, scale, *(t for t, _ in more.values()))
    return D, dt, 1 if res_type == torch.bfloat16 else 0, res_type


def kla_add_norm_fwd(x, weight, residual=None, scale=None, eps=1e-6, residual_dtype=None, out=None, residual_out=None):
    """r' = residual + scale x and y = weight * (RMS norm of r'), over the last dimension of x [...,D]; returns (y, r').  residual and r'
    are fp32 or of the type of x (residual_dtype where there is no residual yet: then r' = scale x)."""
    if residual_dtype in (None, torch.float32):
        r = _native("add_norm_fwd", "kla_add_norm_fwd", x, weight, residual, scale, eps, residual_dtype is not None, out, residual_out)
        if r is not None:
            return r
    D, dt, res_dt, res_type = _add_norm_check(x, weight, residual, scale, residual_dtype, out=(out, None), residual_out=(residual_out, "r"))
    ld = _rows("x", x)
    given = out, residual_out
    if out is None:
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    if residual_out is None:
        residual_out = torch.empty(x.shape, dtype=res_type, device=x.device)
    _call("kla_add_norm_fwd", _ptr(x), ld, _ptr(residual), _ptr(scale), _ptr(weight), float(eps), _ptr(out), _ptr(residual_out),
          x.numel() // D if D else 0, D, dt, res_dt, _stream())
    _written(*given)
    return out, residual_out


def kla_add_norm_bwd(x, weight, d_y, residual=None, scale=None, eps=1e-6, d_residual_out=None, residual_dtype=None):
    """Backward of kla_add_norm_fwd: a dict of dx, dweight, dresidual, dscale (None where the input is)."""
    D, dt, res_dt, _ = _add_norm_check(x, weight, residual, scale, residual_dtype, d_y=(d_y, None), d_residual_out=(d_residual_out, "r"))
    if d_y is None:
        raise ValueError("d_y is required")
    ld, M = _rows("x", x), x.numel() // D if D else 0
    ws = _workspace(int(lib().kla_add_norm_bwd_workspace_bytes(M, D, dt)), x)
    g = dict(dx=torch.empty(x.shape, dtype=x.dtype, device=x.device), dweight=torch.empty_like(weight),
             dresidual=None if residual is None else torch.empty_like(residual), dscale=None if scale is None else torch.empty_like(scale))
    _call("kla_add_norm_bwd", _ptr(x), ld, _ptr(residual), _ptr(scale), _ptr(weight), float(eps), _ptr(d_y), _ptr(d_residual_out), _ptr(g["dx"]),
          _ptr(g["dresidual"]), _ptr(g["dscale"]), _ptr(g["dweight"]), M, D, dt, res_dt, _ptr(ws), _ws_bytes(ws), _stream())
    return g


class _AddNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, residual, scale, eps, residual_dtype):
        y, r = kla_add_norm_fwd(x, weight, residual, scale, eps, residual_dtype)
        ctx.save_for_backward(x, weight, residual, scale)
        ctx.set_materialize_grads(False)
        ctx.misc = (eps, r.dtype)
        return y, r

    @staticmethod
    def backward(ctx, d_y, d_r):
        _no_second("kla_add_norm")
        x, weight, residual, scale = ctx.saved_tensors
        eps, res_type = ctx.misc
        d_y = x.new_zeros(x.shape) if d_y is None else d_y.contiguous()
        g = kla_add_norm_bwd(x, weight, d_y, residual, scale, eps, None if d_r is None else d_r.contiguous(), res_type)
        return g["dx"], g["dweight"], g["dresidual"], g["dscale"], None, None


def kla_add_norm(x, weight, residual=None, scale=None, eps=1e-6, residual_dtype=None):
    """Differentiable kla_add_norm_fwd: (y, r'), gradients with respect to x, weight, residual and scale."""
    if residual_dtype in (None, torch.float32) and _eager():
        r = _native("add_norm_train", "kla_add_norm_fwd", x, weight, residual, scale, eps, residual_dtype is not None)
        if r is not None:
            return r
    return _AddNorm.apply(x, weight, residual, scale, float(eps), residual_dtype)


def _gate_bits(activation, gate_first):
    if activation not in ("silu", "sigmoid"):
        raise ValueError("activation must be silu or sigmoid, got %r" % (activation,))
    return (KLA_LAYER_SIGMOID if activation == "sigmoid" else 0) | (KLA_LAYER_GATE_FIRST if gate_first else 0)


def _gated_norm_check(x, gate, weight, activation, gate_first, **more):
    if x.dim() < 2:
        raise ValueError("x, gate must be [..., H, D]")
    bits = _gate_bits(activation, gate_first)
    H, D = x.shape[-2:]
    dt = _dt(x)
    _check("gate", gate, x.shape, x.dtype)
    _check("weight", weight, (D,), torch.float32)
    for name, t in more.items():
        _check(name, t, x.shape, x.dtype)
    _sizes(H, D)
    _on_gpu(x, gate, weight, *more.values())
    _dev(weight, *more.values())
    return H, D, x.numel() // (H * D) if H * D else 0, dt, _rows("x", x, 2), _rows("gate", gate, 2), bits


def kla_gated_norm_fwd(x, gate, weight, eps=1e-6, activation="silu", gate_first=False, out=None):
    """weight * (RMS norm of x over the last dimension) * act(gate) for x, gate [...,H,D], weight [D] fp32, act "silu" or "sigmoid";
    gate_first: weight * (RMS norm of x act(gate))."""
    bits = _gate_bits(activation, gate_first)
    r = _native("gated_norm_fwd", "kla_gated_norm_fwd", x, gate, weight, eps, bits, out)
    if r is not None:
        return r
    H, D, M, dt, ld_x, ld_gate, bits = _gated_norm_check(x, gate, weight, activation, gate_first, out=out)
    given = out
    if out is None:
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    _call("kla_gated_norm_fwd", _ptr(x), ld_x, _ptr(gate), ld_gate, _ptr(weight), float(eps), _ptr(out), M, H, D, dt, _stream(), bits)
    _written(given)
    return out


def kla_gated_norm_bwd(x, gate, weight, d_y, eps=1e-6, activation="silu", gate_first=False):
    """Backward of kla_gated_norm_fwd: a dict of dx, dgate, dweight."""
    if d_y is None:
        raise ValueError("d_y is required")
    H, D, M, dt, ld_x, ld_gate, bits = _gated_norm_check(x, gate, weight, activation, gate_first, d_y=d_y)
    ws = _workspace(int(lib().kla_gated_norm_bwd_workspace_bytes(M, H, D, dt)), x)
    g = dict(dx=torch.empty(x.shape, dtype=x.dtype, device=x.device), dgate=torch.empty(x.shape, dtype=x.dtype, device=x.device),
             dweight=torch.empty_like(weight))
    _call("kla_gated_norm_bwd", _ptr(x), ld_x, _ptr(gate), ld_gate, _ptr(weight), float(eps), _ptr(d_y), _ptr(g["dx"]), _ptr(g["dgate"]),
          _ptr(g["dweight"]), M, H, D, dt, _ptr(ws), _ws_bytes(ws), _stream(), bits)
    return g


class _GatedNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gate, weight, eps, activation, gate_first):
        y = kla_gated_norm_fwd(x, gate, weight, eps, activation, gate_first)
        ctx.save_for_backward(x, gate, weight)
        ctx.misc = (eps, activation, gate_first)
        return y

    @staticmethod
    def backward(ctx, d_y):
        _no_second("kla_gated_norm")
        g = kla_gated_norm_bwd(*ctx.saved_tensors, d_y.contiguous(), *ctx.misc)
        return g["dx"], g["dgate"], g["dweight"], None, None, None


def kla_gated_norm(x, gate, weight, eps=1e-6, activation="silu", gate_first=False):
    """Differentiable kla_gated_norm_fwd: gradients with respect to x, gate and weight."""
    if _eager():
        r = _native("gated_norm_train", "kla_gated_norm_fwd", x, gate, weight, eps, _gate_bits(activation, gate_first))
        if r is not None:
            return r
    return _GatedNorm.apply(x, gate, weight, float(eps), activation, bool(gate_first))
