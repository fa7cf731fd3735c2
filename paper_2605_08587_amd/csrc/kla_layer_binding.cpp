// The launching half of the Python binding for the operators around the recurrence, as kla_binding.cpp is for the recurrence: every entry
// checks the tensors of a call, allocates, calls the C ABI on the current stream and returns None for what it does not take.  The
// differentiable calls are C++ nodes of the autograd graph.
#include "kla_binding_rows.hpp"

namespace kla_binding {
namespace {

struct Api {
    decltype(&kla_conv_fwd) conv_fwd;
    decltype(&kla_conv_bwd_workspace_bytes) conv_bwd_bytes;
    decltype(&kla_conv_bwd) conv_bwd;
    decltype(&kla_conv_step) conv_step;
    decltype(&kla_ssm_fwd_workspace_bytes) ssm_fwd_bytes;
    decltype(&kla_ssm_saved_bytes) ssm_saved_bytes;
    decltype(&kla_ssm_fwd) ssm_fwd;
    decltype(&kla_ssm_bwd_workspace_bytes) ssm_bwd_bytes;
    decltype(&kla_ssm_bwd) ssm_bwd;
    decltype(&kla_ssm_step) ssm_step;
    decltype(&kla_add_norm_fwd) add_fwd;
    decltype(&kla_add_norm_bwd_workspace_bytes) add_bwd_bytes;
    decltype(&kla_add_norm_bwd) add_bwd;
    decltype(&kla_gated_norm_fwd) gated_fwd;
    decltype(&kla_gated_norm_bwd_workspace_bytes) gated_bwd_bytes;
    decltype(&kla_gated_norm_bwd) gated_bwd;
} api = {};

PyObject* bind_layer(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 16) { PyErr_SetString(PyExc_TypeError, "bind_layer takes sixteen addresses"); return nullptr; }
    Api b;
    if (!address(a[0], &b.conv_fwd) || !address(a[1], &b.conv_bwd_bytes) || !address(a[2], &b.conv_bwd) || !address(a[3], &b.conv_step) ||
        !address(a[4], &b.ssm_fwd_bytes) || !address(a[5], &b.ssm_saved_bytes) || !address(a[6], &b.ssm_fwd) || !address(a[7], &b.ssm_bwd_bytes) ||
        !address(a[8], &b.ssm_bwd) || !address(a[9], &b.ssm_step) || !address(a[10], &b.add_fwd) || !address(a[11], &b.add_bwd_bytes) ||
        !address(a[12], &b.add_bwd) || !address(a[13], &b.gated_fwd) || !address(a[14], &b.gated_bwd_bytes) || !address(a[15], &b.gated_bwd))
        return nullptr;
    api = b;
    Py_RETURN_NONE;
}

// ---- short convolution ----------------------------------------------------------------------------------------------------------------
struct Conv {
    const at::Tensor *x, *w, *b, *st;
    Offsets cu;
    int64_t N, T, D, W, n_states;
    long ld;
    kla_dtype dt;
    at::ScalarType type;
    unsigned opts;

    template <typename O> bool take(const O& x_, const O& w_, const O& b_, const O& st_, const O& cu_, const O& host_, bool silu)
    {
        x = plain(x_);
        w = on_gpu(w_);
        if (!x || !w || x->dim() != 3 || w->dim() != 2 || !type_of(*x, &dt) || !cu.take(cu_, host_)) return false;
        type = x->scalar_type();
        N = x->size(0); T = x->size(1); D = x->size(2); W = w->size(1);
        n_states = cu.n_seq ? cu.n_seq : N;
        opts = silu ? KLA_LAYER_SILU : 0;
        return ints({N, T, D, W}) && rows(x_, type, x->sizes(), 1, &ld) && gpu(w_, at::kFloat, {D, W}) && gpu_or_none(b_, at::kFloat, {D}, &b) &&
               gpu_or_none(st_, type, {n_states, W - 1, D}, &st) && together({x, w, b, st, cu.dev});
    }
    void fwd(at::Tensor& y, at::Tensor& last, bool want_state) const
    {
        if (!y.defined()) y = fresh(*x, x->sizes(), type);
        if (!last.defined() && want_state) last = fresh(*x, {n_states, W - 1, D}, type);
        check(api.conv_fwd(ptr(x), ld, fptr(w), fptr(b), ptr(st), at_of(y), at_of(last), cu.device(), cu.host, cu.n_seq, (int)N, (int)T, (int)D, (int)W, dt,
                           stream(), opts));
    }
    void bwd(const at::Tensor& d_y, const at::Tensor& d_last, bool want_dst, at::Tensor (&g)[4]) const
    {
        const at::Tensor ws = bytes(*x, api.conv_bwd_bytes((int)N, (int)T, (int)D, (int)W));
        g[0] = fresh(*x, x->sizes(), type);
        g[1] = fresh(w);
        g[2] = fresh(b);
        if (want_dst) g[3] = fresh(st);
        check(api.conv_bwd(ptr(x), ld, fptr(w), fptr(b), ptr(st), d_y.data_ptr(), at_of(d_last), at_of(g[0]), f_of(g[1]), f_of(g[2]), at_of(g[3]),
                           cu.device(), cu.host, cu.n_seq, (int)N, (int)T, (int)D, (int)W, dt, at_of(ws), size_of(ws), stream(), opts));
    }
};

struct ConvNode : public torch::autograd::Function<ConvNode> {
    static torch::autograd::variable_list forward(torch::autograd::AutogradContext* ctx, const at::Tensor& x, const at::Tensor& w,
                                                  const std::optional<at::Tensor>& b, const std::optional<at::Tensor>& st, const Conv* c,
                                                  const at::Tensor* host, bool want_state)
    {
        at::Tensor y, last;
        c->fwd(y, last, want_state);
        ctx->save_for_backward({x, w, value(c->b), value(c->st)});
        ctx->set_materialize_grads(false);
        ctx->saved_data["opts"] = (int64_t)c->opts;
        ctx->saved_data["dst"] = c->st && c->st->requires_grad();
        c->cu.keep(ctx, host);
        if (want_state) return {y, last};
        return {y};
    }
    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads)
    {
        KLA_BACKWARD("kla_conv");
        const auto s = ctx->get_saved_variables();
        at::Tensor cu, host, g[4];
        Offsets::back(ctx, &cu, &host);
        Conv c;
        taken(c.take(s[0], s[1], s[2], s[3], cu, host, ctx->saved_data["opts"].toInt() & KLA_LAYER_SILU), "kla_conv");
        const at::Tensor d_y = grads[0].defined() ? grads[0].contiguous() : at::zeros(c.x->sizes(), c.x->options());
        const at::Tensor d_last = grads.size() > 1 && grads[1].defined() ? grads[1].contiguous() : at::Tensor();
        refused("kla_conv_bwd", [&] { c.bwd(d_y, d_last, ctx->saved_data["dst"].toBool(), g); });
        return {g[0], g[1], g[2], g[3], at::Tensor(), at::Tensor(), at::Tensor()};
    }
};

// conv_fwd(x, weight, bias, state, cu, cu_host, silu, want_state, out, state_out) -> (y, state_out)
PyObject* conv_fwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Conv c;
    const at::Tensor *out, *last;
    if (n != 10 || !api.conv_fwd || !c.take(a[0], a[1], a[2], a[3], a[4], a[5], a[6] == Py_True) || !gpu_or_none(a[8], c.type, c.x->sizes(), &out) ||
        !gpu_or_none(a[9], c.type, {c.n_states, c.W - 1, c.D}, &last) || !together({out, last}))
        Py_RETURN_NONE;
    at::Tensor y = value(out), l = value(last);
    try {
        const NoGil no_gil;
        c.fwd(y, l, a[7] == Py_True);
    } catch (const Refused& e) { return PyLong_FromLong(e.code); }
    written({out, last});
    return pair(y, l);
    END_HANDLE_TH_ERRORS
}
// conv_train(x, weight, bias, state, cu, cu_host, silu, want_state) -> (y, state_out), differentiable
PyObject* conv_train(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Conv c;
    if (n != 8 || !api.conv_fwd || !c.take(a[0], a[1], a[2], a[3], a[4], a[5], a[6] == Py_True)) Py_RETURN_NONE;
    const bool want_state = a[7] == Py_True;
    at::Tensor y, last;
    try {
        const at::Tensor* host = c.cu.dev ? &THPVariable_Unpack(a[5]) : nullptr;
        const NoGil no_gil;
        if (wants({c.x, c.w, c.b, c.st})) {
            const auto r = ConvNode::apply(*c.x, *c.w, maybe(c.b), maybe(c.st), &c, host, want_state);
            y = r[0];
            if (want_state) last = r[1];
        } else c.fwd(y, last, want_state);
    } catch (const Refused& e) { return PyLong_FromLong(e.code); }
    return pair(y, last);
    END_HANDLE_TH_ERRORS
}
// conv_step(x, weight, state, bias, silu, out) -> y
PyObject* conv_step(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const at::Tensor *x, *w, *b, *st, *out;
    kla_dtype dt;
    long ld;
    if (n != 6 || !api.conv_step || !(x = plain(a[0])) || !(w = on_gpu(a[1])) || x->dim() != 2 || w->dim() != 2 || !type_of(*x, &dt)) Py_RETURN_NONE;
    const int64_t B = x->size(0), D = x->size(1), W = w->size(1);
    const at::ScalarType type = x->scalar_type();
    if (!ints({B, D, W}) || !rows(a[0], type, x->sizes(), 1, &ld) || !gpu(a[1], at::kFloat, {D, W}) || !(st = gpu(a[2], type, {B, W - 1, D})) ||
        !gpu_or_none(a[3], at::kFloat, {D}, &b) || !gpu_or_none(a[5], type, x->sizes(), &out) || !together({x, w, b, st, out}))
        Py_RETURN_NONE;
    at::Tensor y = value(out);
    int rc;
    {
        const NoGil no_gil;
        if (!y.defined()) y = fresh(*x, x->sizes(), type);
        rc = api.conv_step(ptr(x), ld, fptr(w), fptr(b), ptr(st), at_of(y), (int)B, (int)D, (int)W, dt, stream(), a[4] == Py_True ? KLA_LAYER_SILU : 0);
    }
    if (rc != KLA_OK) return PyLong_FromLong(rc);
    written({st, out});
    return wrap(y);
    END_HANDLE_TH_ERRORS
}

// ---- selective scan -------------------------------------------------------------------------------------------------------------------
struct Ssm {
    const at::Tensor *u, *delta, *A, *B, *C, *skip, *z, *bias, *h0;
    Offsets cu;
    int64_t N, T, D, G, S, n_states;
    long ld_u, ld_d, ld_B, ld_C, ld_z;
    kla_dtype dt;
    at::ScalarType type;
    unsigned opts;

    // lead: leading dimensions, [N, T] or (a step) [N]
    template <typename O>
    bool take(int lead, const O& u_, const O& delta_, const O& A_, const O& B_, const O& C_, const O& skip_, const O& z_, const O& bias_, bool softplus)
    {
        u = plain(u_);
        B = plain(B_);
        if (!u || !B || u->dim() != lead + 1 || B->dim() != lead + 2 || !type_of(*u, &dt)) return false;
        type = u->scalar_type();
        N = u->size(0); T = lead == 2 ? u->size(1) : 1; D = u->size(lead); G = B->size(lead); S = B->size(lead + 1);
        n_states = N;
        opts = softplus ? KLA_LAYER_SOFTPLUS : 0;
        const at::DimVector bc = lead == 2 ? at::DimVector({N, T, G, S}) : at::DimVector({N, G, S});
        return ints({N, T, D, G, S}) && rows(u_, type, u->sizes(), 1, &ld_u) && (delta = rows(delta_, type, u->sizes(), 1, &ld_d)) &&
               (A = gpu(A_, at::kFloat, {D, S})) && rows(B_, type, bc, 2, &ld_B) && (C = rows(C_, type, bc, 2, &ld_C)) &&
               gpu_or_none(skip_, at::kFloat, {D}, &skip) && rows_or_none(z_, type, u->sizes(), 1, &ld_z, &z) &&
               gpu_or_none(bias_, at::kFloat, {D}, &bias) && together({u, delta, A, B, C, skip, z, bias});
    }
    template <typename O> bool take_batch(const O& h0_, const O& cu_, const O& host_)
    {
        if (!cu.take(cu_, host_)) return false;
        if (cu.n_seq) n_states = cu.n_seq;
        return gpu_or_none(h0_, at::kFloat, {n_states, D, S}, &h0) && together({h0, cu.dev});
    }
    size_t saved_bytes() const { return api.ssm_saved_bytes((int)N, (int)T, (int)D, (int)G, (int)S, cu.host, cu.n_seq); }
    void fwd(at::Tensor& y, at::Tensor& hT, bool want_hT, const at::Tensor& saved) const
    {
        const at::Tensor ws = bytes(*u, api.ssm_fwd_bytes((int)N, (int)T, (int)D, (int)G, (int)S, cu.host, cu.n_seq));
        if (!y.defined()) y = fresh(*u, u->sizes(), type);
        if (!hT.defined() && want_hT) hT = fresh(*u, {n_states, D, S}, at::kFloat);
        check(api.ssm_fwd(ptr(u), ld_u, ptr(delta), ld_d, fptr(A), ptr(B), ld_B, ptr(C), ld_C, fptr(skip), ptr(z), ld_z, fptr(bias), fptr(h0), at_of(y),
                          f_of(hT), f_of(saved), size_of(saved), cu.device(), cu.host, cu.n_seq, (int)N, (int)T, (int)D, (int)G, (int)S, dt, at_of(ws),
                          size_of(ws), stream(), opts));
    }
    // g: of u, delta, A, B, C, skip, z, delta_bias, h0
    void bwd(const at::Tensor& d_y, const at::Tensor& d_hT, const at::Tensor* saved, bool want_dh0, at::Tensor (&g)[9]) const
    {
        const at::Tensor ws = bytes(*u, api.ssm_bwd_bytes((int)N, (int)T, (int)D, (int)G, (int)S, cu.host, cu.n_seq, saved != nullptr));
        const at::Tensor* like[9] = {u, delta, A, B, C, skip, z, bias, want_dh0 ? h0 : nullptr};
        for (int i = 0; i < 9; ++i) g[i] = fresh(like[i]);
        check(api.ssm_bwd(ptr(u), ld_u, ptr(delta), ld_d, fptr(A), ptr(B), ld_B, ptr(C), ld_C, fptr(skip), ptr(z), ld_z, fptr(bias), fptr(h0), d_y.data_ptr(),
                          f_of(d_hT), fptr(saved), saved ? saved->nbytes() : 0, at_of(g[0]), at_of(g[1]), f_of(g[2]), at_of(g[3]), at_of(g[4]), f_of(g[5]),
                          at_of(g[6]), f_of(g[7]), f_of(g[8]), cu.device(), cu.host, cu.n_seq, (int)N, (int)T, (int)D, (int)G, (int)S, dt, at_of(ws),
                          size_of(ws), stream(), opts));
    }
};

struct SsmNode : public torch::autograd::Function<SsmNode> {
    static torch::autograd::variable_list forward(torch::autograd::AutogradContext* ctx, const at::Tensor& u, const at::Tensor& delta, const at::Tensor& A,
                                                  const at::Tensor& B, const at::Tensor& C, const std::optional<at::Tensor>& skip,
                                                  const std::optional<at::Tensor>& z, const std::optional<at::Tensor>& bias,
                                                  const std::optional<at::Tensor>& h0, const Ssm* c, const at::Tensor* host, bool save)
    {
        at::Tensor y, hT, saved;
        if (save) {
            // no memory for it: the backward forms the states again
            try { saved = bytes(u, c->saved_bytes()); } catch (const c10::OutOfMemoryError&) {}
        }
        c->fwd(y, hT, true, saved);
        ctx->save_for_backward({u, delta, A, B, C, value(c->skip), value(c->z), value(c->bias), value(c->h0), saved});
        ctx->set_materialize_grads(false);
        ctx->saved_data["opts"] = (int64_t)c->opts;
        ctx->saved_data["dh0"] = c->h0 && c->h0->requires_grad();
        c->cu.keep(ctx, host);
        return {y, hT};
    }
    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads)
    {
        KLA_BACKWARD("kla_ssm");
        const auto s = ctx->get_saved_variables();
        at::Tensor cu, host, g[9];
        Offsets::back(ctx, &cu, &host);
        Ssm c;
        const at::Tensor* saved;
        taken(c.take(2, s[0], s[1], s[2], s[3], s[4], s[5], s[6], s[7], ctx->saved_data["opts"].toInt() & KLA_LAYER_SOFTPLUS) &&
              c.take_batch(s[8], cu, host) && saved_or_none(s[9], *c.u, &saved), "kla_ssm");
        const at::Tensor d_y = grads[0].defined() ? grads[0].contiguous() : at::zeros(c.u->sizes(), c.u->options());
        const at::Tensor d_hT = grads[1].defined() ? grads[1].contiguous() : at::Tensor();
        refused("kla_ssm_bwd", [&] { c.bwd(d_y, d_hT, saved, ctx->saved_data["dh0"].toBool(), g); });
        return {g[0], g[1], g[2], g[3], g[4], g[5], g[6], g[7], g[8], at::Tensor(), at::Tensor(), at::Tensor()};
    }
};

// ssm_fwd(u, delta, A, B, C, skip, z, delta_bias, softplus, h0, cu, cu_host, want_hT, out, hT) -> (y, hT)
PyObject* ssm_fwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Ssm c;
    const at::Tensor *out, *last;
    if (n != 15 || !api.ssm_fwd || !c.take(2, a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8] == Py_True) || !c.take_batch(a[9], a[10], a[11]) ||
        !gpu_or_none(a[13], c.type, c.u->sizes(), &out) || !gpu_or_none(a[14], at::kFloat, {c.n_states, c.D, c.S}, &last) || !together({out, last}))
        Py_RETURN_NONE;
    at::Tensor y = value(out), hT = value(last);
    try {
        const NoGil no_gil;
        c.fwd(y, hT, a[12] == Py_True, at::Tensor());
    } catch (const Refused& e) { return PyLong_FromLong(e.code); }
    written({out, last});
    return pair(y, hT);
    END_HANDLE_TH_ERRORS
}
// ssm_train(u, delta, A, B, C, skip, z, delta_bias, softplus, h0, cu, cu_host, save) -> (y, hT), differentiable
PyObject* ssm_train(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Ssm c;
    if (n != 13 || !api.ssm_fwd || !c.take(2, a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8] == Py_True) || !c.take_batch(a[9], a[10], a[11]))
        Py_RETURN_NONE;
    at::Tensor y, hT;
    try {
        const at::Tensor* host = c.cu.dev ? &THPVariable_Unpack(a[11]) : nullptr;
        const NoGil no_gil;
        if (wants({c.u, c.delta, c.A, c.B, c.C, c.skip, c.z, c.bias, c.h0})) {
            const auto r = SsmNode::apply(*c.u, *c.delta, *c.A, *c.B, *c.C, maybe(c.skip), maybe(c.z), maybe(c.bias), maybe(c.h0), &c, host, a[12] == Py_True);
            y = r[0];
            hT = r[1];
        } else c.fwd(y, hT, true, at::Tensor());
    } catch (const Refused& e) { return PyLong_FromLong(e.code); }
    return pair(y, hT);
    END_HANDLE_TH_ERRORS
}
// ssm_step(u, delta, A, B, C, h, skip, z, delta_bias, softplus, out) -> y
PyObject* ssm_step(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Ssm c;
    const at::Tensor *h, *out;
    if (n != 11 || !api.ssm_step || !c.take(1, a[0], a[1], a[2], a[3], a[4], a[6], a[7], a[8], a[9] == Py_True) || !(h = gpu(a[5], at::kFloat, {c.N, c.D, c.S})) ||
        !gpu_or_none(a[10], c.type, c.u->sizes(), &out) || !together({h, out}))
        Py_RETURN_NONE;
    at::Tensor y = value(out);
    int rc;
    {
        const NoGil no_gil;
        if (!y.defined()) y = fresh(*c.u, c.u->sizes(), c.type);
        rc = api.ssm_step(ptr(c.u), c.ld_u, ptr(c.delta), c.ld_d, fptr(c.A), ptr(c.B), c.ld_B, ptr(c.C), c.ld_C, fptr(c.skip), ptr(c.z), c.ld_z, fptr(c.bias),
                          fptr(h), at_of(y), (int)c.N, (int)c.D, (int)c.G, (int)c.S, c.dt, stream(), c.opts);
    }
    if (rc != KLA_OK) return PyLong_FromLong(rc);
    written({h, out});
    return wrap(y);
    END_HANDLE_TH_ERRORS
}

// ---- norms ----------------------------------------------------------------------------------------------------------------------------
struct AddNorm {
    const at::Tensor *x, *w, *r, *s;
    int64_t M, D;
    long ld;
    double eps;
    kla_dtype dt, res_dt;
    at::ScalarType type, res_type;

    template <typename O> bool take(const O& x_, const O& w_, const O& r_, const O& s_, double eps_, at::ScalarType without)
    {
        x = plain(x_);
        eps = eps_;
        if (!x || x->dim() < 1 || !type_of(*x, &dt)) return false;
        type = x->scalar_type();
        D = x->size(-1);
        if (D <= 0 || D > INT_MAX) return false;
        M = x->numel() / D;
        r = nullptr;
        if (!is_none(r_) && !(r = on_gpu(r_))) return false;
        res_type = r ? r->scalar_type() : without;
        res_dt = res_type == at::kBFloat16 ? KLA_BF16 : KLA_F32;
        return (res_type == type || res_type == at::kFloat) && rows(x_, type, x->sizes(), 1, &ld) && (w = gpu(w_, at::kFloat, {D})) &&
               (!r || r->sizes() == x->sizes()) && gpu_or_none(s_, at::kFloat, {D}, &s) && together({x, w, r, s});
    }
    void fwd(at::Tensor& y, at::Tensor& r2) const
    {
        if (!y.defined()) y = fresh(*x, x->sizes(), type);
        if (!r2.defined()) r2 = fresh(*x, x->sizes(), res_type);
        check(api.add_fwd(ptr(x), ld, ptr(r), fptr(s), fptr(w), (float)eps, at_of(y), at_of(r2), (long)M, (int)D, dt, res_dt, stream()));
    }
    // g: of x, weight, residual, scale
    void bwd(const at::Tensor& d_y, const at::Tensor& d_r, at::Tensor (&g)[4]) const
    {
        const at::Tensor ws = bytes(*x, api.add_bwd_bytes((long)M, (int)D, dt));
        g[0] = fresh(*x, x->sizes(), type);
        g[1] = fresh(w);
        g[2] = fresh(r);
        g[3] = fresh(s);
        check(api.add_bwd(ptr(x), ld, ptr(r), fptr(s), fptr(w), (float)eps, d_y.data_ptr(), at_of(d_r), at_of(g[0]), at_of(g[2]), f_of(g[3]), f_of(g[1]),
                          (long)M, (int)D, dt, res_dt, at_of(ws), size_of(ws), stream()));
    }
};
struct AddNormNode : public torch::autograd::Function<AddNormNode> {
    static torch::autograd::variable_list forward(torch::autograd::AutogradContext* ctx, const at::Tensor& x, const at::Tensor& w,
                                                  const std::optional<at::Tensor>& r, const std::optional<at::Tensor>& s, const AddNorm* c)
    {
        at::Tensor y, r2;
        c->fwd(y, r2);
        ctx->save_for_backward({x, w, value(c->r), value(c->s)});
        ctx->set_materialize_grads(false);
        ctx->saved_data["eps"] = c->eps;
        ctx->saved_data["f32"] = c->res_type == at::kFloat;
        return {y, r2};
    }
    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads)
    {
        KLA_BACKWARD("kla_add_norm");
        const auto v = ctx->get_saved_variables();
        at::Tensor g[4];
        AddNorm c;
        taken(c.take(v[0], v[1], v[2], v[3], ctx->saved_data["eps"].toDouble(), ctx->saved_data["f32"].toBool() ? at::kFloat : at::kBFloat16), "kla_add_norm");
        const at::Tensor d_y = grads[0].defined() ? grads[0].contiguous() : at::zeros(c.x->sizes(), c.x->options());
        const at::Tensor d_r = grads[1].defined() ? grads[1].contiguous() : at::Tensor();
        refused("kla_add_norm_bwd", [&] { c.bwd(d_y, d_r, g); });
        return {g[0], g[1], g[2], g[3], at::Tensor()};
    }
};
// The type of a stream that there is not yet: fp32 (True) or that of x (False)
bool take_add_norm(AddNorm& c, PyObject* const* a)
{
    double eps;
    const at::Tensor* x = plain(a[0]);
    return x && number(a[4], &eps) && c.take(a[0], a[1], a[2], a[3], eps, a[5] == Py_True ? at::kFloat : x->scalar_type());
}
// add_norm_fwd(x, weight, residual, scale, eps, fp32, out, residual_out) -> (y, r')
PyObject* add_norm_fwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    AddNorm c;
    const at::Tensor *out, *r2;
    if (n != 8 || !api.add_fwd || !take_add_norm(c, a) || !gpu_or_none(a[6], c.type, c.x->sizes(), &out) ||
        !gpu_or_none(a[7], c.res_type, c.x->sizes(), &r2) || !together({out, r2}))
        Py_RETURN_NONE;
    at::Tensor y = value(out), r = value(r2);
    try {
        const NoGil no_gil;
        c.fwd(y, r);
    } catch (const Refused& e) { return PyLong_FromLong(e.code); }
    written({out, r2});
    return pair(y, r);
    END_HANDLE_TH_ERRORS
}
// add_norm_train(x, weight, residual, scale, eps, fp32) -> (y, r'), differentiable
PyObject* add_norm_train(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    AddNorm c;
    if (n != 6 || !api.add_fwd || !take_add_norm(c, a)) Py_RETURN_NONE;
    at::Tensor y, r;
    try {
        const NoGil no_gil;
        if (wants({c.x, c.w, c.r, c.s})) {
            const auto v = AddNormNode::apply(*c.x, *c.w, maybe(c.r), maybe(c.s), &c);
            y = v[0];
            r = v[1];
        } else c.fwd(y, r);
    } catch (const Refused& e) { return PyLong_FromLong(e.code); }
    return pair(y, r);
    END_HANDLE_TH_ERRORS
}

struct GatedNorm {
    const at::Tensor *x, *gate, *w;
    int64_t M, H, D;
    long ld_x, ld_g;
    double eps;
    kla_dtype dt;
    at::ScalarType type;
    unsigned opts;

    template <typename O> bool take(const O& x_, const O& gate_, const O& w_, double eps_, unsigned opts_)
    {
        x = plain(x_);
        eps = eps_;
        opts = opts_;
        if (!x || x->dim() < 2 || !type_of(*x, &dt)) return false;
        type = x->scalar_type();
        H = x->size(-2); D = x->size(-1);
        if (H <= 0 || D <= 0 || !ints({H, D})) return false;
        M = x->numel() / (H * D);
        return rows(x_, type, x->sizes(), 2, &ld_x) && (gate = rows(gate_, type, x->sizes(), 2, &ld_g)) && (w = gpu(w_, at::kFloat, {D})) &&
               together({x, gate, w});
    }
    void fwd(at::Tensor& y) const
    {
        if (!y.defined()) y = fresh(*x, x->sizes(), type);
        check(api.gated_fwd(ptr(x), ld_x, ptr(gate), ld_g, fptr(w), (float)eps, at_of(y), (long)M, (int)H, (int)D, dt, stream(), opts));
    }
    void bwd(const at::Tensor& d_y, at::Tensor (&g)[3]) const
    {
        const at::Tensor ws = bytes(*x, api.gated_bwd_bytes((long)M, (int)H, (int)D, dt));
        g[0] = fresh(*x, x->sizes(), type);
        g[1] = fresh(*x, x->sizes(), type);
        g[2] = fresh(w);
        check(api.gated_bwd(ptr(x), ld_x, ptr(gate), ld_g, fptr(w), (float)eps, d_y.data_ptr(), at_of(g[0]), at_of(g[1]), f_of(g[2]), (long)M, (int)H, (int)D,
                            dt, at_of(ws), size_of(ws), stream(), opts));
    }
};
struct GatedNormNode : public torch::autograd::Function<GatedNormNode> {
    static torch::autograd::variable_list forward(torch::autograd::AutogradContext* ctx, const at::Tensor& x, const at::Tensor& gate, const at::Tensor& w,
                                                  const GatedNorm* c)
    {
        at::Tensor y;
        c->fwd(y);
        ctx->save_for_backward({x, gate, w});
        ctx->saved_data["eps"] = c->eps;
        ctx->saved_data["opts"] = (int64_t)c->opts;
        return {y};
    }
    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads)
    {
        KLA_BACKWARD("kla_gated_norm");
        const auto v = ctx->get_saved_variables();
        at::Tensor g[3];
        GatedNorm c;
        taken(c.take(v[0], v[1], v[2], ctx->saved_data["eps"].toDouble(), (unsigned)ctx->saved_data["opts"].toInt()), "kla_gated_norm");
        const at::Tensor d_y = grads[0].contiguous();
        refused("kla_gated_norm_bwd", [&] { c.bwd(d_y, g); });
        return {g[0], g[1], g[2], at::Tensor()};
    }
};
// gated_norm_fwd(x, gate, weight, eps, opts, out) -> y;  gated_norm_train(x, gate, weight, eps, opts) -> y, differentiable
PyObject* gated_norm_fwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    GatedNorm c;
    const at::Tensor* out;
    double eps;
    long opts;
    if (n != 6 || !api.gated_fwd || !number(a[3], &eps) || !integer(a[4], 0, UINT_MAX, &opts) || !c.take(a[0], a[1], a[2], eps, (unsigned)opts) ||
        !gpu_or_none(a[5], c.type, c.x->sizes(), &out) || !together({out}))
        Py_RETURN_NONE;
    at::Tensor y = value(out);
    try {
        const NoGil no_gil;
        c.fwd(y);
    } catch (const Refused& e) { return PyLong_FromLong(e.code); }
    written({out});
    return wrap(y);
    END_HANDLE_TH_ERRORS
}
PyObject* gated_norm_train(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    GatedNorm c;
    double eps;
    long opts;
    if (n != 5 || !api.gated_fwd || !number(a[3], &eps) || !integer(a[4], 0, UINT_MAX, &opts) || !c.take(a[0], a[1], a[2], eps, (unsigned)opts))
        Py_RETURN_NONE;
    at::Tensor y;
    try {
        const NoGil no_gil;
        if (wants({c.x, c.gate, c.w})) y = GatedNormNode::apply(*c.x, *c.gate, *c.w, &c)[0];
        else c.fwd(y);
    } catch (const Refused& e) { return PyLong_FromLong(e.code); }
    return wrap(y);
    END_HANDLE_TH_ERRORS
}

}  // namespace

PyMethodDef layer_methods[] = {KLA_FASTCALL(bind_layer), KLA_FASTCALL(conv_fwd), KLA_FASTCALL(conv_train), KLA_FASTCALL(conv_step), KLA_FASTCALL(ssm_fwd),
                               KLA_FASTCALL(ssm_train), KLA_FASTCALL(ssm_step), KLA_FASTCALL(add_norm_fwd), KLA_FASTCALL(add_norm_train),
                               KLA_FASTCALL(gated_norm_fwd), KLA_FASTCALL(gated_norm_train), {nullptr, nullptr, 0, nullptr}};

}  // namespace kla_binding
