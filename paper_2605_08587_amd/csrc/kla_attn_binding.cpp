// The launching half of the Python binding for softmax attention, as kla_layer_binding.cpp is for the operators around the recurrence.
#include "kla_binding_rows.hpp"

namespace kla_binding {
namespace {

struct Api {
    decltype(&kla_attn_fwd) fwd;
    decltype(&kla_attn_bwd_workspace_bytes) bwd_bytes;
    decltype(&kla_attn_bwd) bwd;
    decltype(&kla_attn_extend_workspace_bytes) extend_bytes;
    decltype(&kla_attn_extend) extend;
    decltype(&kla_attn_step) step;
} api = {};

PyObject* bind_attn(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 6) { PyErr_SetString(PyExc_TypeError, "bind_attn takes six addresses"); return nullptr; }
    Api b;
    if (!address(a[0], &b.fwd) || !address(a[1], &b.bwd_bytes) || !address(a[2], &b.bwd) || !address(a[3], &b.extend_bytes) || !address(a[4], &b.extend) ||
        !address(a[5], &b.step))
        return nullptr;
    api = b;
    Py_RETURN_NONE;
}

constexpr long kMaxStride = 1L << 24;                    // elements from one token to the next (beyond: Python's half copies or refuses)

// Queries, keys and values of new tokens; lead: leading dimensions, [N, T] or (a step) [B]
struct Heads {
    const at::Tensor *q, *k, *v;
    int64_t N, T, H, Hk, D;
    long ld_q, ld_k, ld_v;
    kla_dtype dt;
    at::ScalarType type;
    float scale;

    template <typename O> bool take(int lead, const O& q_, const O& k_, const O& v_)
    {
        q = plain(q_);
        k = plain(k_);
        if (!q || !k || q->dim() != lead + 2 || k->dim() != lead + 2 || !type_of(*q, &dt)) return false;
        type = q->scalar_type();
        N = q->size(0); T = lead == 2 ? q->size(1) : 1; H = q->size(lead); D = q->size(lead + 1); Hk = k->size(lead);
        const at::DimVector keys = lead == 2 ? at::DimVector({N, T, Hk, D}) : at::DimVector({N, Hk, D});
        return ints({N, T, H, Hk, D}) && Hk > 0 && H % Hk == 0 && rows(q_, type, q->sizes(), 2, &ld_q) && (k = rows(k_, type, keys, 2, &ld_k)) &&
               (v = rows(v_, type, keys, 2, &ld_v)) && ld_q <= kMaxStride && ld_k <= kMaxStride && ld_v <= kMaxStride;
    }
    bool scaled(PyObject* o)
    {
        double x;
        if (!number(o, &x)) return false;
        scale = (float)x;
        return true;
    }
};

// ---- whole sequences ------------------------------------------------------------------------------------------------------------------
struct Attn : Heads {
    Offsets cu;
    int window;
    unsigned opts;

    template <typename O> bool take(const O& q_, const O& k_, const O& v_, const O& cu_, const O& host_)
    {
        return cu.take(cu_, host_) && Heads::take(2, q_, k_, v_) && together({q, k, v, cu.dev});
    }
    bool options(PyObject* scale_, PyObject* causal, PyObject* window_)
    {
        long w;
        if (!scaled(scale_) || !integer(window_, INT_MIN, INT_MAX, &w)) return false;
        window = (int)w;
        opts = causal == Py_True ? KLA_ATTN_CAUSAL : 0;
        return true;
    }
    void fwd(at::Tensor& o, at::Tensor& lse, bool want_lse, const at::Tensor& rest = at::Tensor()) const
    {
        if (!o.defined()) o = fresh(*q, q->sizes(), type);
        if (!lse.defined() && want_lse) lse = fresh(*q, {N, T, H}, at::kFloat);
        check(api.fwd(ptr(q), ld_q, ptr(k), ld_k, ptr(v), ld_v, at_of(o), f_of(lse), at_of(rest), scale, window, cu.device(), cu.host, cu.n_seq, (int)N, (int)T,
                      (int)H, (int)Hk, (int)D, dt, stream(), opts));
    }
    void bwd(const at::Tensor& o, const at::Tensor& lse, const at::Tensor* rest, const at::Tensor& d_o, at::Tensor (&g)[3]) const
    {
        const at::Tensor ws = bytes(*q, api.bwd_bytes((int)N, (int)T, (int)H, (int)Hk, (int)D, cu.host, cu.n_seq, dt));
        g[0] = fresh(*q, q->sizes(), type);
        g[1] = fresh(*k, k->sizes(), type);
        g[2] = fresh(*v, v->sizes(), type);
        check(api.bwd(ptr(q), ld_q, ptr(k), ld_k, ptr(v), ld_v, o.data_ptr(), f_of(lse), ptr(rest), d_o.data_ptr(), at_of(g[0]), at_of(g[1]), at_of(g[2]), scale, window,
                      cu.device(), cu.host, cu.n_seq, (int)N, (int)T, (int)H, (int)Hk, (int)D, dt, at_of(ws), size_of(ws), stream(), opts));
    }
};

// Contiguous and at a multiple of 16 bytes: a gradient can be a piece of a larger tensor, wherever it begins.
at::Tensor at_16_bytes(const at::Tensor& t)
{
    const at::Tensor c = t.contiguous();
    return reinterpret_cast<uintptr_t>(c.data_ptr()) % 16 ? c.clone() : c;
}

struct AttnNode : public torch::autograd::Function<AttnNode> {
    static torch::autograd::variable_list forward(torch::autograd::AutogradContext* ctx, const at::Tensor& q, const at::Tensor& k, const at::Tensor& v,
                                                  const Attn* c, const at::Tensor* host)
    {
        at::Tensor o, lse, rest;
        if (c->dt == KLA_BF16) rest = fresh(q, q.sizes(), c->type);
        c->fwd(o, lse, true, rest);
        ctx->save_for_backward({q, k, v, o, lse, rest});
        ctx->saved_data["scale"] = (double)c->scale;
        ctx->saved_data["window"] = (int64_t)c->window;
        ctx->saved_data["opts"] = (int64_t)c->opts;
        c->cu.keep(ctx, host);
        return {o};
    }
    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads)
    {
        KLA_BACKWARD("kla_attn");
        const auto s = ctx->get_saved_variables();
        at::Tensor cu, host, g[3];
        Offsets::back(ctx, &cu, &host);
        Attn c;
        taken(c.take(s[0], s[1], s[2], cu, host), "kla_attn");
        c.scale = (float)ctx->saved_data["scale"].toDouble();
        c.window = (int)ctx->saved_data["window"].toInt();
        c.opts = (unsigned)ctx->saved_data["opts"].toInt();
        const at::Tensor *o = gpu(s[3], c.type, c.q->sizes()), *lse = gpu(s[4], at::kFloat, {c.N, c.T, c.H}), *rest;
        taken(o && lse && gpu_or_none(s[5], at::kBFloat16, c.q->sizes(), &rest) && together({o, lse, rest}), "kla_attn");
        if (!grads[0].defined()) return {at::Tensor(), at::Tensor(), at::Tensor(), at::Tensor(), at::Tensor()};
        refused("kla_attn_bwd", [&] { c.bwd(*o, *lse, rest, at_16_bytes(grads[0]), g); });
        return {g[0], g[1], g[2], at::Tensor(), at::Tensor()};
    }
};

// attn_fwd(q, k, v, scale, causal, window, cu, cu_host, want_lse, out, lse, rest) -> (o, lse)
PyObject* attn_fwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Attn c;
    const at::Tensor *out, *lse, *rest;
    if (n != 12 || !api.fwd || !c.take(a[0], a[1], a[2], a[6], a[7]) || !c.options(a[3], a[4], a[5]) || !gpu_or_none(a[9], c.type, c.q->sizes(), &out) ||
        !gpu_or_none(a[10], at::kFloat, {c.N, c.T, c.H}, &lse) || !gpu_or_none(a[11], at::kBFloat16, c.q->sizes(), &rest) || !together({out, lse, rest}))
        Py_RETURN_NONE;
    at::Tensor o = value(out), l = value(lse);
    try {
        const NoGil no_gil;
        c.fwd(o, l, a[8] == Py_True, value(rest));
    } catch (const Refused& e) { return PyLong_FromLong(e.code); }
    written({out, lse, rest});
    return pair(o, l);
    END_HANDLE_TH_ERRORS
}
// attn_train(q, k, v, scale, causal, window, cu, cu_host) -> o, differentiable
PyObject* attn_train(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Attn c;
    if (n != 8 || !api.fwd || !c.take(a[0], a[1], a[2], a[6], a[7]) || !c.options(a[3], a[4], a[5])) Py_RETURN_NONE;
    at::Tensor o, lse;
    try {
        const at::Tensor* host = c.cu.dev ? &THPVariable_Unpack(a[7]) : nullptr;
        const NoGil no_gil;
        if (wants({c.q, c.k, c.v})) o = AttnNode::apply(*c.q, *c.k, *c.v, &c, host)[0];
        else c.fwd(o, lse, false);
    } catch (const Refused& e) { return PyLong_FromLong(e.code); }
    return wrap(o);
    END_HANDLE_TH_ERRORS
}

// ---- over a paged cache ---------------------------------------------------------------------------------------------------------------
struct Cache {
    const at::Tensor *k, *v, *table, *cached;
    int64_t n_pages, page, max_pages;
    long ld_table;

    bool take(const Heads& h, int64_t n, PyObject* k_, PyObject* v_, PyObject* table_, PyObject* cached_)
    {
        k = plain(k_);
        table = plain(table_);
        if (!k || !table || k->dim() != 4 || table->dim() != 2) return false;
        n_pages = k->size(0); page = k->size(2); max_pages = table->size(1);
        return ints({n_pages, page, max_pages, max_pages * page}) && (k = gpu(k_, h.type, {n_pages, h.Hk, page, h.D})) &&
               (v = gpu(v_, h.type, {n_pages, h.Hk, page, h.D})) && (table = rows(table_, at::kInt, {n, max_pages}, 1, &ld_table)) &&
               (cached = gpu(cached_, at::kInt, {n})) && together({k, v, table, cached, h.q});
    }
    // the caller's bound of the lengths, or what the table has room for
    bool bound(PyObject* o, int* most) const
    {
        long x = max_pages * page;
        if (!is_none(o) && !integer(o, INT_MIN, INT_MAX, &x)) return false;
        *most = (int)x;
        return true;
    }
};
const int32_t* ints_of(const at::Tensor* t) { return static_cast<const int32_t*>(ptr(t)); }

// attn_extend(q, k, v, k_cache, v_cache, page_table, cached, scale, window, cu, cu_host, max_len, want_lse, out, lse) -> (o, lse)
PyObject* attn_extend(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Attn c;
    Cache s;
    const at::Tensor *out, *lse;
    int most;
    if (n != 15 || !api.extend || !c.take(a[0], a[1], a[2], a[9], a[10]) || !c.options(a[7], Py_True, a[8]) ||
        !s.take(c, c.cu.n_seq ? c.cu.n_seq : c.N, a[3], a[4], a[5], a[6]) || !s.bound(a[11], &most) || !gpu_or_none(a[13], c.type, c.q->sizes(), &out) ||
        !gpu_or_none(a[14], at::kFloat, {c.N, c.T, c.H}, &lse) || !together({out, lse}))
        Py_RETURN_NONE;
    at::Tensor o = value(out), l = value(lse);
    try {
        const NoGil no_gil;
        if (!o.defined()) o = fresh(*c.q, c.q->sizes(), c.type);
        if (!l.defined() && a[12] == Py_True) l = fresh(*c.q, {c.N, c.T, c.H}, at::kFloat);
        const at::Tensor ws = bytes(*c.q, api.extend_bytes((int)c.N, (int)c.T, (int)c.H, (int)c.Hk, (int)c.D, c.cu.host, c.cu.n_seq, c.window, most, c.dt));
        check(api.extend(ptr(c.q), c.ld_q, ptr(c.k), c.ld_k, ptr(c.v), c.ld_v, ptr(s.k), ptr(s.v), ints_of(s.table), s.ld_table, ints_of(s.cached), at_of(o), f_of(l),
                         c.scale, c.window, c.cu.device(), c.cu.host, c.cu.n_seq, (int)c.N, (int)c.T, (int)c.H, (int)c.Hk, (int)c.D, (int)s.n_pages, (int)s.page,
                         (int)s.max_pages, most, c.dt, at_of(ws), size_of(ws), stream()));
    } catch (const Refused& e) { return PyLong_FromLong(e.code); }
    written({s.k, s.v, out, lse});
    return pair(o, l);
    END_HANDLE_TH_ERRORS
}
// attn_step(q, k, v, k_cache, v_cache, page_table, cached, scale, window, max_len, out) -> o
PyObject* attn_step(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Heads c;
    Cache s;
    const at::Tensor* out;
    int most;
    long window;
    if (n != 11 || !api.step || !c.take(1, a[0], a[1], a[2]) || !c.scaled(a[7]) || !integer(a[8], INT_MIN, INT_MAX, &window) ||
        !s.take(c, c.N, a[3], a[4], a[5], a[6]) || !s.bound(a[9], &most) || !gpu_or_none(a[10], c.type, c.q->sizes(), &out) || !together({c.q, c.k, c.v, out}))
        Py_RETURN_NONE;
    at::Tensor o = value(out);
    try {
        const NoGil no_gil;
        if (!o.defined()) o = fresh(*c.q, c.q->sizes(), c.type);
        const at::Tensor ws = bytes(*c.q, api.extend_bytes((int)c.N, 1, (int)c.H, (int)c.Hk, (int)c.D, nullptr, 0, (int)window, most, c.dt));
        check(api.step(ptr(c.q), c.ld_q, ptr(c.k), c.ld_k, ptr(c.v), c.ld_v, ptr(s.k), ptr(s.v), ints_of(s.table), s.ld_table, ints_of(s.cached), at_of(o), c.scale,
                       (int)window, (int)c.N, (int)c.H, (int)c.Hk, (int)c.D, (int)s.n_pages, (int)s.page, (int)s.max_pages, most, c.dt, at_of(ws), size_of(ws),
                       stream()));
    } catch (const Refused& e) { return PyLong_FromLong(e.code); }
    written({s.k, s.v, out});
    return wrap(o);
    END_HANDLE_TH_ERRORS
}

}  // namespace

PyMethodDef attn_methods[] = {KLA_FASTCALL(bind_attn), KLA_FASTCALL(attn_fwd), KLA_FASTCALL(attn_train), KLA_FASTCALL(attn_extend), KLA_FASTCALL(attn_step),
                              {nullptr, nullptr, 0, nullptr}};

}  // namespace kla_binding
