// C ABI of the operators around the recurrence (declared in include/kla.h): argument validation, workspace carving and launch
// sequencing.  No allocation, no state, nothing read from the environment; everything is enqueued on the caller's stream.
#include <limits.h>
#include <type_traits>

#include "kla_args.hpp"

namespace {

using kla::bf16_t;

static_assert(KLA_LAYER_SILU == (int)kla::kLayerSilu && KLA_LAYER_SOFTPLUS == (int)kla::kLayerSoftplus &&
              KLA_LAYER_SIGMOID == (int)kla::kLayerSigmoid && KLA_LAYER_GATE_FIRST == (int)kla::kLayerGateFirst, "option bits");

// ---- short convolution ------------------------------------------------------------------------------------------------------------
constexpr int kMaxConv = 1 << 30;                        // (a row rounded up to whole workgroups is an int)
int conv_check(const void* x, long ld_x, const float* weight, int D, int W, int dt, unsigned opts)
{
    if (!dt_ok(dt)) return KLA_ERR_DTYPE;
    if (D <= 0 || D > kMaxConv || W < 2 || W > 4 || ld_x < D || (opts & ~(unsigned)KLA_LAYER_SILU)) return KLA_ERR_SHAPE;
    if (!weight) return KLA_ERR_NULL;
    (void)x;
    return KLA_OK;
}
template <typename T> kla::ConvArgs<T> conv_args(const void* x, long ld_x, const float* weight, const float* bias, const void* state, const kla::Seqs& s,
                                                 long M, int D)
{
    kla::ConvArgs<T> a = {};
    a.x = static_cast<const T*>(x); a.ld_x = ld_x; a.weight = weight; a.bias = bias; a.state = static_cast<const T*>(state);
    a.seqs = s; a.M = M; a.D = D;
    return a;
}

// ---- selective scan ---------------------------------------------------------------------------------------------------------------
// (a lane's offset from the first of 16 rows fits 32 bits; a step has one row of a sequence and no such offsets)
constexpr int kMaxSsmRow = 1 << 24;
constexpr int kMaxSsmSeqs = 65535;                       // sequences, and groups: a launch's second dimension
bool ssm_shape_ok(int D, int G, int S) { return D > 0 && D <= kMaxSsmRow && G > 0 && D % G == 0 && (S == 8 || S == 16 || S == 32 || S == 64); }
// Tokens per segment.  A wave takes 8 channels of one segment and its tokens one after the other, about 70 ns each when it has its SIMD to
// itself; segments cost a second pass over most of the tokens for their maps.  4096 waves run at twice the tokens per second of 1024, one
// for each SIMD.  So batches of fewer than 768 waves are cut into segments until 4096 run; up to 255 tokens the additional launches cost more than they
// save.  At 768 waves forward calls are about even: 2048 tokens and 16 states, whole and in segments, three sequences of 2048 channels 132 and 127 us, six
// of 1024 126 and 128, twelve of 512 132 and 139; three of 512 tokens 36 and 42 us; 8, 32 and 64 states 98 and 110, 196 and 206, 314 and 356 us.  Both
// directions together, cut alike, still gain there where sequences are long (447 and 393 us, of 8192 tokens 1751 and 1489) and lose where they are
// short or have 64 states (300 tokens 92 and 107 us; 1258 and 1293).  Kernels of both: one sequence 443 and 168 us, two 447 and 297, four 490 and 551.
// Segments are whole pairs of tiles, and 64 tokens at least (in multiples of 64 one sequence of 7000 tokens x 1024 channels took 82 us forward instead
// of 74).  In a packed batch the longest sequence decides: it would run on alone.
int ssm_segment(long M, int n_states, int D, long longest)
{
    const int whole = INT_MAX / 32 * 32;
    const long per = ((long)D + 7) / 8;                  // waves of one sequence
    if (n_states == 0 || longest < 256 || M * per >= 768 * longest) return whole;
    const long len = (M * per / 4096 + 31) / 32 * 32;
    return (int)(len < 64 ? 64 : len < whole ? len : whole);
}
struct SsmPlan { int Lseg; long slots, checkpoints; int channels; };
SsmPlan ssm_plan(const kla::Seqs& s, const int32_t* cu_host, long M, int D, int G, int S)
{
    SsmPlan p;
    long longest = s.T;
    if (s.cu) {
        longest = 0;
        for (int i = 0; i < s.n_seq; ++i) if (cu_host[i + 1] - cu_host[i] > longest) longest = cu_host[i + 1] - cu_host[i];
    }
    p.Lseg = ssm_segment(M, s.n_seq, D, longest);
    p.channels = 64;
    const int ck = kla::ssm_checkpoint(S);
    if (s.cu) {
        p.slots = M / p.Lseg + s.n_seq;
        p.checkpoints = M / ck + s.n_seq;
    } else {
        const long per = ((long)s.T + p.Lseg - 1) / p.Lseg;
        p.slots = (per > 0 ? per : 1) * s.n_seq;
        p.checkpoints = ((long)s.T + ck - 1) / ck * s.n_seq;
    }
    // The forward's workgroups have 64 channels (half as many bring in the rows of B and C) unless 32 spread more evenly over the CUs, where
    // they may be more than a tenth slower.  (bf16, 2048 channels, 2048 tokens, 64 and 32: 8 sequences 225 and 244 us, 16 sequences 404
    // and 456 us, 12 sequences 378 and 334 us, 4 sequences 205 and 142 us; 8 sequences with 64 states 579 and 548 us: there it is 32.)
    auto rounds = [&](int channels) { return ((long)G * ((D / G + channels - 1) / channels) * p.slots + 255) / 256; };
    if (S == 64 || 20 * rounds(64) > 11 * rounds(32)) p.channels = 32;
    return p;
}
// What the queries know: the sizes, and the offsets of a packed batch on the host
int ssm_sizes(int N, int T, int D, int G, int S, const int32_t* cu_host, int n_seq, kla::Seqs* s, long* M)
{
    if (!ssm_shape_ok(D, G, S) || N > kMaxSsmSeqs || n_seq > kMaxSsmSeqs || G > kMaxSsmSeqs) return KLA_ERR_SHAPE;
    return take_seqs(n_seq > 0 ? cu_host : nullptr, cu_host, n_seq, N, T, s, M);
}
bool ssm_split(const kla::Seqs& s, const SsmPlan& p) { return p.slots > s.n_seq; }
size_t ssm_saved(const SsmPlan& p, int D, int S) { return round256((size_t)p.checkpoints * D * S * sizeof(float)); }
struct SsmWork { float *seg_state, *seg_delta, *saved, *part_bc, *part_p; size_t bytes; };
SsmWork ssm_work(char* base, const kla::Seqs& s, const SsmPlan& p, long M, int D, int G, int S, bool bwd, bool keeps)
{
    Carve c{base};
    SsmWork w = {};
    if (ssm_split(s, p)) {
        w.seg_state = c.take<float>((size_t)p.slots * D * S);
        w.seg_delta = c.take<float>((size_t)p.slots * D);
    }
    if (bwd) {
        const long blocks = (long)G * ((D / G + kla::kSsmBwdChannels - 1) / kla::kSsmBwdChannels);
        if (!keeps) w.saved = c.take<float>((size_t)p.checkpoints * D * S);
        w.part_bc = c.take<float>((size_t)blocks * M * 2 * S);
        w.part_p = c.take<float>((size_t)p.slots * D * (S + 2));
    }
    w.bytes = c.used;
    return w;
}
int ssm_check(const void* u, long ld_u, const void* delta, long ld_delta, const float* A, const void* B, long ld_B, const void* C, long ld_C, const void* z,
              long ld_z, int D, int G, int S, int dt, unsigned opts, long most)
{
    if (!dt_ok(dt)) return KLA_ERR_DTYPE;
    if (!ssm_shape_ok(D, G, S) || ld_u < D || ld_delta < D || ld_B < (long)G * S || ld_C < (long)G * S || (z && ld_z < D) ||
        ld_u > most || ld_delta > most || ld_B > most || ld_C > most || (z && ld_z > most) || (opts & ~(unsigned)KLA_LAYER_SOFTPLUS))
        return KLA_ERR_SHAPE;
    if (!A) return KLA_ERR_NULL;
    (void)u; (void)delta; (void)B; (void)C;
    return KLA_OK;
}
template <typename T>
kla::SsmArgs<T> ssm_args(const void* u, long ld_u, const void* delta, long ld_delta, const float* A, const void* B, long ld_B, const void* C, long ld_C,
                         const float* skip, const void* z, long ld_z, const float* delta_bias, const float* h0, const kla::Seqs& s, long M, int D, int G,
                         const SsmPlan& p, unsigned opts)
{
    kla::SsmArgs<T> a = {};
    a.u = static_cast<const T*>(u); a.ld_u = ld_u; a.delta = static_cast<const T*>(delta); a.ld_delta = ld_delta; a.A = A;
    a.B = static_cast<const T*>(B); a.ld_B = ld_B; a.C = static_cast<const T*>(C); a.ld_C = ld_C;
    a.skip = skip; a.z = static_cast<const T*>(z); a.ld_z = ld_z; a.delta_bias = delta_bias; a.h0 = h0;
    a.seqs = s; a.M = M; a.D = D; a.G = G; a.Lseg = p.Lseg; a.slots = p.slots; a.channels = p.channels;
    a.softplus = (opts & KLA_LAYER_SOFTPLUS) != 0;
    return a;
}

// ---- norms ------------------------------------------------------------------------------------------------------------------------
constexpr int kMaxNorm = 8192;
bool norm_shape_ok(long M, int D, float eps) { return M >= 0 && D > 0 && D <= kMaxNorm && eps >= 0.f; }   // (a NaN is not)
template <typename T, typename R>
kla::AddNormArgs<T, R> add_norm_args(const void* x, long ld_x, const void* residual, const float* scale, const float* weight, float eps, long M, int D)
{
    kla::AddNormArgs<T, R> a = {};
    a.x = static_cast<const T*>(x); a.ld_x = ld_x; a.residual = static_cast<const R*>(residual); a.scale = scale; a.weight = weight; a.eps = eps;
    a.M = M; a.D = D;
    return a;
}
template <typename T>
kla::GatedNormArgs<T> gated_norm_args(const void* x, long ld_x, const void* gate, long ld_gate, const float* weight, float eps, long M, int H, int D,
                                      unsigned opts)
{
    kla::GatedNormArgs<T> a = {};
    a.x = static_cast<const T*>(x); a.ld_x = ld_x; a.gate = static_cast<const T*>(gate); a.ld_gate = ld_gate; a.weight = weight; a.eps = eps;
    a.M = M; a.H = H; a.D = D; a.opts = opts;
    return a;
}
int add_norm_check(const void* x, long ld_x, const float* weight, float eps, long M, int D, int dt, int res_dt)
{
    if (!dt_ok(dt) || !dt_ok(res_dt) || (dt == KLA_F32 && res_dt != KLA_F32)) return KLA_ERR_DTYPE;
    if (!norm_shape_ok(M, D, eps) || ld_x < D) return KLA_ERR_SHAPE;
    if (!weight || (M > 0 && !x)) return KLA_ERR_NULL;
    return KLA_OK;
}
int gated_norm_check(const void* x, long ld_x, const void* gate, long ld_gate, const float* weight, float eps, long M, int H, int D, int dt, unsigned opts)
{
    if (!dt_ok(dt)) return KLA_ERR_DTYPE;
    if (!norm_shape_ok(M, D, eps) || H <= 0 || ld_x < (long)H * D || ld_gate < (long)H * D || (opts & ~(unsigned)(KLA_LAYER_SIGMOID | KLA_LAYER_GATE_FIRST)))
        return KLA_ERR_SHAPE;
    if (!weight || (M > 0 && (!x || !gate))) return KLA_ERR_NULL;
    return KLA_OK;
}

}  // namespace

extern "C" {

int kla_conv_fwd(const void* x, long ld_x, const float* weight, const float* bias, const void* state, void* y, void* state_out,
                 const int32_t* cu_seqlens_dev, const int32_t* cu_seqlens_host, int n_seq, int N, int T, int D, int W, kla_dtype dt, void* hip_stream,
                 unsigned opts)
{
    kla::Seqs s;
    long M;
    if (const int e = conv_check(x, ld_x, weight, D, W, dt, opts)) return e;
    if (const int e = take_seqs(cu_seqlens_dev, cu_seqlens_host, n_seq, N, T, &s, &M)) return e;
    if (M > 0 && (!x || !y)) return KLA_ERR_NULL;
    // written while others read it: a token's inputs are those of earlier tokens too
    if ((state_out && state_out == state) || (M > 0 && y == x)) return KLA_ERR_SHAPE;
    const size_t e = elem_bytes(dt);
    if (!aligned(e, {x, state, y, state_out}) || !aligned(4, {weight, bias})) return KLA_ERR_ALIGN;
    const bool silu = opts & KLA_LAYER_SILU;
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    auto run = [&](auto a) {
        a.y = static_cast<decltype(a.y)>(y);
        a.state_out = static_cast<decltype(a.y)>(state_out);
        return status(kla::launch_conv_fwd(a, W, silu, st));
    };
    return dt == KLA_BF16 ? run(conv_args<bf16_t>(x, ld_x, weight, bias, state, s, M, D)) : run(conv_args<float>(x, ld_x, weight, bias, state, s, M, D));
}

size_t kla_conv_bwd_workspace_bytes(int N, int T, int D, int W)
{
    if (N < 0 || T < 0 || D <= 0 || D > kMaxConv || W < 2 || W > 4) return 0;
    return round256((size_t)kla::conv_bwd_plan((long)N * T, D).blocks_t * D * (W + 1) * sizeof(float));
}

int kla_conv_bwd(const void* x, long ld_x, const float* weight, const float* bias, const void* state, const void* d_y, const void* d_state_out, void* dx,
                 float* dweight, float* dbias, void* d_state, const int32_t* cu_seqlens_dev, const int32_t* cu_seqlens_host, int n_seq, int N, int T, int D,
                 int W, kla_dtype dt, void* workspace, size_t workspace_bytes, void* hip_stream, unsigned opts)
{
    kla::Seqs s;
    long M;
    if (const int e = conv_check(x, ld_x, weight, D, W, dt, opts)) return e;
    if (const int e = take_seqs(cu_seqlens_dev, cu_seqlens_host, n_seq, N, T, &s, &M)) return e;
    if (!dweight || (M > 0 && (!x || !d_y || !dx))) return KLA_ERR_NULL;
    if ((M > 0 && (dx == x || dx == d_y)) || (d_state && (d_state == state || d_state == d_state_out))) return KLA_ERR_SHAPE;    // (as y and x)
    const size_t e = elem_bytes(dt);
    if (!aligned(e, {x, state, d_y, d_state_out, dx, d_state}) || !aligned(4, {weight, bias, dweight, dbias})) return KLA_ERR_ALIGN;
    if (const int r = take_workspace(workspace, workspace_bytes, kla_conv_bwd_workspace_bytes(N, T, D, W))) return r;
    const bool silu = opts & KLA_LAYER_SILU;
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    auto run = [&](auto a) {
        using P = decltype(a.x);
        using Q = decltype(a.y);
        a.d_y = static_cast<P>(d_y); a.d_state_out = static_cast<P>(d_state_out); a.dx = static_cast<Q>(dx); a.d_state = static_cast<Q>(d_state);
        a.partial = static_cast<float*>(workspace);
        return status(kla::launch_conv_bwd(a, W, silu, dweight, dbias, st));
    };
    return dt == KLA_BF16 ? run(conv_args<bf16_t>(x, ld_x, weight, bias, state, s, M, D)) : run(conv_args<float>(x, ld_x, weight, bias, state, s, M, D));
}

int kla_conv_step(const void* x, long ld_x, const float* weight, const float* bias, void* state, void* y, int B, int D, int W, kla_dtype dt, void* hip_stream,
                  unsigned opts)
{
    if (const int e = conv_check(x, ld_x, weight, D, W, dt, opts)) return e;
    if (B < 0) return KLA_ERR_SHAPE;
    if (B > 0 && (!x || !state || !y)) return KLA_ERR_NULL;
    if (!aligned(elem_bytes(dt), {x, state, y}) || !aligned(4, {weight, bias})) return KLA_ERR_ALIGN;
    const bool silu = opts & KLA_LAYER_SILU;
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    auto run = [&](auto* px) {
        using E = std::remove_const_t<std::remove_pointer_t<decltype(px)>>;
        return status(kla::launch_conv_step<E>(px, ld_x, weight, bias, static_cast<E*>(state), static_cast<E*>(y), B, D, W, silu, st));
    };
    return dt == KLA_BF16 ? run(static_cast<const bf16_t*>(x)) : run(static_cast<const float*>(x));
}

size_t kla_ssm_fwd_workspace_bytes(int N, int T, int D, int G, int S, const int32_t* cu_seqlens_host, int n_seq)
{
    kla::Seqs s;
    long M;
    if (ssm_sizes(N, T, D, G, S, cu_seqlens_host, n_seq, &s, &M)) return 0;
    return ssm_work(nullptr, s, ssm_plan(s, cu_seqlens_host, M, D, G, S), M, D, G, S, false, false).bytes;
}
size_t kla_ssm_saved_bytes(int N, int T, int D, int G, int S, const int32_t* cu_seqlens_host, int n_seq)
{
    kla::Seqs s;
    long M;
    if (ssm_sizes(N, T, D, G, S, cu_seqlens_host, n_seq, &s, &M)) return 0;
    return ssm_saved(ssm_plan(s, cu_seqlens_host, M, D, G, S), D, S);
}
size_t kla_ssm_bwd_workspace_bytes(int N, int T, int D, int G, int S, const int32_t* cu_seqlens_host, int n_seq, int has_saved)
{
    kla::Seqs s;
    long M;
    if (ssm_sizes(N, T, D, G, S, cu_seqlens_host, n_seq, &s, &M)) return 0;
    return ssm_work(nullptr, s, ssm_plan(s, cu_seqlens_host, M, D, G, S), M, D, G, S, true, has_saved != 0).bytes;
}

int kla_ssm_fwd(const void* u, long ld_u, const void* delta, long ld_delta, const float* A, const void* B, long ld_B, const void* C, long ld_C,
                const float* skip, const void* z, long ld_z, const float* delta_bias, const float* h0, void* y, float* hT, float* saved, size_t saved_bytes,
                const int32_t* cu_seqlens_dev, const int32_t* cu_seqlens_host, int n_seq, int N, int T, int D, int G, int S, kla_dtype dt, void* workspace,
                size_t workspace_bytes, void* hip_stream, unsigned opts)
{
    kla::Seqs s;
    long M;
    if (const int e = ssm_check(u, ld_u, delta, ld_delta, A, B, ld_B, C, ld_C, z, ld_z, D, G, S, dt, opts, kMaxSsmRow)) return e;
    if (const int e = take_seqs(cu_seqlens_dev, cu_seqlens_host, n_seq, N, T, &s, &M)) return e;
    if (M > 0 && (!u || !delta || !B || !C || !y)) return KLA_ERR_NULL;
    if (!aligned(elem_bytes(dt), {u, delta, B, C, z, y}) || !aligned(16, {A, h0, hT, saved}) || !aligned(4, {skip, delta_bias})) return KLA_ERR_ALIGN;
    if (s.n_seq > kMaxSsmSeqs || G > kMaxSsmSeqs) return KLA_ERR_SHAPE;
    const SsmPlan p = ssm_plan(s, cu_seqlens_host, M, D, G, S);
    if (saved && saved_bytes < ssm_saved(p, D, S)) return KLA_ERR_WORKSPACE;
    const SsmWork w = ssm_work(static_cast<char*>(workspace), s, p, M, D, G, S, false, false);
    if (const int e = take_workspace(workspace, workspace_bytes, w.bytes)) return e;
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    auto run = [&](auto a) {
        a.y = static_cast<decltype(a.y)>(y); a.hT = hT; a.saved = saved; a.seg_state = w.seg_state; a.seg_delta = w.seg_delta;
        return status(kla::launch_ssm_fwd(a, S, true, st));
    };
    return dt == KLA_BF16 ? run(ssm_args<bf16_t>(u, ld_u, delta, ld_delta, A, B, ld_B, C, ld_C, skip, z, ld_z, delta_bias, h0, s, M, D, G, p, opts))
                          : run(ssm_args<float>(u, ld_u, delta, ld_delta, A, B, ld_B, C, ld_C, skip, z, ld_z, delta_bias, h0, s, M, D, G, p, opts));
}

int kla_ssm_bwd(const void* u, long ld_u, const void* delta, long ld_delta, const float* A, const void* B, long ld_B, const void* C, long ld_C,
                const float* skip, const void* z, long ld_z, const float* delta_bias, const float* h0, const void* d_y, const float* d_hT, const float* saved,
                size_t saved_bytes, void* du, void* ddelta, float* dA, void* dB, void* dC, float* dskip, void* dz, float* ddelta_bias, float* dh0,
                const int32_t* cu_seqlens_dev, const int32_t* cu_seqlens_host, int n_seq, int N, int T, int D, int G, int S, kla_dtype dt, void* workspace,
                size_t workspace_bytes, void* hip_stream, unsigned opts)
{
    kla::Seqs s;
    long M;
    if (const int e = ssm_check(u, ld_u, delta, ld_delta, A, B, ld_B, C, ld_C, z, ld_z, D, G, S, dt, opts, kMaxSsmRow)) return e;
    if (const int e = take_seqs(cu_seqlens_dev, cu_seqlens_host, n_seq, N, T, &s, &M)) return e;
    if (!dA || (M > 0 && (!u || !delta || !B || !C || !d_y || !du || !ddelta || !dB || !dC || (z && !dz)))) return KLA_ERR_NULL;
    if (!aligned(elem_bytes(dt), {u, delta, B, C, z, d_y, du, ddelta, dB, dC, dz}) || !aligned(16, {A, h0, d_hT, saved, dA, dh0}) ||
        !aligned(4, {skip, delta_bias, dskip, ddelta_bias}))
        return KLA_ERR_ALIGN;
    if (s.n_seq > kMaxSsmSeqs || G > kMaxSsmSeqs) return KLA_ERR_SHAPE;
    const SsmPlan p = ssm_plan(s, cu_seqlens_host, M, D, G, S);
    if (saved && saved_bytes < ssm_saved(p, D, S)) return KLA_ERR_WORKSPACE;
    const SsmWork w = ssm_work(static_cast<char*>(workspace), s, p, M, D, G, S, true, saved != nullptr);
    if (const int e = take_workspace(workspace, workspace_bytes, w.bytes)) return e;
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    auto run = [&](auto a) {
        using P = decltype(a.u);
        using Q = decltype(a.y);
        using E = std::remove_pointer_t<Q>;
        a.seg_state = w.seg_state; a.seg_delta = w.seg_delta;
        a.saved = saved ? const_cast<float*>(saved) : w.saved;
        if (!saved) {
            if (const hipError_t e = kla::launch_ssm_fwd(a, S, false, st)) return status(e);
        }
        a.d_y = static_cast<P>(d_y); a.d_hT = d_hT;
        a.du = static_cast<Q>(du); a.ddelta = static_cast<Q>(ddelta); a.dz = static_cast<Q>(dz); a.dh0 = dh0;
        a.part_bc = w.part_bc; a.part_p = w.part_p;
        return status(kla::launch_ssm_bwd<E>(a, S, dA, static_cast<Q>(dB), static_cast<Q>(dC), dskip, ddelta_bias, st));
    };
    return dt == KLA_BF16 ? run(ssm_args<bf16_t>(u, ld_u, delta, ld_delta, A, B, ld_B, C, ld_C, skip, z, ld_z, delta_bias, h0, s, M, D, G, p, opts))
                          : run(ssm_args<float>(u, ld_u, delta, ld_delta, A, B, ld_B, C, ld_C, skip, z, ld_z, delta_bias, h0, s, M, D, G, p, opts));
}

int kla_ssm_step(const void* u, long ld_u, const void* delta, long ld_delta, const float* A, const void* B, long ld_B, const void* C, long ld_C,
                 const float* skip, const void* z, long ld_z, const float* delta_bias, float* h, void* y, int N, int D, int G, int S, kla_dtype dt,
                 void* hip_stream, unsigned opts)
{
    if (const int e = ssm_check(u, ld_u, delta, ld_delta, A, B, ld_B, C, ld_C, z, ld_z, D, G, S, dt, opts, LONG_MAX)) return e;
    if (N < 0) return KLA_ERR_SHAPE;
    if (N > 0 && (!u || !delta || !B || !C || !h || !y)) return KLA_ERR_NULL;
    if (!aligned(elem_bytes(dt), {u, delta, B, C, z, y}) || !aligned(16, {A, h}) || !aligned(4, {skip, delta_bias})) return KLA_ERR_ALIGN;
    const kla::Seqs s = {nullptr, N, 1};
    const SsmPlan p = {1, N, N, 64};
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    auto run = [&](auto a) {
        a.y = static_cast<decltype(a.y)>(y);
        return status(kla::launch_ssm_step(a, h, N, S, st));
    };
    return dt == KLA_BF16 ? run(ssm_args<bf16_t>(u, ld_u, delta, ld_delta, A, B, ld_B, C, ld_C, skip, z, ld_z, delta_bias, nullptr, s, N, D, G, p, opts))
                          : run(ssm_args<float>(u, ld_u, delta, ld_delta, A, B, ld_B, C, ld_C, skip, z, ld_z, delta_bias, nullptr, s, N, D, G, p, opts));
}

int kla_add_norm_fwd(const void* x, long ld_x, const void* residual, const float* scale, const float* weight, float eps, void* y, void* residual_out, long M,
                     int D, kla_dtype dt, kla_dtype res_dt, void* hip_stream)
{
    if (const int e = add_norm_check(x, ld_x, weight, eps, M, D, dt, res_dt)) return e;
    if (M > 0 && !y) return KLA_ERR_NULL;
    const size_t e = elem_bytes(dt), r = elem_bytes(res_dt);
    if (!aligned(e, {x, y}) || !aligned(r, {residual, residual_out}) || !aligned(4, {scale, weight})) return KLA_ERR_ALIGN;
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    auto run = [&](auto a) {
        a.y = static_cast<decltype(a.y)>(y);
        a.residual_out = static_cast<decltype(a.residual_out)>(residual_out);
        return status(kla::launch_add_norm_fwd(a, st));
    };
    if (dt == KLA_F32) return run(add_norm_args<float, float>(x, ld_x, residual, scale, weight, eps, M, D));
    return res_dt == KLA_F32 ? run(add_norm_args<bf16_t, float>(x, ld_x, residual, scale, weight, eps, M, D))
                             : run(add_norm_args<bf16_t, bf16_t>(x, ld_x, residual, scale, weight, eps, M, D));
}

static int norm_blocks(long rows, int D, int dt) { return kla::norm_bwd_blocks(rows, D, dt == KLA_BF16 ? 8 : 4); }
size_t kla_add_norm_bwd_workspace_bytes(long M, int D, kla_dtype dt)
{
    if (!dt_ok(dt) || !norm_shape_ok(M, D, 0.f)) return 0;
    return round256((size_t)norm_blocks(M, D, dt) * 2 * D * sizeof(float));
}

int kla_add_norm_bwd(const void* x, long ld_x, const void* residual, const float* scale, const float* weight, float eps, const void* d_y,
                     const void* d_residual_out, void* dx, void* d_residual, float* dscale, float* dweight, long M, int D, kla_dtype dt, kla_dtype res_dt,
                     void* workspace, size_t workspace_bytes, void* hip_stream)
{
    if (const int e = add_norm_check(x, ld_x, weight, eps, M, D, dt, res_dt)) return e;
    if (!dweight || (M > 0 && (!d_y || !dx))) return KLA_ERR_NULL;
    const size_t e = elem_bytes(dt), r = elem_bytes(res_dt);
    if (!aligned(e, {x, d_y, dx}) || !aligned(r, {residual, d_residual_out, d_residual}) || !aligned(4, {scale, weight, dscale, dweight}))
        return KLA_ERR_ALIGN;
    if (const int q = take_workspace(workspace, workspace_bytes, kla_add_norm_bwd_workspace_bytes(M, D, dt))) return q;
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    auto run = [&](auto a) {
        a.d_y = static_cast<decltype(a.d_y)>(d_y);
        a.d_residual_out = static_cast<decltype(a.d_residual_out)>(d_residual_out);
        a.dx = static_cast<decltype(a.dx)>(dx);
        a.d_residual = static_cast<decltype(a.d_residual)>(d_residual);
        a.partial = static_cast<float*>(workspace);
        return status(kla::launch_add_norm_bwd(a, dweight, dscale, st));
    };
    if (dt == KLA_F32) return run(add_norm_args<float, float>(x, ld_x, residual, scale, weight, eps, M, D));
    return res_dt == KLA_F32 ? run(add_norm_args<bf16_t, float>(x, ld_x, residual, scale, weight, eps, M, D))
                             : run(add_norm_args<bf16_t, bf16_t>(x, ld_x, residual, scale, weight, eps, M, D));
}

int kla_gated_norm_fwd(const void* x, long ld_x, const void* gate, long ld_gate, const float* weight, float eps, void* y, long M, int H, int D, kla_dtype dt,
                       void* hip_stream, unsigned opts)
{
    if (const int e = gated_norm_check(x, ld_x, gate, ld_gate, weight, eps, M, H, D, dt, opts)) return e;
    if (M > 0 && !y) return KLA_ERR_NULL;
    const size_t e = elem_bytes(dt);
    if (!aligned(e, {x, gate, y}) || !aligned(4, {weight})) return KLA_ERR_ALIGN;
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    auto run = [&](auto a) {
        a.y = static_cast<decltype(a.y)>(y);
        return status(kla::launch_gated_norm_fwd(a, st));
    };
    return dt == KLA_BF16 ? run(gated_norm_args<bf16_t>(x, ld_x, gate, ld_gate, weight, eps, M, H, D, opts))
                          : run(gated_norm_args<float>(x, ld_x, gate, ld_gate, weight, eps, M, H, D, opts));
}

size_t kla_gated_norm_bwd_workspace_bytes(long M, int H, int D, kla_dtype dt)
{
    if (!dt_ok(dt) || !norm_shape_ok(M, D, 0.f) || H <= 0) return 0;
    return round256((size_t)norm_blocks(M * H, D, dt) * D * sizeof(float));
}

int kla_gated_norm_bwd(const void* x, long ld_x, const void* gate, long ld_gate, const float* weight, float eps, const void* d_y, void* dx, void* d_gate,
                       float* dweight, long M, int H, int D, kla_dtype dt, void* workspace, size_t workspace_bytes, void* hip_stream, unsigned opts)
{
    if (const int e = gated_norm_check(x, ld_x, gate, ld_gate, weight, eps, M, H, D, dt, opts)) return e;
    if (!dweight || (M > 0 && (!d_y || !dx || !d_gate))) return KLA_ERR_NULL;
    const size_t e = elem_bytes(dt);
    if (!aligned(e, {x, gate, d_y, dx, d_gate}) || !aligned(4, {weight, dweight})) return KLA_ERR_ALIGN;
    if (const int q = take_workspace(workspace, workspace_bytes, kla_gated_norm_bwd_workspace_bytes(M, H, D, dt))) return q;
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    auto run = [&](auto a) {
        a.d_y = static_cast<decltype(a.d_y)>(d_y);
        a.dx = static_cast<decltype(a.dx)>(dx);
        a.d_gate = static_cast<decltype(a.dx)>(d_gate);
        a.partial = static_cast<float*>(workspace);
        return status(kla::launch_gated_norm_bwd(a, dweight, st));
    };
    return dt == KLA_BF16 ? run(gated_norm_args<bf16_t>(x, ld_x, gate, ld_gate, weight, eps, M, H, D, opts))
                          : run(gated_norm_args<float>(x, ld_x, gate, ld_gate, weight, eps, M, H, D, opts));
}

}  // extern "C"
