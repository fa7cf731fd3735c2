// The two norms of a block, forward and backward:
//   add_norm    r' = r + s x,  y = w n,  n = f r',  f = 1/sqrt(mean(r'^2) + eps)
//   gated_norm  y = w n g, n = f x  (or: n = f (x g), y = w n),  g = gate sigmoid(gate) or sigmoid(gate), per head
// Backward of a norm: with e = w dy (dy times the gate's activation where it stands behind), the gradient of what is normalised is
//   f (e - n mean(e n)),  and  d_w = sum over the rows of dy n.
// A row stays in the registers of its TPR threads between the sum and its use, so that every element is read once and written
// once; nothing but the inputs is kept for the backward, which forms f again.  Bound by memory: bf16, 32768 rows of 1024 with an fp32 stream
// forward 74 us (403 MB, 5.4 TB/s), backward 119 us (604 MB, 5.1 TB/s); 262144 heads of 256 with their gates forward 78 us (403 MB, 5.2 TB/s),
// backward 135 us (671 MB, 5.0 TB/s); a large copy 4.8 TB/s.
#include <algorithm>

#include "kla_layer.hpp"

namespace kla {

// Sum over the TPR threads of a row, in every one of them; red: TPR/64 floats, behind a barrier that the next use of red needs too.
template <int TPR> __device__ __forceinline__ float row_sum(float x, float* red)
{
    if constexpr (TPR == 16) return row_sum16(x);
    if constexpr (TPR == 32) {
        x = row_sum16(x);
        return x + __shfl_xor(x, 16, 64);
    }
    if constexpr (TPR == 64) return wave_sum_rows(x);
    if constexpr (TPR > 64) {
        x = wave_sum_rows(x);
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
        __syncthreads();
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < TPR / 64; ++i) s += red[i];
        __syncthreads();
        return s;
    }
}
// 1/sqrt(mean + eps); 0 for a row of zeros with eps = 0, whose norm is then zeros and not 0/0.  The hardware's root takes a denormal for 0
// and gives infinity: such a mean is brought into its range first.
__device__ __forceinline__ float inv_rms(float sum, float inv_d, float eps)
{
    const float m = fmaf(sum, inv_d, eps);
    const bool low = m < 0x1p-126f;
    const float f = __builtin_amdgcn_rsqf(low ? m * 0x1p64f : m);
    return m == 0.f ? 0.f : low ? f * 0x1p32f : f;
}
// the activated gate and its derivative
__device__ __forceinline__ void gate_of(float t, bool plain_sigmoid, float* g, float* slope)
{
    const float s = sigmoid(t);
    *g = plain_sigmoid ? s : t * s;
    *slope = plain_sigmoid ? s * (1.f - s) : s * fmaf(t, 1.f - s, 1.f);
}

// A thread's elements of a row of D >= V: vector v of it stands at column (v * TPR + lane) * V, the row's last vector at D - V.  That one may
// hold columns of the vector before it too: they are left out of the sums, and come to the same in both.
template <int V, int NV> struct Row { float v[NV][V]; };
#define KLA_EACH_VEC(v) _Pragma("unroll") for (int v = 0; v < NV; ++v)
#define KLA_EACH(v, i) KLA_EACH_VEC(v) _Pragma("unroll") for (int i = 0; i < V; ++i)
template <int TPR, int V, int NV> struct Columns {
    int c[NV], twice;                                    // first columns; how many of the last vector are the one's before it
    bool on[NV];
    __device__ __forceinline__ Columns(int lane, int D)
    {
        KLA_EACH_VEC(v) {
            const int place = (v * TPR + lane) * V;
            on[v] = place < D;
            c[v] = min(place, D - V);
            if (v == NV - 1) twice = place - c[v];
        }
    }
    // x, or 0 where the vector before has it too: of both factors of a product, as 0 times an infinity is none.  (The last vector is one of the
    // threads' last: by_width.)
    __device__ __forceinline__ float once(int v, int i, float x) const { return v == NV - 1 && i < twice ? 0.f : x; }
    template <typename T> __device__ __forceinline__ Row<V, NV> load(const T* p, float fill = 0.f) const
    {
        Row<V, NV> r;
        KLA_EACH_VEC(v) {
            if (on[v]) {
                const Floats<V> f = load_vec<T, V>(p + c[v]);
#pragma unroll
                for (int i = 0; i < V; ++i) r.v[v][i] = f.v[i];
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) r.v[v][i] = fill;
            }
        }
        return r;
    }
    template <typename T> __device__ __forceinline__ void store(T* p, const Row<V, NV>& r) const
    {
        KLA_EACH_VEC(v) {
            if (on[v]) {
                Floats<V> f;
#pragma unroll
                for (int i = 0; i < V; ++i) f.v[i] = r.v[v][i];
                store_vec<T, V>(p + c[v], f);
            }
        }
    }
};

constexpr int block_threads(int TPR) { return TPR < 256 ? 256 : TPR; }

template <typename T, typename R, int TPR, int V, int NV>
__global__ __launch_bounds__(block_threads(TPR)) void add_norm_fwd_kernel(AddNormArgs<T, R> a)
{
    constexpr int ROWS = block_threads(TPR) / TPR;
    __shared__ float red[TPR > 64 ? TPR / 64 : 1];
    const Columns<TPR, V, NV> at(threadIdx.x % TPR, a.D);
    const long row = (long)blockIdx.x * ROWS + threadIdx.x / TPR;
    if (row >= a.M) return;                              // (TPR > 64: ROWS is 1 and no row is beyond the last)
    Row<V, NV> x = at.load(a.x + row * a.ld_x);
    if (a.residual) {
        const Row<V, NV> r = at.load(a.residual + row * a.D);
        if (a.scale) {
            const Row<V, NV> s = at.load(a.scale);
            KLA_EACH(v, i) x.v[v][i] = fmaf(s.v[v][i], x.v[v][i], r.v[v][i]);
        } else {
            KLA_EACH(v, i) x.v[v][i] += r.v[v][i];
        }
    } else if (a.scale) {
        const Row<V, NV> s = at.load(a.scale);
        KLA_EACH(v, i) x.v[v][i] *= s.v[v][i];
    }
    const Row<V, NV> w = at.load(a.weight);
    float sum = 0.f;
    KLA_EACH(v, i) {
        const float o = at.once(v, i, x.v[v][i]);
        sum = fmaf(o, o, sum);
    }
    const float f = inv_rms(row_sum<TPR>(sum, red), 1.f / (float)a.D, a.eps);
    // Behind the sum's barrier: residual_out may be residual, and the row's last vector has columns of another wave's, which has to have read
    // them by then (up to TPR = 64 one wave has the row, and its loads stand ahead of its stores).
    if (a.residual_out) at.store(a.residual_out + row * a.D, x);
    KLA_EACH(v, i) x.v[v][i] *= f * w.v[v][i];
    at.store(a.y + row * a.D, x);
}

// Sums over the rows that a workgroup took, from the registers of its threads: one row of partial[.][n_out * D] per workgroup, part p
// of it at p * D.
template <int TPR, int V, int NV> __device__ __forceinline__ void leave_partial(float* out, float* red, const Columns<TPR, V, NV>& at, int group, int D,
                                                                                const Row<V, NV>& s)
{
    constexpr int ROWS = block_threads(TPR) / TPR, LONG = NV * TPR * V;
    if constexpr (ROWS == 1) {
        at.store(out, s);
    } else {
        KLA_EACH_VEC(v) {
            if (at.on[v]) {
#pragma unroll
                for (int i = 0; i < V; ++i) red[group * LONG + at.c[v] + i] = s.v[v][i];
            }
        }
        __syncthreads();
        for (int c = threadIdx.x; c < D; c += block_threads(TPR)) {
            float t = 0.f;
            for (int g = 0; g < ROWS; ++g) t += red[g * LONG + c];
            out[c] = t;
        }
        __syncthreads();
    }
}

template <typename T, typename R, int TPR, int V, int NV>
__global__ __launch_bounds__(block_threads(TPR)) void add_norm_bwd_kernel(AddNormArgs<T, R> a)
{
    constexpr int ROWS = block_threads(TPR) / TPR;
    __shared__ float red[ROWS == 1 ? (TPR > 64 ? TPR / 64 : 1) : ROWS * NV * TPR * V];
    const int group = threadIdx.x / TPR;
    const Columns<TPR, V, NV> at(threadIdx.x % TPR, a.D);
    const Row<V, NV> w = at.load(a.weight);
    Row<V, NV> sc, dw, ds;
    if (a.scale) sc = at.load(a.scale, 1.f);
    else { KLA_EACH(v, i) sc.v[v][i] = 1.f; }
    KLA_EACH(v, i) dw.v[v][i] = ds.v[v][i] = 0.f;
    const float inv_d = 1.f / (float)a.D;
    for (long row = (long)blockIdx.x * ROWS + group; row < a.M; row += (long)gridDim.x * ROWS) {
        const Row<V, NV> x = at.load(a.x + row * a.ld_x);
        Row<V, NV> n, dy = at.load(a.d_y + row * a.D), d;
        if (a.residual) n = at.load(a.residual + row * a.D);
        else { KLA_EACH(v, i) n.v[v][i] = 0.f; }
        if (a.d_residual_out) d = at.load(a.d_residual_out + row * a.D);
        else { KLA_EACH(v, i) d.v[v][i] = 0.f; }
        float sq = 0.f, en = 0.f;
        KLA_EACH(v, i) {
            const float t = fmaf(sc.v[v][i], x.v[v][i], n.v[v][i]);
            n.v[v][i] = t;
            const float o = at.once(v, i, t);
            sq = fmaf(o, o, sq);
            en = fmaf(at.once(v, i, dy.v[v][i] * w.v[v][i]), o, en);
        }
        sq = row_sum<TPR>(sq, red);
        en = row_sum<TPR>(en, red);
        const float f = inv_rms(sq, inv_d, a.eps), m = en * f * inv_d;       // mean(e n)
        KLA_EACH(v, i) {
            const float u = n.v[v][i] * f;
            dw.v[v][i] = fmaf(dy.v[v][i], u, dw.v[v][i]);
            const float g = fmaf(f, fmaf(dy.v[v][i], w.v[v][i], -u * m), d.v[v][i]);
            ds.v[v][i] = fmaf(g, x.v[v][i], ds.v[v][i]);
            d.v[v][i] = g;
        }
        if (a.d_residual) at.store(a.d_residual + row * a.D, d);
        KLA_EACH(v, i) d.v[v][i] *= sc.v[v][i];
        at.store(a.dx + row * a.D, d);
    }
    if constexpr (TPR > 64 || ROWS > 1) __syncthreads();
    float* out = a.partial + (long)blockIdx.x * 2 * a.D;
    leave_partial<TPR, V, NV>(out, red, at, group, a.D, dw);
    leave_partial<TPR, V, NV>(out + a.D, red, at, group, a.D, ds);
}

template <typename T, int TPR, int V, int NV>
__global__ __launch_bounds__(block_threads(TPR)) void gated_norm_fwd_kernel(GatedNormArgs<T> a)
{
    constexpr int ROWS = block_threads(TPR) / TPR;
    __shared__ float red[TPR > 64 ? TPR / 64 : 1];
    const Columns<TPR, V, NV> at(threadIdx.x % TPR, a.D);
    const long row = (long)blockIdx.x * ROWS + threadIdx.x / TPR;
    if (row >= a.M * a.H) return;
    const long m = row / a.H, h = row - m * a.H;
    Row<V, NV> x = at.load(a.x + m * a.ld_x + h * a.D);
    Row<V, NV> g = at.load(a.gate + m * a.ld_gate + h * a.D);
    const Row<V, NV> w = at.load(a.weight);
    const bool first = a.opts & kLayerGateFirst, plain = a.opts & kLayerSigmoid;
    float sum = 0.f;
    KLA_EACH(v, i) {
        float s;
        gate_of(g.v[v][i], plain, &g.v[v][i], &s);
        if (first) { x.v[v][i] *= g.v[v][i]; g.v[v][i] = 1.f; }
        const float o = at.once(v, i, x.v[v][i]);
        sum = fmaf(o, o, sum);
    }
    const float f = inv_rms(row_sum<TPR>(sum, red), 1.f / (float)a.D, a.eps);
    KLA_EACH(v, i) x.v[v][i] *= f * w.v[v][i] * g.v[v][i];
    at.store(a.y + row * a.D, x);
}

template <typename T, int TPR, int V, int NV>
__global__ __launch_bounds__(block_threads(TPR)) void gated_norm_bwd_kernel(GatedNormArgs<T> a)
{
    constexpr int ROWS = block_threads(TPR) / TPR;
    __shared__ float red[ROWS == 1 ? (TPR > 64 ? TPR / 64 : 1) : ROWS * NV * TPR * V];
    const int group = threadIdx.x / TPR;
    const Columns<TPR, V, NV> at(threadIdx.x % TPR, a.D);
    const Row<V, NV> w = at.load(a.weight);
    Row<V, NV> dw;
    KLA_EACH(v, i) dw.v[v][i] = 0.f;
    const bool first = a.opts & kLayerGateFirst, plain = a.opts & kLayerSigmoid;
    const float inv_d = 1.f / (float)a.D;
    const long rows = a.M * a.H;
    for (long row = (long)blockIdx.x * ROWS + group; row < rows; row += (long)gridDim.x * ROWS) {
        const long m = row / a.H, h = row - m * a.H;
        Row<V, NV> x = at.load(a.x + m * a.ld_x + h * a.D);
        const Row<V, NV> t = at.load(a.gate + m * a.ld_gate + h * a.D);
        Row<V, NV> dy = at.load(a.d_y + row * a.D);
        float sq = 0.f, en = 0.f;
        KLA_EACH(v, i) {
            float g, s;
            gate_of(t.v[v][i], plain, &g, &s);
            const float q = first ? x.v[v][i] * g : x.v[v][i];       // what is normalised
            const float e = (first ? dy.v[v][i] : dy.v[v][i] * g) * w.v[v][i];
            const float o = at.once(v, i, q);
            sq = fmaf(o, o, sq);
            en = fmaf(at.once(v, i, e), o, en);
        }
        sq = row_sum<TPR>(sq, red);
        en = row_sum<TPR>(en, red);
        const float f = inv_rms(sq, inv_d, a.eps), mean = en * f * inv_d;
        KLA_EACH(v, i) {
            float g, s;
            gate_of(t.v[v][i], plain, &g, &s);
            const float q = first ? x.v[v][i] * g : x.v[v][i], u = q * f;
            const float out = first ? dy.v[v][i] : dy.v[v][i] * g;
            dw.v[v][i] = fmaf(out, u, dw.v[v][i]);
            const float dq = f * fmaf(out, w.v[v][i], -u * mean);
            const float dg = first ? dq * x.v[v][i] : dy.v[v][i] * u * w.v[v][i];
            x.v[v][i] = first ? dq * g : dq;
            dy.v[v][i] = dg * s;
        }
        at.store(a.dx + row * a.D, x);
        at.store(a.d_gate + row * a.D, dy);
    }
    if constexpr (TPR > 64 || ROWS > 1) __syncthreads();
    leave_partial<TPR, V, NV>(a.partial + (long)blockIdx.x * a.D, red, at, group, a.D, dw);
}

// Threads per row and vectors per thread for a row of n_vec vectors: f(threads per row, elements per vector, vectors per thread).  At most
// 16 elements per thread, which leaves the backward without a spilled register.  A row of fewer elements than a vector has one per thread.
// (Rows of odd widths in vectors too and not an element at a time: bf16, 16384 gated rows of 2047, both directions 132 against 282 us.)
template <int V, typename F> static hipError_t by_width(long n_vec, F&& f)
{
    if (n_vec <= 16) return f(IntC<16>(), IntC<V>(), IntC<1>());
    if (n_vec <= 32) return f(IntC<32>(), IntC<V>(), IntC<1>());
    if (n_vec <= 64) return f(IntC<64>(), IntC<V>(), IntC<1>());
    if (n_vec <= 128) return f(IntC<64>(), IntC<V>(), IntC<2>());
    if (n_vec <= 256) return f(IntC<256>(), IntC<V>(), IntC<1>());
    if (n_vec <= 512) return f(IntC<256>(), IntC<V>(), IntC<2>());
    if (n_vec <= 1024) return f(IntC<512>(), IntC<V>(), IntC<2>());
    if constexpr (V < 8) {
        if (n_vec <= 2048) return f(IntC<1024>(), IntC<V>(), IntC<2>());
    }
    return hipErrorInvalidConfiguration;
}
static int threads_per_row(long n_vec)
{
    return n_vec <= 16 ? 16 : n_vec <= 32 ? 32 : n_vec <= 128 ? 64 : n_vec <= 512 ? 256 : n_vec <= 1024 ? 512 : 1024;
}

// Workgroups of the backward, each of which takes rows one after the other and leaves sums for the parameters.  Two for each CU, and four for
// rows of up to a wave's vectors, whose threads have little under way (bf16, 512 and 1024 workgroups, with the sums: 262144 gated heads of 256
// 197 and 134 us, 131072 of 128 48 and 39 us; add_norm 32768 x 1024 124 and 127 us, 4096 x 8192 137 and 151 us; 2048 always cost more).
int norm_bwd_blocks(long rows, int D, int vec_len)
{
    const long n_vec = (D + vec_len - 1) / vec_len;
    const int tpr = threads_per_row(n_vec);
    const long per = block_threads(tpr) / tpr, want = (rows + per - 1) / per, most = n_vec <= 64 ? 1024 : 512;
    return (int)(want < most ? want : most);
}

template <typename T, typename F> static hipError_t for_rows(int D, F&& f)
{
    if (D < kVec<T>) return f(IntC<16>(), IntC<1>(), IntC<1>());
    return by_width<kVec<T>>((D + kVec<T> - 1) / kVec<T>, f);
}
template <typename T, typename R> hipError_t launch_add_norm_fwd(const AddNormArgs<T, R>& a, hipStream_t st)
{
    return for_rows<T>(a.D, [&](auto tpr, auto v, auto nv) {
        constexpr int threads = block_threads(tpr.value), rows = threads / tpr.value;
        AddNormArgs<T, R> b = a;
        for (long done = 0; done < a.M; done += b.M) {
            b.M = std::min(a.M - done, most_blocks(threads) * rows);
            b.x = a.x + done * a.ld_x;
            b.y = a.y + done * a.D;
            if (a.residual) b.residual = a.residual + done * a.D;
            if (a.residual_out) b.residual_out = a.residual_out + done * a.D;
            hipLaunchKernelGGL((add_norm_fwd_kernel<T, R, tpr.value, v.value, nv.value>), dim3((unsigned)((b.M + rows - 1) / rows)), dim3(threads), 0, st, b);
            if (const hipError_t e = hipGetLastError()) return e;
        }
        return hipSuccess;
    });
}
template <typename T, typename R> hipError_t launch_add_norm_bwd(const AddNormArgs<T, R>& a, float* dweight, float* dscale, hipStream_t st)
{
    const int blocks = norm_bwd_blocks(a.M, a.D, kVec<T>);
    if (blocks > 0) {
        const hipError_t e = for_rows<T>(a.D, [&](auto tpr, auto v, auto nv) {
            hipLaunchKernelGGL((add_norm_bwd_kernel<T, R, tpr.value, v.value, nv.value>), dim3(blocks), dim3(block_threads(tpr.value)), 0, st, a);
            return hipGetLastError();
        });
        if (e) return e;
    }
    return launch_column_sums(a.partial, blocks, {{a.D, a.D, 0}, {dweight, dscale, nullptr}}, st);
}
template <typename T> hipError_t launch_gated_norm_fwd(const GatedNormArgs<T>& a, hipStream_t st)
{
    return for_rows<T>(a.D, [&](auto tpr, auto v, auto nv) {
        constexpr int threads = block_threads(tpr.value), rows = threads / tpr.value;
        const long piece = most_blocks(threads) * rows / a.H;            // tokens of a launch
        if (piece == 0) return hipErrorInvalidConfiguration;
        GatedNormArgs<T> b = a;
        for (long done = 0; done < a.M; done += b.M) {
            b.M = std::min(a.M - done, piece);
            b.x = a.x + done * a.ld_x;
            b.gate = a.gate + done * a.ld_gate;
            b.y = a.y + done * a.H * a.D;
            hipLaunchKernelGGL((gated_norm_fwd_kernel<T, tpr.value, v.value, nv.value>), dim3((unsigned)((b.M * a.H + rows - 1) / rows)), dim3(threads), 0,
                               st, b);
            if (const hipError_t e = hipGetLastError()) return e;
        }
        return hipSuccess;
    });
}
template <typename T> hipError_t launch_gated_norm_bwd(const GatedNormArgs<T>& a, float* dweight, hipStream_t st)
{
    const int blocks = norm_bwd_blocks(a.M * a.H, a.D, kVec<T>);
    if (blocks > 0) {
        const hipError_t e = for_rows<T>(a.D, [&](auto tpr, auto v, auto nv) {
            hipLaunchKernelGGL((gated_norm_bwd_kernel<T, tpr.value, v.value, nv.value>), dim3(blocks), dim3(block_threads(tpr.value)), 0, st, a);
            return hipGetLastError();
        });
        if (e) return e;
    }
    return launch_column_sums(a.partial, blocks, {{a.D, 0, 0}, {dweight, nullptr, nullptr}}, st);
}

#define KLA_ADD_NORM(T, R)                                                                                       \
    template hipError_t launch_add_norm_fwd<T, R>(const AddNormArgs<T, R>&, hipStream_t);                  \
    template hipError_t launch_add_norm_bwd<T, R>(const AddNormArgs<T, R>&, float*, float*, hipStream_t);
KLA_ADD_NORM(float, float)
KLA_ADD_NORM(bf16_t, float)
KLA_ADD_NORM(bf16_t, bf16_t)
#define KLA_GATED_NORM(T)                                                                                        \
    template hipError_t launch_gated_norm_fwd<T>(const GatedNormArgs<T>&, hipStream_t);                    \
    template hipError_t launch_gated_norm_bwd<T>(const GatedNormArgs<T>&, float*, hipStream_t);
KLA_GATED_NORM(float)
KLA_GATED_NORM(bf16_t)

}  // namespace kla
