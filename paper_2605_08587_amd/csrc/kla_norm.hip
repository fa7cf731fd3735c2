// The two norms of a block, forward and backward:
//   add_norm    r' = r + s x,  y = w n,  n = f r',  f = 1/sqrt(mean(r'^2) + eps)
//   gated_norm  y = w n g, n = f x  (or: n = f (x g), y = w n),  g = gate sigmoid(gate) or sigmoid(gate), per head
// Backward of a norm: with e = w dy (dy times the gate's activation where it stands behind), the gradient of what is normalised is
//   f (e - n mean(e n)),  and  d_w = sum over the rows of dy n.
// A row stays in the registers of its TPR threads between the sum and its use, so that every element is read once and written
// once; nothing but the inputs is kept for the backward, which forms f again.  Bound by memory.
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
// 1/sqrt(mean + eps); 0 for a row of zeros with eps = 0, whose norm is then zeros and not 0/0
__device__ __forceinline__ float inv_rms(float sum, float inv_d, float eps)
{
    const float m = fmaf(sum, inv_d, eps);
    return m == 0.f ? 0.f : __builtin_amdgcn_rsqf(m);
}
// the activated gate and its derivative
__device__ __forceinline__ void gate_of(float t, bool plain_sigmoid, float* g, float* slope)
{
    const float s = sigmoid(t);
    *g = plain_sigmoid ? s : t * s;
    *slope = plain_sigmoid ? s * (1.f - s) : s * fmaf(t, 1.f - s, 1.f);
}

// A thread's elements of a row: vector v of it stands at column (v * TPR + lane) * V.
template <int V, int NV> struct Row { float v[NV][V]; };
#define KLA_EACH_VEC(v) _Pragma("unroll") for (int v = 0; v < NV; ++v)
#define KLA_EACH(v, i) KLA_EACH_VEC(v) _Pragma("unroll") for (int i = 0; i < V; ++i)
template <typename T, int TPR, int V, int NV> __device__ __forceinline__ Row<V, NV> load_row(const T* p, int lane, int D, float fill = 0.f)
{
    Row<V, NV> r;
    KLA_EACH_VEC(v) {
        const int c = (v * TPR + lane) * V;
        if (c < D) {
            const Floats<V> f = load_vec<T, V>(p + c);
#pragma unroll
            for (int i = 0; i < V; ++i) r.v[v][i] = f.v[i];
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) r.v[v][i] = fill;
        }
    }
    return r;
}
template <typename T, int TPR, int V, int NV> __device__ __forceinline__ void store_row(T* p, int lane, int D, const Row<V, NV>& r)
{
    KLA_EACH_VEC(v) {
        const int c = (v * TPR + lane) * V;
        if (c < D) {
            Floats<V> f;
#pragma unroll
            for (int i = 0; i < V; ++i) f.v[i] = r.v[v][i];
            store_vec<T, V>(p + c, f);
        }
    }
}

constexpr int block_threads(int TPR) { return TPR < 256 ? 256 : TPR; }

template <typename T, typename R, int TPR, int V, int NV>
__global__ __launch_bounds__(block_threads(TPR)) void add_norm_fwd_kernel(AddNormArgs<T, R> a)
{
    constexpr int ROWS = block_threads(TPR) / TPR;
    __shared__ float red[TPR > 64 ? TPR / 64 : 1];
    const int lane = threadIdx.x % TPR;
    const long row = (long)blockIdx.x * ROWS + threadIdx.x / TPR;
    if (row >= a.M) return;                              // (TPR > 64: ROWS is 1 and no row is beyond the last)
    Row<V, NV> x = load_row<T, TPR, V, NV>(a.x + row * a.ld_x, lane, a.D);
    if (a.residual) {
        const Row<V, NV> r = load_row<R, TPR, V, NV>(a.residual + row * a.D, lane, a.D);
        if (a.scale) {
            const Row<V, NV> s = load_row<float, TPR, V, NV>(a.scale, lane, a.D);
            KLA_EACH(v, i) x.v[v][i] = fmaf(s.v[v][i], x.v[v][i], r.v[v][i]);
        } else {
            KLA_EACH(v, i) x.v[v][i] += r.v[v][i];
        }
    } else if (a.scale) {
        const Row<V, NV> s = load_row<float, TPR, V, NV>(a.scale, lane, a.D);
        KLA_EACH(v, i) x.v[v][i] *= s.v[v][i];
    }
    const Row<V, NV> w = load_row<float, TPR, V, NV>(a.weight, lane, a.D);
    if (a.residual_out) store_row<R, TPR, V, NV>(a.residual_out + row * a.D, lane, a.D, x);
    float sum = 0.f;
    KLA_EACH(v, i) sum = fmaf(x.v[v][i], x.v[v][i], sum);
    const float f = inv_rms(row_sum<TPR>(sum, red), 1.f / (float)a.D, a.eps);
    KLA_EACH(v, i) x.v[v][i] *= f * w.v[v][i];
    store_row<T, TPR, V, NV>(a.y + row * a.D, lane, a.D, x);
}

// Sums over the rows that a workgroup took, from the registers of its threads: one row of partial[.][n_out * D] per workgroup, part p
// of it at p * D.
template <int TPR, int V, int NV> __device__ __forceinline__ void leave_partial(float* out, float* red, int lane, int group, int D, const Row<V, NV>& s)
{
    constexpr int ROWS = block_threads(TPR) / TPR;
    if constexpr (ROWS == 1) {
        store_row<float, TPR, V, NV>(out, lane, D, s);
    } else {
        KLA_EACH(v, i) red[(group * NV + v) * (TPR * V) + lane * V + i] = s.v[v][i];
        __syncthreads();
        for (int c = threadIdx.x; c < D; c += block_threads(TPR)) {
            float t = 0.f;
            for (int g = 0; g < ROWS; ++g) t += red[g * (NV * TPR * V) + c];
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
    const int lane = threadIdx.x % TPR, group = threadIdx.x / TPR;
    const Row<V, NV> w = load_row<float, TPR, V, NV>(a.weight, lane, a.D);
    Row<V, NV> sc, dw, ds;
    if (a.scale) sc = load_row<float, TPR, V, NV>(a.scale, lane, a.D, 1.f);
    else { KLA_EACH(v, i) sc.v[v][i] = 1.f; }
    KLA_EACH(v, i) dw.v[v][i] = ds.v[v][i] = 0.f;
    const float inv_d = 1.f / (float)a.D;
    for (long row = (long)blockIdx.x * ROWS + group; row < a.M; row += (long)gridDim.x * ROWS) {
        const Row<V, NV> x = load_row<T, TPR, V, NV>(a.x + row * a.ld_x, lane, a.D);
        Row<V, NV> n, dy = load_row<T, TPR, V, NV>(a.d_y + row * a.D, lane, a.D), d;
        if (a.residual) n = load_row<R, TPR, V, NV>(a.residual + row * a.D, lane, a.D);
        else { KLA_EACH(v, i) n.v[v][i] = 0.f; }
        if (a.d_residual_out) d = load_row<R, TPR, V, NV>(a.d_residual_out + row * a.D, lane, a.D);
        else { KLA_EACH(v, i) d.v[v][i] = 0.f; }
        float sq = 0.f, en = 0.f;
        KLA_EACH(v, i) {
            const float t = fmaf(sc.v[v][i], x.v[v][i], n.v[v][i]);
            n.v[v][i] = t;
            sq = fmaf(t, t, sq);
            en = fmaf(dy.v[v][i] * w.v[v][i], t, en);
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
        if (a.d_residual) store_row<R, TPR, V, NV>(a.d_residual + row * a.D, lane, a.D, d);
        KLA_EACH(v, i) d.v[v][i] *= sc.v[v][i];
        store_row<T, TPR, V, NV>(a.dx + row * a.D, lane, a.D, d);
    }
    if constexpr (TPR > 64 || ROWS > 1) __syncthreads();
    float* out = a.partial + (long)blockIdx.x * 2 * a.D;
    leave_partial<TPR, V, NV>(out, red, lane, group, a.D, dw);
    leave_partial<TPR, V, NV>(out + a.D, red, lane, group, a.D, ds);
}

template <typename T, int TPR, int V, int NV>
__global__ __launch_bounds__(block_threads(TPR)) void gated_norm_fwd_kernel(GatedNormArgs<T> a)
{
    constexpr int ROWS = block_threads(TPR) / TPR;
    __shared__ float red[TPR > 64 ? TPR / 64 : 1];
    const int lane = threadIdx.x % TPR;
    const long row = (long)blockIdx.x * ROWS + threadIdx.x / TPR;
    if (row >= a.M * a.H) return;
    const long m = row / a.H, h = row - m * a.H;
    Row<V, NV> x = load_row<T, TPR, V, NV>(a.x + m * a.ld_x + h * a.D, lane, a.D);
    Row<V, NV> g = load_row<T, TPR, V, NV>(a.gate + m * a.ld_gate + h * a.D, lane, a.D);
    const Row<V, NV> w = load_row<float, TPR, V, NV>(a.weight, lane, a.D);
    const bool first = a.opts & kLayerGateFirst, plain = a.opts & kLayerSigmoid;
    float sum = 0.f;
    KLA_EACH(v, i) {
        float s;
        gate_of(g.v[v][i], plain, &g.v[v][i], &s);
        if (first) { x.v[v][i] *= g.v[v][i]; g.v[v][i] = 1.f; }
        sum = fmaf(x.v[v][i], x.v[v][i], sum);
    }
    const float f = inv_rms(row_sum<TPR>(sum, red), 1.f / (float)a.D, a.eps);
    KLA_EACH(v, i) x.v[v][i] *= f * w.v[v][i] * g.v[v][i];
    store_row<T, TPR, V, NV>(a.y + row * a.D, lane, a.D, x);
}

template <typename T, int TPR, int V, int NV>
__global__ __launch_bounds__(block_threads(TPR)) void gated_norm_bwd_kernel(GatedNormArgs<T> a)
{
    constexpr int ROWS = block_threads(TPR) / TPR;
    __shared__ float red[ROWS == 1 ? (TPR > 64 ? TPR / 64 : 1) : ROWS * NV * TPR * V];
    const int lane = threadIdx.x % TPR, group = threadIdx.x / TPR;
    const Row<V, NV> w = load_row<float, TPR, V, NV>(a.weight, lane, a.D);
    Row<V, NV> dw;
    KLA_EACH(v, i) dw.v[v][i] = 0.f;
    const bool first = a.opts & kLayerGateFirst, plain = a.opts & kLayerSigmoid;
    const float inv_d = 1.f / (float)a.D;
    const long rows = a.M * a.H;
    for (long row = (long)blockIdx.x * ROWS + group; row < rows; row += (long)gridDim.x * ROWS) {
        const long m = row / a.H, h = row - m * a.H;
        Row<V, NV> x = load_row<T, TPR, V, NV>(a.x + m * a.ld_x + h * a.D, lane, a.D);
        const Row<V, NV> t = load_row<T, TPR, V, NV>(a.gate + m * a.ld_gate + h * a.D, lane, a.D);
        Row<V, NV> dy = load_row<T, TPR, V, NV>(a.d_y + row * a.D, lane, a.D);
        float sq = 0.f, en = 0.f;
        KLA_EACH(v, i) {
            float g, s;
            gate_of(t.v[v][i], plain, &g, &s);
            const float q = first ? x.v[v][i] * g : x.v[v][i];       // what is normalised
            const float e = (first ? dy.v[v][i] : dy.v[v][i] * g) * w.v[v][i];
            sq = fmaf(q, q, sq);
            en = fmaf(e, q, en);
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
        store_row<T, TPR, V, NV>(a.dx + row * a.D, lane, a.D, x);
        store_row<T, TPR, V, NV>(a.d_gate + row * a.D, lane, a.D, dy);
    }
    if constexpr (TPR > 64 || ROWS > 1) __syncthreads();
    leave_partial<TPR, V, NV>(a.partial + (long)blockIdx.x * a.D, red, lane, group, a.D, dw);
}

// Threads per row and vectors per thread for a row of n_vec vectors: f(threads per row, elements per vector, vectors per thread).  At most
// 16 elements per thread, which leaves the backward without a spilled register.
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
    if constexpr (V == 1) {
        if (n_vec <= 4096) return f(IntC<1024>(), IntC<V>(), IntC<4>());
        if (n_vec <= 8192) return f(IntC<1024>(), IntC<V>(), IntC<8>());
    }
    return hipErrorInvalidConfiguration;
}
static int threads_per_row(long n_vec)
{
    return n_vec <= 16 ? 16 : n_vec <= 32 ? 32 : n_vec <= 128 ? 64 : n_vec <= 512 ? 256 : n_vec <= 1024 ? 512 : 1024;
}

int norm_bwd_blocks(long rows, int D, bool vec, int vec_len)
{
    const int tpr = threads_per_row(vec ? (D + vec_len - 1) / vec_len : D);
    const long per = block_threads(tpr) / tpr, want = (rows + per - 1) / per, most = tpr > 256 ? 512 : 1024;
    return (int)(want < most ? want : most);
}

template <typename T, typename F> static hipError_t for_rows(long rows, int D, bool vec, F&& f)
{
    return vec ? by_width<kVec<T>>((D + kVec<T> - 1) / kVec<T>, f) : by_width<1>(D, f);
}
template <typename T, typename R> hipError_t launch_add_norm_fwd(const AddNormArgs<T, R>& a, bool vec, hipStream_t st)
{
    if (a.M == 0) return hipSuccess;
    return for_rows<T>(a.M, a.D, vec, [&](auto tpr, auto v, auto nv) {
        constexpr int rows = block_threads(tpr.value) / tpr.value;
        const long blocks = (a.M + rows - 1) / rows;
        if (blocks > 0x7fffffffL) return hipErrorInvalidConfiguration;
        hipLaunchKernelGGL((add_norm_fwd_kernel<T, R, tpr.value, v.value, nv.value>), dim3((unsigned)blocks), dim3(block_threads(tpr.value)), 0, st, a);
        return hipGetLastError();
    });
}
template <typename T, typename R> hipError_t launch_add_norm_bwd(const AddNormArgs<T, R>& a, bool vec, float* dweight, float* dscale, hipStream_t st)
{
    const int blocks = norm_bwd_blocks(a.M, a.D, vec, kVec<T>);
    if (blocks > 0) {
        const hipError_t e = for_rows<T>(a.M, a.D, vec, [&](auto tpr, auto v, auto nv) {
            hipLaunchKernelGGL((add_norm_bwd_kernel<T, R, tpr.value, v.value, nv.value>), dim3(blocks), dim3(block_threads(tpr.value)), 0, st, a);
            return hipGetLastError();
        });
        if (e) return e;
    }
    return launch_column_sums(a.partial, blocks, {{a.D, a.D, 0}, {dweight, dscale, nullptr}}, st);
}
template <typename T> hipError_t launch_gated_norm_fwd(const GatedNormArgs<T>& a, bool vec, hipStream_t st)
{
    if (a.M == 0) return hipSuccess;
    return for_rows<T>(a.M * a.H, a.D, vec, [&](auto tpr, auto v, auto nv) {
        constexpr int rows = block_threads(tpr.value) / tpr.value;
        const long blocks = (a.M * a.H + rows - 1) / rows;
        if (blocks > 0x7fffffffL) return hipErrorInvalidConfiguration;
        hipLaunchKernelGGL((gated_norm_fwd_kernel<T, tpr.value, v.value, nv.value>), dim3((unsigned)blocks), dim3(block_threads(tpr.value)), 0, st, a);
        return hipGetLastError();
    });
}
template <typename T> hipError_t launch_gated_norm_bwd(const GatedNormArgs<T>& a, bool vec, float* dweight, hipStream_t st)
{
    const int blocks = norm_bwd_blocks(a.M * a.H, a.D, vec, kVec<T>);
    if (blocks > 0) {
        const hipError_t e = for_rows<T>(a.M * a.H, a.D, vec, [&](auto tpr, auto v, auto nv) {
            hipLaunchKernelGGL((gated_norm_bwd_kernel<T, tpr.value, v.value, nv.value>), dim3(blocks), dim3(block_threads(tpr.value)), 0, st, a);
            return hipGetLastError();
        });
        if (e) return e;
    }
    return launch_column_sums(a.partial, blocks, {{a.D, 0, 0}, {dweight, nullptr, nullptr}}, st);
}

#define KLA_ADD_NORM(T, R)                                                                                       \
    template hipError_t launch_add_norm_fwd<T, R>(const AddNormArgs<T, R>&, bool, hipStream_t);                  \
    template hipError_t launch_add_norm_bwd<T, R>(const AddNormArgs<T, R>&, bool, float*, float*, hipStream_t);
KLA_ADD_NORM(float, float)
KLA_ADD_NORM(bf16_t, float)
KLA_ADD_NORM(bf16_t, bf16_t)
#define KLA_GATED_NORM(T)                                                                                        \
    template hipError_t launch_gated_norm_fwd<T>(const GatedNormArgs<T>&, bool, hipStream_t);                    \
    template hipError_t launch_gated_norm_bwd<T>(const GatedNormArgs<T>&, bool, float*, hipStream_t);
KLA_GATED_NORM(float)
KLA_GATED_NORM(bf16_t)

}  // namespace kla
