// Short causal convolution of every channel with its activation, forward, backward and for single tokens:
//   p_t = b + sum_j w_j x_{t-W+1+j},  y_t = p_t sigmoid(p_t)  (or p_t)
// and backward, with p'_t = d_y_t dy_t/dp_t:
//   d_x_s = sum_j w_j p'_{s+W-1-j},  d_w_j = sum_t p'_t x_{t-W+1+j},  d_b = sum_t p'_t.
// Before a sequence's first token stands its state, the last W - 1 inputs of earlier tokens (or zeros); nothing of another
// sequence is ever multiplied, not even by zero.  Two passes over the elements forward, three backward: bound by memory.  bf16, 2048 channels,
// 8 x 4096 tokens: forward 54 us (268 MB, 5.0 TB/s), backward 93 us (403 MB, 4.3 TB/s) and 5 us for the sums; a large copy 4.8 TB/s.
#include <algorithm>

#include "kla_layer.hpp"

namespace kla {

template <bool SILU> __device__ __forceinline__ float act(float p) { return SILU ? p * sigmoid(p) : p; }
template <bool SILU> __device__ __forceinline__ float act_slope(float p)
{
    if constexpr (!SILU) return 1.f;
    const float s = sigmoid(p);
    return s * fmaf(p, 1.f - s, 1.f);
}

// Threads of a workgroup along a row, a power of two up to a wave: V channels each.
static int row_threads(long n_vec)
{
    int tx = 1;
    while (tx < 64 && tx < n_vec) tx *= 2;
    return tx;
}

// The first of a thread's V channels, from its place in the row: those of the last thread are the last V, some of them the previous one's
// too, and both write the same there.  (D >= V.)
template <int V> __device__ __forceinline__ int channels_at(int place, int D) { return min(place, D - V); }

// Taps and bias of V channels, and the W - 1 inputs ahead of token t of sequence p.
template <int W, int V> struct Taps {
    float w[W][V], b[V];
    __device__ __forceinline__ void load(const float* weight, const float* bias, int c)
    {
#pragma unroll
        for (int i = 0; i < V; ++i) {
#pragma unroll
            for (int j = 0; j < W; ++j) w[j][i] = weight[(long)(c + i) * W + j];
            b[i] = bias ? bias[c + i] : 0.f;
        }
    }
};
template <typename T, int W, int V> __device__ __forceinline__ void load_window(const ConvArgs<T>& a, const Place& p, long t, int c, Floats<V> (&win)[W])
{
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
        const long s = t - (W - 1) + j;
        if (s >= p.first) win[j] = load_vec<T, V>(a.x + s * a.ld_x + c);
        else if (a.state) win[j] = load_vec<T, V>(a.state + ((long)p.n * (W - 1) + (W - 1) + (s - p.first)) * a.D + c);
        else {
#pragma unroll
            for (int i = 0; i < V; ++i) win[j].v[i] = 0.f;
        }
    }
}

// Row of threads of a workgroup.  WAVE: a row is a whole wave, and its strip, tokens and sequences are scalars.
template <bool WAVE> __device__ __forceinline__ int thread_row(int tx)
{
    return WAVE ? __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) : (int)threadIdx.x / tx;
}

constexpr int kFwdAhead = 8;                             // rows in flight per thread

// A thread takes V channels (16 bytes) of L consecutive tokens with the window in registers: every row is read once, W - 1 of a strip twice, and
// a workgroup's strips follow each other, so that those come from the caches.  Rows are asked for eight ahead of their use.  Workgroups from
// n_main on write the states instead.  A row of 2047 channels takes 1.1 times as long as one of 2048 (with one channel per thread: 1.4).
template <typename T, int W, int V, bool SILU, bool WAVE>
__global__ __launch_bounds__(256) void conv_fwd_kernel(ConvArgs<T> a, int tx, int L, int blocks_c, unsigned n_main)
{
    const int lane = threadIdx.x % tx, row = thread_row<WAVE>(tx), ty = 256 / tx;
    const unsigned blk = blockIdx.x < n_main ? blockIdx.x : blockIdx.x - n_main;
    const int place = ((int)(blk % blocks_c) * tx + lane) * V, c = channels_at<V>(place, a.D);
    const long strip = (long)(blk / blocks_c) * ty + row;
    if (place >= a.D) return;
    if (blockIdx.x >= n_main) {                          // strip: the sequence whose state is written
        if (strip >= a.seqs.n_seq) return;
        const Place p = sequence(a.seqs, (int)strip);
        Floats<V> win[W];
        load_window<T, W, V>(a, p, p.end, c, win);
#pragma unroll
        for (int j = 0; j < W - 1; ++j) store_vec<T, V>(a.state_out + ((long)p.n * (W - 1) + j) * a.D + c, win[j]);
        return;
    }
    const long t0 = strip * L, t1 = min(t0 + L, a.M);
    if (t0 >= t1) return;
    // the first rows are asked for ahead of all that has to be found out about them
    Raw<T, V> in[kFwdAhead];
#pragma unroll
    for (int r = 0; r < kFwdAhead; ++r) in[r] = load_raw<T, V>(a.x + min(t0 + r, t1 - 1) * a.ld_x + c);
    Taps<W, V> k;
    k.load(a.weight, a.bias, c);
    Place p = sequence_of(a.seqs, t0);
    Floats<V> win[W];
    load_window<T, W, V>(a, p, t0, c, win);
    for (long base = t0; base < t1; base += kFwdAhead) {
        if (base > t0) {
#pragma unroll
            for (int r = 0; r < kFwdAhead; ++r) in[r] = load_raw<T, V>(a.x + min(base + r, t1 - 1) * a.ld_x + c);
        }
#pragma unroll
        for (int r = 0; r < kFwdAhead; ++r) {
            const long t = base + r;
            if (t < t1) {
                if (t == p.end) {
                    p = sequence_of(a.seqs, t);
                    load_window<T, W, V>(a, p, t, c, win);
                }
                win[W - 1] = floats_of<T, V>(in[r]);
                Floats<V> out;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    float s = k.b[i];
#pragma unroll
                    for (int j = 0; j < W; ++j) s = fmaf(k.w[j][i], win[j].v[i], s);
                    out.v[i] = act<SILU>(s);
                }
                store_vec<T, V>(a.y + t * a.D + c, out);
#pragma unroll
                for (int j = 0; j < W - 1; ++j) win[j] = win[j + 1];
            }
        }
    }
}

constexpr int kRowsAhead = 8;                            // rows in flight per thread, of x and of d_y

// Backward: the same strips; p' is formed once per token of the strip and again for the W - 1 tokens behind it, whose
// gradients reach into it.  acc[j] gathers d_x of token t - (W - 1) + j; the sums for the taps stay in registers, are joined over the
// workgroup's strips and leave one row of partial[blocks_t][D W + D] per workgroup.  Workgroups from n_main on form the gradients of
// the states instead.  Four channels per thread: window, gradients under way and sums for the taps fill 128 registers, four waves per SIMD
// (the bound keeps bf16 there; without scalar tokens it would spill: 128 channels 33 us instead of 16).
template <typename T, int W, int V, bool SILU, bool WAVE>
__global__ __launch_bounds__(256, WAVE && sizeof(T) == 2 ? 4 : 1) void conv_bwd_kernel(ConvArgs<T> a, int tx, int L, int blocks_c, unsigned n_main)
{
    const int lane = threadIdx.x % tx, row = thread_row<WAVE>(tx), ty = 256 / tx;
    const unsigned blk = blockIdx.x < n_main ? blockIdx.x : blockIdx.x - n_main;
    const int place = ((int)(blk % blocks_c) * tx + lane) * V, c = channels_at<V>(place, a.D);
    const long strip = (long)(blk / blocks_c) * ty + row;
    const bool mine = place < a.D;
    Taps<W, V> k;
    if (mine) k.load(a.weight, a.bias, c);

    if (blockIdx.x >= n_main) {
        if (!mine || strip >= a.seqs.n_seq) return;
        const Place p = sequence(a.seqs, (int)strip);
        const long len = p.end - p.first;
        Floats<V> win[W], ds[W - 1];
        load_window<T, W, V>(a, p, p.first, c, win);
#pragma unroll
        for (int i = 0; i < W - 1; ++i) {
#pragma unroll
            for (int e = 0; e < V; ++e) ds[i].v[e] = 0.f;
            // entry i is an entry of the state behind the sequence too where the sequence has fewer than W - 1 tokens
            if (a.d_state_out && i >= len) ds[i] = load_vec<T, V>(a.d_state_out + ((long)p.n * (W - 1) + (i - len)) * a.D + c);
        }
#pragma unroll
        for (int r = 0; r < W - 1; ++r) {
            if (r >= len) break;
            win[W - 1] = load_vec<T, V>(a.x + (p.first + r) * a.ld_x + c);
            const Floats<V> dy = load_vec<T, V>(a.d_y + (p.first + r) * (long)a.D + c);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                float s = k.b[e];
#pragma unroll
                for (int j = 0; j < W; ++j) s = fmaf(k.w[j][e], win[j].v[e], s);
                const float dp = dy.v[e] * act_slope<SILU>(s);
#pragma unroll
                for (int j = 0; j + r < W - 1; ++j) ds[j + r].v[e] = fmaf(k.w[j][e], dp, ds[j + r].v[e]);
            }
#pragma unroll
            for (int j = 0; j < W - 1; ++j) win[j] = win[j + 1];
        }
#pragma unroll
        for (int i = 0; i < W - 1; ++i) store_vec<T, V>(a.d_state + ((long)p.n * (W - 1) + i) * a.D + c, ds[i]);
        return;
    }

    float dw[W][V], db[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        db[e] = 0.f;
#pragma unroll
        for (int j = 0; j < W; ++j) dw[j][e] = 0.f;
    }
    const long t0 = strip * L, t1 = min(t0 + L, a.M);
    if (mine && t0 < t1) {
        const long t2 = min(t1 + W - 1, a.M);
        // (the first rows ahead of all that has to be found out about them)
        Raw<T, V> xin[kRowsAhead], gin[kRowsAhead];
        auto load = [&](long base) {
#pragma unroll
            for (int r = 0; r < kRowsAhead; ++r) {
                const long at = min(base + r, t2 - 1);
                xin[r] = load_raw<T, V>(a.x + at * a.ld_x + c);
                gin[r] = load_raw<T, V>(a.d_y + at * a.D + c);
            }
        };
        load(t0);
        Place p = sequence_of(a.seqs, t0);
        Floats<V> win[W], acc[W];
        load_window<T, W, V>(a, p, t0, c, win);
        auto clear = [&]() {
#pragma unroll
            for (int j = 0; j < W; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e) acc[j].v[e] = 0.f;
        };
        // d_x of token s, where it is this strip's and of the present sequence
        auto emit = [&](long s, Floats<V> g) {
            if (s < t0 || s < p.first || s >= t1) return;
            const long i = s - (p.end - (W - 1));
            if (a.d_state_out && i >= 0) {
                const Floats<V> d = load_vec<T, V>(a.d_state_out + ((long)p.n * (W - 1) + i) * a.D + c);
#pragma unroll
                for (int e = 0; e < V; ++e) g.v[e] += d.v[e];
            }
            store_vec<T, V>(a.dx + s * (long)a.D + c, g);
        };
        clear();
        long t = t0;
        bool on = true;
        for (long base = t0; base < t2 && on; base += kRowsAhead) {
            if (base > t0) load(base);
#pragma unroll
            for (int r = 0; r < kRowsAhead; ++r) {
                t = base + r;
                if (t < t2 && on) {
                    if (t == p.end) {
#pragma unroll
                        for (int j = 0; j < W - 1; ++j) emit(t - (W - 1) + j, acc[j]);
                        clear();
                        if (t >= t1) on = false;
                        else {
                            p = sequence_of(a.seqs, t);
                            load_window<T, W, V>(a, p, t, c, win);
                        }
                    }
                    if (on) {
                        win[W - 1] = floats_of<T, V>(xin[r]);
                        const Floats<V> grad = floats_of<T, V>(gin[r]);
                        const bool own = t < t1;
#pragma unroll
                        for (int e = 0; e < V; ++e) {
                            float s = k.b[e];
#pragma unroll
                            for (int j = 0; j < W; ++j) s = fmaf(k.w[j][e], win[j].v[e], s);
                            const float dp = grad.v[e] * act_slope<SILU>(s);
#pragma unroll
                            for (int j = 0; j < W; ++j) acc[j].v[e] = fmaf(k.w[j][e], dp, acc[j].v[e]);
                            if (own) {
                                db[e] += dp;
#pragma unroll
                                for (int j = 0; j < W; ++j) dw[j][e] = fmaf(dp, win[j].v[e], dw[j][e]);
                            }
                        }
                        emit(t - (W - 1), acc[0]);
#pragma unroll
                        for (int j = 0; j < W - 1; ++j) { acc[j] = acc[j + 1]; win[j] = win[j + 1]; }
#pragma unroll
                        for (int e = 0; e < V; ++e) acc[W - 1].v[e] = 0.f;
                    }
                }
            }
        }
        if (on) {                                        // the batch ends within W - 1 tokens: nothing follows these
#pragma unroll
            for (int j = 0; j < W - 1; ++j) emit(t2 - (W - 1) + j, acc[j]);
        }
    }
    __shared__ float red[256][V * (W + 1) + 1];
#pragma unroll
    for (int e = 0; e < V; ++e) {
#pragma unroll
        for (int j = 0; j < W; ++j) red[threadIdx.x][e * W + j] = dw[j][e];
        red[threadIdx.x][V * W + e] = db[e];
    }
    __syncthreads();
    const int nc = min(tx * V, a.D - (int)(blk % blocks_c) * tx * V);    // channels of this workgroup
    float* out = a.partial + (long)(blk / blocks_c) * ((long)a.D * (W + 1));
    const int c0 = (int)(blk % blocks_c) * tx * V;
    for (int i = threadIdx.x; i < nc * (W + 1); i += 256) {
        const bool tap = i < nc * W;
        const int ch = tap ? i / W : i - nc * W, e = c0 + ch - channels_at<V>(c0 + ch / V * V, a.D);      // element e of thread ch / V
        const int at = tap ? e * W + i % W : V * W + e;
        float s = 0.f;
        for (int r = 0; r < ty; ++r) s += red[r * tx + ch / V][at];
        out[tap ? (long)c0 * W + i : (long)a.D * W + c0 + ch] = s;
    }
}

// One token for B sequences: a thread per channel and sequence; all loads are independent.  One sequence of 2048 channels: 2.3 us, a launch
// that does nothing takes as long.
template <typename T, int W>
__global__ __launch_bounds__(256) void conv_step_kernel(const T* __restrict__ x, long ld_x, const float* __restrict__ weight,
                                                        const float* __restrict__ bias, T* __restrict__ state, T* __restrict__ y, int D,
                                                        int blocks_c, bool silu)
{
    const int c = (blockIdx.x % blocks_c) * 256 + threadIdx.x;
    const long b = blockIdx.x / blocks_c;
    if (c >= D) return;
    T* st = state + b * (W - 1) * D + c;
    T line[W];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) line[j] = st[(long)j * D];
    line[W - 1] = x[b * ld_x + c];
    float s = bias ? bias[c] : 0.f;
#pragma unroll
    for (int j = 0; j < W; ++j) s = fmaf(weight[(long)c * W + j], to_float(line[j]), s);
    y[b * D + c] = from_float<T>(silu ? s * sigmoid(s) : s);
#pragma unroll
    for (int j = 0; j < W - 1; ++j) st[(long)j * D] = line[j + 1];
}

ConvBwdPlan conv_bwd_plan(long M, int D)
{
    // (for four channels per thread; a row of fewer is one thread's)
    ConvBwdPlan p;
    p.tx = row_threads((D + 3) / 4);
    p.ty = 256 / p.tx;
    // (bf16, 2048 channels, strips of 64 and 16: 32768 tokens 90 against 102 us, 16384 tokens 54 and 52 us, 4096 tokens 37 against 20 us)
    p.L = (M / 64) * ((D + 255) / 256) > 2048 ? 64 : 16;
    const long strips = (M + p.L - 1) / p.L;
    p.blocks_t = (strips + p.ty - 1) / p.ty;
    return p;
}

template <typename T, int W, int V, bool SILU> static hipError_t conv_fwd(const ConvArgs<T>& a, hipStream_t st)
{
    const long n_vec = (a.D + V - 1) / V;
    const int tx = row_threads(n_vec), ty = 256 / tx, blocks_c = (int)((n_vec + tx - 1) / tx);
    // Strips of 32 tokens read few rows twice; where they would be fewer than four waves for each CU, strips of 8 use more of them
    // (bf16, 2048 channels: 32768 tokens 54 against 65 us, 8192 tokens 22 and 21 us, 2048 tokens 16 against 10 us).
    const int L = (a.M / 32) * ((n_vec + 63) / 64) > 1024 ? 32 : 8;
    const long strips = (a.M + L - 1) / L, n_main = (strips + ty - 1) / ty * blocks_c;
    const long n_state = a.state_out ? (a.seqs.n_seq + (long)ty - 1) / ty * blocks_c : 0;
    if (n_main + n_state == 0) return hipSuccess;
    if (n_main + n_state > most_blocks(256)) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)(n_main + n_state)), block(256);
    if (tx == 64) hipLaunchKernelGGL((conv_fwd_kernel<T, W, V, SILU, true>), grid, block, 0, st, a, tx, L, blocks_c, (unsigned)n_main);
    else          hipLaunchKernelGGL((conv_fwd_kernel<T, W, V, SILU, false>), grid, block, 0, st, a, tx, L, blocks_c, (unsigned)n_main);
    return hipGetLastError();
}
template <typename T, int W, int V, bool SILU> static hipError_t conv_bwd(const ConvArgs<T>& a, float* dweight, float* dbias, hipStream_t st)
{
    const ConvBwdPlan p = conv_bwd_plan(a.M, a.D);
    const int blocks_c = (a.D + p.tx * V - 1) / (p.tx * V);
    const long n_main = p.blocks_t * blocks_c, n_state = a.d_state ? (a.seqs.n_seq + (long)p.ty - 1) / p.ty * blocks_c : 0;
    if (n_main + n_state > most_blocks(256)) return hipErrorInvalidConfiguration;
    if (n_main + n_state > 0) {
        const dim3 grid((unsigned)(n_main + n_state)), block(256);
        if (p.tx == 64) hipLaunchKernelGGL((conv_bwd_kernel<T, W, V, SILU, true>), grid, block, 0, st, a, p.tx, p.L, blocks_c, (unsigned)n_main);
        else            hipLaunchKernelGGL((conv_bwd_kernel<T, W, V, SILU, false>), grid, block, 0, st, a, p.tx, p.L, blocks_c, (unsigned)n_main);
        if (const hipError_t e = hipGetLastError()) return e;
    }
    return launch_column_sums(a.partial, p.blocks_t, {{(long)a.D * W, a.D, 0}, {dweight, dbias, nullptr}}, st);
}

template <typename T, int V, typename F> static hipError_t by_taps(int W, bool silu, F&& f)
{
    switch (W * 2 + (silu ? 1 : 0)) {
        case 4: return f(IntC<2>(), IntC<V>(), IntC<0>());
        case 5: return f(IntC<2>(), IntC<V>(), IntC<1>());
        case 6: return f(IntC<3>(), IntC<V>(), IntC<0>());
        case 7: return f(IntC<3>(), IntC<V>(), IntC<1>());
        case 8: return f(IntC<4>(), IntC<V>(), IntC<0>());
        default: return f(IntC<4>(), IntC<V>(), IntC<1>());
    }
}
// (one channel per thread where a row has fewer than a vector)
template <typename T> hipError_t launch_conv_fwd(const ConvArgs<T>& a, int W, bool silu, hipStream_t st)
{
    auto f = [&](auto w, auto v, auto s) { return conv_fwd<T, w.value, v.value, (s.value != 0)>(a, st); };
    return a.D >= kVec<T> ? by_taps<T, kVec<T>>(W, silu, f) : by_taps<T, 1>(W, silu, f);
}
template <typename T> hipError_t launch_conv_bwd(const ConvArgs<T>& a, int W, bool silu, float* dweight, float* dbias, hipStream_t st)
{
    auto f = [&](auto w, auto v, auto s) { return conv_bwd<T, w.value, v.value, (s.value != 0)>(a, dweight, dbias, st); };
    return a.D >= 4 ? by_taps<T, 4>(W, silu, f) : by_taps<T, 1>(W, silu, f);
}
template <typename T> hipError_t launch_conv_step(const T* x, long ld_x, const float* weight, const float* bias, T* state, T* y, int B, int D, int W,
                                                  bool silu, hipStream_t st)
{
    const int blocks_c = (D + 255) / 256;
    const dim3 block(256);
    const int piece = (int)std::min<long>(most_blocks(256) / blocks_c, B);           // sequences of a launch
    for (int done = 0, n; done < B; done += n) {
        n = std::min(piece, B - done);
        const dim3 grid((unsigned)((long)blocks_c * n));
        switch (W) {
            case 2:  hipLaunchKernelGGL((conv_step_kernel<T, 2>), grid, block, 0, st, x, ld_x, weight, bias, state, y, D, blocks_c, silu); break;
            case 3:  hipLaunchKernelGGL((conv_step_kernel<T, 3>), grid, block, 0, st, x, ld_x, weight, bias, state, y, D, blocks_c, silu); break;
            default: hipLaunchKernelGGL((conv_step_kernel<T, 4>), grid, block, 0, st, x, ld_x, weight, bias, state, y, D, blocks_c, silu); break;
        }
        if (const hipError_t e = hipGetLastError()) return e;
        x += n * ld_x;
        state += (long)n * (W - 1) * D;
        y += (long)n * D;
    }
    return hipSuccess;
}

#define KLA_CONV(T)                                                                                                                       \
    template hipError_t launch_conv_fwd<T>(const ConvArgs<T>&, int, bool, hipStream_t);                                             \
    template hipError_t launch_conv_bwd<T>(const ConvArgs<T>&, int, bool, float*, float*, hipStream_t);                             \
    template hipError_t launch_conv_step<T>(const T*, long, const float*, const float*, T*, T*, int, int, int, bool, hipStream_t);
KLA_CONV(float)
KLA_CONV(bf16_t)

}  // namespace kla
