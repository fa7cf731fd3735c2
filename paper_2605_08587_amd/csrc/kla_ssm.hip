// Selective state space scan, forward and for single tokens.  Per channel d with states n = 0..S-1:
//   delta_t = softplus(raw_t + bias),  a_t[n] = exp(delta_t A[n]),  h_t[n] = a_t[n] h_{t-1}[n] + delta_t u_t B_t[n],
//   y_t = (sum_n C_t[n] h_t[n] + skip u_t) z_t sigmoid(z_t)
// with B, C shared by the channels of a group.  Everything is fp32 in registers.  Per token, channel and state: an exponential, two
// products, two products with sums; the vector ALU bounds it, the exponential at a quarter of its rate.
#include "kla_ssm_ops.hpp"

namespace kla {

constexpr int kTok = 16;                                 // tokens per tile

// What a lane takes of a tile: tokens 8 i + o of its channel, raw until they are used.  Nothing is read beyond the segment.
template <typename T, bool HASZ> struct TileTok {
    T u[2], raw[2], z[2];
    __device__ __forceinline__ void load(const SsmArgs<T>& a, int c, int o, long t, long t1)
    {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const long at = min(t + 8 * i + o, t1 - 1);
            u[i] = a.u[at * a.ld_u + c];
            raw[i] = a.delta[at * a.ld_delta + c];
            if constexpr (HASZ) z[i] = a.z[at * a.ld_z + c];
        }
    }
};

enum SsmMode { kSsmOutputs, kSsmStates, kSsmMaps };      // y (and checkpoints); checkpoints alone; the maps of the segments

// One workgroup: 64 channels of one segment, tiles of 16 tokens one after the other, two tiles on their way.
template <typename T, int S, SsmMode MODE, bool HASZ>
__global__ __launch_bounds__(kSsmThreads) void ssm_fwd_kernel(SsmArgs<T> a, int blocks_c)
{
    constexpr int K = S / 8, CK = ssm_checkpoint(S);
    __shared__ __align__(16) float lds[2][2 * kTok * S];
    const int o = threadIdx.x & 7;
    const int block = blockIdx.x % blocks_c;
    const long slot = blockIdx.x / blocks_c;
    Segment g;
    if (!segment_of(a, slot, &g)) return;
    if (MODE == kSsmMaps && g.last) return;              // nothing follows it
    const Channels ch = channels_of(block, a.D, a.G);
    const int c = ch.c;
    const long mine = ((long)c * S) + o * K;             // this lane's states of [D][S]

    float A2[K], h[K];
    load_states<K>(A2, a.A + mine);
#pragma unroll
    for (int k = 0; k < K; ++k) { A2[k] *= kLog2e; h[k] = 0.f; }
    const float skip = a.skip ? a.skip[c] : 0.f, bias = a.delta_bias ? a.delta_bias[c] : 0.f;
    if (MODE != kSsmMaps) {
        if (a.seg_state) load_states<K>(h, a.seg_state + slot * a.D * S + mine);
        else if (a.h0) load_states<K>(h, a.h0 + (long)g.seq.n * a.D * S + mine);
    }
    float sum_delta = 0.f;

    TileBC<T, S, kTok> bc[2];
    TileTok<T, HASZ> tk[2];
    auto tile = [&](auto which, long t) {
        constexpr int w = which.value;
        bc[w].store(lds[w]);
        const TileTok<T, HASZ> now = tk[w];
        __syncthreads();
        if (t + 2 * kTok < g.t1) {
            bc[w].load(a, ch.g, t + 2 * kTok, g.t1);
            tk[w].load(a, c, o, t + 2 * kTok, g.t1);
        }
        const float* row = lds[w] + o * 2 * K;
        float y[2];
        static_for<2>([&](auto i) {
            if (MODE != kSsmMaps && (8 * i.value) % CK == 0 && a.saved && t + 8 * i.value < g.t1 && ch.mine)
                store_states<K>(a.saved + checkpoint_at(a, g.seq, t + 8 * i.value, CK) * a.D * S + mine, h);
            // a token beyond the segment decays nothing and adds nothing
            const bool in = t + 8 * i.value + o < g.t1;
            const float u = to_float(now.u[i.value]), raw = to_float(now.raw[i.value]) + bias, soft = softplus(raw);
            const float delta = in ? (a.softplus ? soft : raw) : 0.f;
            const Oct ds = oct_of(delta), us = oct_of(in ? delta * u : 0.f);
            float acc[8];
            static_for<8>([&](auto j) {
                const float dj = oct_bcast<j.value>(ds), uj = oct_bcast<j.value>(us);
                const StateBC<K> m = lds_bc<K>(row + (8 * i.value + j.value) * 2 * S);
                float s = 0.f;
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    h[k] = fmaf(exp2_hw(dj * A2[k]), h[k], uj * m.b[k]);
                    if (MODE == kSsmOutputs) s = k ? fmaf(m.c[k], h[k], s) : m.c[k] * h[k];
                }
                acc[j.value] = s;
            });
            if (MODE == kSsmMaps) sum_delta += delta;
            if (MODE == kSsmOutputs) {
                y[i.value] = fmaf(skip, u, oct_sum_own(acc, o));
                if constexpr (HASZ) {
                    const float z = to_float(now.z[i.value]);
                    y[i.value] *= z * sigmoid(z);
                }
            }
        });
        if (MODE == kSsmOutputs && ch.mine) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const long at = t + 8 * i + o;
                if (at < g.t1) a.y[at * a.D + c] = from_float<T>(y[i]);
            }
        }
    };
    if (g.t0 < g.t1) {
        bc[0].load(a, ch.g, g.t0, g.t1);
        tk[0].load(a, c, o, g.t0, g.t1);
        if (g.t0 + kTok < g.t1) {
            bc[1].load(a, ch.g, g.t0 + kTok, g.t1);
            tk[1].load(a, c, o, g.t0 + kTok, g.t1);
        }
    }
    for (long t = g.t0; t < g.t1; t += 2 * kTok) {
        tile(IntC<0>(), t);
        if (t + kTok < g.t1) tile(IntC<1>(), t + kTok);
    }
    if (MODE == kSsmMaps) sum_delta = oct_sum(sum_delta);
    if (!ch.mine) return;
    if (MODE == kSsmMaps) {
        store_states<K>(a.seg_state + slot * a.D * S + mine, h);
        if (o == 0) a.seg_delta[slot * a.D + c] = sum_delta;
    } else if (a.hT && g.last) {
        store_states<K>(a.hT + (long)g.seq.n * a.D * S + mine, h);
    }
}

// The states between segments: seg_state of slot s, the state a segment leaves from zeros, becomes the state it starts from.
template <typename T>
__global__ __launch_bounds__(256) void ssm_join_kernel(SsmArgs<T> a, int S)
{
    const long e = (long)blockIdx.x * 256 + threadIdx.x, DS = (long)a.D * S;
    if (e >= DS) return;
    const Place p = sequence(a.seqs, blockIdx.y);
    const long base = first_slot(a, p);
    const long n = (p.end - p.first + a.Lseg - 1) / a.Lseg;
    const float A2 = kLog2e * a.A[e];
    const int c = (int)(e / S);
    float h = a.h0 ? a.h0[p.n * DS + e] : 0.f;
    for (long k = 0; k + 1 < n; ++k) {                   // (of the last segment there is no map)
        const float own = a.seg_state[(base + k) * DS + e], d = a.seg_delta[(base + k) * a.D + c];
        a.seg_state[(base + k) * DS + e] = h;
        h = fmaf(exp2_hw(A2 * d), h, own);
    }
    a.seg_state[(base + max(n - 1, 0L)) * DS + e] = h;
}

// One token for B sequences: four lanes per channel, the state updated in place.  Bound by the traffic of the states.
template <typename T, int S>
__global__ __launch_bounds__(256) void ssm_step_kernel(SsmArgs<T> a, float* __restrict__ state, int blocks_c)
{
    constexpr int K = S / 4;
    const int q = threadIdx.x & 3, c = (int)(blockIdx.x % blocks_c) * 64 + (threadIdx.x >> 2);
    const long b = blockIdx.x / blocks_c;
    if (c >= a.D) return;                                // whole quads
    const int g = c / (a.D / a.G);
    float* st = state + (b * a.D + c) * S + q * K;
    float h[K];
#pragma unroll
    for (int k = 0; k < K; ++k) h[k] = st[k];
    const float u = to_float(a.u[b * a.ld_u + c]);
    const float raw = to_float(a.delta[b * a.ld_delta + c]) + (a.delta_bias ? a.delta_bias[c] : 0.f);
    const float delta = a.softplus ? softplus(raw) : raw, du = delta * u;
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int n = q * K + k;
        h[k] = fmaf(exp2_hw(delta * (kLog2e * a.A[(long)c * S + n])), h[k], du * to_float(a.B[b * a.ld_B + g * S + n]));
        s = fmaf(to_float(a.C[b * a.ld_C + g * S + n]), h[k], s);
        st[k] = h[k];
    }
    s += quad_xor1(s);
    s += quad_xor2(s);
    if (q == 0) {
        s = fmaf(a.skip ? a.skip[c] : 0.f, u, s);
        if (a.z) { const float z = to_float(a.z[b * a.ld_z + c]); s *= z * sigmoid(z); }
        a.y[b * a.D + c] = from_float<T>(s);
    }
}

template <typename T, int S> static hipError_t ssm_fwd(const SsmArgs<T>& a, bool outputs, hipStream_t st)
{
    const int blocks_c = ssm_channel_blocks(a.D, a.G);
    const long blocks = blocks_c * a.slots;
    if (blocks == 0) return hipSuccess;
    if (blocks > 0x7fffffffL || a.seqs.n_seq > 65535) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)blocks), block(kSsmThreads);
    if (a.seg_state) {
        hipLaunchKernelGGL((ssm_fwd_kernel<T, S, kSsmMaps, false>), grid, block, 0, st, a, blocks_c);
        if (const hipError_t e = hipGetLastError()) return e;
        hipLaunchKernelGGL((ssm_join_kernel<T>), dim3((unsigned)(((long)a.D * S + 255) / 256), a.seqs.n_seq), dim3(256), 0, st, a, S);
        if (const hipError_t e = hipGetLastError()) return e;
    }
    if (!outputs) hipLaunchKernelGGL((ssm_fwd_kernel<T, S, kSsmStates, false>), grid, block, 0, st, a, blocks_c);
    else if (a.z) hipLaunchKernelGGL((ssm_fwd_kernel<T, S, kSsmOutputs, true>), grid, block, 0, st, a, blocks_c);
    else          hipLaunchKernelGGL((ssm_fwd_kernel<T, S, kSsmOutputs, false>), grid, block, 0, st, a, blocks_c);
    return hipGetLastError();
}
template <typename T> hipError_t launch_ssm_fwd(const SsmArgs<T>& a, int S, bool outputs, hipStream_t st)
{
    switch (S) {
        case 8:  return ssm_fwd<T, 8>(a, outputs, st);
        case 16: return ssm_fwd<T, 16>(a, outputs, st);
        case 32: return ssm_fwd<T, 32>(a, outputs, st);
        default: return ssm_fwd<T, 64>(a, outputs, st);
    }
}
template <typename T> hipError_t launch_ssm_step(const SsmArgs<T>& a, float* h, int B, int S, hipStream_t st)
{
    const int blocks_c = (a.D + 63) / 64;
    const long blocks = (long)blocks_c * B;
    if (blocks == 0) return hipSuccess;
    if (blocks > 0x7fffffffL) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)blocks), block(256);
    switch (S) {
        case 8:  hipLaunchKernelGGL((ssm_step_kernel<T, 8>), grid, block, 0, st, a, h, blocks_c); break;
        case 16: hipLaunchKernelGGL((ssm_step_kernel<T, 16>), grid, block, 0, st, a, h, blocks_c); break;
        case 32: hipLaunchKernelGGL((ssm_step_kernel<T, 32>), grid, block, 0, st, a, h, blocks_c); break;
        default: hipLaunchKernelGGL((ssm_step_kernel<T, 64>), grid, block, 0, st, a, h, blocks_c); break;
    }
    return hipGetLastError();
}

#define KLA_SSM(T)                                                                                       \
    template hipError_t launch_ssm_fwd<T>(const SsmArgs<T>&, int, bool, hipStream_t);                    \
    template hipError_t launch_ssm_step<T>(const SsmArgs<T>&, float*, int, int, hipStream_t);
KLA_SSM(float)
KLA_SSM(bf16_t)

}  // namespace kla
