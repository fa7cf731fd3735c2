// Selective state space scan, forward and for single tokens.  Per channel d with states n = 0..S-1:
//   delta_t = softplus(raw_t + bias),  a_t[n] = exp(delta_t A[n]),  h_t[n] = a_t[n] h_{t-1}[n] + delta_t u_t B_t[n],
//   y_t = (sum_n C_t[n] h_t[n] + skip u_t) z_t sigmoid(z_t)
// with B, C shared by the channels of a group.  Everything is fp32 in registers.  Per token, channel and state: an exponential, two
// products, two products with sums; the vector ALU bounds it, the exponential at a quarter of its rate.
#include "kla_ssm_ops.hpp"

namespace kla {

constexpr int kTok = 16;                                 // tokens per tile

// The rows of B and C of a tile in LDS as fp32, filled by all threads of the workgroup one tile ahead.
template <typename T, int S> struct TileBC {
    static constexpr int N = kTok * S / 256 > 0 ? kTok * S / 256 : 1;    // elements per thread, of each
    float b[N], c[N];
    __device__ __forceinline__ void load(const SsmArgs<T>& a, int g, long t, long t1, bool with_c)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int e = threadIdx.x + 256 * i, tok = e / S, n = e % S;
            b[i] = c[i] = 0.f;
            if (tok < kTok && t + tok < t1) {
                b[i] = to_float(a.B[(t + tok) * a.ld_B + g * S + n]);
                if (with_c) c[i] = to_float(a.C[(t + tok) * a.ld_C + g * S + n]);
            }
        }
    }
    __device__ __forceinline__ void store(float* lds_b, float* lds_c) const
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int e = threadIdx.x + 256 * i;
            if (e < kTok * S) { lds_b[e] = b[i]; lds_c[e] = c[i]; }
        }
    }
};

// What a lane takes of a tile: token 4 i + q of its channel.  Nothing is read beyond the segment.
template <typename T> struct TileTok {
    float u[4], raw[4], z[4];
    __device__ __forceinline__ void load(const SsmArgs<T>& a, int c, int q, long t, long t1, bool with_z)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const long at = min(t + 4 * i + q, t1 - 1);
            u[i] = to_float(a.u[at * a.ld_u + c]);
            raw[i] = to_float(a.delta[at * a.ld_delta + c]);
            z[i] = with_z ? to_float(a.z[at * a.ld_z + c]) : 0.f;
        }
    }
};

enum SsmMode { kSsmOutputs, kSsmStates, kSsmMaps };      // y (and checkpoints); checkpoints alone; the maps of the segments

// One workgroup: 64 channels of one segment, tiles of 16 tokens one after the other.
template <typename T, int S, SsmMode MODE>
__global__ __launch_bounds__(256) void ssm_fwd_kernel(SsmArgs<T> a, int blocks_c)
{
    constexpr int K = S / 4, CK = 256 / S;
    __shared__ float lds[2][2][kTok * S];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, q = lane & 3;
    const int block = blockIdx.x % blocks_c;
    const long slot = blockIdx.x / blocks_c;
    Segment g;
    if (!segment_of(a, slot, &g)) return;
    if (MODE == kSsmMaps && g.last) return;              // nothing follows it
    const Channels ch = channels_of(block, a.D, a.G, wave, lane);
    const int c = ch.c;

    float A2[K], h[K];
#pragma unroll
    for (int k = 0; k < K; ++k) A2[k] = kLog2e * a.A[(long)c * S + q * K + k];
    const float skip = a.skip ? a.skip[c] : 0.f, bias = a.delta_bias ? a.delta_bias[c] : 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        h[k] = 0.f;
        if (MODE != kSsmMaps) {
            if (a.seg_state) h[k] = a.seg_state[(slot * a.D + c) * S + q * K + k];
            else if (a.h0) h[k] = a.h0[((long)g.seq.n * a.D + c) * S + q * K + k];
        }
    }
    float sum_delta = 0.f;

    TileBC<T, S> bc;
    TileTok<T> tk;
    if (g.t0 < g.t1) {
        bc.load(a, ch.g, g.t0, g.t1, MODE == kSsmOutputs);
        tk.load(a, c, q, g.t0, g.t1, MODE == kSsmOutputs && a.z);
    }
    int buf = 0;
    for (long t = g.t0; t < g.t1; t += kTok, buf ^= 1) {
        bc.store(lds[buf][0], lds[buf][1]);
        __syncthreads();
        const TileTok<T> now = tk;
        if (t + kTok < g.t1) {
            bc.load(a, ch.g, t + kTok, g.t1, MODE == kSsmOutputs);
            tk.load(a, c, q, t + kTok, g.t1, MODE == kSsmOutputs && a.z);
        }
        const float* lb = lds[buf][0] + q * K;
        const float* lc = lds[buf][1] + q * K;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const long mine = t + 4 * i + q;
            if (MODE != kSsmMaps && (4 * i) % CK == 0 && (CK <= kTok || (t - g.t0) % CK == 0) && a.saved && t + 4 * i < g.t1 && ch.mine) {
                float* at = a.saved + (checkpoint_at(a, g.seq, t + 4 * i, CK) * a.D + c) * S + q * K;
#pragma unroll
                for (int k = 0; k < K; ++k) at[k] = h[k];
            }
            // a token beyond the segment decays nothing and adds nothing
            const bool in = mine < g.t1;
            const float raw = now.raw[i] + bias;
            const float delta = in ? (a.softplus ? softplus(raw) : raw) : 0.f;
            const float du = in ? delta * now.u[i] : 0.f;
            float acc[4];
            static_for<4>([&](auto j) {
                const float dj = quad_bcast<j.value>(delta), uj = quad_bcast<j.value>(du);
                const float* b = lb + (4 * i + j.value) * S;
                const float* cc = lc + (4 * i + j.value) * S;
                float s = 0.f;
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    h[k] = fmaf(exp2_hw(dj * A2[k]), h[k], uj * b[k]);
                    if (MODE == kSsmOutputs) s = fmaf(cc[k], h[k], s);
                }
                acc[j.value] = s;
            });
            if (MODE == kSsmMaps) sum_delta += delta;
            if (MODE == kSsmOutputs) {
                float y = fmaf(skip, now.u[i], quad_sum_own(acc, q));
                if (a.z) y *= now.z[i] * sigmoid(now.z[i]);
                if (in && ch.mine) a.y[mine * a.D + c] = from_float<T>(y);
            }
        }
    }
    if (!ch.mine) return;
    if (MODE == kSsmMaps) {
        sum_delta = quad_sum(sum_delta);
#pragma unroll
        for (int k = 0; k < K; ++k) a.seg_state[(slot * a.D + c) * S + q * K + k] = h[k];
        if (q == 0) a.seg_delta[slot * a.D + c] = sum_delta;
    } else if (a.hT && g.last) {
#pragma unroll
        for (int k = 0; k < K; ++k) a.hT[((long)g.seq.n * a.D + c) * S + q * K + k] = h[k];
    }
}

// The states between segments: seg_state of slot s, the state a segment leaves from zeros, becomes the state it starts from.
template <typename T>
__global__ __launch_bounds__(256) void ssm_join_kernel(SsmArgs<T> a, int S)
{
    const long e = (long)blockIdx.x * 256 + threadIdx.x, DS = (long)a.D * S;
    if (e >= DS) return;
    const Place p = sequence(a.seqs, blockIdx.y);
    const long base = a.seqs.cu ? p.first / a.Lseg + p.n : (long)p.n * max(1, (a.seqs.T + a.Lseg - 1) / a.Lseg);
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
    s = quad_sum(s);
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
    const dim3 grid((unsigned)blocks), block(256);
    if (a.seg_state) {
        hipLaunchKernelGGL((ssm_fwd_kernel<T, S, kSsmMaps>), grid, block, 0, st, a, blocks_c);
        if (const hipError_t e = hipGetLastError()) return e;
        hipLaunchKernelGGL((ssm_join_kernel<T>), dim3((unsigned)(((long)a.D * S + 255) / 256), a.seqs.n_seq), block, 0, st, a, S);
        if (const hipError_t e = hipGetLastError()) return e;
    }
    if (outputs) hipLaunchKernelGGL((ssm_fwd_kernel<T, S, kSsmOutputs>), grid, block, 0, st, a, blocks_c);
    else         hipLaunchKernelGGL((ssm_fwd_kernel<T, S, kSsmStates>), grid, block, 0, st, a, blocks_c);
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
