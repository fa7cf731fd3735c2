// Backward of the selective scan (kla_ssm.hip).  With c_t = sum_n C_t[n] h_t[n] + skip u_t, y_t = c_t z_t sigmoid(z_t), and
// d_c = d_y z sigmoid(z):
//   g_t[n] = d_c C_t[n] + a_{t+1}[n] g_{t+1}[n]                      gradient of h_t
//   e_t[n] = g_t[n] a_t[n] h_{t-1}[n]                                gradient of the exponent delta_t A[n]
//   d_A[n] = sum_t e_t delta_t,   d_delta = sum_n e A + u sum_n g B,   d_raw = d_delta sigmoid(raw + bias),   d_bias = sum_t d_raw
//   d_u = delta sum_n g B + skip d_c,   d_skip = sum_t d_c u,   d_z = d_y c (z sigmoid(z))'
//   d_B_t[n] = sum over the group's channels of g delta u,   d_C_t[n] = the same of d_c h,   d_h0 = a_1 g_1
// The states come from checkpoints 256/S tokens apart: from each the states and decays of its tokens are formed again and stay in
// registers (64 of each per lane) for the way back.  Sums over channels go through the wave by lane swaps that halve what is left
// at every step, then over the four waves through LDS, then over the workgroups in a kernel of their own: no atomics.
#include "kla_ssm_ops.hpp"

namespace kla {

// rows r = 0..3 of a wave hold, after two swaps, value 4 j + kRowValue[r] of sixteen
__device__ __forceinline__ int row_value(int r) { return ((r & 1) << 1) | (r >> 1); }

__device__ __forceinline__ float swap32_sum(float x, float y)
{
    // lanes 0-31: x of both halves; lanes 32-63: y of both halves
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(y), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float swap16_sum(float x, float y)
{
    // even rows of sixteen lanes: x of both rows; odd rows: y of both rows
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(y), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// MAPS: what a segment adds to the gradient that enters the one before it, from zeros (with the segment's sum of delta).
template <typename T, int S, bool MAPS>
__global__ __launch_bounds__(256) void ssm_bwd_kernel(SsmArgs<T> a, int blocks_c)
{
    constexpr int K = S / 4, CK = 256 / S, NQ = CK / 4;  // tokens per checkpoint, in groups of four
    constexpr int NE = CK * S / 256;                     // elements of a tile of B per thread
    static_assert(NE == 1, "a tile of B or C has one element per thread");
    __shared__ float lds[2][2][CK * S];
    __shared__ float red[MAPS ? 1 : 4][MAPS ? 1 : CK][2 * S];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, q = lane & 3;
    const int block = blockIdx.x % blocks_c;
    const long slot = blockIdx.x / blocks_c;
    Segment g;
    if (!segment_of(a, slot, &g)) return;
    if (MAPS && g.t0 == g.seq.first) return;             // nothing stands before it
    const Channels ch = channels_of(block, a.D, a.G, wave, lane);
    const int c = ch.c;

    float A2[K], dA[K], ag[K];                           // ag: a_{t+1} g_{t+1}
#pragma unroll
    for (int k = 0; k < K; ++k) {
        A2[k] = kLog2e * a.A[(long)c * S + q * K + k];
        dA[k] = ag[k] = 0.f;
        if (!MAPS) {
            if (a.seg_state) ag[k] = a.seg_state[(slot * a.D + c) * S + q * K + k];
            else if (a.d_hT) ag[k] = a.d_hT[((long)g.seq.n * a.D + c) * S + q * K + k];
        }
    }
    const float skip = a.skip ? a.skip[c] : 0.f, bias = a.delta_bias ? a.delta_bias[c] : 0.f;
    float d_skip = 0.f, d_bias = 0.f, sum_delta = 0.f;

    // this thread's element of the tile of B, C, and this lane's tokens 4 i + q
    float in_b, in_c, in_u[NQ], in_raw[NQ], in_z[NQ], in_dy[NQ];
    const int e_tok = threadIdx.x / S, e_n = threadIdx.x % S;
    auto load = [&](long t) {
        const bool in = t + e_tok < g.t1;
        in_b = in ? to_float(a.B[(t + e_tok) * a.ld_B + ch.g * S + e_n]) : 0.f;
        in_c = in ? to_float(a.C[(t + e_tok) * a.ld_C + ch.g * S + e_n]) : 0.f;
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            const long at = min(t + 4 * i + q, g.t1 - 1);
            in_u[i] = to_float(a.u[at * a.ld_u + c]);
            in_raw[i] = to_float(a.delta[at * a.ld_delta + c]);
            in_z[i] = a.z ? to_float(a.z[at * a.ld_z + c]) : 0.f;
            in_dy[i] = to_float(a.d_y[at * a.D + c]);
        }
    };
    const long tiles = (g.t1 - g.t0 + CK - 1) / CK;
    if (tiles > 0) load(g.t0 + (tiles - 1) * CK);
    int buf = 0;
    for (long tile = tiles - 1; tile >= 0; --tile, buf ^= 1) {
        const long t = g.t0 + tile * CK;
        lds[buf][0][threadIdx.x] = in_b;
        lds[buf][1][threadIdx.x] = in_c;
        float u[NQ], raw[NQ], z[NQ], dy[NQ], delta[NQ], du[NQ], dc[NQ], core[NQ];
#pragma unroll
        for (int i = 0; i < NQ; ++i) { u[i] = in_u[i]; raw[i] = in_raw[i] + bias; z[i] = in_z[i]; dy[i] = in_dy[i]; }
        __syncthreads();
        if (tile > 0) load(t - CK);
        // a token beyond the segment decays nothing, adds nothing and has no gradient; nor has a lane without a channel of its own
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            const bool in = t + 4 * i + q < g.t1;
            delta[i] = in ? (a.softplus ? softplus(raw[i]) : raw[i]) : 0.f;
            du[i] = in && ch.mine ? delta[i] * u[i] : 0.f;
            dc[i] = in && ch.mine ? (a.z ? dy[i] * (z[i] * sigmoid(z[i])) : dy[i]) : 0.f;
            if (MAPS) sum_delta += delta[i];
        }
        const float* lb = lds[buf][0] + q * K;
        const float* lc = lds[buf][1] + q * K;
        if constexpr (MAPS) {
            static_for<NQ>([&](auto ii) {
                constexpr int i = NQ - 1 - ii.value;
                static_for<4>([&](auto jj) {
                    constexpr int j = 3 - jj.value;
                    const float dj = quad_bcast<j>(delta[i]), cj = quad_bcast<j>(dc[i]);
#pragma unroll
                    for (int k = 0; k < K; ++k) ag[k] = exp2_hw(dj * A2[k]) * fmaf(cj, lc[(4 * i + j) * S + k], ag[k]);
                });
            });
        } else {
            float h[CK + 1][K], dec[CK][K];
            const float* from = a.saved + (checkpoint_at(a, g.seq, t, CK) * a.D + c) * S + q * K;
#pragma unroll
            for (int k = 0; k < K; ++k) h[0][k] = from[k];
            static_for<NQ>([&](auto i) {
                float acc[4];
                static_for<4>([&](auto j) {
                    constexpr int n = 4 * i.value + j.value;
                    const float dj = quad_bcast<j.value>(delta[i.value]), uj = quad_bcast<j.value>(du[i.value]);
                    float s = 0.f;
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        dec[n][k] = exp2_hw(dj * A2[k]);
                        h[n + 1][k] = fmaf(dec[n][k], h[n][k], uj * lb[n * S + k]);
                        s = fmaf(lc[n * S + k], h[n + 1][k], s);
                    }
                    acc[j.value] = s;
                });
                if (a.z) core[i.value] = fmaf(skip, u[i.value], quad_sum_own(acc, q));
            });
            static_for<NQ>([&](auto ii) {
                constexpr int i = NQ - 1 - ii.value;
                float via_a[4], via_b[4], own[K / 2];
                static_for<4>([&](auto jj) {
                    constexpr int j = 3 - jj.value, n = 4 * i + j;
                    const float dj = quad_bcast<j>(delta[i]), uj = quad_bcast<j>(du[i]), cj = quad_bcast<j>(dc[i]);
                    float val[2 * K], sa = 0.f, sb = 0.f;
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        const float gk = fmaf(cj, lc[n * S + k], ag[k]);
                        const float e = gk * (dec[n][k] * h[n][k]);
                        val[k] = cj * h[n + 1][k];
                        val[K + k] = uj * gk;
                        sb = fmaf(gk, lb[n * S + k], sb);
                        sa = fmaf(e, A2[k], sa);
                        dA[k] = fmaf(e, dj, dA[k]);
                        ag[k] = dec[n][k] * gk;
                    }
                    via_a[j] = sa;
                    via_b[j] = sb;
                    // over the wave's 16 channels: lanes 4 c + q of a row keep the sums over all c, the lanes of c % 4 = j those of token j
#pragma unroll
                    for (int v = 0; v < K / 2; ++v) {
                        const float x = swap32_sum(val[4 * v], val[4 * v + 1]), y = swap32_sum(val[4 * v + 2], val[4 * v + 3]);
                        float s = swap16_sum(x, y);
                        s += dpp_mov<0x128>(s);          // row_ror:8
                        s += dpp_mov<0x124>(s);          // row_ror:4
                        own[v] = ((lane >> 2) & 3) == j ? s : (jj.value == 0 ? 0.f : own[v]);
                    }
                });
#pragma unroll
                for (int v = 0; v < K / 2; ++v) {
                    const int val = 4 * v + row_value(lane >> 4), kk = val < K ? val : val - K;     // < K: of C, else of B
                    red[wave][4 * i + ((lane >> 2) & 3)][(val < K ? 0 : S) + q * K + kk] = own[v];
                }
                const float sa = quad_sum_own(via_a, q) * kLn2, sb = quad_sum_own(via_b, q);
                const bool in = t + 4 * i + q < g.t1;
                float d_raw = fmaf(u[i], sb, sa);
                if (a.softplus) d_raw *= sigmoid(raw[i]);
                if (in) {
                    d_bias += d_raw;
                    d_skip = fmaf(dc[i], u[i], d_skip);
                    if (ch.mine) {
                        const long at = (t + 4 * i + q) * a.D + c;
                        a.du[at] = from_float<T>(fmaf(delta[i], sb, skip * dc[i]));
                        a.ddelta[at] = from_float<T>(d_raw);
                        if (a.z) {
                            const float s = sigmoid(z[i]);
                            a.dz[at] = from_float<T>(dy[i] * core[i] * (s * fmaf(z[i], 1.f - s, 1.f)));
                        }
                    }
                }
            });
            __syncthreads();
            // the four waves' channels together: [token][2 S], C first
            float* out = a.part_bc + ((long)block * a.M + t) * (2 * S);
            const int n_out = (int)min((long)CK, g.t1 - t) * 2 * S;
            for (int e = threadIdx.x; e < n_out; e += 256) {
                const float* r = &red[0][0][0] + e;
                out[e] = (r[0] + r[CK * 2 * S]) + (r[2 * CK * 2 * S] + r[3 * CK * 2 * S]);
            }
            // (red is written again behind the next tile's barrier)
        }
    }
    if (!ch.mine) return;
    if constexpr (MAPS) {
        sum_delta = quad_sum(sum_delta);
#pragma unroll
        for (int k = 0; k < K; ++k) a.seg_state[(slot * a.D + c) * S + q * K + k] = ag[k];
        if (q == 0) a.seg_delta[slot * a.D + c] = sum_delta;
    } else {
        if (a.dh0 && g.t0 == g.seq.first) {
#pragma unroll
            for (int k = 0; k < K; ++k) a.dh0[((long)g.seq.n * a.D + c) * S + q * K + k] = ag[k];
        }
        float* p = a.part_p + slot * ((long)a.D * (S + 2));
#pragma unroll
        for (int k = 0; k < K; ++k) p[(long)c * S + q * K + k] = dA[k];
        d_skip = quad_sum(d_skip);
        d_bias = quad_sum(d_bias);
        if (q == 0) {
            p[(long)a.D * S + c] = d_skip;
            p[(long)a.D * (S + 1) + c] = d_bias;
        }
    }
}

// The gradients that enter the segments from behind: seg_state of slot s, what the segment adds from zeros, becomes what enters it.
template <typename T>
__global__ __launch_bounds__(256) void ssm_join_bwd_kernel(SsmArgs<T> a, int S)
{
    const long e = (long)blockIdx.x * 256 + threadIdx.x, DS = (long)a.D * S;
    if (e >= DS) return;
    const Place p = sequence(a.seqs, blockIdx.y);
    const long base = a.seqs.cu ? p.first / a.Lseg + p.n : (long)p.n * max(1, (a.seqs.T + a.Lseg - 1) / a.Lseg);
    const long n = (p.end - p.first + a.Lseg - 1) / a.Lseg;
    const float A2 = kLog2e * a.A[e];
    const int c = (int)(e / S);
    float g = a.d_hT ? a.d_hT[p.n * DS + e] : 0.f;
    for (long k = n - 1; k > 0; --k) {
        const float own = a.seg_state[(base + k) * DS + e], d = a.seg_delta[(base + k) * a.D + c];
        a.seg_state[(base + k) * DS + e] = g;
        g = fmaf(exp2_hw(A2 * d), g, own);
    }
    a.seg_state[base * DS + e] = g;
}

// Slots without a segment leave their rows of part_p as they are: zeros, for the sums.
template <typename T>
__global__ __launch_bounds__(256) void ssm_clear_kernel(SsmArgs<T> a, long row)
{
    Segment g;
    if (segment_of(a, blockIdx.x, &g)) return;
    for (long e = threadIdx.x; e < row; e += 256) a.part_p[blockIdx.x * row + e] = 0.f;
}

// Gradients of B and C: the sums over the workgroups of a group's channels.
template <typename T, int S>
__global__ __launch_bounds__(256) void ssm_sum_bc_kernel(const float* __restrict__ part, T* __restrict__ dB, T* __restrict__ dC, long M, int G, int blocks)
{
    const long e = (long)blockIdx.x * 256 + threadIdx.x;     // (token, 2 S)
    const int g = blockIdx.y;
    if (e >= M * 2 * S) return;
    float s = 0.f;
#pragma unroll 4
    for (int b = 0; b < blocks; ++b) s += part[((long)g * blocks + b) * M * 2 * S + e];
    const long tok = e / (2 * S);
    const int n = (int)(e % (2 * S));
    if (n < S) dC[(tok * G + g) * S + n] = from_float<T>(s);
    else       dB[(tok * G + g) * S + n - S] = from_float<T>(s);
}

template <typename T, int S> static hipError_t ssm_bwd(const SsmArgs<T>& a, float* dA, T* dB, T* dC, float* dskip, float* ddelta_bias, hipStream_t st)
{
    const int blocks_c = ssm_channel_blocks(a.D, a.G);
    const long blocks = blocks_c * a.slots, row = (long)a.D * (S + 2);
    if (blocks > 0x7fffffffL || a.seqs.n_seq > 65535 || a.G > 65535 || (a.M * 2 * S + 255) / 256 > 0x7fffffffL) return hipErrorInvalidConfiguration;
    if (blocks > 0) {
        const dim3 grid((unsigned)blocks), block(256);
        if (a.seg_state) {
            hipLaunchKernelGGL((ssm_bwd_kernel<T, S, true>), grid, block, 0, st, a, blocks_c);
            if (const hipError_t e = hipGetLastError()) return e;
            hipLaunchKernelGGL((ssm_join_bwd_kernel<T>), dim3((unsigned)(((long)a.D * S + 255) / 256), a.seqs.n_seq), block, 0, st, a, S);
            if (const hipError_t e = hipGetLastError()) return e;
        }
        if (a.seqs.cu) {
            hipLaunchKernelGGL((ssm_clear_kernel<T>), dim3((unsigned)a.slots), block, 0, st, a, row);
            if (const hipError_t e = hipGetLastError()) return e;
        }
        hipLaunchKernelGGL((ssm_bwd_kernel<T, S, false>), grid, block, 0, st, a, blocks_c);
        if (const hipError_t e = hipGetLastError()) return e;
    }
    if (a.M > 0) {
        hipLaunchKernelGGL((ssm_sum_bc_kernel<T, S>), dim3((unsigned)((a.M * 2 * S + 255) / 256), a.G), dim3(256), 0, st, a.part_bc, dB, dC, a.M, a.G,
                           blocks_c / a.G);
        if (const hipError_t e = hipGetLastError()) return e;
    }
    return launch_column_sums(a.part_p, a.slots, {{(long)a.D * S, a.D, a.D}, {dA, dskip, ddelta_bias}}, st);
}
template <typename T> hipError_t launch_ssm_bwd(const SsmArgs<T>& a, int S, float* dA, T* dB, T* dC, float* dskip, float* ddelta_bias, hipStream_t st)
{
    switch (S) {
        case 8:  return ssm_bwd<T, 8>(a, dA, dB, dC, dskip, ddelta_bias, st);
        case 16: return ssm_bwd<T, 16>(a, dA, dB, dC, dskip, ddelta_bias, st);
        case 32: return ssm_bwd<T, 32>(a, dA, dB, dC, dskip, ddelta_bias, st);
        default: return ssm_bwd<T, 64>(a, dA, dB, dC, dskip, ddelta_bias, st);
    }
}
template hipError_t launch_ssm_bwd<float>(const SsmArgs<float>&, int, float*, float*, float*, float*, float*, hipStream_t);
template hipError_t launch_ssm_bwd<bf16_t>(const SsmArgs<bf16_t>&, int, float*, bf16_t*, bf16_t*, float*, float*, hipStream_t);

}  // namespace kla
