// Backward of the selective scan (kla_ssm.hip).  With c_t = sum_n C_t[n] h_t[n] + skip u_t, y_t = c_t z_t sigmoid(z_t), and
// d_c = d_y z sigmoid(z):
//   g_t[n] = d_c C_t[n] + a_{t+1}[n] g_{t+1}[n]                      gradient of h_t
//   e_t[n] = g_t[n] a_t[n] h_{t-1}[n]                                gradient of the exponent delta_t A[n]
//   d_A[n] = sum_t e_t delta_t,   d_delta = sum_n e A + u sum_n g B,   d_raw = d_delta sigmoid(raw + bias),   d_bias = sum_t d_raw
//   d_u = delta sum_n g B + skip d_c,   d_skip = sum_t d_c u,   d_z = d_y c (z sigmoid(z))'
//   d_B_t[n] = sum over the group's channels of g delta u,   d_C_t[n] = the same of d_c h,   d_h0 = a_1 g_1
// The states come from checkpoints 16 tokens apart (8 from S = 32 on): from each the states and decays of its tokens are formed again and
// stay in registers for the way back.  Sums over channels go through the wave by lane swaps that halve what is left
// at every step, then over the four waves through LDS, then over the workgroups in a kernel of their own: no atomics.
// The vector ALU bounds it: 55 instructions per token and wave of 8 channels x 16 states (26 of them the formulas').  bf16, 2048 channels, 16 states:
// 8 x 2048 tokens 520 us with the ALU busy for 92 %, 4 x 2048 tokens 325 us, one wave per SIMD, 72 %; the sums over the workgroups 23 and 13 us.
#include <algorithm>

#include "kla_ssm_ops.hpp"

namespace kla {

// which of four values row r of the wave holds after two swaps
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

// (Bound to two waves per SIMD in fp32 up to S = 32, where the compiler would take more registers: at S = 16, 8 x 999 tokens x 2048 channels,
// 284 against 330 us.  At S = 64 the bound spills and costs twice the time; in bf16 it only moves code, 5 % the worse.)
// MAPS: what a segment adds to the gradient that enters the one before it, from zeros (with the segment's sum of delta).
template <typename T, int S, bool MAPS, bool HASZ>
__global__ __launch_bounds__(kSsmBwdChannels * 8, S < 64 && sizeof(T) == 4 ? 2 : 1) void ssm_bwd_kernel(SsmArgs<T> a, int blocks_c)
{
    constexpr int K = S / 8, CK = ssm_checkpoint(S), NG = CK / 8;    // tokens per checkpoint and tile, in groups of eight
    constexpr int THREADS = kSsmBwdChannels * 8, WAVES = THREADS / 64;
    __shared__ __align__(16) float lds[2][2 * CK * S];
    __shared__ float red[MAPS ? 1 : WAVES][MAPS ? 1 : CK][2 * S];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, o = lane & 7;
    const int block = blockIdx.x % blocks_c;
    const long slot = a.slot0 + blockIdx.x / blocks_c;
    Segment g;
    if (!segment_of(a, slot, &g)) return;
    if (MAPS && g.t0 == g.seq.first) return;             // nothing stands before it
    const Channels ch = channels_of(block, a.D, a.G, THREADS / 8);
    const int c = ch.c, per_group = blocks_c / a.G;
    const long mine = (long)c * S + o * K, DS = (long)a.D * S;

    float A2[K], dA[K], ag[K];                           // ag: a_{t+1} g_{t+1}
    load_rates<K>(A2, a.A + mine);
#pragma unroll
    for (int k = 0; k < K; ++k) dA[k] = ag[k] = 0.f;
    if (!MAPS) {
        if (a.seg_state) load_states<K>(ag, a.seg_state + slot * DS + mine);
        else if (a.d_hT) load_states<K>(ag, a.d_hT + (long)g.seq.n * DS + mine);
    }
    const float skip = a.skip ? a.skip[c] : 0.f, bias = a.delta_bias ? a.delta_bias[c] : 0.f;
    float d_skip = 0.f, d_bias = 0.f, sum_delta = 0.f;

    const int tokens = (int)(g.t1 - g.t0), tiles = (tokens + CK - 1) / CK;
    const long t_last = g.t0 + (long)(tiles - 1) * CK;   // the last tile comes first
    TileBC<T, S, CK, THREADS> bc;
    Tokens<const T, NG> pu, pd, pz, py;
    Tokens<T, NG> qu, qd, qz;
    bc.init(a, ch.g, t_last);
    pu.init(a.u, t_last, (int)a.ld_u, c, o);
    pd.init(a.delta, t_last, (int)a.ld_delta, c, o);
    if constexpr (HASZ) pz.init(a.z, t_last, (int)a.ld_z, c, o);
    py.init(a.d_y, t_last, a.D, c, o);
    if constexpr (!MAPS) {
        qu.init(a.du, t_last, a.D, c, o);
        qd.init(a.ddelta, t_last, a.D, c, o);
        if constexpr (HASZ) qz.init(a.dz, t_last, a.D, c, o);
    }
    const float* saved = MAPS || tiles == 0 ? nullptr : a.saved + (checkpoint_at(a, g.seq, g.t0, CK) + tiles - 1) * DS;
    float* out_bc = MAPS ? nullptr : a.part_bc + ((long)block * a.M + t_last) * (2 * S);
    T in_bc[decltype(bc)::NE], in_u[NG], in_d[NG], in_z[NG], in_y[NG];
    float in_h[K];
    // the tile at the bases, with `last` the last of its tokens
    auto load = [&](auto full, int last) {
        constexpr bool FULL = full.value != 0;
        bc.template load<FULL>(in_bc, last);
        pu.template load<FULL>(in_u, last, o);
        pd.template load<FULL>(in_d, last, o);
        if constexpr (HASZ) pz.template load<FULL>(in_z, last, o);
        py.template load<FULL>(in_y, last, o);
        if constexpr (!MAPS) load_states<K>(in_h, saved + mine);
    };
    // One tile.  FULL: all of its tokens and of the workgroup's channels are there, so that nothing is masked and the number of stores is
    // known: the wait for the loads before them does not wait for them too.
    auto step = [&](auto full, int tile) {
        constexpr bool FULL = full.value != 0;
        const int w = tile & 1, left = FULL ? CK : min(tokens - tile * CK, CK);
        bc.store(lds[w], in_bc);
        if (!FULL && left < CK) bc.clear(lds[w], left);
        float u[NG], raw[NG], z[NG], dy[NG], delta[NG], dc[NG], core[NG];
        float h[MAPS ? 1 : CK + 1][K];
#pragma unroll
        for (int i = 0; i < NG; ++i) {
            u[i] = to_float(in_u[i]);
            raw[i] = to_float(in_d[i]) + bias;
            dy[i] = to_float(in_y[i]);
            settle(u[i]);
            settle(raw[i]);
            settle(dy[i]);
            if constexpr (HASZ) {
                z[i] = to_float(in_z[i]);
                settle(z[i]);
            }
        }
        if constexpr (!MAPS) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                h[0][k] = in_h[k];
                settle(h[0][k]);
            }
        }
        __syncthreads();
        if (tile > 0) {                                  // the tiles before the last have all their tokens
            if constexpr (!MAPS) saved -= DS;
            bc.move(-CK);
            pu.move(-CK);
            pd.move(-CK);
            if constexpr (HASZ) pz.move(-CK);
            py.move(-CK);
        }
        // (where a tile is full the first one is too, and is asked for a second time when it is reached)
        if (FULL || tile > 0) load(IntC<1>(), 0);
        // a token beyond the segment decays nothing, adds nothing and has no gradient; nor has a lane without a channel of its own
        Oct ds[NG], us[NG], cs[NG];
#pragma unroll
        for (int i = 0; i < NG; ++i) {
            const bool live = FULL || 8 * i + o < left, own = FULL || (live && ch.mine);
            const float soft = softplus<T>(raw[i]);
            delta[i] = where(live, a.softplus ? soft : raw[i]);
            float gate = 1.f;
            if constexpr (HASZ) gate = z[i] * sigmoid(z[i]);
            dc[i] = where(own, dy[i] * gate);
            ds[i] = oct_of(delta[i]);
            us[i] = oct_of(where(own, delta[i] * u[i]));
            cs[i] = oct_of(dc[i]);
            if (MAPS) sum_delta += delta[i];
        }
        const float* row = lds[w] + o * 2 * K;
        if constexpr (MAPS) {
            static_for<CK>([&](auto nn) {
                constexpr int n = CK - 1 - nn.value, i = n / 8, j = n % 8;
                const float dj = oct_bcast<j>(ds[i]), cj = oct_bcast<j>(cs[i]);
                const StateBC<K> m = lds_bc<K>(row + n * 2 * S);
#pragma unroll
                for (int k = 0; k < K; ++k) ag[k] = exp2_hw(dj * A2[k]) * fmaf(cj, m.c[k], ag[k]);
            });
        } else {
            // (at S = 64 the decays would not fit the registers with the states: there they are formed a second time)
            constexpr bool KEEP = K < 8;
            float dec[KEEP ? CK : 1][K];
            static_for<NG>([&](auto i) {
                float acc[8];
                static_for<8>([&](auto j) {
                    constexpr int n = 8 * i.value + j.value;
                    const float dj = oct_bcast<j.value>(ds[i.value]), uj = oct_bcast<j.value>(us[i.value]);
                    const StateBC<K> m = lds_bc<K>(row + n * 2 * S);
                    float s = 0.f;
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        const float d = exp2_hw(dj * A2[k]);
                        if constexpr (KEEP) dec[n][k] = d;
                        h[n + 1][k] = fmaf(d, h[n][k], uj * m.b[k]);
                        if constexpr (HASZ) s = k ? fmaf(m.c[k], h[n + 1][k], s) : m.c[k] * h[n + 1][k];
                    }
                    acc[j.value] = s;
                });
                if constexpr (HASZ) core[i.value] = fmaf(skip, u[i.value], oct_sum_own(acc, o));
            });
            static_for<NG>([&](auto ii) {
                constexpr int i = NG - 1 - ii.value;
                float via_a[8], via_b[8], pair[K < 2 ? 1 : K / 2];
                static_for<8>([&](auto jj) {
                    constexpr int j = 7 - jj.value, n = 8 * i + j;
                    const float dj = oct_bcast<j>(ds[i]), uj = oct_bcast<j>(us[i]), cj = oct_bcast<j>(cs[i]);
                    const StateBC<K> m = lds_bc<K>(row + n * 2 * S);
                    float val[2 * K], sa = 0.f, sb = 0.f;
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        const float gk = fmaf(cj, m.c[k], ag[k]);
                        const float d = KEEP ? dec[KEEP ? n : 0][k] : exp2_hw(dj * A2[k]);
                        ag[k] = d * gk;
                        const float e = ag[k] * h[n][k];
                        val[k] = cj * h[n + 1][k];
                        val[K + k] = uj * gk;
                        sb = fmaf(gk, m.b[k], sb);
                        sa = fmaf(e, A2[k], sa);
                        if (FULL || n < left) dA[k] = fmaf(e, dj, dA[k]);    // (e may be infinite where dj is 0)
                    }
                    via_a[j] = sa;
                    via_b[j] = sb;
                    // Over the wave's 8 channels: two swaps that leave row r of 16 lanes with value 4 v + row_value(r), then over the row's two
                    // octets; token j even stays in the first of them, odd in the second.
#pragma unroll
                    for (int v = 0; v < (K < 2 ? 1 : K / 2); ++v) {
                        float x, y;
                        if constexpr (K == 1) x = y = swap32_sum(val[0], val[1]);
                        else { x = swap32_sum(val[4 * v], val[4 * v + 1]); y = swap32_sum(val[4 * v + 2], val[4 * v + 3]); }
                        float s = swap16_sum(x, y);
                        s += dpp_mov<0x128>(s);          // row_ror:8
                        pair[v] = (j & 1) || (lane & 8) == 0 ? s : pair[v];
                        if constexpr ((j & 1) == 0) {
                            const int tok = n + ((lane >> 3) & 1);
                            if constexpr (K == 1) {
                                red[wave][tok][(lane >> 5) * S + o] = pair[v];       // (both rows of a half hold the same)
                            } else {
                                const int at = 4 * v + row_value(lane >> 4);         // < K: of C, else of B
                                red[wave][tok][(at < K ? 0 : S) + o * K + (at < K ? at : at - K)] = pair[v];
                            }
                        }
                    }
                });
                const float sa = oct_sum_own(via_a, o) * kLn2, sb = oct_sum_own(via_b, o);
                float d_raw = fmaf(u[i], sb, sa);
                d_raw *= a.softplus ? sigmoid(raw[i]) : 1.f;
                const T out_u = rounded<T>(fmaf(delta[i], sb, skip * dc[i])), out_d = rounded<T>(d_raw);
                T out_z = {};
                if constexpr (HASZ) {
                    const float s = sigmoid(z[i]);
                    out_z = rounded<T>(dy[i] * core[i] * (s * fmaf(z[i], 1.f - s, 1.f)));
                }
                if (FULL || (8 * i + o < left && ch.mine)) {
                    d_skip = fmaf(dc[i], u[i], d_skip);
                    d_bias += d_raw;
                    qu.store(i, out_u);
                    qd.store(i, out_d);
                    if constexpr (HASZ) qz.store(i, out_z);
                }
            });
            __syncthreads();
            // the waves' channels together: [token][2 S], C first
#pragma unroll
            for (int i = 0; i < (CK * 2 * S + THREADS - 1) / THREADS; ++i) {
                const int e = threadIdx.x + i * THREADS;
                const float* r = &red[0][0][0] + min(e, CK * 2 * S - 1);
                float s = 0.f;
#pragma unroll
                for (int v = 0; v < WAVES; ++v) s += r[v * CK * 2 * S];
                if (FULL && CK * 2 * S % THREADS == 0) out_bc[e] = s;
                else if (e < left * 2 * S) out_bc[e] = s;
            }
            out_bc -= CK * 2 * S;
            qu.move(-CK);
            qd.move(-CK);
            if constexpr (HASZ) qz.move(-CK);
            // (red is written again behind the next tile's barrier)
        }
    };
    if (tiles > 0) {
        const bool whole = (block % per_group + 1) * (THREADS / 8) <= a.D / a.G;     // the workgroup's channels
        load(IntC<0>(), tokens - 1 - (tiles - 1) * CK);
        int tile = tiles - 1;
        for (; tile >= 0 && !(whole && (tile + 1) * CK <= tokens); --tile) step(IntC<0>(), tile);
        for (; tile >= 0; --tile) step(IntC<1>(), tile);
    }
    sum_delta = oct_sum(sum_delta);
    d_skip = oct_sum(d_skip);
    d_bias = oct_sum(d_bias);
    if (!ch.mine) return;
    if constexpr (MAPS) {
        store_states<K>(a.seg_state + slot * DS + mine, ag);
        if (o == 0) a.seg_delta[slot * a.D + c] = sum_delta;
    } else {
        if (a.dh0 && g.t0 == g.seq.first) store_states<K>(a.dh0 + (long)g.seq.n * DS + mine, ag);
        float* p = a.part_p + slot * ((long)a.D * (S + 2));
        store_states<K>(p + mine, dA);
        if (o == 0) {
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
    const long base = first_slot(a, p);
    const long n = (p.end - p.first + a.Lseg - 1) / a.Lseg;
    const float A2 = rate(a.A[e]);
    const int c = (int)(e / S);
    float g = a.d_hT ? a.d_hT[p.n * DS + e] : 0.f;
    constexpr int AHEAD = 8;                             // reads of so many segments at once
    for (long k0 = n - 1; k0 > 0; k0 -= AHEAD) {
        float own[AHEAD], d[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const long k = max(k0 - i, 1L);
            own[i] = a.seg_state[(base + k) * DS + e];
            d[i] = a.seg_delta[(base + k) * a.D + c];
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (k0 - i > 0) {
                a.seg_state[(base + k0 - i) * DS + e] = g;
                g = fmaf(exp2_hw(A2 * d[i]), g, own[i]);
            }
        }
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

// Gradients of B and C: the sums over the workgroups of a group's channels.  A stream: 134 MB in 23 us, 5.8 TB/s.
template <typename T, int S>
__global__ __launch_bounds__(256) void ssm_sum_bc_kernel(const float* __restrict__ part, T* __restrict__ dB, T* __restrict__ dC, long M, int G, int blocks,
                                                         long first)
{
    const long e = first + (long)blockIdx.x * 256 + threadIdx.x;     // (token, 2 S)
    const int g = blockIdx.y;
    if (e >= M * 2 * S) return;
    float s = 0.f;
#pragma unroll 4
    for (int b = 0; b < blocks; ++b) s += part[((long)g * blocks + b) * M * 2 * S + e];
    const long tok = e / (2 * S);
    const int n = (int)(e % (2 * S));
    if (n < S) dC[(tok * G + g) * S + n] = rounded<T>(s);
    else       dB[(tok * G + g) * S + n - S] = rounded<T>(s);
}

template <typename T, int S, bool MAPS, bool HASZ> static hipError_t ssm_bwd_pass(SsmArgs<T> a, int blocks_c, hipStream_t st)
{
    constexpr int THREADS = kSsmBwdChannels * 8;
    for (long n; a.slot0 < a.slots; a.slot0 += n) {
        n = std::min(a.slots - a.slot0, most_blocks(THREADS) / blocks_c);
        hipLaunchKernelGGL((ssm_bwd_kernel<T, S, MAPS, HASZ>), dim3((unsigned)(blocks_c * n)), dim3(THREADS), 0, st, a, blocks_c);
        if (const hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}
template <typename T, int S> static hipError_t ssm_bwd(const SsmArgs<T>& a, float* dA, T* dB, T* dC, float* dskip, float* ddelta_bias, hipStream_t st)
{
    const int blocks_c = ssm_channel_blocks(a.D, a.G, kSsmBwdChannels);
    const long row = (long)a.D * (S + 2);
    if (a.slots > 0) {
        if (a.seg_state) {
            if (const hipError_t e = a.z ? ssm_bwd_pass<T, S, true, true>(a, blocks_c, st) : ssm_bwd_pass<T, S, true, false>(a, blocks_c, st)) return e;
            hipLaunchKernelGGL((ssm_join_bwd_kernel<T>), dim3((unsigned)(((long)a.D * S + 255) / 256), a.seqs.n_seq), dim3(256), 0, st, a, S);
            if (const hipError_t e = hipGetLastError()) return e;
        }
        if (a.seqs.cu) {
            hipLaunchKernelGGL((ssm_clear_kernel<T>), dim3((unsigned)a.slots), dim3(256), 0, st, a, row);
            if (const hipError_t e = hipGetLastError()) return e;
        }
        if (const hipError_t e = a.z ? ssm_bwd_pass<T, S, false, true>(a, blocks_c, st) : ssm_bwd_pass<T, S, false, false>(a, blocks_c, st)) return e;
    }
    for (long first = 0; first < a.M * 2 * S; first += most_blocks(256) * 256) {
        const long blocks = std::min((a.M * 2 * S - first + 255) / 256, most_blocks(256));
        hipLaunchKernelGGL((ssm_sum_bc_kernel<T, S>), dim3((unsigned)blocks, a.G), dim3(256), 0, st, a.part_bc, dB, dC, a.M, a.G, blocks_c / a.G, first);
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
