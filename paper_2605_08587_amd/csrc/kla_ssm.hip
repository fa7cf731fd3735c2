// Selective state space scan, forward and for single tokens.  Per channel d with states n = 0..S-1:
//   delta_t = softplus(raw_t + bias),  a_t[n] = exp(delta_t A[n]),  h_t[n] = a_t[n] h_{t-1}[n] + delta_t u_t B_t[n],
//   y_t = (sum_n C_t[n] h_t[n] + skip u_t) z_t sigmoid(z_t)
// with B, C shared by the channels of a group.  Everything is fp32 in registers.  Per token, channel and state: an exponential, two
// products, two products with sums, that is six slots of the vector ALU (the exponential takes two), which bounds it and not memory.  Eight
// lanes per channel and not one: the scalars of a token (steps, gates) are formed once per channel, and a channel's chain is its own wave's;
// sixteen lanes have twice the scalar work per state (one sequence of 65536 tokens x 1024 channels x 16 states 773 us against 576, both of one early
// form; 548 now).  That sequence: maps and outputs take 13 and 18 vector instructions per token and wave (8 channels) and keep the ALU busy for 96 and
// 93 %.  4 x 2048 tokens x 2048 channels, training: 146 us, one wave per SIMD (71 ns a token), the ALU busy for 56 %; 8 x 2048: 220 us, 76 %.
#include <algorithm>

#include "kla_ssm_ops.hpp"

namespace kla {

constexpr int kTok = 16;                                 // tokens per tile (32: 7 to 20 % slower, the code then exceeds what the instruction cache keeps)

enum SsmMode { kSsmOutputs, kSsmStates, kSsmMaps };      // y (and checkpoints); checkpoints alone; the maps of the segments

// One workgroup: THREADS / 8 channels of one segment, tiles of 16 tokens one after the other, two tiles on their way.  (The bound of two waves per
// SIMD: the compiler would give the maps at S = 64 more registers than two waves have; 16384 tokens x 1024 channels 221 against 260 us.)
template <typename T, int S, SsmMode MODE, bool HASZ, int THREADS>
__global__ __launch_bounds__(THREADS, MODE == kSsmMaps && S == 64 ? 2 : 1) void ssm_fwd_kernel(SsmArgs<T> a, int blocks_c)
{
    constexpr int K = S / 8, CK = ssm_checkpoint(S), NG = kTok / 8;
    __shared__ __align__(16) float lds[2][2 * kTok * S];
    const int o = threadIdx.x & 7;
    const int block = blockIdx.x % blocks_c;
    const long slot = a.slot0 + blockIdx.x / blocks_c;
    Segment g;
    if (!segment_of(a, slot, &g)) return;
    if (MODE == kSsmMaps && g.last) return;              // nothing follows it
    const Channels ch = channels_of(block, a.D, a.G, THREADS / 8);
    const int c = ch.c;
    const long mine = ((long)c * S) + o * K, DS = (long)a.D * S;         // this lane's states of [D][S]

    float A2[K], h[K];
    load_rates<K>(A2, a.A + mine);
#pragma unroll
    for (int k = 0; k < K; ++k) h[k] = 0.f;
    const float skip = a.skip ? a.skip[c] : 0.f, bias = a.delta_bias ? a.delta_bias[c] : 0.f;
    if (MODE != kSsmMaps) {
        if (a.seg_state) load_states<K>(h, a.seg_state + slot * DS + mine);
        else if (a.h0) load_states<K>(h, a.h0 + (long)g.seq.n * DS + mine);
    }
    float sum_delta = 0.f;
    const bool saves = MODE != kSsmMaps && a.saved;
    float* saved = saves ? a.saved + checkpoint_at(a, g.seq, g.t0, CK) * DS : nullptr;

    TileBC<T, S, kTok, THREADS> bc;
    Tokens<const T, NG> pu, pd, pz;
    Tokens<T, NG> py;
    T in_bc[2][decltype(bc)::NE], in_u[2][NG], in_d[2][NG], in_z[2][NG];
    bc.init(a, ch.g, g.t0);
    pu.init(a.u, g.t0, (int)a.ld_u, c, o);
    pd.init(a.delta, g.t0, (int)a.ld_delta, c, o);
    if constexpr (HASZ) pz.init(a.z, g.t0, (int)a.ld_z, c, o);
    py.init(a.y, g.t0, a.D, c, o);
    const int tokens = (int)(g.t1 - g.t0);
    // The next tile of the segment, and the bases on to the one behind it.  The last tile is asked for again where there is none behind it
    // (the bases stay: an offset from them may not be negative): the number of loads on their way is then known, and a wait for the older
    // ones does not wait for the newer.
    int next = 0;                                        // the token at which that tile begins, <= tokens - 1
    auto load = [&](auto which) {
        constexpr int w = which.value;
        auto rows = [&](auto full) {
            constexpr bool FULL = full.value != 0;
            const int last = tokens - 1 - next;
            bc.template load<FULL>(in_bc[w], last);
            pu.template load<FULL>(in_u[w], last, o);
            pd.template load<FULL>(in_d[w], last, o);
            if constexpr (HASZ) pz.template load<FULL>(in_z[w], last, o);
        };
        if (next + kTok <= tokens) rows(IntC<1>());
        else rows(IntC<0>());
        if (next + kTok < tokens) {
            next += kTok;
            bc.move(kTok);
            pu.move(kTok);
            pd.move(kTok);
            if constexpr (HASZ) pz.move(kTok);
        }
    };
    auto tile = [&](auto which, int at) {
        constexpr int w = which.value;
        const int left = tokens - at;
        bc.store(lds[w], in_bc[w]);
        if (MODE != kSsmMaps && left < kTok) bc.clear(lds[w], left);     // (a segment that another follows has whole tiles)
        float u[NG], raw[NG], z[NG], y[NG];
#pragma unroll
        for (int i = 0; i < NG; ++i) {
            u[i] = to_float(in_u[w][i]);
            raw[i] = to_float(in_d[w][i]) + bias;
            settle(u[i]);
            settle(raw[i]);
            if constexpr (HASZ) {
                z[i] = to_float(in_z[w][i]);
                settle(z[i]);
            }
        }
        __syncthreads();
        load(which);
        const float* row = lds[w] + o * 2 * K;
        // In steps, in this order: what eight tokens need from LDS is on its way while steps, gates and decays are formed, and the chain of
        // states finds everything at hand.  (Left to itself the compiler reads each row where it is used and waits.)
        constexpr int AHEAD = K <= 4 ? 8 : 4;
        StateBC<K> m[AHEAD];
        static_for<AHEAD>([&](auto j) { m[j.value] = lds_bc<K>(row + j.value * 2 * S); });
        __builtin_amdgcn_sched_barrier(0);
        // a token beyond the segment decays nothing and adds nothing
        float delta[NG], du[NG], gate[NG];
#pragma unroll
        for (int i = 0; i < NG; ++i) {
            const bool in = 8 * i + o < left;
            const float soft = softplus<T>(raw[i]);
            delta[i] = where(in, a.softplus ? soft : raw[i]);
            du[i] = where(in, delta[i] * u[i]);
            if constexpr (HASZ) gate[i] = z[i] * sigmoid(z[i]);
            if (MODE == kSsmMaps) sum_delta += delta[i];
        }
        static_for<NG>([&](auto i) {
            if (saves && (8 * i.value) % CK == 0) {
                if (8 * i.value < left && ch.mine) store_states<K>(saved + mine, h);
                saved += DS;
            }
            const Oct ds = oct_of(delta[i.value]), us = oct_of(du[i.value]);
            float acc[8];
            static_for<8 / AHEAD>([&](auto part) {
                constexpr int j0 = part.value * AHEAD;
                float dec[AHEAD][K];
                static_for<AHEAD>([&](auto j) {
                    const float dj = oct_bcast<j0 + j.value>(ds);
#pragma unroll
                    for (int k = 0; k < K; ++k) dec[j.value][k] = exp2_hw(dj * A2[k]);
                });
                __builtin_amdgcn_sched_barrier(0);
                static_for<AHEAD>([&](auto j) {
                    const float uj = oct_bcast<j0 + j.value>(us);
                    float s = 0.f;
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        h[k] = fmaf(dec[j.value][k], h[k], uj * m[j.value].b[k]);
                        if (MODE == kSsmOutputs) s = k ? fmaf(m[j.value].c[k], h[k], s) : m[j.value].c[k] * h[k];
                    }
                    acc[j0 + j.value] = s;
                    // the row in its place for the tokens that follow
                    constexpr int n = 8 * i.value + j0 + j.value + AHEAD;
                    if constexpr (n < kTok) m[j.value] = lds_bc<K>(row + n * 2 * S);
                });
            });
            if (MODE == kSsmOutputs) {
                y[i.value] = fmaf(skip, u[i.value], oct_sum_own(acc, o));
                if constexpr (HASZ) y[i.value] *= gate[i.value];
            }
        });
        if (MODE == kSsmOutputs) {
#pragma unroll
            for (int i = 0; i < NG; ++i) {
                const T out = rounded<T>(y[i]);
                if (8 * i + o < left && ch.mine) py.store(i, out);
            }
            py.move(kTok);
        }
    };
    if (tokens > 0) {
        load(IntC<0>());
        load(IntC<1>());
        int at = 0;
        for (; at + kTok < tokens; at += 2 * kTok) {     // (no way out between the two: the compiler would count its loads as the last)
            tile(IntC<0>(), at);
            tile(IntC<1>(), at + kTok);
        }
        if (at < tokens) tile(IntC<0>(), at);
    }
    if (MODE == kSsmMaps) sum_delta = oct_sum(sum_delta);
    if (!ch.mine) return;
    if (MODE == kSsmMaps) {
        store_states<K>(a.seg_state + slot * DS + mine, h);
        if (o == 0) a.seg_delta[slot * a.D + c] = sum_delta;
    } else if (a.hT && g.last) {
        store_states<K>(a.hT + (long)g.seq.n * DS + mine, h);
    }
}

// A thread per channel and state, over the segments one after the other with eight of them read at once: 5 us for 16, 7 us for 32.
// The states between segments: seg_state of slot s, the state a segment leaves from zeros, becomes the state it starts from.
template <typename T>
__global__ __launch_bounds__(256) void ssm_join_kernel(SsmArgs<T> a, int S)
{
    const long e = (long)blockIdx.x * 256 + threadIdx.x, DS = (long)a.D * S;
    if (e >= DS) return;
    const Place p = sequence(a.seqs, blockIdx.y);
    const long base = first_slot(a, p);
    const long n = (p.end - p.first + a.Lseg - 1) / a.Lseg;
    const float A2 = rate(a.A[e]);
    const int c = (int)(e / S);
    float h = a.h0 ? a.h0[p.n * DS + e] : 0.f;
    constexpr int AHEAD = 8;                             // reads of so many segments at once
    for (long k0 = 0; k0 + 1 < n; k0 += AHEAD) {         // (of the last segment there is no map)
        float own[AHEAD], d[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const long k = min(k0 + i, n - 2);
            own[i] = a.seg_state[(base + k) * DS + e];
            d[i] = a.seg_delta[(base + k) * a.D + c];
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (k0 + i + 1 < n) {
                a.seg_state[(base + k0 + i) * DS + e] = h;
                h = fmaf(exp2_hw(A2 * d[i]), h, own[i]);
            }
        }
    }
    a.seg_state[(base + max(n - 1, 0L)) * DS + e] = h;
}

// One token for B sequences: four lanes per channel, the state updated in place.  Bound by the traffic of the states: 64 sequences of 2048
// channels x 16 states 5.6 us (18 MB, 3.2 TB/s; the launch and one trip to memory are half of it).
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
    const float delta = a.softplus ? softplus<T>(raw) : raw, du = delta * u;
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int n = q * K + k;
        h[k] = fmaf(exp2_hw(delta * rate(a.A[(long)c * S + n])), h[k], du * to_float(a.B[b * a.ld_B + g * S + n]));
        s = fmaf(to_float(a.C[b * a.ld_C + g * S + n]), h[k], s);
        st[k] = h[k];
    }
    s += quad_xor1(s);
    s += quad_xor2(s);
    if (q == 0) {
        s = fmaf(a.skip ? a.skip[c] : 0.f, u, s);
        if (a.z) { const float z = to_float(a.z[b * a.ld_z + c]); s *= z * sigmoid(z); }
        a.y[b * a.D + c] = rounded<T>(s);
    }
}

template <typename T, int S, SsmMode MODE, bool HASZ, int THREADS> static hipError_t ssm_fwd_mode(SsmArgs<T> a, hipStream_t st)
{
    const int blocks_c = ssm_channel_blocks(a.D, a.G, THREADS / 8);
    for (long n; a.slot0 < a.slots; a.slot0 += n) {
        n = std::min(a.slots - a.slot0, most_blocks(THREADS) / blocks_c);
        hipLaunchKernelGGL((ssm_fwd_kernel<T, S, MODE, HASZ, THREADS>), dim3((unsigned)(blocks_c * n)), dim3(THREADS), 0, st, a, blocks_c);
        if (const hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}
template <typename T, int S, int THREADS> static hipError_t ssm_fwd_by(const SsmArgs<T>& a, bool outputs, hipStream_t st)
{
    if (a.slots == 0) return hipSuccess;
    if (a.seg_state) {
        if (const hipError_t e = ssm_fwd_mode<T, S, kSsmMaps, false, THREADS>(a, st)) return e;
        hipLaunchKernelGGL((ssm_join_kernel<T>), dim3((unsigned)(((long)a.D * S + 255) / 256), a.seqs.n_seq), dim3(256), 0, st, a, S);
        if (const hipError_t e = hipGetLastError()) return e;
    }
    if (!outputs) return ssm_fwd_mode<T, S, kSsmStates, false, THREADS>(a, st);
    return a.z ? ssm_fwd_mode<T, S, kSsmOutputs, true, THREADS>(a, st) : ssm_fwd_mode<T, S, kSsmOutputs, false, THREADS>(a, st);
}
template <typename T, int S> static hipError_t ssm_fwd(const SsmArgs<T>& a, bool outputs, hipStream_t st)
{
    if constexpr (S < 64) {
        if (a.channels == 64) return ssm_fwd_by<T, S, 512>(a, outputs, st);
    }
    return ssm_fwd_by<T, S, 256>(a, outputs, st);
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
template <typename T> hipError_t launch_ssm_step(SsmArgs<T> a, float* h, int B, int S, hipStream_t st)
{
    const int blocks_c = (a.D + 63) / 64;
    const dim3 block(256);
    const int piece = (int)std::min<long>(most_blocks(256) / blocks_c, B);           // sequences of a launch
    for (int done = 0, n; done < B; done += n) {
        n = std::min(piece, B - done);
        const dim3 grid((unsigned)((long)blocks_c * n));
        switch (S) {
            case 8:  hipLaunchKernelGGL((ssm_step_kernel<T, 8>), grid, block, 0, st, a, h, blocks_c); break;
            case 16: hipLaunchKernelGGL((ssm_step_kernel<T, 16>), grid, block, 0, st, a, h, blocks_c); break;
            case 32: hipLaunchKernelGGL((ssm_step_kernel<T, 32>), grid, block, 0, st, a, h, blocks_c); break;
            default: hipLaunchKernelGGL((ssm_step_kernel<T, 64>), grid, block, 0, st, a, h, blocks_c); break;
        }
        if (const hipError_t e = hipGetLastError()) return e;
        a.u += n * a.ld_u;
        a.delta += n * a.ld_delta;
        a.B += n * a.ld_B;
        a.C += n * a.ld_C;
        if (a.z) a.z += n * a.ld_z;
        a.y += (long)n * a.D;
        h += (long)n * a.D * S;
    }
    return hipSuccess;
}

#define KLA_SSM(T)                                                                                       \
    template hipError_t launch_ssm_fwd<T>(const SsmArgs<T>&, int, bool, hipStream_t);                    \
    template hipError_t launch_ssm_step<T>(SsmArgs<T>, float*, int, int, hipStream_t);
KLA_SSM(float)
KLA_SSM(bf16_t)

}  // namespace kla
