// What the kernels of the selective scan share.  Lanes: a wave holds 8 channels, lane = 8 * channel + o, and lane o of the octet holds the
// states n = o K ... o K + K - 1 of its channel (K = S / 8) in registers.  Per-token scalars of a channel (delta, u, z, ...) live with lane o
// for token 8 i + o of eight: one load, one softplus per token and channel; DPP moves hand them round.
#pragma once
#include <type_traits>

#include "kla_layer.hpp"

namespace kla {

template <int CTRL, int BANKS> __device__ __forceinline__ float dpp_into(float old, float x)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(old), __float_as_int(x), CTRL, 0xf, BANKS, false));
}
template <int I> __device__ __forceinline__ float quad_bcast(float x) { return dpp_mov<I * 0x55>(x); }    // lane I of the quad, in all four
__device__ __forceinline__ float quad_xor1(float x) { return dpp_mov<0xB1>(x); }
__device__ __forceinline__ float quad_xor2(float x) { return dpp_mov<0x4E>(x); }

// The scalars of the octet's eight tokens in both of its quads: of tokens 0-3 (half 0), of tokens 4-7 (half 1), lane q of a quad holding
// that of token q (4 + q).  Rows of 16 lanes are two octets: the quads of tokens 0-3 are banks 0 and 2.
struct Oct { float half[2]; };
__device__ __forceinline__ Oct oct_of(float x)
{
    return {{dpp_into<0x114, 0xA>(x, x), dpp_into<0x104, 0x5>(x, x)}};        // row_shr:4 into banks 1, 3; row_shl:4 into banks 0, 2
}
template <int J> __device__ __forceinline__ float oct_bcast(const Oct& x) { return quad_bcast<(J & 3)>(x.half[J >> 2]); }

// x[j] summed over the quad, for token j = q in lane q
__device__ __forceinline__ float quad_sum_own(float x0, float x1, float x2, float x3, bool odd, bool high)
{
    const float a = (odd ? x1 : x0) + quad_xor1(odd ? x0 : x1);                // tokens 0, 1
    const float b = (odd ? x3 : x2) + quad_xor1(odd ? x2 : x3);                // tokens 2, 3
    return (high ? b : a) + quad_xor2(high ? a : b);
}
// x[j] summed over the octet, for token j = o in lane o
__device__ __forceinline__ float oct_sum_own(const float (&x)[8], int o)
{
    const bool odd = o & 1, high = o & 2;
    const float lo = quad_sum_own(x[0], x[1], x[2], x[3], odd, high), hi = quad_sum_own(x[4], x[5], x[6], x[7], odd, high);
    const float other = dpp_into<0x114, 0xA>(dpp_into<0x104, 0x5>(lo, lo), hi);     // the other quad's: tokens 0-3 to banks 0, 2; 4-7 to 1, 3
    return (o & 4 ? hi : lo) + other;
}
// the octet's sum, in all its lanes
__device__ __forceinline__ float oct_sum(float x)
{
    x += quad_xor1(x);
    x += quad_xor2(x);
    return x + dpp_mov<0x141>(x);                        // row_half_mirror: the quad's lanes are alike
}

// Slot -> the segment it stands for
struct Segment { Place seq; long t0, t1; bool last; };
template <typename T> __device__ __forceinline__ bool segment_of(const SsmArgs<T>& a, long slot, Segment* g)
{
    int n;
    long base;
    if (a.seqs.cu) {
        int lo = 0, hi = a.seqs.n_seq - 1;               // last n with first/Lseg + n <= slot
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (a.seqs.cu[mid] / a.Lseg + mid <= slot) lo = mid; else hi = mid - 1;
        }
        n = lo;
        base = a.seqs.cu[n] / a.Lseg + n;
    } else {
        const int per = max(1, (int)(((long)a.seqs.T + a.Lseg - 1) / a.Lseg));
        n = (int)slot / per;
        base = (long)n * per;
    }
    n = __builtin_amdgcn_readfirstlane(n);               // (one slot per workgroup: all of this is the same for its lanes)
    g->seq = sequence(a.seqs, n);
    g->t0 = g->seq.first + (slot - base) * a.Lseg;
    g->t1 = min(g->t0 + a.Lseg, g->seq.end);
    g->last = g->t0 + a.Lseg >= g->seq.end;
    // a sequence without a token has one segment without one: its state passes through
    return g->t0 < g->seq.end || (slot == base && g->seq.first == g->seq.end);
}
// Slot of a sequence's first segment, and its number of segments
template <typename T> __device__ __forceinline__ long first_slot(const SsmArgs<T>& a, const Place& p)
{
    return a.seqs.cu ? p.first / a.Lseg + p.n : (long)p.n * max(1L, ((long)a.seqs.T + a.Lseg - 1) / a.Lseg);
}
// Where the checkpoint of token t stands (t - first a multiple of ck): like the slots, nothing has to be counted
template <typename T> __device__ __forceinline__ long checkpoint_at(const SsmArgs<T>& a, const Place& p, long t, int ck)
{
    const long base = a.seqs.cu ? p.first / ck + p.n : (long)p.n * ((a.seqs.T + ck - 1) / ck);
    return base + (t - p.first) / ck;
}

// The channels of a workgroup: blocks of `channels` of one group each
struct Channels { int g, c; bool mine; };                // group, this lane's channel (clamped), whether it is one
__device__ __forceinline__ Channels channels_of(int block, int D, int G, int channels)
{
    const int per = D / G, blocks = (per + channels - 1) / channels;
    Channels r;
    r.g = block / blocks;
    const int in = (block - r.g * blocks) * channels + (int)(threadIdx.x >> 3);
    r.mine = in < per;
    r.c = r.g * per + min(in, per - 1);
    return r;
}
inline int ssm_channel_blocks(int D, int G, int channels) { return G * ((D / G + channels - 1) / channels); }

// A value that has to be there at this point: a register that a load is about to fill anew must not be read later, or the load goes
// elsewhere and its result has to be moved, and waited for, at the end of the loop's body.
__device__ __forceinline__ void settle(float& x) { asm volatile("" : "+v"(x)); }

// An element by a base that is the same for the wave and this lane's offset in bytes: no address arithmetic in the vector unit
template <typename T> __device__ __forceinline__ T load_at(const T* base, unsigned bytes)
{
    return *reinterpret_cast<const T*>(reinterpret_cast<const char*>(base) + bytes);
}
template <typename T> __device__ __forceinline__ void store_at(T* base, unsigned bytes, T x)
{
    *reinterpret_cast<T*>(reinterpret_cast<char*>(base) + bytes) = x;
}
// x where the token is one of the segment, else 0: on the bits, so that no branch and no NaN comes of it
__device__ __forceinline__ float where(bool in, float x) { return __int_as_float(__float_as_int(x) & (in ? -1 : 0)); }

// A lane's tokens 8 i + o of the tiles of one input or output [tokens][ld], raw: converted where they are loaded they would be waited for
// there.  The base moves by a tile at a time (a wave alone on its SIMD pays for scalar instructions as for others).  In a tile that the
// segment's end cuts the last row is repeated: nothing is read beyond it.
template <typename T, int NG> struct Tokens {
    T* p; int ld; unsigned off[NG];
    __device__ __forceinline__ void init(T* base, long t, int ld_, int c, int o)
    {
        ld = ld_;
        p = base + t * ld;
#pragma unroll
        for (int i = 0; i < NG; ++i) off[i] = (unsigned)((8 * i + o) * ld + c) * (unsigned)sizeof(T);
    }
    __device__ __forceinline__ void move(int tokens) { p += (long)tokens * ld; }
    template <bool FULL> __device__ __forceinline__ void load(std::remove_const_t<T> (&v)[NG], int last, int o) const
    {
#pragma unroll
        for (int i = 0; i < NG; ++i)
            v[i] = load_at(p, FULL ? off[i] : off[i] - (unsigned)(max(8 * i + o - last, 0) * ld) * (unsigned)sizeof(T));
    }
    __device__ __forceinline__ void store(int i, T x) const { store_at(p, off[i], x); }
};

// The rows of B and C of a tile of TOK tokens, in LDS as fp32: [token][o][B of the lane's K states, then C].  Every thread brings NE elements.
template <typename T, int S, int TOK, int THREADS> struct TileBC {
    static constexpr int K = S / 8, ALL = 2 * TOK * S, NE = (ALL + THREADS - 1) / THREADS;
    static_assert(TOK * S % 64 == 0, "a wave's elements are of B or of C");
    const T* p[NE]; int ld[NE]; unsigned off[NE]; int tok[NE], at[NE];
    __device__ __forceinline__ void init(const SsmArgs<T>& a, int g, long t)
    {
#pragma unroll
        for (int i = 0; i < NE; ++i) {
            const int e = (int)threadIdx.x + THREADS * i;
            const int m = __builtin_amdgcn_readfirstlane(e) / (TOK * S);         // 0: of B, 1: of C, 2: none
            ld[i] = (int)(m == 1 ? a.ld_C : a.ld_B);
            p[i] = (m == 1 ? a.C : a.B) + t * ld[i] + g * S;
            tok[i] = e / S % TOK;
            off[i] = (unsigned)(tok[i] * ld[i] + e % S) * (unsigned)sizeof(T);
            at[i] = m > 1 ? -1 : tok[i] * 2 * S + e % S / K * 2 * K + m * K + e % K;
        }
    }
    __device__ __forceinline__ void move(int tokens)
    {
#pragma unroll
        for (int i = 0; i < NE; ++i) p[i] += (long)tokens * ld[i];
    }
    // (rows beyond the segment repeat its last)
    template <bool FULL> __device__ __forceinline__ void load(T (&v)[NE], int last) const
    {
#pragma unroll
        for (int i = 0; i < NE; ++i)
            v[i] = load_at(p[i], FULL ? off[i] : off[i] - (unsigned)(max(tok[i] - last, 0) * ld[i]) * (unsigned)sizeof(T));
    }
    __device__ __forceinline__ void store(float* lds, const T (&v)[NE]) const
    {
#pragma unroll
        for (int i = 0; i < NE; ++i) if (ALL % THREADS == 0 || at[i] >= 0) lds[at[i]] = to_float(v[i]);
    }
    // Zeros for the rows beyond the segment, `left` of the tile being its own: 0 times what stands there would be a NaN where the segment's
    // last token has an infinity.  (By the threads that stored them; a mask in store instead costs 1 % of a long sequence's time, this 0.2 %.)
    __device__ __forceinline__ void clear(float* lds, int left) const
    {
#pragma unroll
        for (int i = 0; i < NE; ++i) if ((ALL % THREADS == 0 || at[i] >= 0) && tok[i] >= left) lds[at[i]] = 0.f;
    }
};
template <int K> struct StateBC { float b[K], c[K]; };
template <int K> __device__ __forceinline__ StateBC<K> lds_bc(const float* lane_row)
{
    StateBC<K> r;
    if constexpr (K == 1) {
        const float2 x = *reinterpret_cast<const float2*>(lane_row);
        r.b[0] = x.x; r.c[0] = x.y;
    } else if constexpr (K == 2) {
        const float4 x = *reinterpret_cast<const float4*>(lane_row);
        r.b[0] = x.x; r.b[1] = x.y; r.c[0] = x.z; r.c[1] = x.w;
    } else {
#pragma unroll
        for (int k = 0; k < K; k += 4) {
            const float4 x = *reinterpret_cast<const float4*>(lane_row + k), y = *reinterpret_cast<const float4*>(lane_row + K + k);
            r.b[k] = x.x; r.b[k + 1] = x.y; r.b[k + 2] = x.z; r.b[k + 3] = x.w;
            r.c[k] = y.x; r.c[k + 1] = y.y; r.c[k + 2] = y.z; r.c[k + 3] = y.w;
        }
    }
    return r;
}
// K states of a lane in memory, K * 4 bytes aligned so
template <int K> __device__ __forceinline__ void load_states(float (&h)[K], const float* p)
{
    if constexpr (K == 1) h[0] = *p;
    if constexpr (K == 2) { const float2 x = *reinterpret_cast<const float2*>(p); h[0] = x.x; h[1] = x.y; }
    if constexpr (K >= 4) {
#pragma unroll
        for (int k = 0; k < K; k += 4) {
            const float4 x = *reinterpret_cast<const float4*>(p + k);
            h[k] = x.x; h[k + 1] = x.y; h[k + 2] = x.z; h[k + 3] = x.w;
        }
    }
}
// log2(e) A of a state.  One that forgets at once (A = -inf) has the lowest number in its place: a token that is none, with a
// step of 0, then leaves it as it is and does not make it 0 * inf.
__device__ __forceinline__ float rate(float A)
{
    constexpr float kMost = 3.402823466e38f;
    const float A2 = kLog2e * A;
    return fabsf(A2) > kMost ? copysignf(kMost, A2) : A2;                // (a NaN stays one)
}
template <int K> __device__ __forceinline__ void load_rates(float (&A2)[K], const float* p)
{
    load_states<K>(A2, p);
#pragma unroll
    for (int k = 0; k < K; ++k) A2[k] = rate(A2[k]);
}
template <int K> __device__ __forceinline__ void store_states(float* p, const float (&h)[K])
{
    if constexpr (K == 1) *p = h[0];
    if constexpr (K == 2) *reinterpret_cast<float2*>(p) = make_float2(h[0], h[1]);
    if constexpr (K >= 4) {
#pragma unroll
        for (int k = 0; k < K; k += 4) *reinterpret_cast<float4*>(p + k) = make_float4(h[k], h[k + 1], h[k + 2], h[k + 3]);
    }
}

}  // namespace kla
