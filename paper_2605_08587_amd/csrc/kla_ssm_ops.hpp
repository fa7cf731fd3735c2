// What the kernels of the selective scan share.  Lanes: a wave holds 16 channels, lane = 4 * channel + q, and lane q holds the
// states n = q K ... q K + K - 1 of its channel (K = S / 4) in registers.  Per-token scalars of a channel (delta, u, z, ...) live with the
// lane q of token 4 i + q of four: one load and one softplus per token and channel; the quad hands them round by DPP.
#pragma once
#include "kla_layer.hpp"

namespace kla {

template <int I> __device__ __forceinline__ float quad_bcast(float x) { return dpp_mov<I * 0x55>(x); }    // lane I of the quad, in all four
__device__ __forceinline__ float quad_xor1(float x) { return dpp_mov<0xB1>(x); }
__device__ __forceinline__ float quad_xor2(float x) { return dpp_mov<0x4E>(x); }
__device__ __forceinline__ float quad_sum(float x)
{
    x += quad_xor1(x);
    return x + quad_xor2(x);
}
// x[i] summed over the quad, for token i = q in lane q
__device__ __forceinline__ float quad_sum_own(const float (&x)[4], int q)
{
    const bool odd = q & 1, high = q & 2;
    const float a = (odd ? x[1] : x[0]) + quad_xor1(odd ? x[0] : x[1]);        // tokens 0, 1
    const float b = (odd ? x[3] : x[2]) + quad_xor1(odd ? x[2] : x[3]);        // tokens 2, 3
    return (high ? b : a) + quad_xor2(high ? a : b);
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
        const int per = max(1, (a.seqs.T + a.Lseg - 1) / a.Lseg);
        n = (int)(slot / per);
        base = (long)n * per;
    }
    g->seq = sequence(a.seqs, n);
    g->t0 = g->seq.first + (slot - base) * a.Lseg;
    g->t1 = min(g->t0 + a.Lseg, g->seq.end);
    g->last = g->t0 + a.Lseg >= g->seq.end;
    // a sequence without a token has one segment without one: its state passes through
    return g->t0 < g->seq.end || (slot == base && g->seq.first == g->seq.end);
}
// Where the checkpoint of token t stands (t - first a multiple of ck): like the slots, nothing has to be counted
template <typename T> __device__ __forceinline__ long checkpoint_at(const SsmArgs<T>& a, const Place& p, long t, int ck)
{
    const long base = a.seqs.cu ? p.first / ck + p.n : (long)p.n * ((a.seqs.T + ck - 1) / ck);
    return base + (t - p.first) / ck;
}

// The channels of a workgroup: blocks of kSsmTile channels of one group each
struct Channels { int g, c, most; bool mine; };          // group, this lane's channel (clamped), whether it is one
__device__ __forceinline__ Channels channels_of(int block, int D, int G, int wave, int lane)
{
    const int per = D / G, blocks = (per + kSsmTile - 1) / kSsmTile;
    Channels r;
    r.g = block / blocks;
    const int in = (block - r.g * blocks) * kSsmTile + wave * 16 + (lane >> 2);
    r.mine = in < per;
    r.c = r.g * per + min(in, per - 1);
    r.most = blocks;
    return r;
}
inline int ssm_channel_blocks(int D, int G) { return G * ((D / G + kSsmTile - 1) / kSsmTile); }

}  // namespace kla
