// What the operators around the recurrence share (short convolution, selective scan, norms): where a token lies in its batch,
// vector loads, activations, and the launchers' arguments.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kla_common.hpp"

namespace kla {

// option bits (the values of KLA_LAYER_* in include/kla.h)
constexpr unsigned kLayerSilu = 1u, kLayerSoftplus = 2u, kLayerSigmoid = 4u, kLayerGateFirst = 8u;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// 2^x and 1/x in hardware (1 ulp each)
__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float rcp_hw(float x) { return __builtin_amdgcn_rcpf(x); }
__device__ __forceinline__ float sigmoid(float x) { return rcp_hw(1.f + exp2_hw(-kLog2e * x)); }
// log(1 + e^x) = max(x, 0) + log1p(e^-|x|), the second term as 2 atanh(s) = 2 s (1 + s^2/3 + ...), s = e/(2 + e) <= 1/3: digits are kept
// where the result is as small as e^x itself (a logarithm of 1 + e loses them there).  The coefficients are a least
// largest relative error's over s^2 <= 1/9, 5e-9 before rounding.  The exponent's product with log2(e) is rounded, which costs 5e-7 of the result
// at x = -7, 9e-7 at -20 and 3.4e-6 at -85 (measured): of no weight beside bf16 inputs.  For fp32 ones it is put back, e^-|x| = 2^t e^r with
// r = -|x| - t ln 2, and 3.5e-7 is the most (three instructions, 1 % of an fp32 scan's time; a bf16 one's is 2 %).
template <typename T> __device__ __forceinline__ float softplus(float x)
{
    const float t = -kLog2e * fabsf(x);
    float e = exp2_hw(t);
    // (where t is infinite r is too, or a NaN: bounded, as e is 0)
    if constexpr (sizeof(T) == 4) e = fmaf(e, __builtin_amdgcn_fmed3f(fmaf(t, -kLn2, -fabsf(x)), -1.f, 1.f), e);
    const float s = e * rcp_hw(2.f + e), q = s * s;
    float p = 0.140059933f;
    p = fmaf(p, q, 0.140009031f);
    p = fmaf(p, q, 0.200107634f);
    p = fmaf(p, q, 0.333332092f);
    p = fmaf(p, q, 1.f);
    // (a NaN stays one: fmaxf alone would drop it, the sum with p does not)
    return fmaf(2.f * s, p, fmaxf(x, 0.f));
}

// One value of T: bf16 by the hardware's conversion (nearest even), of which it makes pairs
template <typename T> __device__ __forceinline__ T rounded(float x);
template <> __device__ __forceinline__ float rounded<float>(float x) { return x; }
template <> __device__ __forceinline__ bf16_t rounded<bf16_t>(float x) { return {(uint16_t)pack_bf16x2(x, x)}; }

// V consecutive elements, as they are (a load is waited for where it is converted) and as fp32 registers.  They stand at any element: rows
// of odd widths and column ranges of wider tensors are no different, and one load or store of up to 16 bytes takes them all the same.
template <int V> struct Floats { float v[V]; };
template <typename T, int V> struct alignas(V * sizeof(T) < 16 ? V * sizeof(T) : 16) Raw { T v[V]; };
template <typename T, int V> __device__ __forceinline__ Raw<T, V> load_raw(const T* p) 
{
    Raw<T, V> r;
    __builtin_memcpy(&r, p, sizeof r);
    return r;
}
template <typename T, int V> __device__ __forceinline__ Floats<V> floats_of(const Raw<T, V>& x)
{
    Floats<V> r;
#pragma unroll
    for (int i = 0; i < V; ++i) r.v[i] = to_float(x.v[i]);
    return r;
}
template <typename T, int V> __device__ __forceinline__ Floats<V> load_vec(const T* p) { return floats_of<T, V>(load_raw<T, V>(p)); }
template <typename T, int V> __device__ __forceinline__ void store_vec(T* p, const Floats<V>& r)
{
    if constexpr (V == 1) {
        *p = rounded<T>(r.v[0]);
    } else if constexpr (sizeof(T) == 4) {
        __builtin_memcpy(p, r.v, sizeof r.v);
    } else {
        uint32_t pairs[V / 2];
#pragma unroll
        for (int i = 0; i < V / 2; ++i) pairs[i] = pack_bf16x2(r.v[2 * i], r.v[2 * i + 1]);
        __builtin_memcpy(p, pairs, sizeof pairs);
    }
}
// Elements of T in 16 bytes
template <typename T> constexpr int kVec = 16 / (int)sizeof(T);

// The sequences of a batch of flattened tokens: offsets cu[n_seq + 1] of a packed batch, or cu = NULL and n_seq sequences of T tokens.
struct Seqs { const int* cu; int n_seq; int T; };
struct Place { int n; long first, end; };                // a sequence: its number, first token, token after its last
__device__ __forceinline__ Place sequence(const Seqs& s, int n)
{
    if (s.cu) return {n, s.cu[n], s.cu[n + 1]};
    return {n, (long)n * s.T, ((long)n + 1) * s.T};
}
// the sequence of token t (sequences without a token hold none)
__device__ __forceinline__ Place sequence_of(const Seqs& s, long t)
{
    if (!s.cu) return sequence(s, t >> 31 ? (int)(t / s.T) : (int)((unsigned)t / (unsigned)s.T));     // (32 bits divide faster)
    int lo = 0, hi = s.n_seq - 1;                        // last n with cu[n] <= t
    while (lo < hi) { const int mid = (lo + hi + 1) >> 1; if (s.cu[mid] <= t) lo = mid; else hi = mid - 1; }
    return sequence(s, lo);
}

// A launch's threads are counted in 32 bits: one of more runs what is left of the number, without an error.
inline long most_blocks(int threads) { return 0xffffffffL / threads; }

// ---- launchers ------------------------------------------------------------------------------------------------------------------
// Sums over the rows of partial[P][n0 + n1 + n2] in a fixed order, the columns to up to three outputs (each may be NULL).
struct ColumnSums { long n[3]; float* out[3]; };
hipError_t launch_column_sums(const float* partial, long P, const ColumnSums& s, hipStream_t st);

template <typename T> struct ConvArgs {
    const T* x; long ld_x; const float* weight; const float* bias; const T* state;      // bias, state: or NULL
    T* y; T* state_out;                                                                   // state_out: or NULL
    const T* d_y; const T* d_state_out; T* dx; T* d_state; float* partial;               // backward
    Seqs seqs; long M; int D;
};
// Threads along a row of D channels and rows of threads (strips) of one workgroup of the backward, and its strips' tokens: what
// lays out the partial sums.
struct ConvBwdPlan { int tx, ty, L; long blocks_t; };
ConvBwdPlan conv_bwd_plan(long M, int D);
template <typename T> hipError_t launch_conv_fwd(const ConvArgs<T>& a, int W, bool silu, hipStream_t st);
template <typename T> hipError_t launch_conv_bwd(const ConvArgs<T>& a, int W, bool silu, float* dweight, float* dbias, hipStream_t st);
template <typename T> hipError_t launch_conv_step(const T* x, long ld_x, const float* weight, const float* bias, T* state, T* y, int B, int D, int W,
                                                  bool silu, hipStream_t st);

// T: type of x, y; R: type of the residual stream
template <typename T, typename R> struct AddNormArgs {
    const T* x; long ld_x; const R* residual; const float* scale; const float* weight; float eps;   // residual, scale: or NULL
    T* y; R* residual_out;                                                                           // residual_out: or NULL
    const T* d_y; const R* d_residual_out; T* dx; R* d_residual; float* partial;                    // backward; d_residual_out, d_residual: or NULL
    long M; int D;
};
template <typename T> struct GatedNormArgs {
    const T* x; long ld_x; const T* gate; long ld_gate; const float* weight; float eps;
    T* y;
    const T* d_y; T* dx; T* d_gate; float* partial;
    long M; int H, D;                                    // M tokens of H rows of D
    unsigned opts;                                       // kLayerSigmoid | kLayerGateFirst
};
// Workgroups of a norm's backward, each of which leaves a row of partial sums
int norm_bwd_blocks(long rows, int D, int vec_len);
template <typename T, typename R> hipError_t launch_add_norm_fwd(const AddNormArgs<T, R>& a, hipStream_t st);
template <typename T, typename R> hipError_t launch_add_norm_bwd(const AddNormArgs<T, R>& a, float* dweight, float* dscale, hipStream_t st);
template <typename T> hipError_t launch_gated_norm_fwd(const GatedNormArgs<T>& a, hipStream_t st);
template <typename T> hipError_t launch_gated_norm_bwd(const GatedNormArgs<T>& a, float* dweight, hipStream_t st);

// Selective scan.  The tokens of a sequence are taken in segments of Lseg (a multiple of the checkpoint distance); segment k of
// sequence n has the slot first/Lseg + n + k (packed) or n * ceil(T/Lseg) + k, which nothing has to count: a few slots stay empty.
template <typename T> struct SsmArgs {
    const T* u; long ld_u; const T* delta; long ld_delta; const float* A;
    const T* B; long ld_B; const T* C; long ld_C;
    const float* skip; const T* z; long ld_z; const float* delta_bias; const float* h0;  // each of these or NULL
    T* y; float* hT;                                     // hT: or NULL
    float* saved;                                        // states at every checkpoint, or NULL
    float* seg_state; float* seg_delta;                  // per slot: [D][S] and [D]; NULL: one segment per sequence
    Seqs seqs; long M; int D, G, Lseg; long slots;
    long slot0;                                          // of a launch that takes not all of them
    bool softplus;
    int channels;                                        // of a workgroup of the forward: 32 or 64
    // backward
    const T* d_y; const float* d_hT;
    T* du; T* ddelta; T* dz; float* dh0;
    float* part_bc;                                      // [channel block][token][2 S]: gradients of C, then of B
    float* part_p;                                       // [slot][D S + 2 D]: gradients of A, skip, delta_bias
};
// Channels of a workgroup of the backward.  With 64 there are half the sums for the gradients of B and C, but eight waves at once that wait for
// each other and take all registers of a CU (bf16, S = 16, 2048 channels, 2048 tokens, both kernels: 8 sequences 548 us with 32 and 573 with
// 64, 12 sequences 798 and 1079; at S = 8 454 and 430).
constexpr int kSsmBwdChannels = 32;
constexpr int ssm_checkpoint(int S) { return S > 16 ? 8 : 16; }     // tokens between checkpoints
template <typename T> hipError_t launch_ssm_fwd(const SsmArgs<T>& a, int S, bool outputs, hipStream_t st);
template <typename T> hipError_t launch_ssm_bwd(const SsmArgs<T>& a, int S, float* dA, T* dB, T* dC, float* dskip, float* ddelta_bias, hipStream_t st);
template <typename T> hipError_t launch_ssm_step(SsmArgs<T> a, float* h, int B, int S, hipStream_t st);

}  // namespace kla
