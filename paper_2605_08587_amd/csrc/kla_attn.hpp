// What the attention kernels share: 32x32 matrix products on 16-byte operands, swizzled tiles of rows in LDS, where a tile of query rows
// lies in its batch, and the launchers' arguments.
//
// All products are 32x32 tiles accumulated in fp32.  A lane is (n, h) = (lane % 32, lane / 32).
//
//   accumulator     : lane (n, h) holds rows 8 (e / 4) + 4 h + e % 4 of column n, e = 0..15
//   "slot" (16 B)   : of operand row n (A) or operand column n (B), contraction indices
//                       rows of memory : the 16-byte piece 2 c + h of row n, c = 0, 1, ..
//                       from registers : of an accumulator whose row index is the next contraction index, registers 8 c .. 8 c + 7 rounded
//                                        to bf16, or 4 c .. 4 c + 3 in fp32: rows 16 c + 4 h + {0..3, 8..11}, or 8 c + 4 h + {0..3}
//
// The hardware pairs element i of an A slot with element i of a B slot, half by half, so any order of the contraction index serves as long as both
// use the same.  Scores are formed transposed, S^T = K Q^T: a lane then has one query, its softmax needs one exchange between the halves
// of a wave, and exp(S^T) is the B operand of O^T += V^T P^T as it lies.
#pragma once
#include "kla_bf16_ops.hpp"
#include "kla_layer.hpp"

namespace kla {

typedef float floatx16 __attribute__((ext_vector_type(16)));

constexpr unsigned kAttnCausal = 1u;                     // (the value of KLA_ATTN_CAUSAL in include/kla.h)

// ---- products ---------------------------------------------------------------------------------------------------------------------
template <typename T> __device__ __forceinline__ void mma32x32(floatx16& acc, u32x4 a, u32x4 b)
{
    if constexpr (sizeof(T) == 2) {
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), acc, 0, 0, 0);
    } else {
        const floatx4 x = __builtin_bit_cast(floatx4, a), y = __builtin_bit_cast(floatx4, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(x[i], y[i], acc, 0, 0, 0);
    }
}
// Rows of an accumulator that one slot holds per half: an accumulator gives 16 / kSlot<T> slots of kSlot<T> registers
template <typename T> constexpr int kSlot = 16 / (int)sizeof(T);
template <typename T, int C> __device__ __forceinline__ u32x4 slot_of(const floatx16& s)
{
    if constexpr (sizeof(T) == 2) {
        const u32x4 r = {pack_bf16x2(s[8 * C], s[8 * C + 1]), pack_bf16x2(s[8 * C + 2], s[8 * C + 3]), pack_bf16x2(s[8 * C + 4], s[8 * C + 5]),
                         pack_bf16x2(s[8 * C + 6], s[8 * C + 7])};
        return r;
    } else {
        const floatx4 r = {s[4 * C], s[4 * C + 1], s[4 * C + 2], s[4 * C + 3]};
        return __builtin_bit_cast(u32x4, r);
    }
}
// the accumulator row of register e is acc_row(e) + 4 h
__host__ __device__ constexpr int acc_row(int e) { return 8 * (e >> 2) + (e & 3); }

// Where an operand's row that a mask hides holds an infinity or a NaN, its zero weight does not hide it: 0 x inf.  Kernels that find their result not
// finite compute it again with products that keep such rows apart: the elements of a that are not finite are zeros in `fin`, and two more products count
// what a column takes in, into one accumulator: `sgn` (4096 times the sign of an infinity) times the signs of b plus `bad` (1) times the mask's ones.
template <typename T> struct Apart { u32x4 fin, sgn, bad; };
template <typename T> __device__ __forceinline__ Apart<T> apart(u32x4 a)
{
    Apart<T> r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 2) {
            uint32_t fin = 0, sgn = 0, bad = 0;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const uint32_t x = (a[i] >> (16 * j)) & 0xffffu;
                const bool b = (x & 0x7f80u) == 0x7f80u, inf = (x & 0x7fffu) == 0x7f80u;
                fin |= (b ? 0u : x) << (16 * j);
                sgn |= (inf ? 0x4580u | (x & 0x8000u) : 0u) << (16 * j);
                bad |= (b ? 0x3f80u : 0u) << (16 * j);
            }
            r.fin[i] = fin; r.sgn[i] = sgn; r.bad[i] = bad;
        } else {
            const uint32_t x = a[i];
            const bool b = (x & 0x7f800000u) == 0x7f800000u, inf = (x & 0x7fffffffu) == 0x7f800000u;
            r.fin[i] = b ? 0u : x;
            r.sgn[i] = inf ? 0x45800000u | (x & 0x80000000u) : 0u;
            r.bad[i] = b ? 0x3f800000u : 0u;
        }
    }
    return r;
}
// +-1 for values that are not zero (0 for NaN: what they meet becomes one)
__device__ __forceinline__ float sign_of(float x) { return x > 0.f ? 1.f : x < 0.f ? -1.f : 0.f; }
// what a column takes in, of an accumulator of the two products: all of its infinities of one sign and no NaN, or a NaN
__device__ __forceinline__ float not_finite(float x)
{
    const float signs = rintf(x * (1.f / 4096.f)), count = fmaf(signs, -4096.f, x);      // (at most 64 terms)
    return count == 0.f ? 0.f : signs == count ? __builtin_inff() : signs == -count ? -__builtin_inff() : __builtin_nanf("");
}
__device__ __forceinline__ bool finite(const floatx16& x)
{
    float t = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) t = fmaf(x[e], 0.f, t);
    return t == 0.f;
}

// ---- tiles of rows in LDS ---------------------------------------------------------------------------------------------------------
// Rows of D elements stand as pieces of 16 bytes; piece p of a row is at position p ^ row_swz(row).  Slot reads of 32 rows (16 lanes a cycle:
// rows {0-3, 12-15, 20-27} or the others) and transposing reads (32 lanes a cycle: four rows of 64 bytes) both then spread over the banks.
template <int PIECES> __host__ __device__ constexpr int row_swz(int row)
{
    if (PIECES == 8) return ((row >> 1 & 1) << 2) | (row >> 2 & 3);
    return ((row & 3) << 2) | (row >> 2 & 3);
}
// what all lanes have alike, in a scalar register (quotients come out of the vector ALU, and what is formed from them stays there)
__device__ __forceinline__ int wave_uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ long wave_uniform(long x)
{
    return (long)((uint64_t)(uint32_t)wave_uniform((int)x) | (uint64_t)(uint32_t)wave_uniform((int)(x >> 32)) << 32);
}
__device__ __forceinline__ const char* wave_uniform(const char* p) { return reinterpret_cast<const char*>(wave_uniform((long)p)); }
__device__ __forceinline__ uint32_t lds_place(char* wave_base)
{
    return (uint32_t)wave_uniform((int)(uint32_t)(uintptr_t)((__attribute__((address_space(3))) char*)wave_base));
}
// 16 bytes per lane from the lane's address to LDS at lds_wave_base + 16 lane (as dma16, with an address of 64 bits)
__device__ __forceinline__ void dma16_from(const char* lane_address, char* lds_wave_base)
{
    const uint32_t m = (uint32_t)(uintptr_t)((__attribute__((address_space(3))) char*)lds_wave_base);
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(lane_address), "s"(m) : "memory");
}
// from base + lane_off, base the wave's (as dma16, where the compiler has formed the places on the vector ALU)
__device__ __forceinline__ void dma16_at(const char* base, int lane_off, char* lds_wave_base)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(lane_off), "s"(wave_uniform(base)), "s"(lds_place(lds_wave_base)) : "memory");
}
// 4 bytes per lane, to lds_wave_base + 4 lane
__device__ __forceinline__ void dma4_from(const void* lane_address, char* lds_wave_base)
{
    const uint32_t m = lds_place(lds_wave_base);
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(lane_address), "s"(m) : "memory");
}
// A tile of rows of D elements of T
template <typename T, int D> struct RowTile {
    static constexpr int RB = D * (int)sizeof(T);        // bytes of a row
    static constexpr int PIECES = RB / 16;
    static constexpr int NC = RB / 32;                   // slots of a row per half
    static constexpr int RPI = 1024 / RB;                // rows of one copy instruction
    // Row slots: offset of row n, piece 2 c + h (rows 32 i + n: + 32 i RB)
    static __device__ __forceinline__ int row_offset(int n, int h) { return n * RB + ((h ^ row_swz<PIECES>(n)) * 16); }
    static __device__ __forceinline__ u32x4 row_slot(const char* tile, int row_off, int c) { return ld16(tile + (row_off ^ (32 * c))); }
    // Column slots, the contraction along rows: column 32 dt + n, rows as an accumulator's registers give them
    static __device__ __forceinline__ int col_offset(int lane)
    {
        const int n = lane & 31, h = lane >> 5;
        if constexpr (sizeof(T) == 2) {
            // source lane (a, c) of sixteen: row 4 h + a, columns 4 c .. 4 c + 3 of sixteen
            const int a = lane >> 2 & 3, c = lane & 3, s = lane >> 4 & 1, row = 4 * h + a;
            return row * RB + (((2 * s + (c >> 1)) ^ row_swz<PIECES>(row)) * 16) + (c & 1) * 8;
        } else {
            return 4 * h * RB + (((n >> 2) ^ h) * 16) + (n & 3) * 4;
        }
    }
    // slot C of the 32 rows from `tile` on
    template <int C, int DT> static __device__ __forceinline__ u32x4 col_slot(const char* tile, int col_off)
    {
        if constexpr (sizeof(T) == 2) {
            const u32x2 lo = lds_read_tr(tile + (col_off ^ (64 * DT)) + 16 * C * RB), hi = lds_read_tr(tile + (col_off ^ (64 * DT) ^ 32) + (16 * C + 8) * RB);
            return u32x4{lo.x, lo.y, hi.x, hi.y};
        } else {
            u32x4 r;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                r[i] = *reinterpret_cast<const uint32_t*>(tile + (col_off ^ (64 * i) ^ (32 * (C & 1)) ^ (128 * DT)) + (8 * C + i) * RB);
            return r;
        }
    }
};
static_assert(row_swz<16>(8) == 2 && row_swz<8>(8) == 2 && row_swz<16>(16) == 0 && row_swz<8>(16) == 0, "col_slot's constants");

// acc += (32 rows of a tile)^T b, b an accumulator of weights.  Where the block is masked, rows that are not finite count for what `seen(e)` (e: of b)
// says sees them.
template <bool CAREFUL, typename T, int D, int NDT, typename Seen>
__device__ __forceinline__ void add_product(floatx16 (&acc)[NDT], const char* tile, int col_off, const floatx16& b, bool masked, Seen&& seen)
{
    using Tile = RowTile<T, D>;
    constexpr int NS = 16 / kSlot<T>;
    if constexpr (CAREFUL) {
        if (masked) {
            floatx16 sgn, ones;
#pragma unroll
            for (int e = 0; e < 16; ++e) { sgn[e] = sign_of(b[e]); ones[e] = seen(e) ? 1.f : 0.f; }
            static_for<NDT>([&](auto dt) {
                floatx16 x;
#pragma unroll
                for (int e = 0; e < 16; ++e) x[e] = 0.f;
                static_for<NS>([&](auto c) {
                    const Apart<T> a = apart<T>(Tile::template col_slot<c, dt>(tile, col_off));
                    mma32x32<T>(acc[dt], a.fin, slot_of<T, c>(b));
                    mma32x32<T>(x, a.sgn, slot_of<T, c>(sgn));
                    mma32x32<T>(x, a.bad, slot_of<T, c>(ones));
                });
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[dt][e] += not_finite(x[e]);
            });
            return;
        }
    }
    static_for<NS>([&](auto c) {
        const u32x4 s = slot_of<T, c>(b);
        static_for<NDT>([&](auto dt) { mma32x32<T>(acc[dt], Tile::template col_slot<c, dt>(tile, col_off), s); });
    });
}

// All of this wave's copies have landed, and its LDS reads are done; then every wave's.
__device__ __forceinline__ void wait_copies() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void wait_copies_and_barrier() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// This thread, for a second run of a workgroup's work behind a first: what is derived from it anew is not kept in registers through the first.
__device__ __forceinline__ int thread_again()
{
    int t = threadIdx.x;
    asm volatile("" : "+v"(t));
    return t;
}

// What was loaded is there: without this the compiler, which does not know of the copies, would wait for such loads inside the loop over the tiles, and
// with them for the copies issued since.
__device__ __forceinline__ void settle(u32x4& x) { asm volatile("" : "+v"(x)); }
__device__ __forceinline__ void settle(int& x) { asm volatile("" : "+v"(x)); }
__device__ __forceinline__ void settle(float& x) { asm volatile("" : "+v"(x)); }
// Accumulators stay what they are here: registers behind each other (as 16 values each, a loop that scales them moved every one to another register)
template <int N> __device__ __forceinline__ void keep_whole(floatx16 (&x)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(x[i]));
}
// row i of rows `stride` bytes apart (one multiplication of 32 bits)
__device__ __forceinline__ const char* row_at(const char* p, int i, uint32_t stride) { return p + (uint64_t)(uint32_t)i * stride; }

// max and sum over the two halves of a wave, in every lane
__device__ __forceinline__ float halves_max(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float halves_sum(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// ---- rows of a batch --------------------------------------------------------------------------------------------------------------
// The query heads of one key head are rows of their own: row r of (sequence, key head) is token r / G, head hk G + r % G, and a key head's rows are taken in
// tiles of ROWS.  Fixed lengths: tiles of one number of all sequences beside each other, `per` for each sequence.  Packed: tile k of sequence n
// has the place floor(cu[n] G / ROWS) + n + k, which nothing has to count (some places stay empty); a wave looks at 64 sequences at once.  false: an empty place.
struct RowPlace { int n; int tile; int len; long tok0; };
template <int ROWS> __device__ __forceinline__ bool find_rows(const Seqs& s, int G, long per, long idx, int lane, RowPlace* p)
{
    if (!s.cu) {
        p->n = (int)(idx % s.n_seq);
        p->tile = (int)(idx / s.n_seq);
        p->len = s.T;
        p->tok0 = (long)p->n * s.T;
        return p->tile < per;
    }
    // the last sequence whose first place is at most idx (places grow with every sequence, and the first one's is 0)
    int lo = 0, step = (s.n_seq + 63) / 64;
    for (;;) {
        const int n = (int)min(lo + (long)lane * step, (long)s.n_seq);                // (cu has n_seq + 1 entries)
        const int c0 = s.cu[n];
        const long first = (long)c0 * G / ROWS + n;
        const int l = 63 - __builtin_clzll(__ballot(n < s.n_seq && first <= idx));
        lo = __builtin_amdgcn_readlane(n, l);
        if (step == 1) {
            p->n = lo;
            p->tok0 = __builtin_amdgcn_readlane(c0, l);
            break;
        }
        step = (step + 63) / 64;
    }
    p->len = s.cu[p->n + 1] - (int)p->tok0;
    const long k = idx - (p->tok0 * G / ROWS + p->n);
    p->tile = (int)k;
    return k < ((long)p->len * G + ROWS - 1) / ROWS;
}
inline long row_places(const Seqs& s, long M, int G, int rows, long* per)
{
    *per = ((long)s.T * G + rows - 1) / rows;
    if (M == 0) return 0;
    return s.cu ? M * G / rows + s.n_seq : *per * s.n_seq;
}

// ---- launchers --------------------------------------------------------------------------------------------------------------------
template <typename T> struct AttnArgs {
    const T* q; long ld_q; const T* k; long ld_k; const T* v; long ld_v;                  // rows of new tokens
    T* o; float* lse; T* rest;                           // lse, rest: or NULL; rest: what o's rounding leaves out
    Seqs seqs; int H, Hk, G;
    float scale; int window; bool causal;
    // the cache of earlier tokens: pages [n_pages][Hk][1 << page_shift][D]; table [n_seq][max_pages], rows ld_table apart
    T* k_cache; T* v_cache; const int* table; long ld_table; const int* cached; int n_pages, page_shift, max_pages;
    // keys in up to `splits` (at most 64) parts of at least `chunk` each (a multiple of 128): part_o [splits][tokens H][D] and part_lse [splits][tokens H] (base 2), where there are
    // several; part_count [tokens H]: how many there are
    int splits, chunk; float* part_o; float* part_lse; int* part_count; long M;
    long tiles, per;                                     // places of tiles of query rows of a key head: in all; of one sequence (fixed lengths)
    long unit0;                                          // first workgroup of this launch
};
// Backward: d_o, dq like o, dk, dv [tokens][Hk][D]; row_lse, row_delta [tokens][H]: the rows' lse (base 2) and -<d_o, o>; part_dk, part_dv
// [parts][tokens][Hk][D] where the query rows of a tile of keys are taken in `parts` parts.
template <typename T> struct AttnBwdArgs {
    AttnArgs<T> f;                                       // (o, lse, rest: the forward's; tiles, per, unit0: of a launch)
    const T* d_o; T* dq; T* dk; T* dv;
    float* row_lse; float* row_delta;
    int parts; float* part_dk; float* part_dv;
    bool beside;                                         // dk, dv and dq in one launch, rows of dq in tiles of 64 (else of 128: f.tiles)
    long key_tiles, key_per;                             // places of tiles of 128 keys: in all; of one sequence (fixed lengths)
};
template <typename T> hipError_t launch_attn_bwd(const AttnBwdArgs<T>& a, int D, hipStream_t st);

// How the forward's work is cut: rows of a tile (128: four waves of 32 rows that share tiles of keys; 32: four waves that share the rows and divide the
// keys), parts of the keys and their least length.
struct AttnPlan { int rows; int splits; int chunk; };
template <typename T> hipError_t launch_attn_fwd(const AttnArgs<T>& a, int D, const AttnPlan& p, bool paged, hipStream_t st);
template <typename T> hipError_t launch_attn_join(const AttnArgs<T>& a, int D, hipStream_t st);

}  // namespace kla
