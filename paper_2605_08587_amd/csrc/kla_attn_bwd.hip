// Softmax attention, backward.  With p_ij = exp(s_ij - lse_i), formed again from the forward's lse:
//
//     delta_i = <do_i, o_i>,   dp_ij = <do_i, v_j>,   ds_ij = p_ij (dp_ij - delta_i)
//     dv_j = sum_i p_ij do_i,   dk_j = scale sum_i ds_ij q_i,   dq_i = scale sum_j ds_ij k_j
//
// Two kernels behind a small one for delta, so that every sum has one owner and no atomics: one has tiles of 128 keys and goes over the query rows of
// all heads that share them (dk, dv: four products per tile), one has tiles of 128 query rows and goes over the keys (dq: three).  They form s and dp
// twice, 7 products where one kernel with sums in memory has 5; that one's dq would be added up by all workgroups in no fixed order.  A wave holds 32
// keys (or rows) as the columns of its accumulators; p and ds come out of S = Q K^T as the B operands of the products behind it.  p and ds are fp32
// and rounded to the inputs' type where they enter a product; sums are fp32.
//
// bf16, 8 x 4096 tokens, 8 heads of 128, causal: dk, dv 618 us (0.89 PFLOP/s), dq 441 us (0.94), delta 32 us (200 MB at 6.3 TB/s);
// at 1.7 GHz and with the matrix pipe busy 47 and 49 % of the cycles (counted).  No pipe is full (the vector ALU issues in 37 and 33 % of the cycles, 45 % with an
// exponential as four): a SIMD has two waves, and they stand at waits and barriers for 34 and 41 % of their time.  6 sequences of 1000 to 5000 tokens, window
// 1024, 16 heads over 4 of 64: dk, dv 251 us, where 572 workgroups with keys come to 512 places (1.3 waves to a SIMD on the average), dq 123 us.
#include "kla_attn.hpp"

namespace kla {

namespace {

// delta and lse in units of log 2.  16 lanes to a row.  (The rounding of o to bf16 would be most of the error of dq and dk: where a row sees few keys its
// o is as large as v, and delta's error is the whole row's.  With o's remainder their error is 2.4e-3, as p's and their own rounding give, without it 3.2e-3.)
template <typename T, int D> __global__ __launch_bounds__(256) void attn_rows_kernel(const AttnBwdArgs<T> a, long row0)
{
    constexpr int V = kVec<T>, N = D / (16 * V) > 0 ? D / (16 * V) : 1, LANES = D / (N * V);
    const long rows = a.f.M * a.f.H, row = row0 + (long)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
    const int l = threadIdx.x % LANES;
    float sum = 0.f;
    if (row < rows) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const Floats<V> x = load_vec<T, V>(a.d_o + row * D + (i * LANES + l) * V);
            Floats<V> y = load_vec<T, V>(a.f.o + row * D + (i * LANES + l) * V);
            if (a.f.rest) {
                const Floats<V> z = load_vec<T, V>(a.f.rest + row * D + (i * LANES + l) * V);
#pragma unroll
                for (int e = 0; e < V; ++e) y.v[e] += z.v[e];
            }
#pragma unroll
            for (int e = 0; e < V; ++e) sum = fmaf(x.v[e], y.v[e], sum);
        }
    }
#pragma unroll
    for (int d = LANES / 2; d >= 1; d >>= 1) sum += __shfl_xor(sum, d, 64);
    if (row < rows && l == 0) {
        a.row_delta[row] = -sum;                         // (where the sums of dp begin)
        a.row_lse[row] = a.f.lse[row] * kLog2e;
    }
}

template <int NDT> __device__ __forceinline__ void clear(floatx16 (&x)[NDT])
{
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) x[dt][e] = 0.f;
}
template <int NDT> __device__ __forceinline__ bool all_finite(const floatx16 (&x)[NDT])
{
    bool f = true;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) f = f && finite(x[dt]);
    return f;
}
// a lane's column of O^T-like accumulators: features 32 dt + 8 i + 4 h .. + 3 of one row
template <typename E, int NDT> __device__ __forceinline__ void store_row(E* row, const floatx16 (&x)[NDT], float f, int h)
{
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const Floats<4> v = {{x[dt][4 * i] * f, x[dt][4 * i + 1] * f, x[dt][4 * i + 2] * f, x[dt][4 * i + 3] * f}};
            store_vec<E, 4>(row + 32 * dt + 8 * i + 4 * h, v);
        }
}

// ---- dk, dv -----------------------------------------------------------------------------------------------------------------------
template <typename T, int D> struct Dkv {
    using Tile = RowTile<T, D>;
    static constexpr bool VL = sizeof(T) == 2 && D == 128;                // the tile's rows of V stand in LDS, not in registers
    static constexpr int BM = sizeof(T) == 4 || VL ? 32 : 64;             // query rows of a tile
    static constexpr int TILE = BM * Tile::RB, STAGE = 2 * TILE, VECS = 2 * STAGE, VROWS = VECS + 2 * 512, LDS = VROWS + (VL ? 128 * Tile::RB : 0);
    static constexpr int NDT = D / 32;

    struct Place { int len, rows; long tok0; int hk; };
    // The first row of a tile, and which head of which token it is: it goes on by BM, without a division
    struct Front {
        int m0, token, head;
        __device__ __forceinline__ void next(int G)
        {
            m0 += BM;
            token += BM / G;
            head += BM % G;
            if (head >= G) { head -= G; ++token; }
        }
    };

    static __device__ __forceinline__ void copy(const AttnBwdArgs<T>& a, const Place& p, const Front& f, char* lds, int stage, int wave, int lane)
    {
        constexpr int RPI = Tile::RPI, ROWS = BM / 4, NI = ROWS / RPI;
        const uint32_t ld = (uint32_t)(a.f.ld_q * sizeof(T)), ldo = (uint32_t)a.f.H * Tile::RB;      // (63 of them fit 31 bits, as strides at most 2^24 elements do)
        const char* q = reinterpret_cast<const char*>(a.f.q) + (p.tok0 + f.token) * (long)ld + (long)p.hk * a.f.G * Tile::RB;
        const char* g = reinterpret_cast<const char*>(a.d_o) + ((p.tok0 + f.token) * a.f.H + (long)p.hk * a.f.G) * Tile::RB;
        char* at = lds + stage * STAGE;
        // Whole tokens, all of them there: what a lane takes of a tile does not depend on the tile.  (Heads told apart by division in every tile: 55 vector
        // instructions of 220 instead of 14; 8 x 4096 tokens, 8 heads of 128, both directions 1400 us instead of 1373.)
        if (BM % a.f.G == 0 && f.m0 + BM <= p.rows) {
            const int sh = __builtin_ctz(a.f.G), mask = a.f.G - 1;
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const int first = wave * ROWS + i * RPI, row = first + lane / Tile::PIECES, t = row >> sh, head = row & mask;
                const int piece = ((lane % Tile::PIECES) ^ row_swz<Tile::PIECES>(row)) * 16 + head * Tile::RB;
                dma16_at(q, (int)(t * ld) + piece, at + first * Tile::RB);
                dma16_at(g, (int)(t * ldo) + piece, at + TILE + first * Tile::RB);
            }
            if (wave < 2) {
                const float* row0 = (wave ? a.row_delta : a.row_lse) + (p.tok0 + f.token) * a.f.H + (long)p.hk * a.f.G;
                const int row = min(lane, BM - 1);
                dma4_from(row0 + ((row >> sh) * a.f.H + (row & mask)), lds + VECS + stage * 512 + wave * 256);
            }
            return;
        }
        // row f.m0 + i as a token and a head of it: (x + 1/2) / G is at least 1/2G from any whole number, far more than x below 2^17 loses in fp32
        const float over = 1.f / (float)a.f.G;
        auto split = [&](int i, int* head) {
            const int x = f.head + min(i, p.rows - 1 - f.m0), t = (int)(((float)x + 0.5f) * over);
            *head = x - t * a.f.G;
            return t;
        };
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int first = wave * ROWS + i * RPI, row = first + lane / Tile::PIECES;
            int head;
            const int t = split(row, &head), piece = ((lane % Tile::PIECES) ^ row_swz<Tile::PIECES>(row)) * 16 + head * Tile::RB;
            dma16_at(q, (int)(t * ld) + piece, at + first * Tile::RB);
            dma16_at(g, (int)(t * ldo) + piece, at + TILE + first * Tile::RB);
        }
        if (wave < 2) {
            int head;
            const int t = split(lane, &head);
            const long row = (p.tok0 + f.token + t) * a.f.H + (long)p.hk * a.f.G + head;
            dma4_from((wave ? a.row_delta : a.row_lse) + row, lds + VECS + stage * 512 + wave * 256);
        }
    }

    struct Keys { u32x4 k[Tile::NC], v[VL ? 1 : Tile::NC]; const char* rows; int lo, hi; int lo_least, lo_most, hi_least, hi_most; float c; };

    template <bool CAREFUL>
    static __device__ __forceinline__ void block(const Keys& key, floatx16 (&dk)[NDT], floatx16 (&dv)[NDT], const char* q, const char* g, const float* vecs, int m0,
                                                 int row_off, int col_off, int h)
    {
        // rows m0 .. m0 + 31 against the rows lo .. hi - 1 that see this lane's key
        const bool masked = m0 < key.lo_most || m0 + 32 > key.hi_least;
        const int lo = key.lo - m0 - 4 * h, hi = key.hi - m0 - 4 * h;
        auto seen = [&](int e) { return acc_row(e) >= lo && acc_row(e) < hi; };
        floatx16 s, ds;
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
        for (int c = 0; c < Tile::NC; ++c) mma32x32<T>(s, Tile::row_slot(q, row_off, c), key.k[c]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const floatx4 d = *reinterpret_cast<const floatx4*>(vecs + 64 + 8 * i + 4 * h);
#pragma unroll
            for (int e = 0; e < 4; ++e) ds[4 * i + e] = d[e];
        }
#pragma unroll
        for (int c = 0; c < Tile::NC; ++c) mma32x32<T>(ds, Tile::row_slot(g, row_off, c), VL ? Tile::row_slot(key.rows, row_off, c) : key.v[VL ? 0 : c]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const floatx4 l = *reinterpret_cast<const floatx4*>(vecs + 8 * i + 4 * h);
#pragma unroll
            for (int e = 0; e < 4; ++e) s[4 * i + e] = exp2_hw(fmaf(s[4 * i + e], key.c, -l[e]));
        }
        if (masked) {
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] = seen(e) ? s[e] : 0.f;
        }
        __builtin_amdgcn_sched_barrier(0);
        add_product<CAREFUL, T, D>(dv, g, col_off, s, masked, seen);
#pragma unroll
        for (int e = 0; e < 16; ++e) ds[e] *= s[e];
        if (masked) {                                    // (0 times what is not finite)
#pragma unroll
            for (int e = 0; e < 16; ++e) ds[e] = seen(e) ? ds[e] : 0.f;
        }
        __builtin_amdgcn_sched_barrier(0);
        add_product<CAREFUL, T, D>(dk, q, col_off, ds, masked, seen);
    }

    template <bool CAREFUL>
    static __device__ __forceinline__ void pass(const AttnBwdArgs<T>& a, const Place& p, const Keys& key, floatx16 (&dk)[NDT], floatx16 (&dv)[NDT], int tb, int te,
                                                char* lds, int wave, int lane)
    {
        const int h = lane >> 5, row_off = Tile::row_offset(lane & 31, h), col_off = Tile::col_offset(lane);
        clear(dk);
        clear(dv);
        Front front = {tb * BM, wave_uniform(tb * BM / a.f.G), wave_uniform(tb * BM % a.f.G)};
        if (tb < te) copy(a, p, front, lds, 0, wave, lane);
        for (int t = tb; t < te; ++t) {
            wait_copies_and_barrier();
            const int stage = (t - tb) & 1;
            front.next(a.f.G);
            if (t + 1 < te) copy(a, p, front, lds, stage ^ 1, wave, lane);
#pragma unroll 1
            for (int b = 0; b < BM / 32; ++b) {
                const int m0 = t * BM + 32 * b;
                if (m0 + 31 < key.lo_least || m0 >= key.hi_most) continue;
                const char* q = lds + stage * STAGE + 32 * b * Tile::RB;
                block<CAREFUL>(key, dk, dv, q, q + TILE, reinterpret_cast<const float*>(lds + VECS + stage * 512) + 32 * b, m0, row_off, col_off, h);
            }
        }
    }

    // false: something is not finite, nothing was stored (CAREFUL stores whatever comes out)
    template <bool CAREFUL> static __device__ __forceinline__ bool run(const AttnBwdArgs<T>& a, long unit, int thread, char* lds)
    {
        const int lane = thread & 63, wave = __builtin_amdgcn_readfirstlane(thread >> 6);
        const int n = lane & 31, h = lane >> 5;
        // the first keys of a sequence are seen by the most rows: they go first
        const int part = (int)(unit % a.parts);
        Place p;
        p.hk = wave_uniform((int)(unit / a.parts % a.f.Hk));
        RowPlace at;
        if (!find_rows<128>(a.f.seqs, 1, a.key_per, unit / a.parts / a.f.Hk, lane, &at)) return true;
        p.len = wave_uniform(at.len); p.tok0 = wave_uniform(at.tok0); p.rows = p.len * a.f.G;
        const int k0 = wave_uniform(at.tile) * 128, G = a.f.G, window = a.f.window ? min(a.f.window, p.len) : 0;
        // the rows that see key j: lo .. hi - 1
        auto lo_of = [&](int j) { return a.f.causal ? j * G : 0; };
        auto hi_of = [&](int j) { return window ? min(p.len, j + window) * G : p.rows; };
        const int k1 = min(k0 + 127, p.len - 1);
        const int t0 = lo_of(k0) / BM, t1 = (hi_of(k1) + BM - 1) / BM;
        const int tb = wave_uniform(t0 + (int)((long)(t1 - t0) * part / a.parts)), te = wave_uniform(t0 + (int)((long)(t1 - t0) * (part + 1) / a.parts));
        const int w0 = k0 + 32 * wave, j = min(w0 + n, p.len - 1);
        Keys key;
        key.c = a.f.scale * kLog2e;
        {
            const char* kp = reinterpret_cast<const char*>(a.f.k + (p.tok0 + j) * a.f.ld_k + (long)p.hk * D);
            const char* vp = reinterpret_cast<const char*>(a.f.v + (p.tok0 + j) * a.f.ld_v + (long)p.hk * D);
#pragma unroll
            for (int c = 0; c < Tile::NC; ++c) {
                key.k[c] = ld16(kp + (2 * c + h) * 16);
                if constexpr (!VL) key.v[c] = ld16(vp + (2 * c + h) * 16);
            }
        }
#pragma unroll
        for (int c = 0; c < Tile::NC; ++c) {
            settle(key.k[c]);
            if constexpr (!VL) settle(key.v[c]);
        }
        key.rows = lds + VROWS + 32 * wave * Tile::RB;
        if constexpr (VL) {                              // each wave its own (awaited with the first tile)
#pragma unroll
            for (int i = 0; i < 32 / Tile::RPI; ++i) {
                const int row = i * Tile::RPI + lane / Tile::PIECES;
                const char* vp = reinterpret_cast<const char*>(a.f.v + (p.tok0 + min(w0 + row, p.len - 1)) * a.f.ld_v + (long)p.hk * D);
                dma16_from(vp + ((lane % Tile::PIECES) ^ row_swz<Tile::PIECES>(row)) * 16, lds + VROWS + (32 * wave + i * Tile::RPI) * Tile::RB);
            }
        }
        const int j0 = min(w0, p.len - 1), j1 = min(w0 + 31, p.len - 1);
        key.lo = lo_of(j); key.hi = hi_of(j);
        key.lo_least = lo_of(j0); key.lo_most = lo_of(j1);
        key.hi_least = hi_of(j0); key.hi_most = w0 >= p.len ? -1 : hi_of(j1);        // (a wave without keys passes over every tile)
        floatx16 dk[NDT], dv[NDT];
        pass<CAREFUL>(a, p, key, dk, dv, tb, te, lds, wave, lane);
        if constexpr (!CAREFUL) {
            if (__syncthreads_or(!all_finite(dk) || !all_finite(dv))) return false;
        }
        if (w0 + n >= p.len) return true;
        const long row = (p.tok0 + j) * a.f.Hk + p.hk;
        if (a.parts > 1) {
            const long to = ((long)part * a.f.M * a.f.Hk + row) * D;
            store_row<float>(a.part_dk + to, dk, a.f.scale, h);
            store_row<float>(a.part_dv + to, dv, 1.f, h);
        } else {
            store_row<T>(a.dk + row * D, dk, a.f.scale, h);
            store_row<T>(a.dv + row * D, dv, 1.f, h);
        }
        return true;
    }
};

// ---- dq ---------------------------------------------------------------------------------------------------------------------------
// Four waves: RW of 32 rows each, which share tiles of keys, times KW = 4 / RW that divide the tiles, in step, and add up what they have.
template <typename T, int D, int RW> struct Dq {
    using Tile = RowTile<T, D>;
    static constexpr int KW = 4 / RW;
    static constexpr int BN = sizeof(T) == 4 || KW > 1 ? 32 : 64;         // keys of a tile
    static constexpr int TILE = BN * Tile::RB, STAGE = 2 * TILE, LDS = KW * 2 * STAGE;
    static constexpr int NDT = D / 32;
    static_assert(KW == 1 || (KW - 1) * RW * 32 * D * 4 <= LDS, "room for the other waves' sums");

    struct Place { int len, rows; long tok0; int hk; };

    static __device__ __forceinline__ void copy(const AttnBwdArgs<T>& a, const Place& p, int j0, int last, char* at, int wave, int lane)
    {
        constexpr int RPI = Tile::RPI, ROWS = BN / RW, NI = ROWS / RPI;
        const uint32_t ldk = (uint32_t)(a.f.ld_k * sizeof(T)), ldv = (uint32_t)(a.f.ld_v * sizeof(T));
        const char* k = reinterpret_cast<const char*>(a.f.k) + p.tok0 * (long)ldk + (long)p.hk * Tile::RB;
        const char* v = reinterpret_cast<const char*>(a.f.v) + p.tok0 * (long)ldv + (long)p.hk * Tile::RB;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int first = wave * ROWS + i * RPI, row = first + lane / Tile::PIECES, j = min(j0 + row, last);
            const int piece = ((lane % Tile::PIECES) ^ row_swz<Tile::PIECES>(row)) * 16;
            dma16_from(row_at(k, j, ldk) + piece, at + first * Tile::RB);
            dma16_from(row_at(v, j, ldv) + piece, at + TILE + first * Tile::RB);
        }
    }

    struct Rows { u32x4 q[Tile::NC], g[Tile::NC]; int lo, hi; int lo_least, lo_most, hi_least, hi_most; float c, lse; floatx16 delta; };

    template <bool CAREFUL>
    static __device__ __forceinline__ void block(const Rows& r, floatx16 (&dq)[NDT], const char* k, const char* v, int j0, int last, int row_off, int col_off, int h)
    {
        floatx16 s, ds = r.delta;
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
        for (int c = 0; c < Tile::NC; ++c) mma32x32<T>(s, Tile::row_slot(k, row_off, c), r.q[c]);
#pragma unroll
        for (int c = 0; c < Tile::NC; ++c) mma32x32<T>(ds, Tile::row_slot(v, row_off, c), r.g[c]);
#pragma unroll
        for (int e = 0; e < 16; ++e) ds[e] *= exp2_hw(fmaf(s[e], r.c, -r.lse));
        const bool masked = j0 + 31 > min(r.hi_least, last) || j0 < r.lo_most;
        const int hi = min(r.hi, last) - j0 - 4 * h, lo = r.lo - j0 - 4 * h;
        auto seen = [&](int e) { return acc_row(e) <= hi && acc_row(e) >= lo; };
        if (masked) {
#pragma unroll
            for (int e = 0; e < 16; ++e) ds[e] = seen(e) ? ds[e] : 0.f;
        }
        add_product<CAREFUL, T, D>(dq, k, col_off, ds, masked, seen);
    }

    // Tiles tb .. te - 1: in step i the waves of part kw have tile tb + KW i + kw
    template <bool CAREFUL>
    static __device__ __forceinline__ void pass(const AttnBwdArgs<T>& a, const Place& p, const Rows& r, floatx16 (&dq)[NDT], int tb, int te, int last, char* lds,
                                                int rw, int kw, int lane)
    {
        const int h = lane >> 5, row_off = Tile::row_offset(lane & 31, h), col_off = Tile::col_offset(lane);
        clear(dq);
        char* ring = lds + kw * 2 * STAGE;
        if (tb + kw < te) copy(a, p, (tb + kw) * BN, last, ring, rw, lane);
        int stage = 0;
        for (int t = tb + kw; t - kw < te; t += KW, stage ^= 1) {
            wait_copies_and_barrier();
            if (t + KW < te) copy(a, p, (t + KW) * BN, last, ring + (stage ^ 1) * STAGE, rw, lane);
            if (t >= te) continue;
#pragma unroll 1
            for (int b = 0; b < BN / 32; ++b) {
                const int j0 = t * BN + 32 * b;
                if (j0 > min(r.hi_most, last) || j0 + 31 < r.lo_least) continue;
                const char* k = ring + stage * STAGE + 32 * b * Tile::RB;
                block<CAREFUL>(r, dq, k, k + TILE, j0, last, row_off, col_off, h);
            }
        }
        if constexpr (KW > 1) {                          // [kw - 1][rw][D][32]
            __syncthreads();
            float* part = reinterpret_cast<float*>(lds);
            const int n = lane & 31;
            if (kw > 0) {
#pragma unroll
                for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
                    for (int e = 0; e < 16; ++e) part[(((kw - 1) * RW + rw) * D + 32 * dt + acc_row(e) + 4 * h) * 32 + n] = dq[dt][e];
            }
            __syncthreads();
            if (kw == 0) {
#pragma unroll
                for (int w = 1; w < KW; ++w)
#pragma unroll
                    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
                        for (int e = 0; e < 16; ++e) dq[dt][e] += part[(((w - 1) * RW + rw) * D + 32 * dt + acc_row(e) + 4 * h) * 32 + n];
            }
            __syncthreads();
        }
    }

    // false: something is not finite, nothing was stored (CAREFUL stores whatever comes out)
    template <bool CAREFUL> static __device__ __forceinline__ bool run(const AttnBwdArgs<T>& a, long unit, int thread, char* lds)
    {
        const int lane = thread & 63, wave = __builtin_amdgcn_readfirstlane(thread >> 6);
        const int rw = wave % RW, kw = wave / RW;
        const int n = lane & 31, h = lane >> 5;
        Place p;
        p.hk = (int)(unit % a.f.Hk);
        RowPlace at;
        if (!find_rows<32 * RW>(a.f.seqs, a.f.G, a.f.per, a.f.tiles - 1 - unit / a.f.Hk, lane, &at)) return true;
        p.len = at.len; p.tok0 = at.tok0; p.rows = at.len * a.f.G;
        const int G = a.f.G, window = a.f.window ? min(a.f.window, p.len) : p.len;
        const int row0 = at.tile * 32 * RW, t_first = row0 / G, t_last = min(row0 + 32 * RW - 1, p.rows - 1) / G;
        auto lo_of = [&](int t) { return max(0, t - window + 1) * (int)a.f.causal; };
        auto hi_of = [&](int t) { return a.f.causal ? t : p.len - 1; };
        const int last = hi_of(t_last), tb = lo_of(t_first) / BN, te = last / BN + 1;
        const int w0 = row0 + 32 * rw, row = min(w0 + n, p.rows - 1), t = row / G;
        const long to = (p.tok0 + t) * a.f.H + (long)p.hk * G + (row - t * G);
        Rows r;
        r.c = a.f.scale * kLog2e;
        r.lse = a.row_lse[to];
        float delta = a.row_delta[to];
        {
            const char* q = reinterpret_cast<const char*>(a.f.q + (p.tok0 + t) * a.f.ld_q + (long)(p.hk * G + (row - t * G)) * D);
            const char* g = reinterpret_cast<const char*>(a.d_o + to * D);
#pragma unroll
            for (int c = 0; c < Tile::NC; ++c) { r.q[c] = ld16(q + (2 * c + h) * 16); r.g[c] = ld16(g + (2 * c + h) * 16); }
        }
#pragma unroll
        for (int c = 0; c < Tile::NC; ++c) { settle(r.q[c]); settle(r.g[c]); }
        settle(r.lse);
        settle(delta);
#pragma unroll
        for (int e = 0; e < 16; ++e) r.delta[e] = delta;
        const int u0 = min(w0, p.rows - 1) / G, u1 = min(w0 + 31, p.rows - 1) / G;
        r.lo = lo_of(t); r.lo_least = lo_of(u0); r.lo_most = lo_of(u1);
        r.hi = hi_of(t); r.hi_least = hi_of(u0); r.hi_most = w0 >= p.rows ? -1 : hi_of(u1);
        floatx16 dq[NDT];
        pass<CAREFUL>(a, p, r, dq, tb, te, last, lds, rw, kw, lane);
        if constexpr (!CAREFUL) {
            if (__syncthreads_or(!all_finite(dq))) return false;
        }
        if (kw == 0 && w0 + n < p.rows) store_row<T>(a.dq + to * D, dq, a.f.scale, h);
        return true;
    }
};

// dk and dv of all parts of the query rows, in order
template <typename T> __global__ __launch_bounds__(256) void attn_parts_kernel(const float* part_dk, const float* part_dv, T* dk, T* dv, int parts, long n, long block0)
{
    const long i = ((block0 + blockIdx.x) * 256 + threadIdx.x) * 4;
    if (i >= 2 * n) return;
    const bool second = i >= n;
    const long at = second ? i - n : i;
    const float* p = second ? part_dv : part_dk;
    Floats<4> x = load_vec<float, 4>(p + at);
    for (int s = 1; s < parts; ++s) {
        const Floats<4> y = load_vec<float, 4>(p + s * n + at);
#pragma unroll
        for (int e = 0; e < 4; ++e) x.v[e] += y.v[e];
    }
    store_vec<T, 4>((second ? dv : dk) + at, x);
}

template <typename K, typename A> __device__ __forceinline__ void run_unit(const A& a, long unit, char* lds)
{
    if (!K::template run<false>(a, unit, threadIdx.x, lds)) K::template run<true>(a, unit, thread_again(), lds);
}
template <typename T, int D> __global__ __launch_bounds__(256, sizeof(T) == 4 && D == 128 ? 1 : 2) void attn_dkv_kernel(const AttnBwdArgs<T> a)
{
    extern __shared__ char lds[];
    run_unit<Dkv<T, D>>(a, a.f.unit0 + blockIdx.x, lds);
}
template <typename T, int D> __global__ __launch_bounds__(256, sizeof(T) == 4 ? (D == 128 ? 1 : 2) : D == 64 ? 3 : 2) void attn_dq_kernel(const AttnBwdArgs<T> a)
{
    extern __shared__ char lds[];
    run_unit<Dq<T, D, 4>>(a, a.f.unit0 + blockIdx.x, lds);
}
// Both beside each other, dq's rows in smaller tiles: where neither fills the GPU
template <typename T, int D> __global__ __launch_bounds__(256, sizeof(T) == 4 && D == 128 ? 1 : 2) void attn_bwd_kernel(const AttnBwdArgs<T> a)
{
    extern __shared__ char lds[];
    const long dq = a.f.tiles * a.f.Hk, unit = a.f.unit0 + blockIdx.x;
    if (unit < dq) run_unit<Dq<T, D, 2>>(a, unit, lds);
    else run_unit<Dkv<T, D>>(a, unit - dq, lds);
}

template <typename A, typename K> hipError_t launch_units(A& a, K kernel, int lds, long units, hipStream_t st)
{
    const long most = most_blocks(256);
    for (a.f.unit0 = 0; a.f.unit0 < units; a.f.unit0 += most) {
        kernel<<<dim3((unsigned)(units - a.f.unit0 < most ? units - a.f.unit0 : most)), dim3(256), lds, st>>>(a);
        if (const hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

template <typename T, int D> hipError_t bwd(AttnBwdArgs<T> a, hipStream_t st)
{
    constexpr int PER = 256 / (D / kVec<T> < 16 ? D / kVec<T> : 16);      // rows of a workgroup
    const long most = most_blocks(256), blocks = (a.f.M * a.f.H + PER - 1) / PER;
    for (long b = 0; b < blocks; b += most) {
        attn_rows_kernel<T, D><<<dim3((unsigned)(blocks - b < most ? blocks - b : most)), dim3(256), 0, st>>>(a, b * PER);
        if (const hipError_t e = hipGetLastError()) return e;
    }
    if (a.beside) {
        constexpr int LDS = Dkv<T, D>::LDS > Dq<T, D, 2>::LDS ? Dkv<T, D>::LDS : Dq<T, D, 2>::LDS;
        if (const hipError_t e = launch_units(a, attn_bwd_kernel<T, D>, LDS, (a.key_tiles * a.parts + a.f.tiles) * a.f.Hk, st)) return e;
    } else {
        if (const hipError_t e = launch_units(a, attn_dkv_kernel<T, D>, Dkv<T, D>::LDS, a.key_tiles * a.f.Hk * a.parts, st)) return e;
        if (const hipError_t e = launch_units(a, attn_dq_kernel<T, D>, Dq<T, D, 4>::LDS, a.f.tiles * a.f.Hk, st)) return e;
    }
    if (a.parts > 1) {
        const long n = a.f.M * a.f.Hk * D, sums = (2 * n / 4 + 255) / 256;
        for (long b = 0; b < sums; b += most) {
            attn_parts_kernel<T><<<dim3((unsigned)(sums - b < most ? sums - b : most)), dim3(256), 0, st>>>(a.part_dk, a.part_dv, a.dk, a.dv, a.parts, n, b);
            if (const hipError_t e = hipGetLastError()) return e;
        }
    }
    return hipSuccess;
}

}  // namespace

template <typename T> hipError_t launch_attn_bwd(const AttnBwdArgs<T>& a, int D, hipStream_t st)
{
    if (a.f.tiles == 0) return hipSuccess;
    return D == 64 ? bwd<T, 64>(a, st) : bwd<T, 128>(a, st);
}
template hipError_t launch_attn_bwd<float>(const AttnBwdArgs<float>&, int, hipStream_t);
template hipError_t launch_attn_bwd<bf16_t>(const AttnBwdArgs<bf16_t>&, int, hipStream_t);

}  // namespace kla
