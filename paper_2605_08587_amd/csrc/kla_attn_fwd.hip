// Softmax attention, forward: whole sequences, and new tokens over a paged cache.
//
//     s_ij = scale q_i . k_j over the keys j that query i sees,  m_i >= max_j s_ij - log 2,  p_ij = exp(s_ij - m_i)
//     l_i = sum_j p_ij,  o_i = (sum_j p_ij v_j) / l_i,  lse_i = m_i + log l_i
//
// One pass over the keys: a wave has 32 query rows, and for every tile of keys forms S^T = K Q^T, p, and O^T += V^T p^T on the matrix pipe, with
// the running reference m, the sum l and O^T in registers.  Scores, p, l and O are fp32; p is rounded to the inputs' type where it enters the product with V
// (bf16: 2^-8 of each weight at most, as much as the rounding of the output).  O^T is scaled anew where some row's maximum has grown to more than twice
// exp(m).  (The quotient does not depend on m.  A factor of 2^8 in place of 2 saves 3 % of the time, but then a row's largest weights are rounded like the others
// instead of being powers of two: error of o 2.1e-3 of its norm instead of 1.8e-3, of dq behind it 2.7e-3 instead of 2.4e-3; a factor of 1 is no better than 2.)
//
// bf16, D = 128, 16 heads over 4, 16384 tokens: 1.06 PFLOP/s, 8192 tokens both ways 1.04, where a matrix product of 8192^3 reaches 1.39 on the same card; D = 64: 0.87,
// bound by the exponentials and the other 4.5 instructions per score.  Tried and left: scores formed a tile ahead and interleaved with this tile's
// exponentials (two workgroups to a CU do as much: 3 to 10 % slower with a barrier per 32 keys), eight waves to a tile (1 %), tiles of 64 rows
// (no gain at any size), priorities around the products (none), two groups of four waves half a tile apart, so that one's products stand beside the
// other's exponentials (none; D = 64: 10 % slower), three stages of keys (D = 64: 6 % slower).
#include "kla_attn.hpp"

namespace kla {

namespace {

// RW waves of 32 rows each that share tiles of keys (KW = 1), or KW waves that divide the keys of 32 rows (RW = 1).
template <typename T, int D, int RW, int KW, bool PAGED> struct Fwd {
    static_assert(RW == 1 || KW == 1, "one way to share the work");
    using Tile = RowTile<T, D>;
    static constexpr int W = RW * KW;
    static constexpr int BN = sizeof(T) == 4 || KW > 1 ? 32 : 64;         // keys of a tile
    static constexpr int KT = BN / 32;
    static constexpr int TILE = BN * Tile::RB;
    static constexpr int STAGE = 2 * TILE;
    static constexpr int LDS = KW * 2 * STAGE;
    static constexpr int NDT = D / 32;
    static_assert(KW == 1 || KW * (D + 2) * 32 * 4 <= LDS, "room for the waves' results");

    struct Keys { int n; int cached; int total; long tok0; int hk; };

    static constexpr int ROWS = BN / RW;                 // of a tile that one wave copies
    static constexpr int GROUPS = (ROWS + 15) / 16;      // of rows of one page: pages begin at multiples of 16 keys
    // The table's entries for this wave's rows of the tile at j0, lane g that of group g.  They are asked for a tile ahead of the copies that need them.
    static __device__ __forceinline__ int entries(const AttnArgs<T>& a, const Keys& k, int j0, int last, int wave, int lane)
    {
        if (!PAGED) return 0;
        // (one that is there in any case: no condition, and no move of the value, stands between the load and the wait for it)
        const int j = max(min(min(j0 + wave * ROWS + 16 * (lane % GROUPS), last), k.cached - 1), 0);
        return a.table[k.n * a.ld_table + (j >> a.page_shift)];
    }
    // Copies of the K and V rows of keys j0 .. j0 + BN - 1 (those beyond `last` repeat it) by the waves of a team
    static __device__ __forceinline__ void copy(const AttnArgs<T>& a, const Keys& k, int j0, int last, int ids, char* stage, int wave, int lane)
    {
        constexpr int RPI = Tile::RPI, NI = ROWS / RPI;
        static_assert(ROWS % RPI == 0 && 16 % RPI == 0, "whole copy instructions");
        // (strides at most 2^26 bytes: 63 of them fit 32 bits)
        const uint32_t ldk = (uint32_t)(a.ld_k * sizeof(T)), ldv = (uint32_t)(a.ld_v * sizeof(T));
        const char* kn = reinterpret_cast<const char*>(a.k) + k.tok0 * (long)ldk + (long)k.hk * Tile::RB;
        const char* vn = reinterpret_cast<const char*>(a.v) + k.tok0 * (long)ldv + (long)k.hk * Tile::RB;
        long pages[GROUPS];                              // where this key head's rows of a group's page begin
#pragma unroll
        for (int g = 0; g < GROUPS && PAGED; ++g)
            pages[g] = (((long)min(max(__builtin_amdgcn_readlane(ids, g), 0), a.n_pages - 1) * a.Hk + k.hk) << a.page_shift) * Tile::RB;
        // Cached keys throughout: an instruction's rows stand behind each other, from a place that the wave has in common.  (With an address formed for every
        // lane these copies are a fifth of the loop's vector instructions: 254 us instead of 218 for four sequences of 300 to 518 new tokens over 4126 to 13917.)
        if (PAGED && j0 + BN - 1 <= min(last, k.cached - 1)) {
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const int first = wave * ROWS + i * RPI, row = first + lane / Tile::PIECES;
                const int off = lane / Tile::PIECES * Tile::RB + ((lane % Tile::PIECES) ^ row_swz<Tile::PIECES>(row)) * 16;
                const long at = pages[(i * RPI) / 16] + (long)((j0 + first) & ((1 << a.page_shift) - 1)) * Tile::RB;
                dma16(reinterpret_cast<const char*>(a.k_cache) + at, off, stage + first * Tile::RB);
                dma16(reinterpret_cast<const char*>(a.v_cache) + at, off, stage + first * Tile::RB + TILE);
            }
            return;
        }
        // Keys that are all there: the same, rows a stride apart.  (8 multiplications of 64 bits less for each tile: 4 x 1500 tokens both ways, heads of 64, 39.5 -> 38.1 us.)
        if (!PAGED && j0 + BN - 1 <= last) {
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const int first = wave * ROWS + i * RPI, row = first + lane / Tile::PIECES;
                const int piece = ((lane % Tile::PIECES) ^ row_swz<Tile::PIECES>(row)) * 16;
                dma16(row_at(kn, j0 + first, ldk), (int)(lane / Tile::PIECES * ldk) + piece, stage + first * Tile::RB);
                dma16(row_at(vn, j0 + first, ldv), (int)(lane / Tile::PIECES * ldv) + piece, stage + first * Tile::RB + TILE);
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int first = wave * ROWS + i * RPI, row = first + lane / Tile::PIECES;
            const int piece = ((lane % Tile::PIECES) ^ row_swz<Tile::PIECES>(row)) * 16;
            char* to = stage + first * Tile::RB;
            if constexpr (PAGED) {
                const int j = min(j0 + row, last), fresh = max(j - k.cached, 0);
                const bool old = j < k.cached;
                const long at = pages[(i * RPI) / 16] + (long)(j & ((1 << a.page_shift) - 1)) * Tile::RB;
                dma16_from((old ? reinterpret_cast<const char*>(a.k_cache) + at : row_at(kn, fresh, ldk)) + piece, to);
                dma16_from((old ? reinterpret_cast<const char*>(a.v_cache) + at : row_at(vn, fresh, ldv)) + piece, to + TILE);
            } else {
                const int j = min(j0 + row, last);
                dma16_from(row_at(kn, j, ldk) + piece, to);
                dma16_from(row_at(vn, j, ldv) + piece, to + TILE);
            }
        }
    }

    // The new tokens whose first row lies in this tile go into their pages.
    static __device__ __forceinline__ void store_new(const AttnArgs<T>& a, const Keys& k, int t0, int t1, int thread)
    {
        constexpr int P = Tile::PIECES;
        for (int i = thread; i < (t1 - t0) * P; i += 64 * W) {
            const int t = t0 + i / P, pos = k.cached + t;
            const long page = (long)pos >> a.page_shift;
            if (page >= a.max_pages) continue;
            const int id = a.table[k.n * a.ld_table + page];
            if (id < 0 || id >= a.n_pages) continue;
            const long at = (((((long)id * a.Hk + k.hk) << a.page_shift) + (pos & ((1 << a.page_shift) - 1))) * Tile::RB) + (i % P) * 16;
            const long from = (long)k.hk * Tile::RB + (i % P) * 16;
            st16(reinterpret_cast<char*>(a.k_cache) + at, ld16(reinterpret_cast<const char*>(a.k) + (k.tok0 + t) * a.ld_k * (long)sizeof(T) + from));
            st16(reinterpret_cast<char*>(a.v_cache) + at, ld16(reinterpret_cast<const char*>(a.v) + (k.tok0 + t) * a.ld_v * (long)sizeof(T) + from));
        }
    }

    struct Rows {                                        // a wave's 32 query rows, lane = row
        u32x4 q[Tile::NC];
        int lo, hi;                                      // first and last key that this lane's row sees
        int lo_most, hi_least;                           // the largest and smallest of the wave's
        int lo_least, hi_most;
        float c;                                         // scores in units of log 2
    };
    struct State { floatx16 o[NDT]; float m, mc, l; };

    template <bool CAREFUL>
    static __device__ __forceinline__ void tile(const Rows& r, State& s, const char* stage, int j0, int last, int row_off, int col_off, int h)
    {
        floatx16 st[KT];
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
#pragma unroll
            for (int e = 0; e < 16; ++e) st[kt][e] = 0.f;
#pragma unroll
            for (int c = 0; c < Tile::NC; ++c) mma32x32<T>(st[kt], Tile::row_slot(stage + 32 * kt * Tile::RB, row_off, c), r.q[c]);
        }
        const bool masked = j0 + BN - 1 > min(r.hi_least, last) || j0 < r.lo_most;
        const int hi = min(r.hi, last) - j0 - 4 * h, lo = r.lo - j0 - 4 * h;
        if (masked) {
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int j = 32 * kt + acc_row(e);
                    st[kt][e] = j <= hi && j >= lo ? st[kt][e] : -__builtin_inff();
                }
        }
        float top = st[0][0];
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, st[kt][e]);
        top = halves_max(top);
        // (nothing seen so far: m is -inf and any score above it makes a reference)
        if (__any(top * r.c > s.m * r.c + 1.f)) {
            const float m = fmaxf(s.m, top), mc = m == -__builtin_inff() ? 0.f : m * r.c;
            // From references as they were rounded: exactly 1 for a row whose own has not moved.  (Never above 1, also where nothing was seen so far: sums of zero.)
            const float f = exp2_hw(fminf(s.mc - mc, 0.f));
            s.m = m; s.mc = mc;
            s.l *= f;
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
                for (int e = 0; e < 16; ++e) s.o[dt][e] *= f;
        }
        float l[2] = {0.f, 0.f};
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                st[kt][e] = exp2_hw(fmaf(st[kt][e], r.c, -s.mc));
                l[e & 1] += st[kt][e];
            }
        s.l += l[0] + l[1];
        static_for<KT>([&](auto kt) {
            add_product<CAREFUL, T, D>(s.o, stage + TILE + 32 * kt * Tile::RB, col_off, st[kt], masked,
                                       [&](int e) { return 32 * kt + acc_row(e) <= hi && 32 * kt + acc_row(e) >= lo; });
        });
    }

    // Tiles tb .. te - 1 of keys, from j_first on, for one wave's rows
    template <bool CAREFUL>
    static __device__ __forceinline__ void pass(const AttnArgs<T>& a, const Keys& k, const Rows& r, State& s, int j_first, int tb, int te, int last, char* ring,
                                                int wave, int lane)
    {
        const int h = lane >> 5, row_off = Tile::row_offset(lane & 31, h), col_off = Tile::col_offset(lane);
        s.m = -__builtin_inff();
        s.mc = s.l = 0.f;
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
            for (int e = 0; e < 16; ++e) s.o[dt][e] = 0.f;
        const int cw = KW > 1 ? 0 : wave;
        int ids = 0;
        if (tb < te) {
            copy(a, k, j_first + tb * BN, last, entries(a, k, j_first + tb * BN, last, cw, lane), ring, cw, lane);
            ids = entries(a, k, j_first + (tb + 1) * BN, last, cw, lane);
        }
        for (int t = tb; t < te; ++t) {
            // the copies of this tile have landed, and the other stage is no longer read
            if constexpr (PAGED) asm volatile("" : "+v"(ids));       // (awaited with the copies, not behind the ones that follow)
            if constexpr (RW > 1) wait_copies_and_barrier();
            else wait_copies();
            if constexpr (RW > 1 || !PAGED) keep_whole(s.o);
            const int j0 = j_first + t * BN;
            char* stage = ring + ((t - tb) & 1) * STAGE;
            if (t + 1 < te) copy(a, k, j0 + BN, last, ids, ring + ((t - tb + 1) & 1) * STAGE, cw, lane);
            ids = entries(a, k, j0 + 2 * BN, last, cw, lane);
            if (j0 > r.hi_most || j0 + BN - 1 < r.lo_least) continue;
            tile<CAREFUL>(r, s, stage, j0, last, row_off, col_off, h);
        }
        s.l = halves_sum(s.l);
    }

    static __device__ __forceinline__ bool all_finite(const State& s)
    {
        bool f = true;
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) f = f && finite(s.o[dt]);
        return f;
    }

    // 4 consecutive features of one row
    static __device__ __forceinline__ void store4(const AttnArgs<T>& a, int split, int parts, long row, int d, float x0, float x1, float x2, float x3)
    {
        const Floats<4> x = {{x0, x1, x2, x3}};
        if (parts > 1) store_vec<float, 4>(a.part_o + ((long)split * a.M * a.H + row) * D + d, x);
        else {
            store_vec<T, 4>(a.o + row * D + d, x);
            if constexpr (sizeof(T) == 2 && !PAGED) {
                if (a.rest) {
                    Floats<4> y;
#pragma unroll
                    for (int e = 0; e < 4; ++e) y.v[e] = x.v[e] - to_float(rounded<T>(x.v[e]));
                    store_vec<T, 4>(a.rest + row * D + d, y);
                }
            }
        }
    }
    // l = 0: scores that are all -inf, whose quotient is a NaN, or no key of a part that this row sees
    static __device__ __forceinline__ float inverse(int parts, float l) { return parts > 1 && l == 0.f ? 0.f : 1.f / l; }
    static __device__ __forceinline__ void store_lse(const AttnArgs<T>& a, int split, int parts, long row, float m, float l)
    {
        const float lse = m + __log2f(l);                // base 2
        if (parts > 1) a.part_lse[(long)split * a.M * a.H + row] = lse;
        else if (a.lse) a.lse[row] = lse * kLn2;
    }

    // false: something is not finite, nothing was stored (CAREFUL stores whatever comes out)
    template <bool CAREFUL> static __device__ __forceinline__ bool run(const AttnArgs<T>& a, int thread, char* lds)
    {
        const int lane = thread & 63, wave = __builtin_amdgcn_readfirstlane(thread >> 6);
        const int n = lane & 31, h = lane >> 5;
        // heaviest tiles (the last ones of their sequences) first; the parts of a tile and the key heads beside each other
        const long unit = a.unit0 + blockIdx.x;
        const int split = (int)(unit % a.splits);
        Keys k;
        k.hk = wave_uniform((int)(unit / a.splits % a.Hk));
        RowPlace at;
        if (!find_rows<32 * RW>(a.seqs, a.G, a.per, a.tiles - 1 - unit / a.splits / a.Hk, lane, &at)) return true;
        k.n = wave_uniform(at.n); k.tok0 = wave_uniform(at.tok0);
        k.cached = 0;
        if constexpr (PAGED) k.cached = (int)min((long)max(a.cached[at.n], 0), (long)a.max_pages << a.page_shift);
        k.total = k.cached + at.len;
        const int rows = at.len * a.G, row0 = at.tile * 32 * RW;
        const int t_first = row0 / a.G, t_last = min(row0 + 32 * RW - 1, rows - 1) / a.G;
        // keys of the tile's rows, and this part of them
        const int k_first = a.window ? max(0, k.cached + t_first - a.window + 1) : 0, k_last = wave_uniform(a.causal ? k.cached + t_last : k.total - 1);
        const int j_first = wave_uniform(k_first / BN * BN), nt = (k_last - j_first) / BN + 1;
        // as many parts as leave a.chunk keys to each, `splits` at most
        const int part = max(a.chunk / BN, (nt + a.splits - 1) / a.splits), s0 = (int)min((long)nt, (long)split * part), s1 = min(nt, s0 + part);
        int tb = s0, te = s1;
        if constexpr (KW > 1) {
            tb = s0 + (int)((long)(s1 - s0) * wave / KW);
            te = s0 + (int)((long)(s1 - s0) * (wave + 1) / KW);
        }
        const long out0 = k.tok0 * a.H + (long)k.hk * a.G;
        auto out_row = [&](int rr) { const int tt = rr / a.G; return out0 + (long)tt * a.H + (rr - tt * a.G); };
        if (s0 >= s1) return true;                       // (the first part is never empty)
        tb = wave_uniform(tb);
        te = wave_uniform(te);
        const int parts = (nt + part - 1) / part;
        if (a.splits > 1 && split == 0 && !CAREFUL)
            for (int i = thread; i < 32 * RW && row0 + i < rows; i += 64 * W) a.part_count[out_row(row0 + i)] = parts;
        // this wave's rows
        const int w0 = row0 + (KW > 1 ? 0 : 32 * wave), row = min(w0 + n, rows - 1);
        const int t = row / a.G, head = k.hk * a.G + (row - t * a.G);
        Rows r;
        r.c = a.scale * kLog2e;
        {
            const char* q = reinterpret_cast<const char*>(a.q + (k.tok0 + t) * a.ld_q + (long)head * D);
#pragma unroll
            for (int c = 0; c < Tile::NC; ++c) r.q[c] = ld16(q + (2 * c + h) * 16);
        }
        const int tw0 = min(w0, rows - 1) / a.G, tw1 = min(w0 + 31, rows - 1) / a.G;
        r.lo = a.window ? max(0, k.cached + t - a.window + 1) : 0;
        r.lo_least = a.window ? max(0, k.cached + tw0 - a.window + 1) : 0;
        r.lo_most = a.window ? max(0, k.cached + tw1 - a.window + 1) : 0;
        r.hi = a.causal ? k.cached + t : k.total - 1;
        r.hi_least = a.causal ? k.cached + tw0 : k.total - 1;
        r.hi_most = w0 >= rows ? -1 : a.causal ? k.cached + tw1 : k.total - 1;       // (no rows of its own: every tile is passed over)
        if constexpr (PAGED) {
            if (split == 0 && !CAREFUL) {                    // tokens whose first row lies in this tile
                const int u0 = (row0 + a.G - 1) / a.G, u1 = min(at.len, (row0 + 32 * RW + a.G - 1) / a.G);
                store_new(a, k, u0, u1, thread);
            }
        }
#pragma unroll
        for (int c = 0; c < Tile::NC; ++c) settle(r.q[c]);
        State s;
        char* ring = lds + (KW > 1 ? wave * 2 * STAGE : 0);
        pass<CAREFUL>(a, k, r, s, j_first, tb, te, k_last, ring, wave, lane);
        if constexpr (!CAREFUL) {
            if (__syncthreads_or(!all_finite(s))) return false;
        }
        const float mc = s.m == -__builtin_inff() ? s.m : s.mc;
        if constexpr (KW == 1) {
            if (w0 + n < rows) {
                const long to = out_row(row);
                const float f = inverse(parts, s.l);
#pragma unroll
                for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        store4(a, split, parts, to, 32 * dt + 8 * i + 4 * h, s.o[dt][4 * i] * f, s.o[dt][4 * i + 1] * f, s.o[dt][4 * i + 2] * f, s.o[dt][4 * i + 3] * f);
                if (h == 0) store_lse(a, split, parts, to, mc, s.l);
            }
        } else {
            // the waves' parts, [wave][D + 2][32]: O^T, reference, sum
            __syncthreads();
            float* part = reinterpret_cast<float*>(lds);
            constexpr int PW = (D + 2) * 32;
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
                for (int e = 0; e < 16; ++e) part[wave * PW + (32 * dt + acc_row(e) + 4 * h) * 32 + n] = s.o[dt][e];
            if (h == 0) {
                part[wave * PW + D * 32 + n] = mc;
                part[wave * PW + (D + 1) * 32 + n] = s.l;
            }
            __syncthreads();
            const int rr = row0 + n, d0 = (thread >> 5) * (D / (2 * KW));
            if (rr < rows) {
                float m = -__builtin_inff(), l = 0.f, w[KW];
#pragma unroll
                for (int i = 0; i < KW; ++i) m = fmaxf(m, part[i * PW + D * 32 + n]);
#pragma unroll
                for (int i = 0; i < KW; ++i) {
                    w[i] = m == -__builtin_inff() ? 0.f : exp2_hw(part[i * PW + D * 32 + n] - m);
                    l = fmaf(w[i], part[i * PW + (D + 1) * 32 + n], l);
                }
                const long to = out_row(rr);
                const float f = inverse(parts, l);
#pragma unroll
                for (int d = 0; d < D / (2 * KW); d += 4) {
                    float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int i = 0; i < KW; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[e] = fmaf(w[i], part[i * PW + (d0 + d + e) * 32 + n], x[e]);
                    store4(a, split, parts, to, d0 + d, x[0] * f, x[1] * f, x[2] * f, x[3] * f);
                }
                if (thread < 32) store_lse(a, split, parts, to, m, l);
            }
        }
        return true;
    }
};

template <typename T, int D, int RW, int KW, bool PAGED>
__global__ __launch_bounds__(64 * RW * KW, KW > 1 ? (D == 64 && sizeof(T) == 2 ? 2 : 1) : D == 64 ? 3 : 2) void attn_fwd_kernel(const AttnArgs<T> a)
{
    extern __shared__ char lds[];
    using F = Fwd<T, D, RW, KW, PAGED>;
    if (!F::template run<false>(a, threadIdx.x, lds)) F::template run<true>(a, thread_again(), lds);
}

template <typename T, int D, int RW, int KW, bool PAGED> hipError_t launch(AttnArgs<T> a, hipStream_t st)
{
    using F = Fwd<T, D, RW, KW, PAGED>;
    const auto kernel = attn_fwd_kernel<T, D, RW, KW, PAGED>;
    const long units = a.tiles * a.Hk * a.splits, most = most_blocks(64 * F::W);
    for (a.unit0 = 0; a.unit0 < units; a.unit0 += most) {
        kernel<<<dim3((unsigned)(units - a.unit0 < most ? units - a.unit0 : most)), dim3(64 * F::W), F::LDS, st>>>(a);
        if (const hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

// The parts of a row joined: sum_s 2^(lse_s - M) o_s / sum_s 2^(lse_s - M).  A row has D / 4 threads for its features times SG for its parts, so that all
// of a row's parts are on their way at once (64 at most: lane s of every wave has part s's weight).  3.6 us for 16 rows, of which most is the launch
// and three trips to memory behind each other, 17 us for 26000 rows of 128.
template <typename T, int D, int SG> __global__ __launch_bounds__(256) void attn_join_kernel(const AttnArgs<T> a, long row0)
{
    constexpr int TPR = D / 4, ROWS = 256 / (TPR * SG), BATCH = 8;
    __shared__ float4 part[256];
    const long rows = a.M * a.H;
    const int lane = threadIdx.x & 63, quad = threadIdx.x % TPR, group = threadIdx.x / TPR % SG;
    static_assert(TPR * SG % 64 == 0, "a wave has one row");
    const long row = row0 + (long)blockIdx.x * ROWS + threadIdx.x / (TPR * SG);
    const bool here = row < rows;
    const int parts = here ? a.part_count[row] : 0;
    float lse = -__builtin_inff();
    if (here && lane < a.splits) lse = a.part_lse[lane * rows + row];
    if (lane >= parts) lse = -__builtin_inff();          // (nothing was written there)
    float m = lse;
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) m = fmaxf(m, __shfl_xor(m, d, 64));
    const float w = lse == -__builtin_inff() ? 0.f : exp2_hw(lse - m);          // (a NaN among parts of -inf, which m does not show, stays one)
    const float l = wave_sum(w);
    Floats<4> x = {{0.f, 0.f, 0.f, 0.f}};
    if (parts > 1)                                       // (one part is the result, and stands in o)
        for (int s0 = 0; s0 < parts; s0 += SG * BATCH) {
            Floats<4> o[BATCH];
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                const int s = s0 + group + i * SG;
                o[i] = Floats<4>{{0.f, 0.f, 0.f, 0.f}};
                if (s < parts) o[i] = load_vec<float, 4>(a.part_o + (s * rows + row) * D + 4 * quad);
            }
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                const float ws = __shfl(w, min(s0 + group + i * SG, 63), 64);       // (0 from `parts` on)
#pragma unroll
                for (int e = 0; e < 4; ++e) x.v[e] = fmaf(ws, o[i].v[e], x.v[e]);
            }
        }
    if constexpr (SG > 1) {
        part[threadIdx.x] = make_float4(x.v[0], x.v[1], x.v[2], x.v[3]);
        __syncthreads();
        if (group) return;
#pragma unroll
        for (int g = 1; g < SG; ++g) {
            const float4 y = part[threadIdx.x + g * TPR];
            x.v[0] += y.x; x.v[1] += y.y; x.v[2] += y.z; x.v[3] += y.w;
        }
    }
    if (parts < 2) return;
    const float f = 1.f / l;                             // (scores that are all -inf: a NaN)
#pragma unroll
    for (int e = 0; e < 4; ++e) x.v[e] *= f;
    store_vec<T, 4>(a.o + row * D + 4 * quad, x);
    if (a.lse && quad == 0) a.lse[row] = (m + __log2f(l)) * kLn2;
}

template <typename T, int D, int SG> hipError_t join(const AttnArgs<T>& a, hipStream_t st)
{
    constexpr long per = 256 / (D / 4 * SG);
    const long blocks = (a.M * a.H + per - 1) / per, most = most_blocks(256);
    for (long b = 0; b < blocks; b += most) {
        attn_join_kernel<T, D, SG><<<dim3((unsigned)(blocks - b < most ? blocks - b : most)), dim3(256), 0, st>>>(a, b * per);
        if (const hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

template <typename T, int D> hipError_t pick(const AttnArgs<T>& a, const AttnPlan& p, bool paged, hipStream_t st)
{
    constexpr int KW = sizeof(T) == 4 && D == 128 ? 2 : 4;
    if (p.rows == 32) return paged ? launch<T, D, 1, KW, true>(a, st) : launch<T, D, 1, KW, false>(a, st);
    return paged ? launch<T, D, 4, 1, true>(a, st) : launch<T, D, 4, 1, false>(a, st);
}

}  // namespace

template <typename T> hipError_t launch_attn_fwd(const AttnArgs<T>& a, int D, const AttnPlan& p, bool paged, hipStream_t st)
{
    if (a.tiles == 0) return hipSuccess;
    return D == 64 ? pick<T, 64>(a, p, paged, st) : pick<T, 128>(a, p, paged, st);
}
template <typename T> hipError_t launch_attn_join(const AttnArgs<T>& a, int D, hipStream_t st)
{
    if (a.splits > 8) return D == 64 ? join<T, 64, 8>(a, st) : join<T, 128, 8>(a, st);
    return D == 64 ? join<T, 64, 4>(a, st) : join<T, 128, 2>(a, st);
}

template hipError_t launch_attn_fwd<float>(const AttnArgs<float>&, int, const AttnPlan&, bool, hipStream_t);
template hipError_t launch_attn_fwd<bf16_t>(const AttnArgs<bf16_t>&, int, const AttnPlan&, bool, hipStream_t);
template hipError_t launch_attn_join<float>(const AttnArgs<float>&, int, hipStream_t);
template hipError_t launch_attn_join<bf16_t>(const AttnArgs<bf16_t>&, int, hipStream_t);

}  // namespace kla
