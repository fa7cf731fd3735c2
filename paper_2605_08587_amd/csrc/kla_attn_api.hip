// C ABI of softmax attention (declared in include/kla.h): argument validation, how the work is cut, workspace carving and launch sequencing.  No
// allocation, no state, nothing read from the environment; everything is enqueued on the caller's stream.
#include <limits.h>
#include <math.h>
#include <type_traits>

#include "kla_args.hpp"
#include "kla_attn.hpp"

namespace {

using kla::bf16_t;

static_assert(KLA_ATTN_CAUSAL == (int)kla::kAttnCausal, "option bits");

constexpr int kMaxAttnRows = 1 << 30;                    // tokens times query heads of a key head, and positions (32-bit numbers)
constexpr int kMaxAttnGroup = 1 << 16;                   // query heads of a key head
constexpr long kMaxAttnStride = 1L << 24;                // elements from one token to the next

struct AttnSizes { int N, T, H, Hk, D; };
int attn_sizes(const AttnSizes& z, int dt)
{
    if (!dt_ok(dt)) return KLA_ERR_DTYPE;
    if (z.N < 0 || z.T < 0 || z.H <= 0 || z.Hk <= 0 || z.H % z.Hk || z.H / z.Hk > kMaxAttnGroup || (z.D != 64 && z.D != 128) || (long)z.H * z.D > kMaxAttnStride ||
        (long)z.T * (z.H / z.Hk) > kMaxAttnRows)
        return KLA_ERR_SHAPE;
    return KLA_OK;
}
int attn_check(const AttnSizes& z, long ld_q, long ld_k, long ld_v, float scale, int window, int dt)
{
    if (const int e = attn_sizes(z, dt)) return e;
    if (ld_q < (long)z.H * z.D || ld_k < (long)z.Hk * z.D || ld_v < (long)z.Hk * z.D || ld_q > kMaxAttnStride || ld_k > kMaxAttnStride || ld_v > kMaxAttnStride ||
        !(scale > 0.f) || isinf(scale * kla::kLog2e) || window < 0)
        return KLA_ERR_SHAPE;
    const long vec = 16 / (long)elem_bytes(dt);
    return ld_q % vec || ld_k % vec || ld_v % vec ? KLA_ERR_ALIGN : KLA_OK;
}
// Tiles of `rows` query rows of one key head
long attn_tiles(const kla::Seqs& s, const int32_t* cu_host, int G, int rows)
{
    if (!s.cu) return ((long)s.T * G + rows - 1) / rows * s.n_seq;
    long tiles = 0;
    for (int i = 0; i < s.n_seq; ++i) tiles += ((long)(cu_host[i + 1] - cu_host[i]) * G + rows - 1) / rows;
    return tiles;
}
int longest(const kla::Seqs& s, const int32_t* cu_host)
{
    if (!s.cu) return s.n_seq ? s.T : 0;
    int most = 0;
    for (int i = 0; i < s.n_seq; ++i) most = cu_host[i + 1] - cu_host[i] > most ? cu_host[i + 1] - cu_host[i] : most;
    return most;
}
// The forward over whole sequences: four waves of 32 rows each to a workgroup, which share every tile of keys, unless that gives too few workgroups
// for the CUs; then four waves share 32 rows and divide the keys.
kla::AttnPlan attn_plan(const kla::Seqs& s, const int32_t* cu_host, int G, int Hk, int D)
{
    const long units = attn_tiles(s, cu_host, G, 128) * Hk;
    return {units >= (D == 64 ? 320 : 256) ? 128 : 32, 1, 128};
}
// New tokens over a cache: a row sees up to `span` keys.
kla::AttnPlan extend_plan(const kla::Seqs& s, const int32_t* cu_host, int G, int Hk, int max_len, int window)
{
    kla::AttnPlan p = {128, 1, 128};
    const int most_new = longest(s, cu_host);
    const long span = window && window + (long)most_new < max_len ? window + most_new : max_len;
    long units = attn_tiles(s, cu_host, G, 128) * Hk;
    // Rows in tiles of 32 with their keys divided among the waves, too, where larger tiles in parts of 256 keys would leave CUs idle (fp32, three
    // sequences of 54 to 160 new tokens over 115 to 852, 8 heads over 2 of 64: 31 us a call in tiles of 128, 20 of 32; bf16, 16 tokens over 1000 17 and 12 us).
    if ((long)most_new * G <= 32 || units * ((span + 255) / 256) < 256) {
        p.rows = 32;
        units = attn_tiles(s, cu_host, G, 32) * Hk;
    }
    if (units == 0) return p;
    // Single tokens and drafts: a workgroup takes about 3 us until its first keys are there, one after the other on a CU (its tiles take all of the LDS), so
    // that few keys to a part cost bandwidth; below one workgroup for each CU parts of 128 keys still gain.  (bf16, D = 128: 32 tokens over 4000 to 32000
    // keys, 4 key heads: parts for 512, 1024 and 2048 workgroups 242, 228 and 230 us; 16 x 5 tokens over 2000 to 8000: 47, 57 and 76 us; one token
    // over 4096: parts of 128 and 256 keys 11.1 and 12.4 us.)  More rows: two workgroups to a CU; parts are written and read in fp32 (four
    // sequences of 300 to 518 new tokens over 4126 to 13917: for 256, 512, 1024 and 2048 workgroups 220, 215, 233 and 261 us).
    if (p.rows == 32) {
        const long fill = (256 + units - 1) / units, most = (span + 1023) / 1024;
        long want = (1024 + units - 1) / units;
        if (want > most) want = most > fill ? most : fill;
        p.chunk = 128;
        p.splits = (int)(want < (span + 127) / 128 ? want : (span + 127) / 128);
    } else {
        p.chunk = 256;
        const long want = (512 + units - 1) / units, most = (span + 255) / 256;
        p.splits = (int)(want < most ? want : most);
    }
    if (p.splits > 64) p.splits = 64;
    if (p.splits < 1) p.splits = 1;
    return p;
}
template <typename T>
kla::AttnArgs<T> attn_args(const void* q, long ld_q, const void* k, long ld_k, const void* v, long ld_v, void* o, float* lse, const kla::Seqs& s, long M,
                           const AttnSizes& z, float scale, int window, unsigned opts)
{
    kla::AttnArgs<T> a = {};
    a.q = static_cast<const T*>(q); a.ld_q = ld_q; a.k = static_cast<const T*>(k); a.ld_k = ld_k; a.v = static_cast<const T*>(v); a.ld_v = ld_v;
    a.o = static_cast<T*>(o); a.lse = lse; a.seqs = s; a.H = z.H; a.Hk = z.Hk; a.G = z.H / z.Hk;
    a.scale = scale; a.window = window; a.causal = opts & KLA_ATTN_CAUSAL; a.splits = 1; a.chunk = 128; a.M = M;
    return a;
}
// Backward: below so many tiles of 128 query rows (two for each CU) dk, dv and dq run beside each other in one launch, dq's tiles half as large and with their keys
// in two parts.  bf16: 2048 tokens, 8 heads of 64 and 128 76 -> 44 and 117 -> 66 us; at 768 tiles 238 and 399 us apart, 248 and 422 beside.  fp32: 777
// tokens, 8 heads over 2 of 64 132 -> 56 us, 2048 tokens and 8 of 128 571 -> 315 us.
constexpr long kAttnBeside = 512;
// The query rows that see a tile of 128 keys are taken in parts where there are fewer than two such tiles for each CU.  (More parts cost more in sums
// than they even out: bf16, D = 128, 4096 tokens, 8 heads, 3 sequences 399 us whole, 471 in two parts.)
int attn_bwd_parts(const kla::Seqs& s, const int32_t* cu_host, int G, int Hk)
{
    const long units = attn_tiles(s, cu_host, 1, 128) * Hk;
    if (units == 0 || units >= 512) return 1;
    const long want = (512 + units - 1) / units, most = ((long)longest(s, cu_host) * G + 255) / 256;
    const long parts = want < most ? want : most;
    return (int)(parts < 1 ? 1 : parts > 16 ? 16 : parts);
}
struct BwdWork { float *row_lse, *row_delta, *part_dk, *part_dv; size_t bytes; };
BwdWork bwd_work(char* base, int parts, long M, const AttnSizes& z)
{
    Carve c{base};
    BwdWork w = {};
    w.row_lse = c.take<float>((size_t)M * z.H);
    w.row_delta = c.take<float>((size_t)M * z.H);
    if (parts > 1) {
        w.part_dk = c.take<float>((size_t)parts * M * z.Hk * z.D);
        w.part_dv = c.take<float>((size_t)parts * M * z.Hk * z.D);
    }
    w.bytes = c.used;
    return w;
}
struct ExtendWork { float *part_o, *part_lse; int* part_count; size_t bytes; };
ExtendWork extend_work(char* base, const kla::AttnPlan& p, long M, int H, int D)
{
    Carve c{base};
    ExtendWork w = {};
    if (p.splits > 1) {
        w.part_o = c.take<float>((size_t)p.splits * M * H * D);
        w.part_lse = c.take<float>((size_t)p.splits * M * H);
        w.part_count = c.take<int>((size_t)M * H);
    }
    w.bytes = c.used;
    return w;
}

}  // namespace

extern "C" {

int kla_attn_fwd(const void* q, long ld_q, const void* k, long ld_k, const void* v, long ld_v, void* o, float* lse, void* rest, float scale, int window,
                 const int32_t* cu_seqlens_dev, const int32_t* cu_seqlens_host, int n_seq, int N, int T, int H, int Hk, int D, kla_dtype dt, void* hip_stream,
                 unsigned opts)
{
    kla::Seqs s;
    long M;
    const AttnSizes z = {N, T, H, Hk, D};
    if (const int e = attn_check(z, ld_q, ld_k, ld_v, scale, window, dt)) return e;
    if ((opts & ~(unsigned)KLA_ATTN_CAUSAL) || (window && !(opts & KLA_ATTN_CAUSAL))) return KLA_ERR_SHAPE;
    if (const int e = take_seqs(cu_seqlens_dev, cu_seqlens_host, n_seq, N, T, &s, &M)) return e;
    if (M > 0 && (!q || !k || !v || !o)) return KLA_ERR_NULL;
    if (M > 0 && (o == q || o == k || o == v)) return KLA_ERR_SHAPE;                   // (other workgroups still read them)
    if (rest && dt != KLA_BF16) return KLA_ERR_DTYPE;
    if (rest && (rest == q || rest == k || rest == v || rest == o)) return KLA_ERR_SHAPE;
    if (!aligned(16, {q, k, v, o, rest}) || !aligned(4, {lse})) return KLA_ERR_ALIGN;
    const kla::AttnPlan p = attn_plan(s, cu_seqlens_host, H / Hk, Hk, D);
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    auto run = [&](auto a) {
        a.rest = static_cast<decltype(a.rest)>(rest);
        a.tiles = kla::row_places(s, M, a.G, p.rows, &a.per);
        return status(kla::launch_attn_fwd(a, D, p, false, st));
    };
    return dt == KLA_BF16 ? run(attn_args<bf16_t>(q, ld_q, k, ld_k, v, ld_v, o, lse, s, M, z, scale, window, opts))
                          : run(attn_args<float>(q, ld_q, k, ld_k, v, ld_v, o, lse, s, M, z, scale, window, opts));
}

size_t kla_attn_bwd_workspace_bytes(int N, int T, int H, int Hk, int D, const int32_t* cu_seqlens_host, int n_seq, kla_dtype dt)
{
    kla::Seqs s;
    long M;
    const AttnSizes z = {N, T, H, Hk, D};
    if (attn_sizes(z, dt) || take_seqs(n_seq > 0 ? cu_seqlens_host : nullptr, cu_seqlens_host, n_seq, N, T, &s, &M)) return 0;
    return bwd_work(nullptr, attn_bwd_parts(s, cu_seqlens_host, H / Hk, Hk), M, z).bytes;
}

int kla_attn_bwd(const void* q, long ld_q, const void* k, long ld_k, const void* v, long ld_v, const void* o, const float* lse, const void* rest, const void* d_o, void* dq,
                 void* dk, void* dv, float scale, int window, const int32_t* cu_seqlens_dev, const int32_t* cu_seqlens_host, int n_seq, int N, int T, int H,
                 int Hk, int D, kla_dtype dt, void* workspace, size_t workspace_bytes, void* hip_stream, unsigned opts)
{
    kla::Seqs s;
    long M;
    const AttnSizes z = {N, T, H, Hk, D};
    if (const int e = attn_check(z, ld_q, ld_k, ld_v, scale, window, dt)) return e;
    if ((opts & ~(unsigned)KLA_ATTN_CAUSAL) || (window && !(opts & KLA_ATTN_CAUSAL))) return KLA_ERR_SHAPE;
    if (const int e = take_seqs(cu_seqlens_dev, cu_seqlens_host, n_seq, N, T, &s, &M)) return e;
    if (M > 0 && (!q || !k || !v || !o || !lse || !d_o || !dq || !dk || !dv)) return KLA_ERR_NULL;
    if (M > 0)
        for (const void* out : {dq, dk, dv})
            for (const void* in : {q, k, v, o, rest, d_o}) if (out == in) return KLA_ERR_SHAPE;
    if (M > 0 && (dq == dk || dq == dv || dk == dv)) return KLA_ERR_SHAPE;
    if (rest && dt != KLA_BF16) return KLA_ERR_DTYPE;
    if (!aligned(16, {q, k, v, o, rest, d_o, dq, dk, dv}) || !aligned(4, {lse})) return KLA_ERR_ALIGN;
    const int parts = attn_bwd_parts(s, cu_seqlens_host, H / Hk, Hk);
    const BwdWork w = bwd_work(static_cast<char*>(workspace), parts, M, z);
    if (const int e = take_workspace(workspace, workspace_bytes, w.bytes)) return e;
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    auto run = [&](auto a) {
        using Q = decltype(a.o);
        using E = std::remove_pointer_t<Q>;
        kla::AttnBwdArgs<E> b = {};
        b.f = a;
        b.f.rest = static_cast<Q>(const_cast<void*>(rest));
        b.d_o = static_cast<const E*>(d_o); b.dq = static_cast<Q>(dq); b.dk = static_cast<Q>(dk); b.dv = static_cast<Q>(dv);
        b.row_lse = w.row_lse; b.row_delta = w.row_delta; b.parts = parts; b.part_dk = w.part_dk; b.part_dv = w.part_dv;
        b.beside = attn_tiles(s, cu_seqlens_host, a.G, 128) * Hk < kAttnBeside;
        b.f.tiles = kla::row_places(s, M, a.G, b.beside ? 64 : 128, &b.f.per);
        b.key_tiles = kla::row_places(s, M, 1, 128, &b.key_per);
        return status(kla::launch_attn_bwd(b, D, st));
    };
    void* out = const_cast<void*>(o);
    float* l = const_cast<float*>(lse);
    return dt == KLA_BF16 ? run(attn_args<bf16_t>(q, ld_q, k, ld_k, v, ld_v, out, l, s, M, z, scale, window, opts))
                          : run(attn_args<float>(q, ld_q, k, ld_k, v, ld_v, out, l, s, M, z, scale, window, opts));
}

size_t kla_attn_extend_workspace_bytes(int N, int T, int H, int Hk, int D, const int32_t* cu_seqlens_host, int n_seq, int window, int max_len, kla_dtype dt)
{
    kla::Seqs s;
    long M;
    if (attn_sizes({N, T, H, Hk, D}, dt) || max_len < 0 || window < 0 || take_seqs(n_seq > 0 ? cu_seqlens_host : nullptr, cu_seqlens_host, n_seq, N, T, &s, &M)) return 0;
    return extend_work(nullptr, extend_plan(s, cu_seqlens_host, H / Hk, Hk, max_len, window), M, H, D).bytes;
}

int kla_attn_extend(const void* q, long ld_q, const void* k, long ld_k, const void* v, long ld_v, void* k_cache, void* v_cache, const int32_t* page_table,
                    long ld_table, const int32_t* cached, void* o, float* lse, float scale, int window, const int32_t* cu_seqlens_dev,
                    const int32_t* cu_seqlens_host, int n_seq, int N, int T, int H, int Hk, int D, int n_pages, int page, int max_pages, int max_len,
                    kla_dtype dt, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    kla::Seqs s;
    long M;
    const AttnSizes z = {N, T, H, Hk, D};
    if (const int e = attn_check(z, ld_q, ld_k, ld_v, scale, window, dt)) return e;
    int shift = 4;
    while (shift < 10 && (1 << shift) < page) ++shift;
    if (page != 1 << shift || n_pages <= 0 || max_pages <= 0 || ((long)max_pages << shift) > kMaxAttnRows || ld_table < max_pages || max_len < 0)
        return KLA_ERR_SHAPE;
    if (const int e = take_seqs(cu_seqlens_dev, cu_seqlens_host, n_seq, N, T, &s, &M)) return e;
    if (M > 0 && (!q || !k || !v || !o || !k_cache || !v_cache || !page_table || !cached)) return KLA_ERR_NULL;
    if (M > 0 && (o == q || o == k || o == v || k_cache == v_cache || k_cache == q || k_cache == k || k_cache == v || k_cache == o || v_cache == q ||
                  v_cache == k || v_cache == v || v_cache == o))
        return KLA_ERR_SHAPE;
    if (!aligned(16, {q, k, v, o, k_cache, v_cache}) || !aligned(4, {lse, page_table, cached})) return KLA_ERR_ALIGN;
    const kla::AttnPlan p = extend_plan(s, cu_seqlens_host, H / Hk, Hk, max_len, window);
    const ExtendWork w = extend_work(static_cast<char*>(workspace), p, M, H, D);
    if (const int e = take_workspace(workspace, workspace_bytes, w.bytes)) return e;
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    auto run = [&](auto a) {
        a.k_cache = static_cast<decltype(a.k_cache)>(k_cache); a.v_cache = static_cast<decltype(a.v_cache)>(v_cache);
        a.table = page_table; a.ld_table = ld_table; a.cached = cached; a.n_pages = n_pages; a.page_shift = shift; a.max_pages = max_pages;
        a.splits = p.splits; a.chunk = p.chunk; a.part_o = w.part_o; a.part_lse = w.part_lse; a.part_count = w.part_count;
        a.tiles = kla::row_places(s, M, a.G, p.rows, &a.per);
        if (const hipError_t e = kla::launch_attn_fwd(a, D, p, true, st)) return status(e);
        return p.splits > 1 ? status(kla::launch_attn_join(a, D, st)) : (int)KLA_OK;
    };
    return dt == KLA_BF16 ? run(attn_args<bf16_t>(q, ld_q, k, ld_k, v, ld_v, o, lse, s, M, z, scale, window, KLA_ATTN_CAUSAL))
                          : run(attn_args<float>(q, ld_q, k, ld_k, v, ld_v, o, lse, s, M, z, scale, window, KLA_ATTN_CAUSAL));
}

int kla_attn_step(const void* q, long ld_q, const void* k, long ld_k, const void* v, long ld_v, void* k_cache, void* v_cache, const int32_t* page_table,
                  long ld_table, const int32_t* cached, void* o, float scale, int window, int B, int H, int Hk, int D, int n_pages, int page, int max_pages,
                  int max_len, kla_dtype dt, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    return kla_attn_extend(q, ld_q, k, ld_k, v, ld_v, k_cache, v_cache, page_table, ld_table, cached, o, nullptr, scale, window, nullptr, nullptr, 0, B, 1, H,
                           Hk, D, n_pages, page, max_pages, max_len, dt, workspace, workspace_bytes, hip_stream);
}

}  // extern "C"
