// What the C ABI's checks share for the operators around the recurrence and attention: element types, alignment, the sequences of a batch, workspaces.
#pragma once
#include <initializer_list>

#include "../../include/kla.h"
#include "kla_layer.hpp"

namespace {

inline size_t round256(size_t x) { return (x + 255) & ~(size_t)255; }
inline size_t elem_bytes(int dt) { return dt == KLA_BF16 ? 2 : 4; }
inline bool dt_ok(int dt) { return dt == KLA_F32 || dt == KLA_BF16; }
// every pointer of the list on a multiple of `to` bytes (NULL is)
inline bool aligned(size_t to, std::initializer_list<const void*> ps)
{
    for (const void* p : ps) if (reinterpret_cast<uintptr_t>(p) % to) return false;
    return true;
}
inline int status(hipError_t e) { return e == hipSuccess ? KLA_OK : KLA_ERR_HIP; }

// The sequences of a batch; KLA_OK or what is wrong with them.  M: tokens in all.
int take_seqs(const int32_t* cu_dev, const int32_t* cu_host, int n_seq, int N, int T, kla::Seqs* s, long* M)
{
    if (N < 0 || T < 0 || n_seq < 0) return KLA_ERR_SHAPE;
    if (n_seq == 0) {
        if (cu_dev || cu_host) return KLA_ERR_SEQLENS;
        *s = {nullptr, N, T};
        *M = (long)N * T;
        return KLA_OK;
    }
    if (N != 1) return KLA_ERR_SHAPE;
    if (!cu_dev || !cu_host) return KLA_ERR_NULL;
    if (cu_host[0] != 0 || cu_host[n_seq] != T) return KLA_ERR_SEQLENS;
    for (int i = 0; i < n_seq; ++i) if (cu_host[i + 1] < cu_host[i]) return KLA_ERR_SEQLENS;
    *s = {cu_dev, n_seq, T};
    *M = T;
    return KLA_OK;
}

struct Carve {
    char* base; size_t used = 0;
    template <typename E> E* take(size_t n)
    {
        E* p = base ? reinterpret_cast<E*>(base + used) : nullptr;
        used += round256(n * sizeof(E));
        return p;
    }
};
int take_workspace(const void* ws, size_t have, size_t need)
{
    if (need == 0) return KLA_OK;
    return !ws || have < need || !aligned(256, {ws}) ? KLA_ERR_WORKSPACE : KLA_OK;
}

}  // namespace
