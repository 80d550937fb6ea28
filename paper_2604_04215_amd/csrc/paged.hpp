// What the paged-cache and head kernels share: division by what the host knows, checks of a paged cache.
#pragma once
#include "common.hpp"

namespace dlm {

// quotient of n < 2^31 by a divisor fixed on the host
struct FastDiv {
    uint32_t mul, shift;
};
inline FastDiv fast_div(uint32_t d) {
    FastDiv f;
    f.shift = 0;
    while ((1ull << f.shift) < d) ++f.shift;
    f.mul = (uint32_t)((((1ull << f.shift) - d) << 32) / d + 1);
    return f;
}
__device__ __forceinline__ uint32_t quotient(uint32_t n, FastDiv f) { return (__umulhi(n, f.mul) + n) >> f.shift; }

// true if a tensor of n[i] steps of stride[i] over rows of `row` entries has no two entries at one place
template <int N>
inline bool apart(const int64_t (&n)[N], const int64_t (&stride)[N], int64_t row) {
    int order[N];
    for (int i = 0; i < N; ++i) order[i] = i;
    for (int i = 1; i < N; ++i)
        for (int j = i; j > 0 && stride[order[j]] < stride[order[j - 1]]; --j) {
            const int t = order[j];
            order[j] = order[j - 1];
            order[j - 1] = t;
        }
    __int128 extent = row;
    for (int i = 0; i < N; ++i) {
        const int k = order[i];
        if (n[k] <= 1) continue;
        if (stride[k] < extent) return false;
        extent += (__int128)stride[k] * (n[k] - 1);
    }
    return true;
}

inline int log2_of(int v) {
    int s = 0;
    while ((1 << s) < v) ++s;
    return s;
}

inline int validate_cache(const dlm_paged_kv& c, int Hkv, int d, const char* who, bool written) {
    if (c.type != DLM_KV_BF16 && c.type != DLM_KV_E4M3) return fail(DLM_ERR_INVALID_ARG, "%s: unknown cache type %d", who, c.type);
    if (c.n_pages < 0) return fail(DLM_ERR_INVALID_ARG, "%s: n_pages < 0", who);
    if (c.page_size < 1 || (c.page_size & (c.page_size - 1)))
        return fail(DLM_ERR_INVALID_ARG, "%s: page_size=%d is not a power of two", who, c.page_size);
    if (c.page_size < 16 || c.page_size > 65536) return fail(DLM_ERR_UNSUPPORTED, "%s: page_size %d (supported: 16 .. 65536)", who, c.page_size);
    if ((int64_t)c.n_pages * c.page_size > 0x7fffffff) return fail(DLM_ERR_UNSUPPORTED, "%s: more than 2^31 slots", who);
    if (c.type == DLM_KV_BF16 && (c.k_scale || c.v_scale)) return fail(DLM_ERR_INVALID_ARG, "%s: scales go with an e4m3 cache", who);
    if (c.n_pages == 0) return DLM_OK;
    if (!c.k || !c.v) return fail(DLM_ERR_INVALID_ARG, "%s: null cache", who);
    if (!aligned16(c.k) || !aligned16(c.v)) return fail(DLM_ERR_UNSUPPORTED, "%s: cache not 16-byte aligned", who);
    const int64_t n[3] = {c.n_pages, Hkv, c.page_size}, st[3] = {c.stride_page, c.stride_h, c.stride_t};
    const int unit = c.type == DLM_KV_E4M3 ? 16 : 8;
    for (int i = 0; i < 3; ++i)
        if (n[i] > 1 && (st[i] % unit || st[i] < 0))
            return fail(DLM_ERR_UNSUPPORTED, "%s: cache strides must be multiples of 16 bytes, not negative", who);
    if (written && !apart(n, st, d)) return fail(DLM_ERR_INVALID_ARG, "%s: rows of the cache overlap", who);
    return DLM_OK;
}

}  // namespace dlm
