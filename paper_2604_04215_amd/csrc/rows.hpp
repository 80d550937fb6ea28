// Rows of 16 or 32 bits: what the embedding and the norms between layers share.
#pragma once
#include "common.hpp"

namespace dlm {

// A lane's unit of a row, 16 bytes: 8 entries of bf16 or 4 of fp32, computed with in fp32.
template <bool F32>
struct Piece {
    static constexpr int E = F32 ? 4 : 8;
    using Raw = u32x4;
    // past the caches: nothing reads it again soon
    static __device__ __forceinline__ Raw stream(const void* base, int64_t entry) {
        return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>((const char*)base + entry * (F32 ? 4 : 2)));
    }
    static __device__ __forceinline__ void open(Raw v, float (&f)[E]) {
        if constexpr (F32) {
#pragma unroll
            for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f[2 * i] = __uint_as_float(v[i] << 16);
                f[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
            }
        }
    }
    static __device__ __forceinline__ Raw close(const float (&f)[E]) {
        Raw v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = F32 ? __float_as_uint(f[i]) : pack_bf16x2(f[(2 * i) % E], f[(2 * i + 1) % E]);
        return v;
    }
    static __device__ __forceinline__ void stream_out(void* base, int64_t entry, Raw v) {
        __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>((char*)base + entry * (F32 ? 4 : 2)));
    }
};
// the E bf16 values that go with a piece
template <int E>
__device__ __forceinline__ void load_bf16(const uint16_t* p, float (&f)[E]) {
    if constexpr (E == 8) {
        Piece<false>::open(*reinterpret_cast<const u32x4*>(p), f);
    } else {
        const u32x2 v = *reinterpret_cast<const u32x2*>(p);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            f[2 * i] = __uint_as_float(v[i] << 16);
            f[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
        }
    }
}

// Checks of rows [n, D] (host): `written`: they are outputs.  `bytes` an entry.
inline int validate_rows(const void* p, int64_t stride, int64_t n, int D, int bytes, bool written, const char* who, const char* name) {
    if (n == 0) return DLM_OK;
    if (!p) return fail(DLM_ERR_INVALID_ARG, "%s: null %s", who, name);
    if (!aligned16(p)) return fail(DLM_ERR_UNSUPPORTED, "%s: %s not 16-byte aligned", who, name);
    if (n > 1 && stride * bytes % 16) return fail(DLM_ERR_UNSUPPORTED, "%s: row stride of %s must be a multiple of 16 bytes", who, name);
    if (n > 1 && stride < 0) return fail(DLM_ERR_UNSUPPORTED, "%s: row stride of %s < 0", who, name);
    if (n > 1 && written && stride < D) return fail(DLM_ERR_INVALID_ARG, "%s: rows of %s overlap", who, name);
    return DLM_OK;
}
inline int row_bytes(int type) { return type == DLM_ROW_F32 ? 4 : 2; }
inline int validate_row_type(int type, const char* who, const char* name) {
    if (type != DLM_ROW_BF16 && type != DLM_ROW_F32) return fail(DLM_ERR_INVALID_ARG, "%s: unknown type %d of %s", who, type, name);
    return DLM_OK;
}

}  // namespace dlm
