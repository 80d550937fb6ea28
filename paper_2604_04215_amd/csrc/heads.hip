// dlm_qk_norm_rope, its gradient, and dlm_paged_append: RMS norm and rotation of query and key heads, stored densely or
// into the pages of a cache.
//
// All three stream heads once and compute a few operations an entry: bound by HBM (large T) or by the chain
// position -> row of the table -> result (small T).
//
// Layout: D/16 lanes own a head, 16 entries each in two pieces of 8 that hold BOTH partners of every rotated pair
// (see Pieces), so the rotation is in-lane and only the sum of squares crosses lanes (two or three cross-lane moves).  A 16-byte load a
// piece: the two loads of a wavefront cover whole lines of 8 (d = 128) or 16 heads.  Queries, keys and values are parts of one launch,
// divided by workgroup, so that what depends on the part (weight, destination, type) is uniform in a wavefront.
#include "paged.hpp"

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

struct Rotation {
    const float* rope;         // NULL: none
    int rope_len, rot;
    const int32_t* positions;
};

// Where a lane's two pieces lie in its head: entries [a, a + 8) and [b, b + 8).  `l`: lane within the head.
//   halves: lane l < rot/16 has 8l.. and its partners rot/2 + 8l..; the other lanes share out the entries behind rot
//   pairs:  16 entries in a row
// Either way the rotated pairs of a lane use the 8 angles from 8l on.
template <bool PAIRS>
struct Pieces {
    int a, b;
    bool turns;
    __device__ __forceinline__ Pieces(int l, int rot) {
        turns = l < (rot >> 4);
        if (PAIRS || !turns) {
            a = 16 * l;
            b = a + 8;
        } else {
            a = 8 * l;
            b = (rot >> 1) + a;
        }
    }
};

__device__ __forceinline__ void unpack8(u32x4 v, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(v[i] << 16);
        f[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ u32x4 pack8(const float (&f)[8]) {
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
    return v;
}
// eight entries of an e4m3 cache: nearest, ties to even (the hardware conversion), larger ones to +-448, NaN kept
__device__ __forceinline__ u32x2 pack8_e4m3(const float (&f)[8], float inv_scale) {
    float g[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float x = f[i] * inv_scale;
        g[i] = x != x ? x : __builtin_fmaxf(__builtin_fminf(x, 448.f), -448.f);
    }
    u32x2 v;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(g[4 * i], g[4 * i + 1], 0, false);
        v[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(g[4 * i + 2], g[4 * i + 3], w, true);
    }
    return v;
}

// sum over the D/16 lanes of a head; every lane gets the same bits
template <int D>
__device__ __forceinline__ float head_sum(float v) {
    static_assert(D == 64 || D == 128, "4 or 8 lanes a head");
    v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0xB1, 0xf, 0xf, true));                    // lane ^ 1
    v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x4E, 0xf, 0xf, true));                    // lane ^ 2
    if (D == 128) v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x141, 0xf, 0xf, true));     // 7 - lane of 8: the other four
    return v;
}

// the 8 cosines and sines of a lane
struct Angles {
    float c[8], s[8];
};
__device__ __forceinline__ void load_angles(const Rotation& r, int token, int l, Angles& g) {
    const int pos = r.positions[token];
    const bool known = (unsigned)pos < (unsigned)r.rope_len;
    const float* row = r.rope + (int64_t)(known ? pos : 0) * r.rot + 8 * l;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const f32x4 c = *reinterpret_cast<const f32x4*>(row + 4 * q), s = *reinterpret_cast<const f32x4*>(row + (r.rot >> 1) + 4 * q);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            g.c[4 * q + e] = known ? c[e] : __builtin_nanf("");
            g.s[4 * q + e] = known ? s[e] : __builtin_nanf("");
        }
    }
}
// BACK: by the opposite angles (the rotation's transpose)
template <bool PAIRS, bool BACK>
__device__ __forceinline__ void turn(const Angles& g, float (&a)[8], float (&b)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float &x = PAIRS ? (e < 4 ? a[2 * (e & 3)] : b[2 * (e & 3)]) : a[e], &y = PAIRS ? (e < 4 ? a[2 * (e & 3) + 1] : b[2 * (e & 3) + 1]) : b[e];
        const float s = BACK ? -g.s[e] : g.s[e], x0 = x;
        x = x0 * g.c[e] - y * s;
        y = y * g.c[e] + x0 * s;
    }
}

// ---- forward and append -------------------------------------------------------------------------------------
struct HeadPart {
    const uint16_t* x;
    int64_t x_st, x_sh;
    void* y;                   // dense destination (strides y_st, y_sh), or the pages (strides y_sp, y_sh, y_st)
    int64_t y_sp, y_st, y_sh;
    const uint16_t* w;
    const float* scale;
    uint32_t rows, heads;      // rows = tokens * heads
    FastDiv by_heads;
    uint32_t first;            // its first workgroup
    int map;                   // norm and rotation (queries, keys) or neither (values)
    int paged;                 // 0: dense, 1: pages of bf16, 2: pages of e4m3
};
struct HeadParams {
    HeadPart part[3];
    Rotation rotation;
    float eps;
    const int32_t* slots;
    uint32_t n_slots;
    int page_shift;
};

template <int D, bool PAIRS>
__global__ __launch_bounds__(256) void head_map_kernel(HeadParams p) {
    constexpr int LPH = D / 16, ROWS = 256 / LPH;
    const HeadPart& t = p.part[blockIdx.x >= p.part[2].first ? 2 : blockIdx.x >= p.part[1].first ? 1 : 0];
    const uint32_t row = (blockIdx.x - t.first) * ROWS + threadIdx.x / LPH;
    const bool live = row < t.rows;          // (lanes of a head are live together)
    const int l = threadIdx.x % LPH;
    const uint32_t token = live ? quotient(row, t.by_heads) : 0, h = live ? row - token * t.heads : 0;
    const int rot = t.map && p.rotation.rope ? p.rotation.rot : 0;
    const Pieces<PAIRS> at(l, rot);
    const uint16_t* x = t.x + (int64_t)token * t.x_st + (int64_t)h * t.x_sh;
    float a[8], b[8];
    const u32x4 ra = *reinterpret_cast<const u32x4*>(x + at.a), rb = *reinterpret_cast<const u32x4*>(x + at.b);
    const int slot = t.paged ? p.slots[token] : 0;
    Angles g;
    if (at.turns) load_angles(p.rotation, token, l, g);
    unpack8(ra, a);
    unpack8(rb, b);
    if (t.map && t.w) {
        float wa[8], wb[8], sum = 0.f;
        unpack8(*reinterpret_cast<const u32x4*>(t.w + at.a), wa);
        unpack8(*reinterpret_cast<const u32x4*>(t.w + at.b), wb);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += a[e] * a[e] + b[e] * b[e];
        const float r = 1.0f / sqrtf(head_sum<D>(sum) * (1.0f / D) + p.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            a[e] *= r * wa[e];
            b[e] *= r * wb[e];
        }
    }
    if (at.turns) turn<PAIRS, false>(g, a, b);
    if (!live) return;
    if (t.paged) {
        if ((uint32_t)slot >= p.n_slots) return;
        const int64_t off = (int64_t)(slot >> p.page_shift) * t.y_sp + (int64_t)(slot & ((1 << p.page_shift) - 1)) * t.y_st + (int64_t)h * t.y_sh;
        if (t.paged == 2) {
            const float inv = t.scale ? 1.0f / t.scale[h] : 1.0f;
            uint8_t* y = (uint8_t*)t.y + off;
            *reinterpret_cast<u32x2*>(y + at.a) = pack8_e4m3(a, inv);
            *reinterpret_cast<u32x2*>(y + at.b) = pack8_e4m3(b, inv);
        } else {
            uint16_t* y = (uint16_t*)t.y + off;
            *reinterpret_cast<u32x4*>(y + at.a) = pack8(a);
            *reinterpret_cast<u32x4*>(y + at.b) = pack8(b);
        }
        return;
    }
    uint16_t* y = (uint16_t*)t.y + (int64_t)token * t.y_st + (int64_t)h * t.y_sh;
    *reinterpret_cast<u32x4*>(y + at.a) = pack8(a);
    *reinterpret_cast<u32x4*>(y + at.b) = pack8(b);
}

// ---- gradient -----------------------------------------------------------------------------------------------
struct GradPart {
    const uint16_t *dy, *x;    // x: only with a weight
    int64_t dy_st, dy_sh, x_st, x_sh;
    uint16_t* dx;
    int64_t dx_st, dx_sh;
    const uint16_t* w;
    float* partial;            // [workgroups][D] sums for the weight's gradient, or NULL
    uint32_t rows, heads;
    FastDiv by_heads;
    uint32_t first, groups;    // its first workgroup and their number
};
struct GradParams {
    GradPart part[2];
    Rotation rotation;
    float eps;
};

// A workgroup walks every groups-th stretch of ROWS heads of its part and keeps the weight's gradient in registers (16 entries a
// lane), so each adds one row of D sums to the workspace.
template <int D, bool PAIRS>
__global__ __launch_bounds__(256) void head_map_grad_kernel(GradParams p) {
    constexpr int LPH = D / 16, ROWS = 256 / LPH;
    __shared__ float sums[4][D];
    const GradPart& t = p.part[blockIdx.x >= p.part[1].first ? 1 : 0];
    const int l = threadIdx.x % LPH, lane = lane_id(), wave = threadIdx.x >> 6;
    const Pieces<PAIRS> at(l, p.rotation.rope ? p.rotation.rot : 0);
    float wa[8], wb[8], dwa[8], dwb[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) dwa[e] = dwb[e] = wa[e] = wb[e] = 0.f;
    if (t.w) {
        unpack8(*reinterpret_cast<const u32x4*>(t.w + at.a), wa);
        unpack8(*reinterpret_cast<const u32x4*>(t.w + at.b), wb);
    }
    for (uint32_t row = (blockIdx.x - t.first) * ROWS + threadIdx.x / LPH; row < t.rows; row += t.groups * ROWS) {
        const uint32_t token = quotient(row, t.by_heads), h = row - token * t.heads;
        const uint16_t* dy = t.dy + (int64_t)token * t.dy_st + (int64_t)h * t.dy_sh;
        float a[8], b[8];
        const u32x4 ra = *reinterpret_cast<const u32x4*>(dy + at.a), rb = *reinterpret_cast<const u32x4*>(dy + at.b);
        u32x4 xa, xb;
        if (t.w) {
            const uint16_t* x = t.x + (int64_t)token * t.x_st + (int64_t)h * t.x_sh;
            xa = *reinterpret_cast<const u32x4*>(x + at.a);
            xb = *reinterpret_cast<const u32x4*>(x + at.b);
        }
        Angles g;
        if (at.turns) load_angles(p.rotation, token, l, g);
        unpack8(ra, a);
        unpack8(rb, b);
        if (at.turns) turn<PAIRS, true>(g, a, b);
        if (t.w) {
            float na[8], nb[8], sum = 0.f, dot = 0.f;
            unpack8(xa, na);
            unpack8(xb, nb);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += na[e] * na[e] + nb[e] * nb[e];
            const float r = 1.0f / sqrtf(head_sum<D>(sum) * (1.0f / D) + p.eps);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                na[e] *= r;
                nb[e] *= r;
                dwa[e] += a[e] * na[e];
                dwb[e] += b[e] * nb[e];
                a[e] *= wa[e];
                b[e] *= wb[e];
                dot += a[e] * na[e] + b[e] * nb[e];
            }
            const float mean = head_sum<D>(dot) * (1.0f / D);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                a[e] = r * (a[e] - na[e] * mean);
                b[e] = r * (b[e] - nb[e] * mean);
            }
        }
        uint16_t* dx = t.dx + (int64_t)token * t.dx_st + (int64_t)h * t.dx_sh;
        *reinterpret_cast<u32x4*>(dx + at.a) = pack8(a);
        *reinterpret_cast<u32x4*>(dx + at.b) = pack8(b);
    }
    if (!t.partial) return;                  // (uniform in the workgroup)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
#pragma unroll
        for (int off = LPH; off < 64; off <<= 1) {
            dwa[e] += shfl_xor(dwa[e], off);
            dwb[e] += shfl_xor(dwb[e], off);
        }
        if (lane < LPH) {
            sums[wave][at.a + e] = dwa[e];
            sums[wave][at.b + e] = dwb[e];
        }
    }
    __syncthreads();
    if (threadIdx.x < D)
        t.partial[(int64_t)(blockIdx.x - t.first) * D + threadIdx.x] =
            (sums[0][threadIdx.x] + sums[1][threadIdx.x]) + (sums[2][threadIdx.x] + sums[3][threadIdx.x]);
}

struct GradSumParams {
    const float* partial[2];
    float* out[2];
    int groups[2];
    int d;
};
// 16 entries of one weight's gradient a workgroup: 64 threads an entry walk the rows of sums, then one adds up in a fixed order
__global__ __launch_bounds__(1024) void head_grad_sum_kernel(GradSumParams p) {
    __shared__ float s[64][17];
    const int which = blockIdx.y, c = threadIdx.x & 15, r = threadIdx.x >> 4;
    if (!p.out[which]) return;
    const float* in = p.partial[which] + blockIdx.x * 16 + c;
    float v = 0.f;
    for (int i = r; i < p.groups[which]; i += 64) v += in[(int64_t)i * p.d];
    s[r][c] = v;
    __syncthreads();
    if (r == 0) {
        v = 0.f;
#pragma unroll
        for (int i = 0; i < 64; ++i) v += s[i][c];
        p.out[which][blockIdx.x * 16 + c] = v;
    }
}

// ---- host ---------------------------------------------------------------------------------------------------
// a [T, H, d] tensor of bf16; `written`: its rows must not overlap
static int validate_heads(const void* x, int64_t st, int64_t sh, int64_t T, int64_t H, int d, bool written, const char* who, const char* name) {
    if (T == 0 || H == 0) return DLM_OK;
    if (!x) return fail(DLM_ERR_INVALID_ARG, "%s: null %s", who, name);
    if (!aligned16(x)) return fail(DLM_ERR_UNSUPPORTED, "%s: %s not 16-byte aligned", who, name);
    if ((T > 1 && st % 8) || (H > 1 && sh % 8)) return fail(DLM_ERR_UNSUPPORTED, "%s: strides of %s must be multiples of 8", who, name);
    const int64_t n[2] = {T, H}, s[2] = {st, sh};
    if (written && !apart(n, s, d)) return fail(DLM_ERR_INVALID_ARG, "%s: rows of %s overlap", who, name);
    return DLM_OK;
}

static int validate_map(const dlm_head_map& m, int T, int Hq, int Hkv, int d, const char* who) {
    if (T < 0 || Hq < 0 || Hkv < 0) return fail(DLM_ERR_INVALID_ARG, "%s: bad sizes T=%d Hq=%d Hkv=%d", who, T, Hq, Hkv);
    if (d != 64 && d != 128) return fail(DLM_ERR_UNSUPPORTED, "%s: head_dim %d (supported: 64, 128)", who, d);
    if ((int64_t)T * (Hq > Hkv ? Hq : Hkv) > 0x7fffffff) return fail(DLM_ERR_UNSUPPORTED, "%s: more than 2^31 heads in all", who);
    if (!(m.eps >= 0.f)) return fail(DLM_ERR_INVALID_ARG, "%s: eps must be >= 0", who);
    if (!aligned16(m.q_weight) || !aligned16(m.k_weight)) return fail(DLM_ERR_UNSUPPORTED, "%s: weights not 16-byte aligned", who);
    if (m.rope) {
        if (m.rope_style != DLM_ROPE_HALVES && m.rope_style != DLM_ROPE_PAIRS)
            return fail(DLM_ERR_INVALID_ARG, "%s: unknown rope_style %d", who, m.rope_style);
        if (m.rot_dim < 16 || m.rot_dim > d || m.rot_dim % 16)
            return fail(DLM_ERR_UNSUPPORTED, "%s: rot_dim %d (supported: multiples of 16 up to d)", who, m.rot_dim);
        if (m.rope_len < 1) return fail(DLM_ERR_INVALID_ARG, "%s: rope_len < 1", who);
        if (!aligned16(m.rope)) return fail(DLM_ERR_UNSUPPORTED, "%s: rope table not 16-byte aligned", who);
        if (!m.positions && T > 0) return fail(DLM_ERR_INVALID_ARG, "%s: a rotation needs positions", who);
    }
    return DLM_OK;
}

static Rotation rotation_of(const dlm_head_map& m) { return Rotation{m.rope, m.rope_len, m.rope ? m.rot_dim : 0, m.positions}; }

// appends a part behind the `groups` workgroups that there are
static void add_part(HeadPart& t, uint32_t& groups, int T, int H, int d, const void* x, int64_t x_st, int64_t x_sh, void* y, int64_t y_sp, int64_t y_st,
                     int64_t y_sh, const void* w, const float* scale, int map, int paged) {
    t = HeadPart{(const uint16_t*)x, x_st, x_sh, y, y_sp, y_st, y_sh, (const uint16_t*)w, scale, (uint32_t)((int64_t)T * H), (uint32_t)(H ? H : 1),
                 fast_div(H ? H : 1), groups, map, paged};
    const uint32_t rows = 256 / (d / 16);
    groups += (t.rows + rows - 1) / rows;
}

static int launch_head_map(const HeadParams& p, uint32_t groups, int d, int style, hipStream_t st) {
    if (groups == 0) return DLM_OK;
    const bool pairs = p.rotation.rope && style == DLM_ROPE_PAIRS;
    if (d == 128) {
        if (pairs) hipLaunchKernelGGL((head_map_kernel<128, true>), dim3(groups), dim3(256), 0, st, p);
        else hipLaunchKernelGGL((head_map_kernel<128, false>), dim3(groups), dim3(256), 0, st, p);
    } else {
        if (pairs) hipLaunchKernelGGL((head_map_kernel<64, true>), dim3(groups), dim3(256), 0, st, p);
        else hipLaunchKernelGGL((head_map_kernel<64, false>), dim3(groups), dim3(256), 0, st, p);
    }
    return check_hip(hipGetLastError(), "head_map_kernel launch");
}

// Workgroups of the gradient for one tensor of T * H heads: one for every stretch of heads, at most 1024 (four a CU), which bounds the
// rows of sums that the second launch reads.
static uint32_t grad_groups(int T, int H, int d) {
    const int64_t per = 256 / (d / 16), n = ((int64_t)T * H + per - 1) / per;
    return (uint32_t)(n < 1024 ? n : 1024);
}

}  // namespace dlm

using namespace dlm;

extern "C" int dlm_qk_norm_rope(const dlm_qk_args* a, void* stream) {
    static const char who[] = "qk_norm_rope";
    if (!a) return fail(DLM_ERR_INVALID_ARG, "%s: null args", who);
    if (a->struct_size != sizeof(dlm_qk_args)) return fail(DLM_ERR_INVALID_ARG, "%s: struct_size %u != %zu", who, a->struct_size, sizeof(dlm_qk_args));
    int rc;
    if ((rc = validate_map(a->map, a->T, a->Hq, a->Hkv, a->d, who)) != DLM_OK) return rc;
    if ((rc = validate_heads(a->q, a->q_stride_t, a->q_stride_h, a->T, a->Hq, a->d, false, who, "q")) != DLM_OK) return rc;
    if ((rc = validate_heads(a->k, a->k_stride_t, a->k_stride_h, a->T, a->Hkv, a->d, false, who, "k")) != DLM_OK) return rc;
    if ((rc = validate_heads(a->q_out, a->qo_stride_t, a->qo_stride_h, a->T, a->Hq, a->d, true, who, "q_out")) != DLM_OK) return rc;
    if ((rc = validate_heads(a->k_out, a->ko_stride_t, a->ko_stride_h, a->T, a->Hkv, a->d, true, who, "k_out")) != DLM_OK) return rc;
    HeadParams p = {};
    uint32_t groups = 0;
    add_part(p.part[0], groups, a->T, a->Hq, a->d, a->q, a->q_stride_t, a->q_stride_h, a->q_out, 0, a->qo_stride_t, a->qo_stride_h, a->map.q_weight, nullptr, 1, 0);
    add_part(p.part[1], groups, a->T, a->Hkv, a->d, a->k, a->k_stride_t, a->k_stride_h, a->k_out, 0, a->ko_stride_t, a->ko_stride_h, a->map.k_weight, nullptr, 1, 0);
    add_part(p.part[2], groups, 0, 0, a->d, nullptr, 0, 0, nullptr, 0, 0, 0, nullptr, nullptr, 0, 0);
    p.rotation = rotation_of(a->map);
    p.eps = a->map.eps;
    return launch_head_map(p, groups, a->d, a->map.rope_style, (hipStream_t)stream);
}

extern "C" int dlm_paged_append(const dlm_append_args* a, void* stream) {
    static const char who[] = "paged_append";
    if (!a) return fail(DLM_ERR_INVALID_ARG, "%s: null args", who);
    if (a->struct_size != sizeof(dlm_append_args))
        return fail(DLM_ERR_INVALID_ARG, "%s: struct_size %u != %zu", who, a->struct_size, sizeof(dlm_append_args));
    int rc;
    if ((rc = validate_map(a->map, a->T, a->Hq, a->Hkv, a->d, who)) != DLM_OK) return rc;
    if (a->Hkv < 1) return fail(DLM_ERR_INVALID_ARG, "%s: Hkv < 1", who);
    if ((rc = validate_cache(a->cache, a->Hkv, a->d, who, true)) != DLM_OK) return rc;
    if ((rc = validate_heads(a->q, a->q_stride_t, a->q_stride_h, a->T, a->Hq, a->d, false, who, "q")) != DLM_OK) return rc;
    if ((rc = validate_heads(a->k, a->k_stride_t, a->k_stride_h, a->T, a->Hkv, a->d, false, who, "k")) != DLM_OK) return rc;
    if ((rc = validate_heads(a->v, a->v_stride_t, a->v_stride_h, a->T, a->Hkv, a->d, false, who, "v")) != DLM_OK) return rc;
    if ((rc = validate_heads(a->q_out, a->qo_stride_t, a->qo_stride_h, a->T, a->Hq, a->d, true, who, "q_out")) != DLM_OK) return rc;
    if (a->T == 0) return DLM_OK;
    if (!a->slots) return fail(DLM_ERR_INVALID_ARG, "%s: null slots", who);
    const dlm_paged_kv& c = a->cache;
    HeadParams p = {};
    uint32_t groups = 0;
    const int kind = c.type == DLM_KV_E4M3 ? 2 : 1;
    add_part(p.part[0], groups, a->T, a->Hq, a->d, a->q, a->q_stride_t, a->q_stride_h, a->q_out, 0, a->qo_stride_t, a->qo_stride_h, a->map.q_weight, nullptr, 1, 0);
    add_part(p.part[1], groups, a->T, a->Hkv, a->d, a->k, a->k_stride_t, a->k_stride_h, c.k, c.stride_page, c.stride_t, c.stride_h, a->map.k_weight, c.k_scale, 1, kind);
    add_part(p.part[2], groups, a->T, a->Hkv, a->d, a->v, a->v_stride_t, a->v_stride_h, c.v, c.stride_page, c.stride_t, c.stride_h, nullptr, c.v_scale, 0, kind);
    p.rotation = rotation_of(a->map);
    p.eps = a->map.eps;
    p.slots = a->slots;
    p.n_slots = (uint32_t)c.n_pages * (uint32_t)c.page_size;
    p.page_shift = log2_of(c.page_size);
    return launch_head_map(p, groups, a->d, a->map.rope_style, (hipStream_t)stream);
}

extern "C" size_t dlm_qk_norm_rope_bwd_workspace_bytes(const dlm_qk_bwd_args* a) {
    if (!a || a->struct_size != sizeof(dlm_qk_bwd_args) || a->T < 0 || a->Hq < 0 || a->Hkv < 0 || (a->d != 64 && a->d != 128)) return 0;
    return (size_t)(grad_groups(a->T, a->Hq, a->d) + grad_groups(a->T, a->Hkv, a->d)) * a->d * sizeof(float);
}

extern "C" int dlm_qk_norm_rope_bwd(const dlm_qk_bwd_args* a, void* stream) {
    static const char who[] = "qk_norm_rope_bwd";
    if (!a) return fail(DLM_ERR_INVALID_ARG, "%s: null args", who);
    if (a->struct_size != sizeof(dlm_qk_bwd_args))
        return fail(DLM_ERR_INVALID_ARG, "%s: struct_size %u != %zu", who, a->struct_size, sizeof(dlm_qk_bwd_args));
    int rc;
    if ((rc = validate_map(a->map, a->T, a->Hq, a->Hkv, a->d, who)) != DLM_OK) return rc;
    if ((rc = validate_heads(a->d_q_out, a->dqo_stride_t, a->dqo_stride_h, a->T, a->Hq, a->d, false, who, "d_q_out")) != DLM_OK) return rc;
    if ((rc = validate_heads(a->d_k_out, a->dko_stride_t, a->dko_stride_h, a->T, a->Hkv, a->d, false, who, "d_k_out")) != DLM_OK) return rc;
    if (a->map.q_weight && (rc = validate_heads(a->q, a->q_stride_t, a->q_stride_h, a->T, a->Hq, a->d, false, who, "q")) != DLM_OK) return rc;
    if (a->map.k_weight && (rc = validate_heads(a->k, a->k_stride_t, a->k_stride_h, a->T, a->Hkv, a->d, false, who, "k")) != DLM_OK) return rc;
    if ((rc = validate_heads(a->d_q, a->dq_stride_t, a->dq_stride_h, a->T, a->Hq, a->d, true, who, "d_q")) != DLM_OK) return rc;
    if ((rc = validate_heads(a->d_k, a->dk_stride_t, a->dk_stride_h, a->T, a->Hkv, a->d, true, who, "d_k")) != DLM_OK) return rc;
    if ((a->d_q_weight && !a->map.q_weight) || (a->d_k_weight && !a->map.k_weight))
        return fail(DLM_ERR_INVALID_ARG, "%s: a weight's gradient needs the weight", who);
    const bool sums = a->d_q_weight || a->d_k_weight;
    if (sums && dlm_qk_norm_rope_bwd_workspace_bytes(a) > 0) {
        if (!a->workspace || a->workspace_bytes < dlm_qk_norm_rope_bwd_workspace_bytes(a))
            return fail(DLM_ERR_WORKSPACE, "%s: workspace of %zu bytes required", who, dlm_qk_norm_rope_bwd_workspace_bytes(a));
        if (!aligned16(a->workspace)) return fail(DLM_ERR_WORKSPACE, "%s: workspace not 16-byte aligned", who);
    }
    const uint32_t gq = grad_groups(a->T, a->Hq, a->d), gk = grad_groups(a->T, a->Hkv, a->d);
    float* part_q = (float*)a->workspace;
    float* part_k = part_q + (size_t)gq * a->d;
    hipStream_t st = (hipStream_t)stream;
    if (gq + gk > 0) {
        GradParams p = {};
        p.part[0] = GradPart{(const uint16_t*)a->d_q_out, (const uint16_t*)a->q, a->dqo_stride_t, a->dqo_stride_h, a->q_stride_t, a->q_stride_h,
                             (uint16_t*)a->d_q, a->dq_stride_t, a->dq_stride_h, (const uint16_t*)a->map.q_weight, a->d_q_weight ? part_q : nullptr,
                             (uint32_t)((int64_t)a->T * a->Hq), (uint32_t)(a->Hq ? a->Hq : 1), fast_div(a->Hq ? a->Hq : 1), 0, gq};
        p.part[1] = GradPart{(const uint16_t*)a->d_k_out, (const uint16_t*)a->k, a->dko_stride_t, a->dko_stride_h, a->k_stride_t, a->k_stride_h,
                             (uint16_t*)a->d_k, a->dk_stride_t, a->dk_stride_h, (const uint16_t*)a->map.k_weight, a->d_k_weight ? part_k : nullptr,
                             (uint32_t)((int64_t)a->T * a->Hkv), (uint32_t)(a->Hkv ? a->Hkv : 1), fast_div(a->Hkv ? a->Hkv : 1), gq, gk};
        p.rotation = rotation_of(a->map);
        p.eps = a->map.eps;
        const bool pairs = p.rotation.rope && a->map.rope_style == DLM_ROPE_PAIRS;
        if (a->d == 128) {
            if (pairs) hipLaunchKernelGGL((head_map_grad_kernel<128, true>), dim3(gq + gk), dim3(256), 0, st, p);
            else hipLaunchKernelGGL((head_map_grad_kernel<128, false>), dim3(gq + gk), dim3(256), 0, st, p);
        } else {
            if (pairs) hipLaunchKernelGGL((head_map_grad_kernel<64, true>), dim3(gq + gk), dim3(256), 0, st, p);
            else hipLaunchKernelGGL((head_map_grad_kernel<64, false>), dim3(gq + gk), dim3(256), 0, st, p);
        }
        if ((rc = check_hip(hipGetLastError(), "head_map_grad_kernel launch")) != DLM_OK) return rc;
    }
    if (!sums) return DLM_OK;
    const GradSumParams s = {{part_q, part_k}, {a->d_q_weight, a->d_k_weight}, {(int)gq, (int)gk}, a->d};
    hipLaunchKernelGGL(head_grad_sum_kernel, dim3(a->d / 16, 2), dim3(1024), 0, st, s);
    return check_hip(hipGetLastError(), "head_grad_sum_kernel launch");
}
