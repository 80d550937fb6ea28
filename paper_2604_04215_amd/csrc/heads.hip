// dlm_qk_norm_rope, its gradient, and dlm_paged_append: RMS norm and rotation of query and key heads, stored densely or
// into the pages of a cache.
//
// All three stream heads once and compute a few operations an entry: bound by HBM (large T) or by the chain position -> row of the
// table -> result (small T).  A SIMD has 16 lanes, so at the rate of a copy a wavefront may spend about 400 instructions on 8
// heads of 128 in and out, and what is not arithmetic on entries is kept out of the loop: see Walk.
//
// Layout: D/16 lanes own a head, 16 entries each in two pieces of 8 that hold BOTH partners of every rotated pair
// (see Pieces), so the rotation is in-lane and only the sum of squares crosses lanes (two or three cross-lane moves).  A 16-byte load a
// piece: the two loads of a wavefront cover whole lines of 8 (d = 128) or 16 heads.  Queries, keys and values are parts of one launch,
// divided by workgroup, so that what depends on the part (weight, destination, type) is uniform in a wavefront.
#include "paged.hpp"

namespace dlm {

// How the wavefronts of a part go over its T * H heads, 1024 / D at a time: with H of at least as many, `per` wavefronts share a token, else a
// wavefront takes `tokens` whole ones.  Either way the addresses of a step are a lane's own constant plus something uniform.
struct Walk {
    uint32_t units, heads;         // steps of a wavefront; H
    FastDiv by_per, by_heads;
    uint32_t per, tokens;
    uint32_t T;
    uint32_t first, groups;        // the part's workgroups
};
inline Walk walk_of(int T, int H, int d) {
    const uint32_t n = 1024 / d, h = H > 0 ? H : 1;
    Walk w = {};
    w.heads = h;
    w.per = h >= n ? (h + n - 1) / n : 1;
    w.tokens = h >= n ? 1 : n / h;
    w.T = H > 0 ? T : 0;
    w.units = w.T ? (uint32_t)(((int64_t)w.T + w.tokens - 1) / w.tokens) * w.per : 0;
    w.by_per = fast_div(w.per);
    w.by_heads = fast_div(h);
    return w;
}
// a lane's place in every step: its token and head from the step's first
template <int D>
struct Place {
    uint32_t l, token, head;
    __device__ __forceinline__ Place(const Walk& w) {
        const uint32_t slot = lane_id() / (D / 16);
        l = lane_id() % (D / 16);
        token = w.tokens > 1 ? quotient(slot, w.by_heads) : 0;
        head = slot - token * w.heads;
    }
};
// a step's first token and head, and whether the lane has a head in it
struct Step {
    uint32_t token, head;
    bool live;
    template <int D>
    __device__ __forceinline__ Step(const Walk& w, const Place<D>& at, uint32_t unit) {
        const uint32_t t = quotient(unit, w.by_per);
        head = (unit - t * w.per) * (1024 / D);
        token = t * w.tokens;
        live = at.token < w.tokens && token + at.token < w.T && head + at.head < w.heads;
    }
};

// sum over the lanes of a wavefront that hold the same entries of its heads; every lane gets it
template <int D>
__device__ __forceinline__ float over_heads(float v) {
    if (D == 64) v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x124, 0xf, 0xf, true));     // rotated by 4 within 16
    v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x128, 0xf, 0xf, true));                   // by 8
    auto w = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(w[0]) + __uint_as_float(w[1]);
    w = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(w[0]) + __uint_as_float(w[1]);
}

struct Rotation {
    const float* rope;         // NULL: none
    int rope_len, rot;
    const int32_t* positions;
};

// Where a lane's two pieces lie in its head: entries [a, a + 8) and [b, b + 8).  `l`: lane within the head.  Neighbouring lanes have neighbouring
// pieces, so that a load or store of the wavefront covers 64 bytes or more in a row (16 of every 32 bytes, two instructions a line: the gradient
// with half the entries rotated 68 -> 78 us under non-temporal loads).
//   halves: lane l < rot/16 has 8l.. and its partners rot/2 + 8l..; the other lanes share out the entries behind rot in the same way
//   pairs:  8l.. and D/2 + 8l..
// The angles of a piece's (or of both pieces') pairs: 4 from i0 on and 4 from i1 on, each where its entries are rotated at all.
template <int D, bool PAIRS>
struct Pieces {
    int a, b, i0, i1;
    bool turns0, turns1;
    __device__ __forceinline__ Pieces(int l, int rot) {
        const int n = rot >> 4;          // (halves) lanes that turn
        if (PAIRS) {
            a = 8 * l;
            b = D / 2 + a;
            i0 = a / 2;
            i1 = b / 2;
            turns0 = a < rot;
            turns1 = b < rot;
        } else {
            turns0 = turns1 = l < n;
            a = turns0 ? 8 * l : rot + 8 * (l - n);
            b = a + (turns0 ? rot : D - rot) / 2;
            i0 = 8 * l;
            i1 = i0 + 4;
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

// the 8 cosines and sines of a lane
struct Angles {
    float c[8], s[8];
};
template <int D, bool PAIRS>
__device__ __forceinline__ void load_angles(const Rotation& r, int pos, const Pieces<D, PAIRS>& at, Angles& g) {
    const bool known = (unsigned)pos < (unsigned)r.rope_len;
    const float* row = r.rope + (int64_t)(known ? pos : 0) * r.rot;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const bool turns = q ? at.turns1 : at.turns0;
        f32x4 c = {1.f, 1.f, 1.f, 1.f}, s = {0.f, 0.f, 0.f, 0.f};
        if (turns) {
            c = *reinterpret_cast<const f32x4*>(row + (q ? at.i1 : at.i0));
            s = *reinterpret_cast<const f32x4*>(row + (r.rot >> 1) + (q ? at.i1 : at.i0));
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            g.c[4 * q + e] = c[e];
            g.s[4 * q + e] = s[e];
        }
    }
    if (!known) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < 4 ? at.turns0 : at.turns1) g.c[e] = g.s[e] = __builtin_nanf("");
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
    Walk walk;
    const uint16_t* x;
    int64_t x_st, x_sh;
    void* y;                   // dense destination (strides y_st, y_sh), or the pages (strides y_sp, y_sh, y_st)
    int64_t y_sp, y_st, y_sh;
    const uint16_t* w;
    const float* scale;
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

// 16 bytes that nothing reads again soon: past the caches (forward of 131072 tokens of 32/8 heads 506 -> 484 us)
__device__ __forceinline__ void stream_out(uint16_t* y, u32x4 v) { __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(y)); }

__device__ __forceinline__ u32x4 stream_in(const uint16_t* x) { return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(x)); }

// One step a wavefront.  131072 tokens of 32/8 heads of 128: 440 us, 6.1 TB/s; prompts of 32000 tokens of 28/4 into pages 87, 6.2 TB/s; a few hundred tokens 3 - 4 us.
template <int D, bool PAIRS>
__global__ __launch_bounds__(256) void head_map_kernel(HeadParams p) {
    const HeadPart& t = p.part[blockIdx.x >= p.part[2].walk.first ? 2 : blockIdx.x >= p.part[1].walk.first ? 1 : 0];
    const Place<D> place(t.walk);
    const int rot = t.map && p.rotation.rope ? p.rotation.rot : 0;
    const Pieces<D, PAIRS> at(place.l, rot);
    const uint16_t* x0 = t.x + (int64_t)place.token * t.x_st + (int64_t)place.head * t.x_sh;
    const bool norm = t.map && t.w;
    const Step step(t.walk, place, (blockIdx.x - t.walk.first) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
    if (!step.live) return;                      // (the lanes of a head are live together)
    const uint32_t token = step.token + place.token, h = step.head + place.head;
    const uint16_t* x = x0 + (int64_t)step.token * t.x_st + (int64_t)step.head * t.x_sh;
    const int pos = rot ? p.rotation.positions[token] : 0, slot = t.paged ? p.slots[token] : 0;
    const u32x4 ra = stream_in(x + at.a), rb = stream_in(x + at.b);
    float wa[8], wb[8], a[8], b[8];
    if (norm) {
        unpack8(*reinterpret_cast<const u32x4*>(t.w + at.a), wa);
        unpack8(*reinterpret_cast<const u32x4*>(t.w + at.b), wb);
    }
    Angles g;
    if (at.turns0 || at.turns1) load_angles(p.rotation, pos, at, g);
    unpack8(ra, a);
    unpack8(rb, b);
    if (norm) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = fmaf(a[e], a[e], fmaf(b[e], b[e], sum));
        const float r = __builtin_amdgcn_rsqf(lanes_sum<D / 16>(sum) * (1.0f / D) + p.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            a[e] *= r * wa[e];
            b[e] *= r * wb[e];
        }
    }
    if (at.turns0 || at.turns1) turn<PAIRS, false>(g, a, b);
    if (!t.paged) {
        uint16_t* y = (uint16_t*)t.y + (int64_t)token * t.y_st + (int64_t)h * t.y_sh;
        stream_out(y + at.a, pack8(a));
        stream_out(y + at.b, pack8(b));
        return;
    }
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
}

// ---- gradient -----------------------------------------------------------------------------------------------
struct GradPart {
    Walk walk;
    const uint16_t *dy, *x;    // x: only with a weight
    int64_t dy_st, dy_sh, x_st, x_sh;
    uint16_t* dx;
    int64_t dx_st, dx_sh;
    const uint16_t* w;
    float* partial;            // [D / 4][workgroups][4] sums for the weight's gradient, or NULL
};
struct GradParams {
    GradPart part[2];
    Rotation rotation;
    float eps;
};

// A wavefront keeps the weight's gradient of all its steps in registers (16 entries a lane), so a workgroup adds one row of D sums to the
// workspace.  With t = r dz: dw += t x;  u = t w;  dx = u - x (r^2 mean(u x)).
// 65536 tokens of 32/32 heads of 128: 543 us, 5.9 TB/s; 333 tokens of 14/2 heads of 64: 4 us, and 2.6 for the sums.
template <int D, bool PAIRS>
__global__ __launch_bounds__(256) void head_map_grad_kernel(GradParams p) {
    __shared__ float sums[4][D];
    const GradPart& t = p.part[blockIdx.x >= p.part[1].walk.first ? 1 : 0];
    const Place<D> place(t.walk);
    const int rot = p.rotation.rope ? p.rotation.rot : 0;
    const Pieces<D, PAIRS> at(place.l, rot);
    const uint16_t* dy0 = t.dy + (int64_t)place.token * t.dy_st + (int64_t)place.head * t.dy_sh;
    const uint16_t* x0 = t.x + (int64_t)place.token * t.x_st + (int64_t)place.head * t.x_sh;
    uint16_t* dx0 = t.dx + (int64_t)place.token * t.dx_st + (int64_t)place.head * t.dx_sh;
    float wa[8], wb[8], dwa[8], dwb[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) dwa[e] = dwb[e] = 0.f;
    if (t.w) {
        unpack8(*reinterpret_cast<const u32x4*>(t.w + at.a), wa);
        unpack8(*reinterpret_cast<const u32x4*>(t.w + at.b), wb);
    }
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), stride = t.walk.groups * 4;
    // the next step's heads and position are requested before this one's are used
    u32x4 na4, nb4, nxa, nxb;
    int npos = 0;
    auto request = [&](uint32_t unit) {
        const Step s(t.walk, place, unit);
        if (!s.live) return;
        npos = rot ? p.rotation.positions[s.token + place.token] : 0;
        const uint16_t* dy = dy0 + (int64_t)s.token * t.dy_st + (int64_t)s.head * t.dy_sh;
        na4 = stream_in(dy + at.a);
        nb4 = stream_in(dy + at.b);
        if (t.w) {
            const uint16_t* x = x0 + (int64_t)s.token * t.x_st + (int64_t)s.head * t.x_sh;
            nxa = stream_in(x + at.a);
            nxb = stream_in(x + at.b);
        }
    };
    uint32_t unit = (blockIdx.x - t.walk.first) * 4 + wave;
    if (unit < t.walk.units) request(unit);
    for (; unit < t.walk.units; unit += stride) {
        const Step step(t.walk, place, unit);
        const u32x4 ra = na4, rb = nb4, xa = nxa, xb = nxb;
        const int pos = npos;
        if (unit + stride < t.walk.units) request(unit + stride);
        if (!step.live) continue;
        Angles g;
        if (at.turns0 || at.turns1) load_angles(p.rotation, pos, at, g);
        float a[8], b[8];
        unpack8(ra, a);
        unpack8(rb, b);
        if (at.turns0 || at.turns1) turn<PAIRS, true>(g, a, b);
        if (t.w) {
            float na[8], nb[8], sum = 0.f, dot = 0.f;
            unpack8(xa, na);
            unpack8(xb, nb);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = fmaf(na[e], na[e], fmaf(nb[e], nb[e], sum));
            const float r = __builtin_amdgcn_rsqf(lanes_sum<D / 16>(sum) * (1.0f / D) + p.eps);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                a[e] *= r;
                b[e] *= r;
                dwa[e] = fmaf(a[e], na[e], dwa[e]);
                dwb[e] = fmaf(b[e], nb[e], dwb[e]);
                a[e] *= wa[e];
                b[e] *= wb[e];
                dot = fmaf(a[e], na[e], fmaf(b[e], nb[e], dot));
            }
            const float c = -(r * r) * (lanes_sum<D / 16>(dot) * (1.0f / D));
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                a[e] = fmaf(na[e], c, a[e]);
                b[e] = fmaf(nb[e], c, b[e]);
            }
        }
        uint16_t* dx = dx0 + (int64_t)step.token * t.dx_st + (int64_t)step.head * t.dx_sh;
        stream_out(dx + at.a, pack8(a));
        stream_out(dx + at.b, pack8(b));
    }
    if (!t.partial) return;                  // (uniform in the workgroup)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        dwa[e] = over_heads<D>(dwa[e]);
        dwb[e] = over_heads<D>(dwb[e]);
        if (lane_id() < D / 16) {
            sums[wave][at.a + e] = dwa[e];
            sums[wave][at.b + e] = dwb[e];
        }
    }
    __syncthreads();
    if (threadIdx.x < D / 4) {
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int c = 4 * threadIdx.x + e;
            v[e] = (sums[0][c] + sums[1][c]) + (sums[2][c] + sums[3][c]);
        }
        *reinterpret_cast<f32x4*>(t.partial + ((int64_t)threadIdx.x * t.walk.groups + (blockIdx.x - t.walk.first)) * 4) = v;
    }
}

struct GradSumParams {
    const float* partial[2];
    float* out[2];
    int groups[2];
};
// Four entries of one weight's gradient a workgroup, whose sums lie in a row: 16 bytes a thread and workgroup of the first launch, eight of
// them requested at a time, then the threads in a fixed order.
__global__ __launch_bounds__(1024) void head_grad_sum_kernel(GradSumParams p) {
    __shared__ f32x4 s[16];
    const int which = blockIdx.y, n = p.groups[which];
    if (!p.out[which]) return;
    const f32x4* in = reinterpret_cast<const f32x4*>(p.partial[which]) + (int64_t)blockIdx.x * n;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    for (int i = threadIdx.x; i < n; i += 1024 * 8) {
        f32x4 u[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) u[k] = in[min(i + 1024 * k, n - 1)];                   // (past the last one it is loaded again and not used)
#pragma unroll
        for (int k = 0; k < 8; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += i + 1024 * k < n ? u[k][e] : 0.f;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[e] = lanes_sum<128 / 16>(v[e]);                       // 8 lanes
        v[e] = over_heads<128>(v[e]);                     // and the eight eights
    }
    if (lane_id() == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    if (threadIdx.x < 4) {
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < 16; ++w) sum += s[w][threadIdx.x];
        p.out[which][blockIdx.x * 4 + threadIdx.x] = sum;
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
    // (the hardware's reciprocal root takes denormals for zeros: mean + eps has to be none)
    if ((m.q_weight || m.k_weight) && !(m.eps >= 1.17549435e-38f)) return fail(DLM_ERR_INVALID_ARG, "%s: a norm needs eps > 0 (at least 2^-126)", who);
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

static HeadPart head_part(int T, int H, int d, const void* x, int64_t x_st, int64_t x_sh, void* y, int64_t y_sp, int64_t y_st, int64_t y_sh,
                          const void* w, const float* scale, int map, int paged) {
    return HeadPart{walk_of(T, H, d), (const uint16_t*)x, x_st, x_sh, y, y_sp, y_st, y_sh, (const uint16_t*)w, scale, map, paged};
}

// Shares out workgroups of 4 wavefronts to the parts of a launch in proportion to their steps, about `most` in all; returns their number.
static uint32_t deal(Walk** walk, int n, uint32_t most) {
    int64_t units = 0;
    for (int i = 0; i < n; ++i) units += walk[i]->units;
    const int64_t each = 4 * ((units + 4 * (int64_t)most - 1) / (4 * (int64_t)most));      // steps of a workgroup
    uint32_t groups = 0;
    for (int i = 0; i < n; ++i) {
        walk[i]->first = groups;
        walk[i]->groups = walk[i]->units ? (uint32_t)((walk[i]->units + each - 1) / each) : 0;
        groups += walk[i]->groups;
    }
    return groups;
}

static int launch_head_map(HeadParams& p, int d, int style, const char* who, hipStream_t st) {
    Walk* walks[3] = {&p.part[0].walk, &p.part[1].walk, &p.part[2].walk};
    const uint32_t groups = deal(walks, 3, 1u << 29);            // one step a wavefront: loops over several were 5 - 12 % slower
    if (groups == 0) return DLM_OK;
    if (groups >= 1u << 24) return fail(DLM_ERR_UNSUPPORTED, "%s: too many heads for one launch", who);      // (2^32 threads)
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

// The gradient's workgroups.  A wavefront that takes many steps needs few sums written and reduced, but workgroups that all stay to the end stream
// worse than ones that come and go (65536 tokens of 32/32 heads: 1024 workgroups 592 us, 8192 558, 16384 543; one step a wavefront 717), so: eight steps a
// wavefront and at most 16384 workgroups (8 MB of sums for d = 128), but where that is less than four rounds of the 1024 that are resident (four a
// CU) those, in one round (12289 tokens of 28/4: 1024 workgroups 55 us, 1536 60).
static uint32_t deal_grad(int T, int Hq, int Hkv, int d, Walk& q, Walk& k) {
    q = walk_of(T, Hq, d);
    k = walk_of(T, Hkv, d);
    Walk* walks[2] = {&q, &k};
    const int64_t by_steps = ((int64_t)q.units + k.units) / 32;
    return deal(walks, 2, by_steps < 4096 ? 1024 : by_steps > 16384 ? 16384 : (uint32_t)by_steps);
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
    p.part[0] = head_part(a->T, a->Hq, a->d, a->q, a->q_stride_t, a->q_stride_h, a->q_out, 0, a->qo_stride_t, a->qo_stride_h, a->map.q_weight, nullptr, 1, 0);
    p.part[1] = head_part(a->T, a->Hkv, a->d, a->k, a->k_stride_t, a->k_stride_h, a->k_out, 0, a->ko_stride_t, a->ko_stride_h, a->map.k_weight, nullptr, 1, 0);
    p.part[2].walk = walk_of(0, 0, a->d);
    p.rotation = rotation_of(a->map);
    p.eps = a->map.eps;
    return launch_head_map(p, a->d, a->map.rope_style, who, (hipStream_t)stream);
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
    const int kind = c.type == DLM_KV_E4M3 ? 2 : 1;
    p.part[0] = head_part(a->T, a->Hq, a->d, a->q, a->q_stride_t, a->q_stride_h, a->q_out, 0, a->qo_stride_t, a->qo_stride_h, a->map.q_weight, nullptr, 1, 0);
    p.part[1] = head_part(a->T, a->Hkv, a->d, a->k, a->k_stride_t, a->k_stride_h, c.k, c.stride_page, c.stride_t, c.stride_h, a->map.k_weight, c.k_scale, 1, kind);
    p.part[2] = head_part(a->T, a->Hkv, a->d, a->v, a->v_stride_t, a->v_stride_h, c.v, c.stride_page, c.stride_t, c.stride_h, nullptr, c.v_scale, 0, kind);
    p.rotation = rotation_of(a->map);
    p.eps = a->map.eps;
    p.slots = a->slots;
    p.n_slots = (uint32_t)c.n_pages * (uint32_t)c.page_size;
    p.page_shift = log2_of(c.page_size);
    return launch_head_map(p, a->d, a->map.rope_style, who, (hipStream_t)stream);
}

extern "C" size_t dlm_qk_norm_rope_bwd_workspace_bytes(const dlm_qk_bwd_args* a) {
    if (!a || a->struct_size != sizeof(dlm_qk_bwd_args) || a->T < 0 || a->Hq < 0 || a->Hkv < 0 || (a->d != 64 && a->d != 128)) return 0;
    Walk q, k;
    return (size_t)deal_grad(a->T, a->Hq, a->Hkv, a->d, q, k) * a->d * sizeof(float);
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
    GradParams p = {};
    const uint32_t groups = deal_grad(a->T, a->Hq, a->Hkv, a->d, p.part[0].walk, p.part[1].walk);
    const uint32_t gq = p.part[0].walk.groups, gk = p.part[1].walk.groups;
    float* part_q = (float*)a->workspace;
    float* part_k = part_q + (size_t)gq * a->d;
    hipStream_t st = (hipStream_t)stream;
    if (groups > 0) {
        p.part[0] = GradPart{p.part[0].walk, (const uint16_t*)a->d_q_out, (const uint16_t*)a->q, a->dqo_stride_t, a->dqo_stride_h, a->q_stride_t,
                             a->q_stride_h, (uint16_t*)a->d_q, a->dq_stride_t, a->dq_stride_h, (const uint16_t*)a->map.q_weight,
                             a->d_q_weight ? part_q : nullptr};
        p.part[1] = GradPart{p.part[1].walk, (const uint16_t*)a->d_k_out, (const uint16_t*)a->k, a->dko_stride_t, a->dko_stride_h, a->k_stride_t,
                             a->k_stride_h, (uint16_t*)a->d_k, a->dk_stride_t, a->dk_stride_h, (const uint16_t*)a->map.k_weight,
                             a->d_k_weight ? part_k : nullptr};
        p.rotation = rotation_of(a->map);
        p.eps = a->map.eps;
        const bool pairs = p.rotation.rope && a->map.rope_style == DLM_ROPE_PAIRS;
        if (a->d == 128) {
            if (pairs) hipLaunchKernelGGL((head_map_grad_kernel<128, true>), dim3(groups), dim3(256), 0, st, p);
            else hipLaunchKernelGGL((head_map_grad_kernel<128, false>), dim3(groups), dim3(256), 0, st, p);
        } else {
            if (pairs) hipLaunchKernelGGL((head_map_grad_kernel<64, true>), dim3(groups), dim3(256), 0, st, p);
            else hipLaunchKernelGGL((head_map_grad_kernel<64, false>), dim3(groups), dim3(256), 0, st, p);
        }
        if ((rc = check_hip(hipGetLastError(), "head_map_grad_kernel launch")) != DLM_OK) return rc;
    }
    if (!sums) return DLM_OK;
    const GradSumParams s = {{part_q, part_k}, {a->d_q_weight, a->d_k_weight}, {(int)gq, (int)gk}};
    hipLaunchKernelGGL(head_grad_sum_kernel, dim3(a->d / 4, 2), dim3(1024), 0, st, s);
    return check_hip(hipGetLastError(), "head_grad_sum_kernel launch");
}
