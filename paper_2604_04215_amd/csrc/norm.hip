// dlm_row_norm and its gradient: RMS or layer norm of the rows between two layers, the residual added on the way in.
//
// Both read every row once and keep it in registers: a team of TPR threads owns a row, N entries each, in 16-byte pieces that lie side by
// side over the team.  Bound by HBM (many rows) or by one chain load -> sum -> store (few).
//
// The mean of a layer norm is taken twice: once over the entries, once over what is left when that mean is subtracted, whose sum would be
// zero without rounding.  Rows of large mean and small deviation (or all equal) so lose nothing to the rounding of the mean, and the second sum
// comes with the sum of squares: no further pass.
//
// Measured: 65536 rows of 3584 fp32, layer norm into bf16 258 us, 5.5 TB/s; the gradient of 65536 rows of 4096 bf16 with d_sum and the weight's 362, 5.9 TB/s (a copy
// reaches 6.2); 256 rows of 4096 with a residual 4.1, of which the GPU works 3; the gradient of 333 rows of 896 8.4, two launches.
#include "rows.hpp"

namespace dlm {

struct NormParams {
    int T, D;
    const void *x, *residual;      // residual NULL: none
    int64_t x_st, r_st;
    void* sum;                     // NULL: not wanted
    int64_t s_st;
    const uint16_t *w, *b;         // NULL: 1, 0
    uint16_t* y;
    int64_t y_st;
    float eps, by_d;               // by_d: 1 / D
    int layer;
};

// Sums over a team of TPR threads; every thread gets the same bits.  Teams of several wavefronts meet in `meet`, of which each call takes the
// other half, so that one barrier a call is enough: a wavefront that writes a half has passed the barrier behind the last reads of it.
template <int TPR, int K>
struct TeamSum {
    static constexpr int W = TPR / WAVE;            // wavefronts of a team (0, 1: no meeting)
    float* meet;                                    // [2][teams][W][K]
    int half;
    __device__ __forceinline__ TeamSum(float* m) : meet(m + (W > 1 ? threadIdx.x / TPR * W * K : 0)), half(0) {}
    template <int N>
    __device__ __forceinline__ void operator()(float (&v)[N]) {
        static_assert(N <= K, "room for K sums");
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = lanes_sum<(TPR < WAVE ? TPR : WAVE)>(v[i]);
        if constexpr (W > 1) {
            constexpr int HALF = 1024 / WAVE * K;
            float* m = meet + half * HALF;
            half ^= 1;
            const int wave = threadIdx.x % TPR / WAVE;
            if (lane_id() == 0) {
#pragma unroll
                for (int i = 0; i < N; ++i) m[wave * K + i] = v[i];
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < N; ++i) {
                float s = m[i];
#pragma unroll
                for (int k = 1; k < W; ++k) s += m[k * K + i];
                v[i] = s;
            }
        }
    }
};

template <bool F32, int N, int TPR>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void norm_kernel(NormParams p) {
    using P = Piece<F32>;
    constexpr int E = P::E, NP = N / E, TEAMS = TPR > 256 ? 1 : 256 / TPR;
    __shared__ float meet[2 * 1024 / WAVE * 2];
    TeamSum<TPR, 2> total(meet);
    const int l = threadIdx.x % TPR;
    const int64_t row0 = (int64_t)blockIdx.x * TEAMS + threadIdx.x / TPR;
    const bool live = row0 < p.T;
    const int64_t row = live ? row0 : p.T - 1;      // (teams behind the last row meet the others, and store nothing)
    typename P::Raw raw[NP], more[NP];
#pragma unroll
    for (int j = 0; j < NP; ++j) {
        raw[j] = more[j] = u32x4{0, 0, 0, 0};
        const int c = (j * TPR + l) * E;
        if (c < p.D) {
            raw[j] = P::stream(p.x, row * p.x_st + c);
            if (p.residual) more[j] = P::stream(p.residual, row * p.r_st + c);
        }
    }
    float v[NP][E], s[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NP; ++j) {
        const int c = (j * TPR + l) * E;
        P::open(raw[j], v[j]);
        if (p.residual) {
            float r[E];
            P::open(more[j], r);
#pragma unroll
            for (int e = 0; e < E; ++e) v[j][e] += r[e];
            const typename P::Raw kept = P::close(v[j]);
            if (p.sum && live && c < p.D) P::stream_out(p.sum, row * p.s_st + c, kept);
            P::open(kept, v[j]);                    // what is normalised is the sum as it is kept
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            s[0] += v[j][e];
            s[1] = fmaf(v[j][e], v[j][e], s[1]);
        }
    }
    total(s);
    float off = 0.f, square = s[1] * p.by_d;
    if (p.layer) {
        const float mean = s[0] * p.by_d;
        float t[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NP; ++j) {
            if ((j * TPR + l) * E < p.D) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    v[j][e] -= mean;
                    t[0] += v[j][e];
                    t[1] = fmaf(v[j][e], v[j][e], t[1]);
                }
            }
        }
        total(t);
        off = t[0] * p.by_d;
        square = fmaxf(t[1] * p.by_d - off * off, 0.f);
        if (t[1] != t[1]) square = t[1];            // (a maximum drops NaN)
    }
    const float r = __builtin_amdgcn_rsqf(square + p.eps);
    if (!live) return;
#pragma unroll
    for (int j = 0; j < NP; ++j) {
        const int c = (j * TPR + l) * E;
        if (c >= p.D) continue;
        float w[E], b[E];
        if (p.w) load_bf16<E>(p.w + c, w);
        if (p.b) load_bf16<E>(p.b + c, b);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            float y = (v[j][e] - off) * r;
            if (p.w) y *= w[e];
            if (p.b) y += b[e];
            v[j][e] = y;
        }
        uint32_t q[E / 2];
#pragma unroll
        for (int i = 0; i < E / 2; ++i) q[i] = pack_bf16x2(v[j][2 * i], v[j][2 * i + 1]);
        uint16_t* y = p.y + row * p.y_st + c;
        if constexpr (E == 8) __builtin_nontemporal_store(u32x4{q[0], q[1], q[2], q[3]}, reinterpret_cast<u32x4*>(y));
        else __builtin_nontemporal_store(u32x2{q[0], q[1]}, reinterpret_cast<u32x2*>(y));
    }
}

// ---- gradient -----------------------------------------------------------------------------------------------
struct NormGradParams {
    int T, D;
    const uint16_t* dy;
    int64_t dy_st;
    const void *x, *ds;            // ds NULL: none
    int64_t x_st, ds_st;
    void* dx;
    int64_t dx_st;
    const uint16_t* w;
    float* part;                   // [workgroups][2][D]: sums for the weight's and the bias' gradients, or NULL
    float eps, by_d;
    int layer;
};

// With n the normalised row, r its factor and g = dy w:  dx = r (g - [layer] mean(g) - n mean(g n)) + ds;  dw = sum of dy n;  db = sum of dy.
// Every team takes one row after the other, the next one's pieces requested before this one's sums are formed, and keeps the sums of its columns in registers;
// norm_sum_kernel adds the workgroups' (5.6 us for 1024 of 4096 columns).
template <bool F32, int N, int TPR>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void norm_grad_kernel(NormGradParams p) {
    using P = Piece<F32>;
    constexpr int E = P::E, NP = N / E, TEAMS = TPR > 256 ? 1 : 256 / TPR, THREADS = TPR > 256 ? TPR : 256;
    constexpr int MEET = 2 * 1024 / WAVE * 3, COLUMNS = TEAMS > 1 ? THREADS * N : 0;
    __shared__ float lds[MEET > COLUMNS ? MEET : COLUMNS];
    TeamSum<TPR, 3> total(lds);
    const int l = threadIdx.x % TPR, team = threadIdx.x / TPR;
    float dw[NP][E], db[NP][E], w[NP][E];
#pragma unroll
    for (int j = 0; j < NP; ++j) {
        const int c = (j * TPR + l) * E;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            dw[j][e] = db[j][e] = 0.f;
            w[j][e] = 1.f;
        }
        if (p.w && c < p.D) load_bf16<E>(p.w + c, w[j]);
    }
    typename P::Raw nx[NP], ns[NP];
    u32x2 ny[NP][E / 4];
    const auto request = [&](int64_t row0) {
        const int64_t row = row0 < p.T ? row0 : p.T - 1;
#pragma unroll
        for (int j = 0; j < NP; ++j) {
            const int c = (j * TPR + l) * E;
            nx[j] = ns[j] = u32x4{0, 0, 0, 0};
#pragma unroll
            for (int h = 0; h < E / 4; ++h) ny[j][h] = u32x2{0, 0};
            if (c < p.D) {
                nx[j] = P::stream(p.x, row * p.x_st + c);
                const uint16_t* dy = p.dy + row * p.dy_st + c;
                if constexpr (E == 8) {
                    const u32x4 q = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(dy));
                    ny[j][0] = u32x2{q[0], q[1]};
                    ny[j][E / 4 - 1] = u32x2{q[2], q[3]};
                } else {
                    ny[j][0] = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(dy));
                }
                if (p.ds) ns[j] = P::stream(p.ds, row * p.ds_st + c);
            }
        }
    };
    const int64_t step = (int64_t)gridDim.x * TEAMS;
    int64_t base = (int64_t)blockIdx.x * TEAMS;     // the same for all teams of a workgroup: they meet
    if (base < p.T) request(base + team);
    for (; base < p.T; base += step) {
        const int64_t row = base + team;
        const bool live = row < p.T;
        float x[NP][E], g[NP][E];
        typename P::Raw s4[NP];
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NP; ++j) {
            P::open(nx[j], x[j]);
            s4[j] = ns[j];
#pragma unroll
            for (int i = 0; i < E / 2; ++i) {
                g[j][2 * i] = __uint_as_float(ny[j][i / 2][i % 2] << 16);
                g[j][2 * i + 1] = __uint_as_float(ny[j][i / 2][i % 2] & 0xffff0000u);
            }
        }
        if (base + step < p.T) request(base + step + team);
        float off = 0.f, mean_g = 0.f, t[3] = {0.f, 0.f, 0.f};      // sums of x^2, g x, x
        if (p.layer) {
#pragma unroll
            for (int j = 0; j < NP; ++j)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    s[0] += x[j][e];
                    s[1] = fmaf(g[j][e], w[j][e], s[1]);
                }
            total(s);
            const float mean = s[0] * p.by_d;
            mean_g = s[1] * p.by_d;
#pragma unroll
            for (int j = 0; j < NP; ++j)
                if ((j * TPR + l) * E < p.D) {
#pragma unroll
                    for (int e = 0; e < E; ++e) x[j][e] -= mean;
                }
        }
#pragma unroll
        for (int j = 0; j < NP; ++j)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                t[0] = fmaf(x[j][e], x[j][e], t[0]);
                t[1] = fmaf(g[j][e] * w[j][e], x[j][e], t[1]);
                t[2] += x[j][e];
            }
        total(t);
        float square = t[0] * p.by_d, gx = t[1] * p.by_d;
        if (p.layer) {
            off = t[2] * p.by_d;
            square = fmaxf(square - off * off, 0.f);
            if (t[0] != t[0]) square = t[0];
            gx -= off * mean_g;
        }
        const float r = __builtin_amdgcn_rsqf(square + p.eps), gn = gx * r;
        if (live) {
#pragma unroll
            for (int j = 0; j < NP; ++j) {
                const int c = (j * TPR + l) * E;
                if (c >= p.D) continue;
                float ds[E], dx[E];
                P::open(s4[j], ds);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float n = (x[j][e] - off) * r;
                    dw[j][e] = fmaf(g[j][e], n, dw[j][e]);
                    db[j][e] += g[j][e];
                    dx[e] = (g[j][e] * w[j][e] - mean_g - n * gn) * r;
                    if (p.ds) dx[e] += ds[e];
                }
                P::stream_out(p.dx, row * p.dx_st + c, P::close(dx));
            }
        }
    }
    if (!p.part) return;
    float* part = p.part + (int64_t)blockIdx.x * 2 * p.D;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        if constexpr (TEAMS > 1) {                  // the teams' sums in their order
            __syncthreads();
#pragma unroll
            for (int j = 0; j < NP; ++j)
#pragma unroll
                for (int e = 0; e < E; ++e) lds[(team * TPR + l) * N + j * E + e] = which ? db[j][e] : dw[j][e];
            __syncthreads();
            if (team == 0) {
#pragma unroll
                for (int j = 0; j < NP; ++j)
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        float a = 0.f;
                        for (int k = 0; k < TEAMS; ++k) a += lds[(k * TPR + l) * N + j * E + e];
                        if (which) db[j][e] = a;
                        else dw[j][e] = a;
                    }
            }
        }
        if (team == 0) {
#pragma unroll
            for (int j = 0; j < NP; ++j) {
                const int c = (j * TPR + l) * E;
                if (c >= p.D) continue;
#pragma unroll
                for (int q = 0; q < E / 4; ++q) {
                    const float* a = which ? &db[j][4 * q] : &dw[j][4 * q];
                    *reinterpret_cast<f32x4*>(part + which * p.D + c + 4 * q) = f32x4{a[0], a[1], a[2], a[3]};
                }
            }
        }
    }
}

// Adds the workgroups' sums: 64 columns a workgroup, its 16 wavefronts one stretch of the rows each, the stretches in their order.
__global__ __launch_bounds__(1024) void norm_sum_kernel(const float* part, int groups, int D, float* dw, float* db) {
    __shared__ float lds[16][WAVE];
    float* out = blockIdx.y ? db : dw;
    if (!out) return;
    const int wave = threadIdx.x / WAVE, c = blockIdx.x * WAVE + lane_id(), at = c < D ? c : D - 1;
    const int each = (groups + 15) / 16, g0 = wave * each, g1 = g0 + each < groups ? g0 + each : groups;
    const float* src = part + (int64_t)blockIdx.y * D + at;
    float a = 0.f;
#pragma unroll 8
    for (int g = g0; g < g1; ++g) a += src[(int64_t)g * 2 * D];
    lds[wave][lane_id()] = a;
    __syncthreads();
    if (wave == 0 && c < D) {
        a = 0.f;
#pragma unroll
        for (int k = 0; k < 16; ++k) a += lds[k][lane_id()];
        out[c] = a;
    }
}

// ---- host ---------------------------------------------------------------------------------------------------
constexpr int NORM_MAX_D = 16384;

static int validate_norm(int T, int D, int kind, float eps, int type, const char* who) {
    if (T < 0 || D <= 0) return fail(DLM_ERR_INVALID_ARG, "%s: bad sizes T=%d D=%d", who, T, D);
    if (D % 8 || D > NORM_MAX_D) return fail(DLM_ERR_UNSUPPORTED, "%s: D=%d (supported: multiples of 8 up to %d)", who, D, NORM_MAX_D);
    if (kind != DLM_NORM_RMS && kind != DLM_NORM_LAYER) return fail(DLM_ERR_INVALID_ARG, "%s: unknown kind %d", who, kind);
    if (!(eps >= 1.17549435e-38f) || eps > 3.0e38f) return fail(DLM_ERR_INVALID_ARG, "%s: eps must be at least 2^-126 and finite", who);
    return validate_row_type(type, who, "x");
}

// Rows written where an input of the same call lies have to be that input's own: an entry is read and written by one thread.
static int validate_in_place(const void* out, int64_t stride, int bytes, const void* in, int64_t in_stride, int in_bytes, int T, const char* who, const char* names) {
    if (!in || out != in) return DLM_OK;
    if (bytes != in_bytes || (T > 1 && stride != in_stride)) return fail(DLM_ERR_INVALID_ARG, "%s: %s are one buffer of different types or strides", who, names);
    return DLM_OK;
}

template <bool F32, int N, int TPR>
static void launch_norm(const NormParams& all, hipStream_t st) {
    constexpr int TEAMS = TPR > 256 ? 1 : 256 / TPR, BYTES = F32 ? 4 : 2;
    constexpr int MOST = 1 << 20;                   // rows a launch: its threads stay below 2^32
    for (int64_t t0 = 0; t0 < all.T; t0 += MOST) {
        NormParams p = all;
        p.T = (int)(all.T - t0 < MOST ? all.T - t0 : MOST);
        p.x = (const char*)all.x + t0 * all.x_st * BYTES;
        if (all.residual) p.residual = (const char*)all.residual + t0 * all.r_st * BYTES;
        if (all.sum) p.sum = (char*)all.sum + t0 * all.s_st * BYTES;
        p.y = all.y + t0 * all.y_st;
        hipLaunchKernelGGL((norm_kernel<F32, N, TPR>), dim3((unsigned)((p.T + TEAMS - 1) / TEAMS)), dim3(TPR > 256 ? TPR : 256), 0, st, p);
    }
}
// As many threads a row as have a piece each; with many rows and nothing to add a wavefront or little more a row, whose threads have more in flight and no
// barrier between them.  us, pieces one a thread / rows on few threads: 65536 rows of 3584 bf16 188 / 152, of 1024 49 / 43, 16384 of 4096 50 / 44, 4096 of 8192 27 / 24; layer norm
// of fp32 rows, 65536 of 3584 274 / 260, 4096 of 8192 44 / 40; 1024 rows of 2048 4.3 / 4.9, 2048 of 2048 5.6 / 6.1.  With a residual: 65536 of 4096 340 / 364, 16384 of 4096
// 85 / 92, fp32 150 / 155, layer norm 87 / 91.
template <bool F32>
static void pick_norm(const NormParams& p, hipStream_t st) {
    const int D = p.D;
    if (D <= 64) launch_norm<F32, 8, 8>(p, st);
    else if (D <= 128) launch_norm<F32, 8, 16>(p, st);
    else if (D <= 256) launch_norm<F32, 8, 32>(p, st);
    else if (D <= 512) launch_norm<F32, 8, 64>(p, st);
    else if (p.T > 2048 && !p.residual) {
        constexpr int N = F32 ? 16 : 32;            // (32 entries of fp32 a thread: 244 registers, 659 us where 16 take 250)
        if (D <= 1024) launch_norm<F32, 16, 64>(p, st);
        else if (D <= 2048) launch_norm<F32, N, 2048 / N>(p, st);
        else if (D <= 4096) launch_norm<F32, N, 4096 / N>(p, st);
        else if (D <= 8192) launch_norm<F32, N, 8192 / N>(p, st);
        else launch_norm<F32, N, 16384 / N>(p, st);
    } else {
        if (D <= 1024) launch_norm<F32, 8, 128>(p, st);
        else if (D <= 2048) launch_norm<F32, 8, 256>(p, st);
        else if (D <= 4096) launch_norm<F32, 8, 512>(p, st);
        else if (D <= 8192) launch_norm<F32, 8, 1024>(p, st);
        else launch_norm<F32, 16, 1024>(p, st);
    }
}

// Threads a row of the gradient, and its workgroups
static int grad_threads(int D) {
    if (D <= 512) return D <= 64 ? 8 : D <= 128 ? 16 : D <= 256 ? 32 : 64;
    int t = 64;
    while (t * 16 < D) t *= 2;
    return t;
}
static int grad_groups(int T, int D) {
    const int tpr = grad_threads(D), teams = tpr > 256 ? 1 : 256 / tpr, most = 1024 * 256 / (tpr > 256 ? tpr : 256);
    const int64_t want = ((int64_t)T + teams - 1) / teams;
    return want < most ? (int)want : most;
}
template <bool F32>
static void pick_norm_grad(const NormGradParams& p, int groups, hipStream_t st) {
#define NORM_GRAD(N, TPR) hipLaunchKernelGGL((norm_grad_kernel<F32, N, TPR>), dim3(groups), dim3(TPR > 256 ? TPR : 256), 0, st, p)
    switch (grad_threads(p.D)) {
        case 8: NORM_GRAD(8, 8); break;
        case 16: NORM_GRAD(8, 16); break;
        case 32: NORM_GRAD(8, 32); break;
        case 64:
            if (p.D <= 512) NORM_GRAD(8, 64);
            else NORM_GRAD(16, 64);
            break;
        case 128: NORM_GRAD(16, 128); break;
        case 256: NORM_GRAD(16, 256); break;
        case 512: NORM_GRAD(16, 512); break;
        default: NORM_GRAD(16, 1024); break;
    }
#undef NORM_GRAD
}

}  // namespace dlm

using namespace dlm;

extern "C" int dlm_row_norm(const dlm_row_norm_args* a, void* stream) {
    static const char who[] = "row_norm";
    if (!a) return fail(DLM_ERR_INVALID_ARG, "%s: null args", who);
    if (a->struct_size != sizeof(dlm_row_norm_args))
        return fail(DLM_ERR_INVALID_ARG, "%s: struct_size %u != %zu", who, a->struct_size, sizeof(dlm_row_norm_args));
    int rc;
    if ((rc = validate_norm(a->T, a->D, a->kind, a->eps, a->x_type, who)) != DLM_OK) return rc;
    if (a->sum_out && !a->residual) return fail(DLM_ERR_INVALID_ARG, "%s: sum_out goes with a residual", who);
    const int bytes = row_bytes(a->x_type);
    if ((rc = validate_rows(a->x, a->x_stride, a->T, a->D, bytes, false, who, "x")) != DLM_OK) return rc;
    if (a->residual && (rc = validate_rows(a->residual, a->residual_stride, a->T, a->D, bytes, false, who, "residual")) != DLM_OK) return rc;
    if (a->sum_out && (rc = validate_rows(a->sum_out, a->sum_stride, a->T, a->D, bytes, true, who, "sum_out")) != DLM_OK) return rc;
    if ((rc = validate_rows(a->out, a->out_stride, a->T, a->D, 2, true, who, "out")) != DLM_OK) return rc;
    if (!aligned16(a->weight) || !aligned16(a->bias)) return fail(DLM_ERR_UNSUPPORTED, "%s: weight / bias not 16-byte aligned", who);
    if (a->T == 0) return DLM_OK;
    if (a->sum_out && a->sum_out == a->out) return fail(DLM_ERR_INVALID_ARG, "%s: sum_out is out", who);
    if ((rc = validate_in_place(a->out, a->out_stride, 2, a->x, a->x_stride, bytes, a->T, who, "out and x")) != DLM_OK) return rc;
    if ((rc = validate_in_place(a->out, a->out_stride, 2, a->residual, a->residual_stride, bytes, a->T, who, "out and residual")) != DLM_OK) return rc;
    if (a->sum_out) {
        if ((rc = validate_in_place(a->sum_out, a->sum_stride, bytes, a->x, a->x_stride, bytes, a->T, who, "sum_out and x")) != DLM_OK) return rc;
        if ((rc = validate_in_place(a->sum_out, a->sum_stride, bytes, a->residual, a->residual_stride, bytes, a->T, who, "sum_out and residual")) != DLM_OK) return rc;
    }
    NormParams p = {a->T, a->D, a->x, a->residual, a->x_stride, a->residual_stride, a->sum_out, a->sum_stride, (const uint16_t*)a->weight,
                    (const uint16_t*)a->bias, (uint16_t*)a->out, a->out_stride, a->eps, 1.0f / (float)a->D, a->kind == DLM_NORM_LAYER};
    if (a->x_type == DLM_ROW_F32) pick_norm<true>(p, (hipStream_t)stream);
    else pick_norm<false>(p, (hipStream_t)stream);
    return check_hip(hipGetLastError(), "norm_kernel launch");
}

extern "C" size_t dlm_row_norm_bwd_workspace_bytes(const dlm_row_norm_bwd_args* a) {
    if (!a || a->struct_size != sizeof(dlm_row_norm_bwd_args) || a->T < 0 || a->D <= 0 || a->D % 8 || a->D > NORM_MAX_D) return 0;
    return (size_t)grad_groups(a->T, a->D) * 2 * a->D * sizeof(float);
}

extern "C" int dlm_row_norm_bwd(const dlm_row_norm_bwd_args* a, void* stream) {
    static const char who[] = "row_norm_bwd";
    if (!a) return fail(DLM_ERR_INVALID_ARG, "%s: null args", who);
    if (a->struct_size != sizeof(dlm_row_norm_bwd_args))
        return fail(DLM_ERR_INVALID_ARG, "%s: struct_size %u != %zu", who, a->struct_size, sizeof(dlm_row_norm_bwd_args));
    int rc;
    if ((rc = validate_norm(a->T, a->D, a->kind, a->eps, a->x_type, who)) != DLM_OK) return rc;
    const int bytes = row_bytes(a->x_type);
    if ((rc = validate_rows(a->d_out, a->d_out_stride, a->T, a->D, 2, false, who, "d_out")) != DLM_OK) return rc;
    if ((rc = validate_rows(a->x, a->x_stride, a->T, a->D, bytes, false, who, "x")) != DLM_OK) return rc;
    if (a->d_sum && (rc = validate_rows(a->d_sum, a->d_sum_stride, a->T, a->D, bytes, false, who, "d_sum")) != DLM_OK) return rc;
    if ((rc = validate_rows(a->d_x, a->d_x_stride, a->T, a->D, bytes, true, who, "d_x")) != DLM_OK) return rc;
    if (!aligned16(a->weight) || !aligned16(a->d_weight) || !aligned16(a->d_bias))
        return fail(DLM_ERR_UNSUPPORTED, "%s: weight / d_weight / d_bias not 16-byte aligned", who);
    if (a->d_weight && a->d_weight == a->d_bias) return fail(DLM_ERR_INVALID_ARG, "%s: d_weight and d_bias are one buffer", who);
    const bool sums = a->d_weight || a->d_bias;
    const size_t need = dlm_row_norm_bwd_workspace_bytes(a);
    if (sums && need > 0) {
        if (!a->workspace || a->workspace_bytes < need) return fail(DLM_ERR_WORKSPACE, "%s: workspace of %zu bytes required", who, need);
        if (!aligned16(a->workspace)) return fail(DLM_ERR_WORKSPACE, "%s: workspace not 16-byte aligned", who);
    }
    if (a->T > 0) {
        if ((rc = validate_in_place(a->d_x, a->d_x_stride, bytes, a->x, a->x_stride, bytes, a->T, who, "d_x and x")) != DLM_OK) return rc;
        if ((rc = validate_in_place(a->d_x, a->d_x_stride, bytes, a->d_sum, a->d_sum_stride, bytes, a->T, who, "d_x and d_sum")) != DLM_OK) return rc;
        if ((rc = validate_in_place(a->d_x, a->d_x_stride, bytes, a->d_out, a->d_out_stride, 2, a->T, who, "d_x and d_out")) != DLM_OK) return rc;
    }
    const int groups = grad_groups(a->T, a->D);
    float* part = sums ? (float*)a->workspace : nullptr;
    hipStream_t st = (hipStream_t)stream;
    if (groups > 0) {
        const NormGradParams p = {a->T, a->D, (const uint16_t*)a->d_out, a->d_out_stride, a->x, a->d_sum, a->x_stride, a->d_sum_stride, a->d_x,
                                  a->d_x_stride, (const uint16_t*)a->weight, part, a->eps, 1.0f / (float)a->D, a->kind == DLM_NORM_LAYER};
        if (a->x_type == DLM_ROW_F32) pick_norm_grad<true>(p, groups, st);
        else pick_norm_grad<false>(p, groups, st);
        if ((rc = check_hip(hipGetLastError(), "norm_grad_kernel launch")) != DLM_OK) return rc;
    }
    if (!sums) return DLM_OK;
    hipLaunchKernelGGL(norm_sum_kernel, dim3((a->D + WAVE - 1) / WAVE, 2), dim3(16 * WAVE), 0, st, part, groups, a->D, a->d_weight, a->d_bias);
    return check_hip(hipGetLastError(), "norm_sum_kernel launch");
}
