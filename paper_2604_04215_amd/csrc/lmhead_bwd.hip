// dlm_lmhead_bwd: gradient of the LM head's log-sum-exp and target logit.
//
// With z = inv_t h w^T and p = exp(z - lse) (lse from the forward pass, so that no row has to be reduced again):
//   dz = inv_t (d_lse p + d_ztarget [v = target]);   d_hidden = dz W;   d_w = dz^T H.
// Three products of 2 M V Dh operations, all bound by the matrix pipes from a few hundred rows on, below that by reading W twice and writing d_w once.
// The logits themselves are never stored; dz is, in 16 bits, for as many columns at a time as the workspace holds (a "chunk"): d_hidden sums over the
// vocabulary and d_w over the rows, so that one of the two would otherwise form all of dz again, a fourth product.
//
// One loop serves the three: C[i][j] = sum over k of A(i, k) B(j, k), on 32 x 32 x 16 MFMA tiles.  An operand comes either with k along its
// rows (hidden and W for the logits; dz for d_hidden) or with k across them (W for d_hidden; dz and hidden for d_w), which is
// turned on the way from LDS into registers by the transposing read, so that nothing is transposed in memory.
//
// Rounding of dz.  One bf16 (8 bits) would make the error of a bf16 gradient 1.4 times that of rounding the gradient alone.  So:
//   bf16 gradients, many rows: one fp16 term, 11 bits, at the same rate.  Its other operands are fp16 too, exact copies of hidden rows and of W
//     but for powers of two (see LmbScale), which costs a pass over W: 3 % of the time of 4096 rows.  Each gradient has a dz of its own, scaled by the rows for
//     d_hidden, by the columns for d_w: a token that is unlikely in every row has a small column of dz, of which all of its row of d_w is summed.
//   bf16 gradients, few rows: two bf16 terms, 16 bits: twice the products where reading W takes longest, and no copy of it.
//   fp32 gradients: three bf16 terms, 24 bits, and sums of 256 products (of a logit 128: an error of one is one of the probability) added up in two floats; the
//     parts of d_hidden's sum, and what its chunks of columns leave in them, are joined in one.  Slower by design; 16 bits of dz and plain sums are 2e-6 off.
//
// Measured, both gradients in bf16: 4096 rows, V = 152064, Dh = 3584 12.1 ms, 1.1 PFLOP/s (W's copy 0.42, dz 4.29 at 1.04, its panels brought together 0.46, the gradients 6.92 at 1.29); 512 rows,
// V = 126464, Dh = 4096 2.05 ms (0.37, 0.57, 0.05, 1.05); 256 rows 1.47, 64 0.73, 4 0.70, of 2.07 GB that it cannot do without.  A register-only loop of these products on such data reaches 1.81.
#include "device.hpp"
#include "rows.hpp"

namespace dlm {

typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) bf16x8 lds_bf16x8;
typedef __attribute__((__vector_size__(8 * sizeof(_Float16)))) _Float16 f16x8;

struct LmbRow {                    // what the logits' kernel knows of a row
    float lse, a, c;               // a = inv_t d_lse, c = inv_t d_ztarget; a row without a has an infinite lse, and so probabilities of zero
    int target;
};
constexpr int LMB_NO_TARGET = -(1 << 28);

// fp16 operands.  With e(x) the exponent of the largest entry of a row (its size lies in [2^e, 2^(e+1))) and 2^(c + 1) above a row's |d_lse| + |d_ztarget|, inv_t
// included, so that |dz| < 2^(c + 1):
//   d_hidden[m] = 2^(S - 27 + c[m]) sum_v D w16[v],   D[m][v] = dz[m][v] 2^(13 - c[m] + f[v] - S),   w16[v] = w[v] 2^(14 - f[v]),   S = max_v f[v]
//   d_w[v] = 2^(L - 27 - 16 k[v]) sum_m E h16[m],   E[m][v] = dz[m][v] 2^(13 + e(h[m]) - L + 16 k[v]),   h16[m] = h[m] 2^(14 - e(h[m])),   L = max_m (e(h[m]) + c[m])
// D and E stay below 2^14 (2^15 where a probability is rounded above one).  f[v] = max(e(w[v]), F), F eight above the largest exponent of 256 rows spread over W:
// nearly always F for all, so that small rows of W do not make their D small (what w16 loses there, 2^-31 of W's largest, counts for nothing in d_hidden).
// k[v], 0 to 7, brings the largest |E| of a column to 2^-1 or more, so that E is 2^-24 of it off at most.  It is known when all rows of dz are: a wavefront scales its
// panel of 32, 64 or 128 rows by the panel's own largest, and lmb_even_kernel brings the panels of a column, where they differ, to the smallest k among them (another
// rounding of what falls below the normal numbers).  One dz for both, scaled by |d_lse| + |d_ztarget| alone, gave zeros for d_w of tokens whose probability is below 2^-39 in
// every row, and few bits below 2^-28: all of a batch whose targets are 40 above the other logits.  What E takes: dz of 4096 rows, V = 152064, Dh = 3584 3960 -> 4290 us,
// lmb_even_kernel 460 (it reads and writes nearly all of E, 5.5 TB/s, since the largest of 128 rows and that of 4096 are mostly over 2^8 apart); of 512 rows, V = 126464,
// Dh = 4096 570 -> 615 and 53.
struct LmbScale {
    int *row_e, *row_c;            // [M rounded up to 64]
    int *hs, *ws;                  // 13 - c;  c + e(h) - L: the powers from dz to D (without f) and from there to E (without k); [M rounded up to 64]
    int* w_f;                      // f, [V rounded up to 256]
    int* col;                      // k, [V rounded up to 256] (LMB_EMPTY: a column of zeros)
    uint8_t* panel;                // k of a panel, [panels][ldz]
    int *row_max, *w_some, *w_max; // by workgroup; exponents of some rows of W; by wavefront
    int* out;                      // S, L
    uint16_t *h16, *w16, *tail16;
    uint16_t* e;                   // E, as dz
};
constexpr int LMB_EMPTY = 255;
constexpr int LMB_ORDER = 64;      // wavefronts that look through row_idx
constexpr int LMB_STATS = 256;     // workgroups that look for a largest exponent
constexpr int LMB_NONE = -100000;  // exponent of a row of zeros

struct LmbParams {
    int M, Dh, V;
    const int32_t* m_dev;
    const uint16_t* hidden;        // as the caller has them
    int64_t h_stride;
    const int32_t* row_idx;
    const uint16_t* w;
    int64_t w_stride;
    float inv_t;
    int forbid, scatter;
    const float *lse, *d_lse, *d_zt;
    const int32_t* target;
    // workspace
    LmbRow* rows;                  // [M rounded up to 64]
    uint16_t* h;                   // the selected hidden rows, [M rounded up to 64][Dh], zeros behind the last
    uint16_t* w_tail;              // [64][Dh]: the last V % 64 rows of W, zeros behind them
    int f16;                       // dz is fp16 and scaled
    LmbScale sc;
    int last_f;                    // the last four of w_f and col
    uint16_t* dz;                  // [terms][M rounded up to 64][ldz]; fp16: D
    int64_t dz_term;               // entries of a term
    int ldz;
    float* part;                   // [splits][terms][M][Dh]
    // the chunk: columns v0 .. v0 + n of dz, n a multiple of 64 but for the end of the vocabulary
    int v0, n, terms_h, terms_w, add;      // add: d_hidden's partial sums are there already
    int splits;                    // parts of d_hidden's sum
    int n2;                        // workgroups of d_hidden (a multiple of 8), where each takes one tile; 0: it is not wanted
    int queued;                    // workgroups take one tile after the other
    int* counters;                 // of three lists of tiles: dz, d_hidden, d_w
    int* order;                    // [LMB_ORDER] not 0: an entry of row_idx does not exceed the one before it
    void* d_hidden;
    int64_t dh_stride;
    int dh_f32;
    void* d_w;
    int64_t dw_stride;
    int dw_f32, accumulate;
};

__device__ __forceinline__ int lmb_rows(const LmbParams& p) { return p.m_dev ? min(p.M, max(__builtin_amdgcn_readfirstlane(*p.m_dev), 0)) : p.M; }

// the largest size of eight entries; NaN and infinities count for nothing
__device__ __forceinline__ float lmb_top8(u32x4 v) {
    float f[8], top = 0.f;
    Piece<false>::open(v, f);
#pragma unroll
    for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(f[e]) < INFINITY ? fabsf(f[e]) : 0.f);
    return top;
}
// the exponent of the largest of a wavefront's sizes
__device__ __forceinline__ int lmb_exponent(float top) {
#pragma unroll
    for (int off = 1; off < WAVE; off *= 2) top = fmaxf(top, shfl_xor(top, off));
    return top > 0.f ? max((int)(__float_as_uint(top) >> 23) - 127, -126) : LMB_NONE;
}
// eight entries times 2^k, zeros if not `any`
__device__ __forceinline__ u32x4 lmb_half8(u32x4 v, bool any, int k) {
    float f[8];
    Piece<false>::open(v, f);
    f16x8 h;
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = (_Float16)(any ? ldexpf(f[e], k) : 0.f);
    return __builtin_bit_cast(u32x4, h);
}

// fp16 operands, first pass: exponents of the selected rows and of their gradients, a wavefront a row; of a row of W a workgroup
__global__ __launch_bounds__(256) void lmb_stat_kernel(LmbParams p) {
    __shared__ int meet[4];
    const int M = lmb_rows(p), lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int most = LMB_NONE;
    for (int r = blockIdx.x * 4 + wave; r < M; r += gridDim.x * 4) {
        const int row = p.row_idx ? p.row_idx[r] : r, at = p.scatter ? row : r;
        const float a = p.d_lse ? fabsf(p.d_lse[at] * p.inv_t) : 0.f, b = p.d_zt ? fabsf(p.d_zt[at] * p.inv_t) : 0.f, g = a + b;
        float top = 0.f;
#pragma unroll 8
        for (int c = lane * 8; c < p.Dh; c += 512) top = fmaxf(top, lmb_top8(*reinterpret_cast<const u32x4*>(p.hidden + row * p.h_stride + c)));
        const int e = lmb_exponent(top);
        const int c = g > 0.f && g < INFINITY ? max((int)(__float_as_uint(g) >> 23) - 127, -126) : LMB_NONE;
        if (lane == 0) {
            p.sc.row_e[r] = e;
            p.sc.row_c[r] = c;
        }
        if (e != LMB_NONE && c != LMB_NONE) most = max(most, e + c);
    }
    if (wave == 0) {
        const uint16_t* w = p.w + (int64_t)blockIdx.x * p.V / LMB_STATS * p.w_stride;
        float top = 0.f;
#pragma unroll 8
        for (int c = lane * 8; c < p.Dh; c += 512) top = fmaxf(top, lmb_top8(*reinterpret_cast<const u32x4*>(w + c)));
        const int e = lmb_exponent(top);
        if (lane == 0) p.sc.w_some[blockIdx.x] = e;
    }
    if (lane == 0) meet[wave] = most;
    __syncthreads();
    if (threadIdx.x == 0) p.sc.row_max[blockIdx.x] = max(max(meet[0], meet[1]), max(meet[2], meet[3]));
}
// largest of n numbers, over the wavefront
__device__ __forceinline__ int lmb_most(const int* v, int n) {
    int m = LMB_NONE;
#pragma unroll 8
    for (int i = threadIdx.x & 63; i < n; i += WAVE) m = max(m, v[i]);
#pragma unroll
    for (int off = 1; off < WAVE; off *= 2) m = max(m, shfl_xor(m, off));
    return m;
}

// Selected hidden rows side by side, what belongs to them, and the rows of W behind the last whole 64: the products then read whole tiles.
// fp16: the scaled copies of both, and of all of W.
__global__ __launch_bounds__(256) void lmb_gather_kernel(LmbParams p) {
    const int M = lmb_rows(p), bound = (p.M + 63) & ~63, r = blockIdx.x;
    if (r == 0 && threadIdx.x < 24) p.counters[threadIdx.x * 16] = 0;
    if (p.f16) {
        for (int v = r * 256 + threadIdx.x; v < p.last_f + 4; v += gridDim.x * 256) p.sc.col[v] = LMB_EMPTY;
    }
    if (r < LMB_ORDER && p.row_idx && threadIdx.x < WAVE) {        // (there are 64 workgroups or more)
        bool falls = false;
#pragma unroll 4
        for (int q = r * WAVE + threadIdx.x; q + 1 < M; q += LMB_ORDER * WAVE) falls |= p.row_idx[q + 1] <= p.row_idx[q];
        const uint64_t any = __ballot(falls);
        if (threadIdx.x == 0) p.order[r] = any != 0;
    }
    if (r >= bound) {
        if (p.f16) {
            // a wavefront a row, its first 4096 entries kept in registers
            int most = LMB_NONE;
            const int some = lmb_most(p.sc.w_some, LMB_STATS), least = some == LMB_NONE ? LMB_NONE : some + 8;
            const int padded = (p.V + 63) & ~63, whole = p.V & ~63, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
            if (r == bound && padded + (int)threadIdx.x < p.last_f + 4) p.sc.w_f[padded + threadIdx.x] = least;      // (columns of the last tiles that no product takes)
            for (int v = (r - bound) * 4 + wave; v < padded; v += LMB_STATS * 8 * 4) {
                uint16_t* dst = v < whole ? p.sc.w16 + (int64_t)v * p.Dh : p.sc.tail16 + (int64_t)(v - whole) * p.Dh;
                const uint16_t* src = p.w + min(v, p.V - 1) * p.w_stride;
                u32x4 kept[8];
                float top = 0.f;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int c = (k * WAVE + lane) * 8;
                    // (past the caches, which cannot hold W: 410 -> 376 us of 126464 x 4096)
                    kept[k] = c < p.Dh ? __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + c)) : u32x4{0, 0, 0, 0};
                }
#pragma unroll
                for (int k = 0; k < 8; ++k) top = fmaxf(top, lmb_top8(kept[k]));
                for (int c = 4096 + lane * 8; c < p.Dh; c += 512) top = fmaxf(top, lmb_top8(*reinterpret_cast<const u32x4*>(src + c)));
                const int e = max(v < p.V ? lmb_exponent(top) : LMB_NONE, least);
                if (lane == 0) p.sc.w_f[v] = e;             // (of the rows behind the last too: their columns of dz are zero times a power of two)
                most = max(most, e);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int c = (k * WAVE + lane) * 8;
                    if (c < p.Dh) __builtin_nontemporal_store(lmb_half8(kept[k], v < p.V && e != LMB_NONE, 14 - e), reinterpret_cast<u32x4*>(dst + c));
                }
                for (int c = 4096 + lane * 8; c < p.Dh; c += 512)
                    *reinterpret_cast<u32x4*>(dst + c) = lmb_half8(*reinterpret_cast<const u32x4*>(src + c), v < p.V && e != LMB_NONE, 14 - e);
            }
            if (lane == 0) p.sc.w_max[(r - bound) * 4 + wave] = most;
            return;
        }
        const int t = r - bound, v = (p.V & ~63) + t;
        for (int c = threadIdx.x * 8; c < p.Dh; c += 2048)
            *reinterpret_cast<u32x4*>(p.w_tail + (int64_t)t * p.Dh + c) =
                v < p.V ? *reinterpret_cast<const u32x4*>(p.w + v * p.w_stride + c) : u32x4{0, 0, 0, 0};
        return;
    }
    if (r >= ((M + 63) & ~63)) return;
    const bool live = r < M;
    const int row = !live ? 0 : p.row_idx ? p.row_idx[r] : r;
    int hs = 0, ws = 0, e = 0;
    if (p.f16 && live) {
        // (a row whose gradient is zero or not finite has any scale; of a hidden row of zeros nothing is to count for the columns' largest)
        const int c = p.sc.row_c[r], most = lmb_most(p.sc.row_max, LMB_STATS);
        e = p.sc.row_e[r];
        if (c != LMB_NONE) hs = 13 - c;
        if (e == LMB_NONE) ws = LMB_NONE;
        else if (c != LMB_NONE) ws = c + e - most;
    }
    for (int c = threadIdx.x * 8; c < p.Dh; c += 2048) {
        const uint16_t* src = p.hidden + row * p.h_stride + c;
        *reinterpret_cast<u32x4*>(p.h + (int64_t)r * p.Dh + c) = live ? *reinterpret_cast<const u32x4*>(src) : u32x4{0, 0, 0, 0};
        if (p.f16) *reinterpret_cast<u32x4*>(p.sc.h16 + (int64_t)r * p.Dh + c) = lmb_half8(live ? *reinterpret_cast<const u32x4*>(src) : u32x4{0, 0, 0, 0}, live && e != LMB_NONE, 14 - e);
    }
    if (threadIdx.x == 0) {
        LmbRow o = {INFINITY, 0.f, 0.f, LMB_NO_TARGET};
        if (live) {
            const int at = p.scatter ? row : r;
            if (p.d_lse) o.a = p.d_lse[at] * p.inv_t;
            if (o.a != 0.f) o.lse = p.lse[at];
            if (p.d_zt) {
                o.c = p.d_zt[at] * p.inv_t;
                const int t = p.target[at];
                o.target = t >= 0 && t < p.V && t != p.forbid ? t : LMB_NO_TARGET;
            }
        }
        p.rows[r] = o;
        if (p.f16) {
            p.sc.hs[r] = hs;
            p.sc.ws[r] = ws;
        }
    }
}
// S and L, from what the workgroups found
__global__ __launch_bounds__(512) void lmb_scale_kernel(LmbParams p) {
    __shared__ int meet[8];
    const int wave = threadIdx.x >> 6, L = lmb_most(p.sc.row_max, LMB_STATS), S0 = p.d_hidden ? lmb_most(p.sc.w_max + wave * LMB_STATS * 4, LMB_STATS * 4) : LMB_NONE;
    if (lane_id() == 0) meet[wave] = S0;
    __syncthreads();
    if (threadIdx.x == 0) {
        int S = meet[0];
        for (int k = 1; k < 8; ++k) S = max(S, meet[k]);
        p.sc.out[0] = S == LMB_NONE ? 0 : S;
        p.sc.out[1] = L == LMB_NONE ? 0 : L;
    }
}

// Tile number -> tile, so that neighbouring numbers form blocks of gi x gj tiles, which share their panels through one XCD's L2 (see lmb_slot).
__device__ __forceinline__ void lmb_tile(int t, int ni, int nj, int gi, int gj, int& i, int& j) {
    const int band = t / (gi * nj), bi = min(gi, ni - band * gi);
    int r = t - band * gi * nj;
    const int col = r / (bi * gj);
    r -= col * bi * gj;
    j = r / bi;
    i = band * gi + r - j * bi;
    j += col * gj;
}
// Workgroups go round the 8 XCDs: each XCD has a stretch of the tile numbers.  With a counter a workgroup takes one tile after the other, in order;
// `ahead` is the one behind the tile at hand, whose operands are requested before that one is done.
struct LmbList {
    int t0, len, index, ahead, later;      // later: what a number from the counter is short of the list's index
    int* counter;                          // NULL: one tile
    __device__ __forceinline__ LmbList(int tiles, int block) {
        const int per = (tiles + 7) >> 3;
        t0 = (block & 7) * per;
        len = max(0, min(per, tiles - t0));
        index = block >> 3;
        ahead = len;
        later = 0;
        counter = nullptr;
    }
};
constexpr int LMB_COUNTERS = 8 * 16;       // of one list: one an XCD, lines apart
__device__ __forceinline__ int lmb_take(int* counter) { return __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

__device__ __forceinline__ void lmb_load_lds16(const void* base, uint32_t offset, uint32_t dst) {   // base: wave-uniform
    uint64_t a;
    // (scalars are read by scalar instructions alone, which wait for whatever wrote them)
    asm volatile("s_mov_b32 m0, %2\n\ts_mov_b64 %0, %3\n\tglobal_load_lds_dwordx4 %1, %0"
                 : "=&s"(a) : "v"(offset), "s"(__builtin_amdgcn_readfirstlane(dst)), "s"(base) : "memory");
}

// Of 16 columns of an accumulator a lane has 0 .. 3 and 8 .. 11 (w[0 .. 1], w[2 .. 3], two a word), lane + 32 the others: eight in a row for each, 0 .. 7
// and 8 .. 15.
__device__ __forceinline__ u32x4 lmb_eight(const uint32_t (&w)[4]) {
    const auto x = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false), y = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
    return u32x4{x[0], y[0], x[1], y[1]};
}

// largest of 32 neighbouring lanes' numbers, for all of them
__device__ __forceinline__ uint32_t lmb_most32(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp(v, 0xB1, 0xf, 0xf, true));       // lane ^ 1
    v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp(v, 0x4E, 0xf, 0xf, true));       // lane ^ 2
    v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp(v, 0x141, 0xf, 0xf, true));      // 7 - lane of 8
    v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp(v, 0x140, 0xf, 0xf, true));      // 15 - lane of 16
    const auto w = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return max((uint32_t)w[0], (uint32_t)w[1]);
}
// Four neighbouring lanes' pieces x[0 .. 3] turned: lane b of the four gets piece b of each, lane u's in x[u].
__device__ __forceinline__ void lmb_turn(u32x4 (&x)[4]) {
    const int l = threadIdx.x;
#pragma unroll
    for (int bit = 1; bit < 4; bit *= 2) {
        const bool up = l & bit;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            if (t & bit) continue;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t a = x[t][k], b = x[t | bit][k], send = up ? a : b;
                const uint32_t got = bit == 1 ? __builtin_amdgcn_mov_dpp(send, 0xB1, 0xf, 0xf, true) : __builtin_amdgcn_mov_dpp(send, 0x4E, 0xf, 0xf, true);
                x[t][k] = up ? got : a;
                x[t | bit][k] = up ? b : got;
            }
        }
    }
}
// fp16 of two numbers, in a word
__device__ __forceinline__ uint32_t lmb_halves(float a, float b) {
    typedef __attribute__((__vector_size__(2 * sizeof(_Float16)))) _Float16 f16x2;
    return __builtin_bit_cast(uint32_t, f16x2{(_Float16)a, (_Float16)b});
}

template <int V, int H, int TV, int TH>
struct LmbShape {
    static constexpr int WV = V, WH = H, TVW = TV, THW = TH;
};
using Lmb256 = LmbShape<2, 2, 4, 4>;       // 256 x 256, one workgroup a CU
using Lmb256x128 = LmbShape<4, 1, 2, 4>;   // one
using Lmb256x64 = LmbShape<4, 1, 2, 2>;    // one
using Lmb128 = LmbShape<2, 2, 2, 2>;       // 128 x 128, two, one with sums in two floats (371 registers)
using Lmb64 = LmbShape<2, 2, 1, 1>;        // 64 x 64, four

// The shape of a workgroup: WV x WH wavefronts of TVW x THW tiles of 32 x 32.
//
// Memory to registers goes through a ring of five LDS stages of 32 k each, without registers in between.  Requests come in pairs of stages, two pairs
// ahead, spread evenly over the MFMAs, and fragments are read one MFMA step ahead, across the barriers (lmhead.hip has the measurements).
// Images of an operand's stage (TILE x 32 entries, 64 TILE bytes):
//   k along the rows: rows of 64 bytes; 16-byte piece c of row r in place c ^ (r / 4 % 4).
//   k across the rows: 32 rows of 2 TILE bytes; 64-byte piece c of row k in place c ^ (k % 4) (TILE = 64: c ^ (k / 2 % 2), TILE = 32: c), so that the four
//   rows that a transposing read touches lie in different banks.
//
// BLOCK > 0: the sums of so many pairs of stages are added up in two floats (a sum, and what its roundings lost).  For dz's logits, whose error is one of the
// probability, two pairs, and the exponent is formed of both floats: gradients of 1656 rows, 1352 columns and a temperature of 0.7 are 6.6e-7 off in the norm, with
// four pairs 9.2e-7, with a rounded logit 1.06e-6 (one pair: 5.6e-7).  1000 rows, V = 32000, Dh = 4096: 3515 us, four pairs 3400, one 3655.
template <bool AROW, bool BROW, bool F16, int BLOCK, int WV, int WH, int TVW, int THW>
struct LmbLoop {
    static constexpr int NW = WV * WH, TI = 32 * TVW * WV, TJ = 32 * THW * WH, STAGE = (TI + TJ) * 64, NS = 5, RING = NS * STAGE;
    static constexpr int IPA = TI / 16 / NW, IPB = TJ / 16 / NW, IPW = IPA + IPB;      // requests of a wavefront and stage
    static_assert(TI / 16 % NW == 0 && TJ / 16 % NW == 0, "requests split evenly over the wavefronts");
    static_assert(RING <= 160 * 1024, "five stages within the 160 KB of LDS");

    unsigned char* ring;
    uint32_t lds0;
    int w, lane;
    uint32_t voff[IPW];            // a lane's place in each request, from the wave-uniform base of its stage
    f32x16 acc[TVW][THW];
    f32x16 low[BLOCK > 0 ? TVW : 1][BLOCK > 0 ? THW : 1];      // what acc, rounded, is short of the two floats

    __device__ __forceinline__ LmbLoop(unsigned char* r) : ring(r) {
        lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)r;
        lane = lane_id();
        w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    }
    // the lane, formed where it stands: what follows from it is not kept in registers over the loop
    __device__ __forceinline__ int lane_here() const {
        int l = lane;
        asm volatile("" : "+v"(l));
        return l;
    }
    static __device__ __forceinline__ int swz(int tile, int k) { return tile >= 128 ? k & 3 : tile == 64 ? k >> 1 & 1 : 0; }
    // Places of operand A's (B's) requests.  k across the rows: row k is `pitch` bytes behind row k - 1, columns end at `last` (a multiple of 8);
    // k along the rows: row r begins at place(r).
    template <int TILE, int IP>
    __device__ __forceinline__ void place_columns(int first, uint32_t pitch, int last) {
        const int l = lane_here();
        constexpr int LPR = TILE / 8, RPI = 64 / LPR;                  // lanes a row, rows a request
#pragma unroll
        for (int j = 0; j < IP; ++j) {
            const int k = (w * IP + j) * RPI + l / LPR, c = l % LPR;
            const int col = ((c >> 2 ^ swz(TILE, k)) << 2 | (c & 3)) * 8;
            voff[first + j] = (uint32_t)k * pitch + (uint32_t)min(col, last) * 2;
        }
    }
    template <int IP, typename Place>
    __device__ __forceinline__ void place_rows(int first, Place&& place) {
        const int l = lane_here();
#pragma unroll
        for (int j = 0; j < IP; ++j) voff[first + j] = place((w * IP + j) * 16 + (l >> 2)) + ((l & 3) ^ (l >> 4 & 3)) * 16;
    }

    struct Bases {
        const char *a0, *a1, *b0, *b1;                                 // of a pair's two stages
    };
    static __device__ __forceinline__ const char* uniform(const char* x) {
        const uint64_t v = (uint64_t)x;
        return (const char*)((uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(v >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)v));
    }
    template <typename Job>
    __device__ __forceinline__ void bases(Job& job, int q, Bases& s) {
        job.pair(*this, q, s);
        s = Bases{uniform(s.a0), uniform(s.a1), uniform(s.b0), uniform(s.b1)};      // (which the compiler does not always see)
    }
    // request jj of a pair (0 .. 2 IPW): even ones into its first stage
    __device__ __forceinline__ void issue(const Bases& s, int jj, uint32_t st0, uint32_t st1) {
        const int j = jj >> 1;
        const char* base = j < IPA ? (jj & 1 ? s.a1 : s.a0) : (jj & 1 ? s.b1 : s.b0);
        const uint32_t at = j < IPA ? (uint32_t)(w * IPA + j) * 1024 : TI * 64 + (uint32_t)(w * IPB + j - IPA) * 1024;
        lmb_load_lds16(base, voff[j], lds0 + (jj & 1 ? st1 : st0) + at);
    }

    // The tiles of a list.  The job knows them: open(t) makes t the tile that requests are for, of np pairs of stages; place(loop) its places; pair(loop, q,
    // bases) the bases of its pair q, asked for in order (and again for the last one); at: what store(loop, at) needs to know of a tile.
    // The requests of a tile's last two pairs are the next tile's first two, so that its first trip to memory hides behind the end of this one; every
    // tile of a list with a counter has two pairs or more.
    template <typename Job>
    __device__ __forceinline__ void run(Job& job, LmbList list) {
        if (list.index >= list.len) return;
        const int n = lane & 31, hi = lane >> 5, s16 = lane & 15, blk = lane >> 4 & 1, wv = w % WV, wh = w / WV;
        // lane offsets of the fragments: one a step (k along the rows), or one a tile
        uint32_t la[AROW ? TVW : 2], lb[BROW ? THW : 2];
#pragma unroll
        for (int h = 0; h < (AROW ? TVW : 2); ++h) {
            if constexpr (AROW) la[h] = lds0 + (8 * hi + (s16 >> 2)) * TI * 2 + ((wv * TVW + h ^ swz(TI, s16 >> 2)) << 6) + 32 * blk + 8 * (s16 & 3);
            else la[h] = lds0 + (wv * TVW * 32 + n) * 64 + ((2 * h + hi ^ (n >> 2 & 3)) << 4);
        }
#pragma unroll
        for (int h = 0; h < (BROW ? THW : 2); ++h) {
            if constexpr (BROW) lb[h] = lds0 + TI * 64 + (8 * hi + (s16 >> 2)) * TJ * 2 + ((wh * THW + h ^ swz(TJ, s16 >> 2)) << 6) + 32 * blk + 8 * (s16 & 3);
            else lb[h] = lds0 + TI * 64 + (wh * THW * 32 + n) * 64 + ((2 * h + hi ^ (n >> 2 & 3)) << 4);
        }
        union Frag {
            s16x4 q[2];
            bf16x8 v;
            f16x8 f;
        };
        Frag fa[2][TVW], fb[2][THW];
        const auto read = [&](int h, uint32_t sb, int f) {
            if (f < TVW) {
                if constexpr (AROW) {
#pragma unroll
                    for (int q = 0; q < 2; ++q)
                        fa[h][f].q[q] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)(la[f % (AROW ? TVW : 2)] + sb + (16 * h + 4 * q) * TI * 2));
                } else {
                    fa[h][f].v = *(const lds_bf16x8*)(uintptr_t)(la[h] + sb + f * 2048);
                }
            } else {
                const int t = f - TVW;
                if constexpr (BROW) {
#pragma unroll
                    for (int q = 0; q < 2; ++q)
                        fb[h][t].q[q] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)(lb[t % (BROW ? THW : 2)] + sb + (16 * h + 4 * q) * TJ * 2));
                } else {
                    fb[h][t].v = *(const lds_bf16x8*)(uintptr_t)(lb[h] + sb + t * 2048);
                }
            }
        };
        constexpr int NF = TVW + THW, NM = TVW * THW, BV = BLOCK > 0 ? TVW : 1, BH = BLOCK > 0 ? THW : 1;
        // half a stage: the products of one MFMA step, behind the first ones the fragments of the next step, between them requests
        Bases src;
        const auto half = [&](auto H, uint32_t rsb, auto PART, uint32_t st0, uint32_t st1) {
            constexpr int h = decltype(H)::value, part = decltype(PART)::value;
#pragma unroll
            for (int i = 0; i < NM; ++i) {
                f32x16& x = acc[i % TVW][i / TVW];
                if constexpr (F16) x = __builtin_amdgcn_mfma_f32_32x32x16_f16(fa[h][i % TVW].f, fb[h][i / TVW].f, x, 0, 0, 0);
                else x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[h][i % TVW].v, fb[h][i / TVW].v, x, 0, 0, 0);
#pragma unroll
                for (int f = 0; f < NF; ++f)
                    if (f * NM / (2 * NF) == i) read(1 - h, rsb, f);
                if constexpr (part != 0) {
#pragma unroll
                    for (int j = 0; j < IPW; ++j)
                        if (j * NM / IPW == i) issue(src, j + (part == 2 ? IPW : 0), st0, st1);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        using I0 = std::integral_constant<int, 0>;
        using I1 = std::integral_constant<int, 1>;
        using I2 = std::integral_constant<int, 2>;
        const auto next = [](uint32_t s) { return s + STAGE == NS * STAGE ? 0u : s + STAGE; };
        job.open(list.t0 + __builtin_amdgcn_readfirstlane(list.index));
        job.place(*this);
        if (job.np > 0) {
            // (a pair past the last one is the last one again, into stages that nobody reads)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                bases(job, min(q, job.np - 1), src);
#pragma unroll
                for (int jj = 0; jj < 2 * IPW; ++jj) issue(src, jj, 2 * q * STAGE, (2 * q + 1) * STAGE);
            }
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * IPW) : "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        }
        uint32_t sb = 0;           // the stage of the pair at hand; the one in front of it is free between tiles
        for (;;) {
            const bool more = list.counter && list.ahead < list.len;
            int taken = 0;
            if (more && threadIdx.x == 0) taken = lmb_take(list.counter);
            const auto at = job.at;
            const int np = job.np;
            f32x16 sum[BV][BH], lost[BV][BH];
#pragma unroll
            for (int a = 0; a < TVW; ++a)
#pragma unroll
                for (int c = 0; c < THW; ++c) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[a][c][i] = 0.f;
                    if constexpr (BLOCK > 0) sum[a][c] = lost[a][c] = acc[a][c];
                }
            if (np > 0) {
#pragma unroll
                for (int f = 0; f < NF; ++f) read(0, sb, f);
            }
            int ask = 2;
            for (int q = 0; q < np;) {
                const int end = BLOCK > 0 ? min(q + BLOCK, np) : np;
#pragma unroll 1
                for (; q < end; ++q) {
                    const uint32_t s1 = next(sb), s2 = next(s1), s3 = next(s2), s4 = next(s3);
                    if (more && q + 2 == np) {
                        job.open(list.t0 + list.ahead);
                        job.place(*this);
                        ask = 0;
                    }
                    bases(job, min(ask, job.np - 1), src);
                    ++ask;
                    half(I0(), sb, I0(), 0, 0);
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                    __builtin_amdgcn_s_barrier();      // every wavefront has read the pair's first stage to the end: it is free
                    asm volatile("" ::: "memory");
                    half(I1(), s1, I1(), s4, sb);
                    half(I0(), s1, I2(), s4, sb);
                    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(2 * IPW) : "memory");      // all but the pair just requested has landed
                    __builtin_amdgcn_s_barrier();
                    asm volatile("" ::: "memory");
                    half(I1(), s2, I0(), 0, 0);
                    sb = s2;
                }
                if constexpr (BLOCK > 0) {
#pragma unroll
                    for (int a = 0; a < TVW; ++a)
#pragma unroll
                        for (int c = 0; c < THW; ++c)
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const float x = acc[a][c][i], s = sum[a][c][i], t = s + x, y = t - s;
                                lost[a][c][i] += (s - (t - y)) + (x - y);
                                sum[a][c][i] = t;
                                acc[a][c][i] = 0.f;
                            }
                }
            }
            if constexpr (BLOCK > 0) {
#pragma unroll
                for (int a = 0; a < TVW; ++a)
#pragma unroll
                    for (int c = 0; c < THW; ++c) {
                        acc[a][c] = sum[a][c] + lost[a][c];
                        low[a][c] = lost[a][c] - (acc[a][c] - sum[a][c]);
                    }
            }
#pragma unroll
            for (int a = 0; a < TVW; ++a)
#pragma unroll
                for (int c = 0; c < THW; ++c) asm volatile("" : "+a"(acc[a][c]));
            job.store(*this, at);
            if (!more) break;
            const uint32_t box = sb == 0 ? (NS - 1) * STAGE : sb - STAGE;
            if (threadIdx.x == 0) *reinterpret_cast<int*>(ring + box) = taken;
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            list.ahead = __builtin_amdgcn_readfirstlane(*reinterpret_cast<const int*>(ring + box)) + list.later;
        }
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");      // requests into the ring end before anything else is put there
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    }
};

// ---- dz of a chunk: rows of W along i, hidden rows along j -----------------------------------------------------
// TERMS bf16 terms; 0: one scaled fp16.
template <int WV, int WH, int TVW, int THW, int TERMS, int BLOCK>
struct LmbDz {
    using Loop = LmbLoop<false, false, false, BLOCK, WV, WH, TVW, THW>;
    struct At {
        int i0, j0;
    };
    const LmbParams& p;
    int padded, ni, nj, gj, np;
    At at;
    const char *wb, *hb;
    __device__ __forceinline__ LmbDz(const LmbParams& q) : p(q) {
        padded = (lmb_rows(p) + 63) & ~63;
        ni = (p.n + Loop::TI - 1) / Loop::TI;
        nj = (padded + Loop::TJ - 1) / Loop::TJ;
        gj = max(min(nj, 8), 1);
        np = p.Dh / 64;
    }
    __device__ __forceinline__ void open(int t) {
        int ti, tj;
        lmb_tile(t, ni, nj, 32 / gj, gj, ti, tj);
        at = At{ti * Loop::TI, tj * Loop::TJ};
        wb = (const char*)(p.w + (int64_t)(p.v0 + at.i0) * p.w_stride);
        hb = (const char*)(p.h + (int64_t)at.j0 * p.Dh);
    }
    __device__ __forceinline__ void place(Loop& loop) const {
        const int last_w = p.V - 1 - p.v0 - at.i0, last_h = padded - 1 - at.j0;
        loop.template place_rows<Loop::IPA>(0, [&](int r) { return (uint32_t)min(r, last_w) * (uint32_t)p.w_stride * 2; });
        loop.template place_rows<Loop::IPB>(Loop::IPA, [&](int r) { return (uint32_t)min(r, last_h) * (uint32_t)p.Dh * 2; });
    }
    __device__ __forceinline__ void pair(Loop&, int q, typename Loop::Bases& b) const {
        b.a0 = wb + q * 128;
        b.a1 = b.a0 + 64;
        b.b0 = hb + q * 128;
        b.b1 = b.b0 + 64;
    }
    // One exponential an entry, and little beside it: the matrix pipes stand still meanwhile.  What few tiles or entries need, the end of the
    // vocabulary, the forbidden token and the target, is behind branches.
    __device__ __forceinline__ void store(Loop& loop, const At& tile) const {
        const int lane = loop.lane_here(), n = lane & 31, hi = lane >> 5, wv = loop.w % WV, wh = loop.w / WV;
        const int first = tile.i0 + wv * TVW * 32 + 4 * hi, v_first = p.v0 + first;                // the lane's first column
        const bool edge = p.v0 + tile.i0 + Loop::TI > p.V || (p.forbid >= p.v0 + tile.i0 && p.forbid < p.v0 + tile.i0 + Loop::TI);
        const float log2e = 1.4426950408889634f, k = p.inv_t * log2e;
        float off[THW], ra[THW], rc[THW], ws[THW];
        int target[THW];
        const int m0 = tile.j0 + wh * THW * 32 + n;            // the lane's first row
#pragma unroll
        for (int c = 0; c < THW; ++c) {
            const int r = min(m0 + c * 32, padded - 1);
            const LmbRow row = p.rows[r];
            off[c] = TERMS == 3 ? -row.lse : -row.lse * log2e;
            const int hs = TERMS == 0 ? p.sc.hs[r] : 0;
            ra[c] = TERMS == 0 ? ldexpf(row.a, hs) : row.a;
            rc[c] = TERMS == 0 ? ldexpf(row.c, hs) : row.c;
            ws[c] = TERMS == 0 ? ldexpf(1.f, p.sc.ws[r]) : 1.f;
            target[c] = row.target - v_first;
        }
        // eight columns of a row, i .. i + 3 and i + 8 .. i + 11
        const auto eight = [&](int a, int g, int c, float (&d)[8]) {
            const int i = first + a * 32 + 8 * g;
#pragma unroll
            for (int q = 0; q < 2; ++q) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float z = loop.acc[a][c][4 * (g + q) + e];
                    // fp32 results: the difference first, a logit and lse are large where their difference is not
                    float x;
                    if constexpr (TERMS == 3) x = fast_exp2(fmaf(loop.low[a][c][4 * (g + q) + e], p.inv_t, fmaf(z, p.inv_t, off[c])) * log2e);
                    else x = fast_exp2(fmaf(z, k, off[c]));
                    d[4 * q + e] = ra[c] * x;
                }
                const uint32_t t = (uint32_t)(target[c] - a * 32 - 8 * (g + q));
                if (t < 4) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) d[4 * q + e] += t == e ? rc[c] : 0.f;
                }
            }
            if (edge) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int v = p.v0 + i + e / 4 * 8 + e % 4;
                    if (v == p.forbid || v >= p.V) d[e] = 0.f;
                }
            }
        };
        if constexpr (TERMS == 0) {
            // Two tiles of 32 columns at a time (one where there is one), for d_hidden and for d_w.  A row's 64 columns are a whole line: four lanes' pieces are turned, so that
            // every store writes lines; some twenty registers of the loop wait in scratch meanwhile.  (Stores of 32 bytes of 32 rows: dz of 4096 rows, V = 50176, Dh = 3584 1600 us, lines 1430; with one dz for both gradients 1300.)
            constexpr int NA = TVW < 2 ? 1 : 2;
            // W's exponents of the columns ahead are asked for before the stores at hand: a load behind stores waits for them
            typedef __attribute__((__vector_size__(4 * sizeof(int)))) int i32x4;
            i32x4 we[NA][4];
            const auto exponents = [&](int a0) {
#pragma unroll
                for (int a = 0; a < NA; ++a)
#pragma unroll
                    for (int g = 0; g < 4; ++g) we[a][g] = *reinterpret_cast<const i32x4*>(p.sc.w_f + min(v_first + (a0 + a) * 32 + 8 * g, p.last_f));
            };
            const int S = p.d_hidden ? p.sc.out[0] : 0;
            if (p.d_hidden) exponents(0);
#pragma unroll
            for (int a0 = 0; a0 < TVW; a0 += NA) {
                u32x4 hold[2][THW][2 * NA];
                uint32_t fs[NA][4];                    // four columns a register
                if (p.d_hidden) {
#pragma unroll
                    for (int a = 0; a < NA; ++a)
#pragma unroll
                        for (int g = 0; g < 4; ++g) {
                            fs[a][g] = 0;
#pragma unroll
                            for (int e = 0; e < 4; ++e) fs[a][g] |= (uint32_t)(we[a][g][e] == LMB_NONE ? 0 : min(S - we[a][g][e], 127)) << 8 * e;
                        }
                }
#pragma unroll
                for (int t = 0; t < 2 * NA; ++t) {
                    const int a = a0 + t / 2, g = t % 2 * 2;
                    float d[THW][8];
#pragma unroll
                    for (int c = 0; c < THW; ++c) eight(a, g, c, d[c]);
                    if (p.d_hidden) {
                        float f[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) f[e] = ldexpf(1.f, -(int)(fs[t / 2][g + e / 4] >> 8 * (e % 4) & 255));
#pragma unroll
                        for (int c = 0; c < THW; ++c) hold[0][c][t] = halves(d[c], f);
                    }
                    if (p.d_w) {
                        float f[8];
                        columns(tile, lane, first + a * 32 + 8 * g, d, ws, f);
#pragma unroll
                        for (int c = 0; c < THW; ++c) hold[1][c][t] = halves(d[c], f);
                    }
                }
                if (p.d_hidden && a0 + NA < TVW) exponents(a0 + NA);
#pragma unroll
                for (int which = 0; which < 2; ++which) {
                    if (!(which ? p.d_w : p.d_hidden)) continue;
                    uint16_t* dst = which ? p.sc.e : p.dz;
#pragma unroll
                    for (int c = 0; c < THW; ++c) {
                        if constexpr (NA == 2) lmb_turn(hold[which][c]);
#pragma unroll
                        for (int u = 0; u < 2 * NA; ++u) {
                            const int row = m0 + c * 32 + (NA == 2 ? u - (n & 3) : 0), col = first - 4 * hi + a0 * 32 + (NA == 2 ? 2 * (n & 3) + hi : 2 * u + hi) * 8;
                            if (row < padded && col < p.ldz) *reinterpret_cast<u32x4*>(dst + (int64_t)row * p.ldz + col) = hold[which][c][u];
                        }
                    }
                }
            }
        } else {
#pragma unroll
            for (int a = 0; a < TVW; ++a)
#pragma unroll
                for (int g = 0; g < 4; g += 2) {
                    const int at8 = first + a * 32 + 8 * g + 4 * hi;        // (lane and lane + 32 share 16 columns, lmb_eight gives each eight of them)
#pragma unroll
                    for (int c = 0; c < THW; ++c) {
                        float d[8];
                        eight(a, g, c, d);
#pragma unroll
                        for (int t = 0; t < TERMS; ++t) {
                            // every term what the ones before it leave, which fp32 holds exactly
                            uint32_t w[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                w[e] = pack_bf16x2(d[2 * e], d[2 * e + 1]);
                                d[2 * e] -= __uint_as_float(w[e] << 16);
                                d[2 * e + 1] -= __uint_as_float(w[e] & 0xffff0000u);
                            }
                            const u32x4 out = lmb_eight(w);
                            if (m0 + c * 32 < padded && at8 < p.ldz) *reinterpret_cast<u32x4*>(p.dz + t * p.dz_term + (int64_t)(m0 + c * 32) * p.ldz + at8) = out;
                        }
                    }
                }
        }
    }
    // eight columns, scaled, in 16 bits
    static __device__ __forceinline__ u32x4 halves(const float (&d)[8], const float (&f)[8]) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = lmb_halves(d[2 * e] * f[2 * e], d[2 * e + 1] * f[2 * e + 1]);
        return lmb_eight(w);
    }
    // d_w's dz of eight columns, i .. i + 3 and i + 8 .. i + 11, of all the wavefront's rows: without the columns' scale in d, the scales in f
    __device__ __forceinline__ void columns(const At& tile, int lane, int i, float (&d)[THW][8], const float (&ws)[THW], float (&f)[8]) const {
        const int n = lane & 31, panel = tile.j0 / (32 * THW) + (int)(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) / WV;
        uint32_t kept[2] = {0, 0};                         // the scales of four columns each
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float most = 0.f;
#pragma unroll
            for (int c = 0; c < THW; ++c) {
                d[c][e] *= ws[c];
                most = fmaxf(most, fabsf(d[c][e]));        // (NaN counts for nothing)
            }
            const uint32_t top = lmb_most32(__float_as_uint(most));        // (of numbers that are not negative the bits have their order)
            const int k = min(max(14 + 127 - (int)(top >> 23), 0) >> 4, 7);
            f[e] = __uint_as_float(0x3f800000u + ((uint32_t)k << 27));     // 2^(16 k)
            kept[e / 4] |= (uint32_t)(top > 0 ? k : LMB_EMPTY) << 8 * (e % 4);
        }
        if (panel * 32 * THW >= padded) return;
        if (n == 0) {
#pragma unroll
            for (int q = 0; q < 2; ++q)
                if (i + 8 * q < p.ldz) *reinterpret_cast<uint32_t*>(p.sc.panel + (int64_t)panel * p.ldz + i + 8 * q) = kept[q];
        }
        const int mine = (n < 4 ? kept[0] : kept[1]) >> 8 * (n & 3) & 255;
        // (the smallest of whole numbers: the same in any order.  Columns behind the vocabulary are empty.)
        if (n < 8 && mine != LMB_EMPTY) __hip_atomic_fetch_min(p.sc.col + p.v0 + i + n / 4 * 8 + n % 4, mine, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
};
template <typename S, int TERMS, int BLOCK>
__global__ __launch_bounds__(64 * S::WV * S::WH, 1) void lmb_dz_kernel(LmbParams p) {
    using Job = LmbDz<S::WV, S::WH, S::TVW, S::THW, TERMS, BLOCK>;
    __shared__ __attribute__((aligned(1024))) unsigned char ring[Job::Loop::RING];
    if (blockIdx.x == 0 && threadIdx.x < 16) p.counters[LMB_COUNTERS + threadIdx.x * 16] = 0;      // the gradients' two lists
    Job job(p);
    LmbList list(job.ni * job.nj, blockIdx.x);
    if (p.queued) {
        list.counter = p.counters + (blockIdx.x & 7) * 16;
        list.later = 2 * (gridDim.x >> 3);
        list.ahead = list.index + (gridDim.x >> 3);
    }
    typename Job::Loop loop(ring);
    loop.run(job, list);
}

// E's panels of `rows` rows whose scale of a column is not the column's.  A lane has eight columns.  (Nearly all of E of some thousand rows: bound by HBM.)
__global__ __launch_bounds__(256) void lmb_even_kernel(LmbParams p, int rows) {
    const int padded = (lmb_rows(p) + 63) & ~63, first = blockIdx.y * rows, c = (blockIdx.x * WAVE + lane_id()) * 8;
    if (first >= padded || c >= p.n) return;
    const uint8_t* k = p.sc.panel + (int64_t)blockIdx.y * p.ldz + c;
    const int* col = p.sc.col + p.v0 + c;
    int down[8], any = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        down[e] = k[e] == LMB_EMPTY ? 0 : 16 * (col[e] - k[e]);
        any |= down[e];
    }
    if (any == 0) return;
    // (`rows` and `padded` are multiples of 32: a wavefront's eight rows are there or not.  All eight are asked for before the first is stored.)
    for (int r = first + (threadIdx.x / WAVE) * 8; r < min(first + rows, padded); r += 32) {
        u32x4* at = reinterpret_cast<u32x4*>(p.sc.e + (int64_t)r * p.ldz + c);
        u32x4 x[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) x[q] = at[(int64_t)q * p.ldz / 8];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const f16x8 v = __builtin_bit_cast(f16x8, x[q]);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[q][e] = lmb_halves(ldexpf((float)v[2 * e], down[2 * e]), ldexpf((float)v[2 * e + 1], down[2 * e + 1]));
            at[(int64_t)q * p.ldz / 8] = x[q];
        }
    }
}

// ---- d_hidden's and d_w's products of a chunk ----------------------------------------------------------------
// d_hidden: columns of Dh along i, rows along j (all of the first term of dz, then the second's, so that W is read once for all), the vocabulary is
// summed over, in `splits` parts.
template <bool F16, int BLOCK, int WV, int WH, int TVW, int THW>
struct LmbHidden {
    using Loop = LmbLoop<true, false, F16, BLOCK, WV, WH, TVW, THW>;
    struct At {
        int i0, j0, s;
    };
    const LmbParams& p;
    int M, padded, rows, ni, nj, gj, np;
    At at;
    int all, whole, q0;                            // pairs of stages; those that W itself holds; the tile's first
    bool tail;
    __device__ __forceinline__ LmbHidden(const LmbParams& q) : p(q) {
        M = lmb_rows(p);
        padded = (M + 63) & ~63;
        rows = padded * p.terms_h;
        ni = (p.Dh + Loop::TI - 1) / Loop::TI;
        nj = (rows + Loop::TJ - 1) / Loop::TJ;
        gj = max(min(nj, 8), 1);
        all = (p.n + 63) >> 6;
        whole = p.n >> 6;
    }
    __device__ __forceinline__ int tiles() const { return ni * nj * p.splits; }
    __device__ __forceinline__ void open(int t) {
        const int s = t / (ni * nj);
        int ti, tj;
        lmb_tile(t - s * ni * nj, ni, nj, 32 / gj, gj, ti, tj);
        at = At{ti * Loop::TI, tj * Loop::TJ, s};
        q0 = all * s / p.splits;                   // (at most 2^18 pairs in at most 64 parts)
        np = all * (s + 1) / p.splits - q0;
        tail = false;
    }
    __device__ __forceinline__ void place_w(Loop& loop) const {
        loop.template place_columns<Loop::TI, Loop::IPA>(0, (uint32_t)(F16 || tail ? p.Dh : p.w_stride) * 2, p.Dh - 8 - at.i0);
    }
    // a row and its term
    __device__ __forceinline__ int split_row(int r, int& m) const {
        const int term = (r >= padded ? 1 : 0) + (r >= 2 * padded ? 1 : 0);
        m = r - term * padded;
        return term;
    }
    __device__ __forceinline__ void place(Loop& loop) const {
        place_w(loop);
        // (dz as a whole is less than 2^32 bytes)
        loop.template place_rows<Loop::IPB>(Loop::IPA, [&](int r) {
            int m;
            const int term = split_row(min(at.j0 + r, rows - 1), m);
            return ((uint32_t)term * (uint32_t)p.dz_term + (uint32_t)m * (uint32_t)p.ldz) * 2;
        });
    }
    __device__ __forceinline__ void pair(Loop& loop, int q, typename Loop::Bases& b) {
        const int k = q + q0;
        if ((k >= whole) != tail) {                // into the rows behind the last whole 64
            tail = !tail;
            if (!F16) place_w(loop);
        }
        const uint16_t *w = F16 ? p.sc.w16 : p.w, *w_tail = F16 ? p.sc.tail16 : p.w_tail;
        const int64_t pitch = F16 || tail ? p.Dh : p.w_stride;
        b.a0 = (const char*)(tail ? w_tail + at.i0 : w + (int64_t)(p.v0 + 64 * k) * pitch + at.i0);
        b.a1 = b.a0 + 64 * pitch;
        b.b0 = (const char*)(p.dz + 64 * k);
        b.b1 = b.b0 + 64;
    }
    __device__ __forceinline__ void store(const Loop& loop, const At& tile) const {
        const int lane = loop.lane_here(), n = lane & 31, hi = lane >> 5, wv = loop.w % WV, wh = loop.w / WV;
#pragma unroll
        for (int c = 0; c < THW; ++c) {
            const int r = tile.j0 + (wh * THW + c) * 32 + n;
            int m;
            const int term = split_row(r, m);
            if (r >= rows || m >= M) continue;
            float* dst = p.part + ((int64_t)(tile.s * p.terms_h + term) * p.M + m) * p.Dh;
#pragma unroll
            for (int a = 0; a < TVW; ++a)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int i = tile.i0 + (wv * TVW + a) * 32 + 8 * g + 4 * hi;
                    if (i >= p.Dh) continue;
                    f32x4 x = {loop.acc[a][c][4 * g], loop.acc[a][c][4 * g + 1], loop.acc[a][c][4 * g + 2], loop.acc[a][c][4 * g + 3]};
                    if (p.add) x += *reinterpret_cast<const f32x4*>(dst + i);
                    *reinterpret_cast<f32x4*>(dst + i) = x;
                }
        }
    }
};

// d_w: columns of Dh along i, the chunk's along j, rows are summed over.
template <bool F16, int BLOCK, int WV, int WH, int TVW, int THW>
struct LmbWeight {
    using Loop = LmbLoop<true, true, F16, BLOCK, WV, WH, TVW, THW>;
    struct At {
        int i0, j0;
    };
    const LmbParams& p;
    int ni, nj, all, np;
    At at;
    __device__ __forceinline__ LmbWeight(const LmbParams& q) : p(q) {
        all = (lmb_rows(p) + 63) >> 6;
        np = all * p.terms_w;
        ni = (p.Dh + Loop::TI - 1) / Loop::TI;
        nj = (p.n + Loop::TJ - 1) / Loop::TJ;
    }
    __device__ __forceinline__ int tiles() const { return ni * nj; }
    __device__ __forceinline__ void open(int t) {
        int ti, tj;
        lmb_tile(t, ni, nj, 4, 8, ti, tj);
        at = At{ti * Loop::TI, tj * Loop::TJ};
    }
    __device__ __forceinline__ void place(Loop& loop) const {
        loop.template place_columns<Loop::TI, Loop::IPA>(0, (uint32_t)p.Dh * 2, p.Dh - 8 - at.i0);
        loop.template place_columns<Loop::TJ, Loop::IPB>(Loop::IPA, (uint32_t)p.ldz * 2, p.ldz - 8 - at.j0);
    }
    __device__ __forceinline__ void pair(Loop&, int q, typename Loop::Bases& b) const {
        const int term = (q >= all ? 1 : 0) + (q >= 2 * all ? 1 : 0), k = q - term * all;
        b.a0 = (const char*)((F16 ? p.sc.h16 : p.h) + (int64_t)64 * k * p.Dh + at.i0);
        b.a1 = b.a0 + (int64_t)64 * p.Dh;
        b.b0 = (const char*)((F16 ? p.sc.e : p.dz) + term * p.dz_term + (int64_t)64 * k * p.ldz + at.j0);
        b.b1 = b.b0 + (int64_t)64 * p.ldz;
    }
    __device__ __forceinline__ void store(const Loop& loop, const At& tile) const {
        const int lane = loop.lane_here(), n = lane & 31, hi = lane >> 5, wv = loop.w % WV, wh = loop.w / WV;
#pragma unroll
        for (int c = 0; c < THW; ++c) {
            const int j = tile.j0 + (wh * THW + c) * 32 + n, v = p.v0 + j;
            const bool live = j < p.n;                                  // (the same for lane and lane + 32)
            int scale = 0;
            if (F16 && all > 0 && live) scale = p.sc.out[1] - 27 - 16 * (p.sc.col[v] & 7);
#pragma unroll
            for (int a = 0; a < TVW; ++a)
#pragma unroll
                for (int g = 0; g < 4; g += 2) {
                    const int i = tile.i0 + (wv * TVW + a) * 32 + 8 * g + 4 * hi;      // and eight further
                    float x[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        x[e] = loop.acc[a][c][4 * g + e];
                        if constexpr (F16) x[e] = ldexpf(x[e], scale);
                    }
                    if (p.dw_f32) {
                        float* dst = (float*)p.d_w + v * p.dw_stride + i;
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            if (!live || i + 8 * q >= p.Dh) continue;
                            f32x4 y = {x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]};
                            if (p.accumulate) y += *reinterpret_cast<const f32x4*>(dst + 8 * q);
                            *reinterpret_cast<f32x4*>(dst + 8 * q) = y;
                        }
                        continue;
                    }
                    if (p.accumulate) {
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            if (!live || i + 8 * q >= p.Dh) continue;
                            float old[4];
                            load_bf16<4>((const uint16_t*)p.d_w + v * p.dw_stride + i + 8 * q, old);
#pragma unroll
                            for (int e = 0; e < 4; ++e) x[4 * q + e] += old[e];
                        }
                    }
                    const uint32_t w[4] = {pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
                    const u32x4 out = lmb_eight(w);
                    if (live && i + 4 * hi < p.Dh) *reinterpret_cast<u32x4*>((uint16_t*)p.d_w + v * p.dw_stride + i + 4 * hi) = out;
                }
        }
    }
};

// Both in one launch: what a workgroup of the first has left over it spends on the second.
template <bool F16, int BLOCK, typename H, typename W>
__global__ __launch_bounds__(64 * H::WV * H::WH, 1) void lmb_grad_kernel(LmbParams p) {
    static_assert(H::WV * H::WH == W::WV * W::WH, "one workgroup size");
    using Hidden = LmbHidden<F16, BLOCK, H::WV, H::WH, H::TVW, H::THW>;
    using Weight = LmbWeight<F16, BLOCK, W::WV, W::WH, W::TVW, W::THW>;
    __shared__ __attribute__((aligned(1024))) unsigned char ring[Hidden::Loop::RING > Weight::Loop::RING ? Hidden::Loop::RING : Weight::Loop::RING];
    if (blockIdx.x == 0 && threadIdx.x < 8) p.counters[threadIdx.x * 16] = 0;          // the next chunk's list of dz
    const int block = blockIdx.x, xcd = block & 7, wgs = gridDim.x >> 3;
    if (p.n2 > 0 && (p.queued || block < p.n2)) {
        Hidden job(p);
        LmbList list(job.tiles(), block);
        if (p.queued) {
            list.counter = p.counters + LMB_COUNTERS + xcd * 16;
            list.later = 2 * wgs;
            list.ahead = list.index + wgs;
        }
        typename Hidden::Loop loop(ring);
        loop.run(job, list);
    }
    if (!p.d_w || (!p.queued && block < p.n2)) return;
    Weight job(p);
    LmbList list(job.tiles(), p.queued ? block : block - p.n2);
    const bool one_pair = p.queued && job.np < 2;      // (few rows, which the device alone knows: tiles by themselves)
    if (p.queued && !one_pair) {
        // in the order in which workgroups come here
        list.counter = p.counters + 2 * LMB_COUNTERS + xcd * 16;
        if (threadIdx.x == 0) {
            const int first = lmb_take(list.counter);
            reinterpret_cast<int*>(ring)[0] = first;
            reinterpret_cast<int*>(ring)[1] = first < list.len ? lmb_take(list.counter) : first;
        }
        __syncthreads();
        list.index = __builtin_amdgcn_readfirstlane(reinterpret_cast<const int*>(ring)[0]);
        list.ahead = __builtin_amdgcn_readfirstlane(reinterpret_cast<const int*>(ring)[1]);
        __syncthreads();
    }
    typename Weight::Loop loop(ring);
    do {
        loop.run(job, list);
        list.index += wgs;
    } while (one_pair && list.index < list.len);
}

// The parts of d_hidden's sum, in order, into the rows that were selected.  A row that is named several times gets all its entries' sums, in their order, from
// the first of them; the others look for an earlier one and find it.  An ascending list has none, and needs no look: `order` says where it is not.
__global__ __launch_bounds__(256) void lmb_join_kernel(LmbParams p) {
    __shared__ uint64_t same[4];
    const int M = lmb_rows(p), r0 = blockIdx.x, wave = threadIdx.x >> 6;
    if (r0 >= M) return;
    const int c = (blockIdx.y * 256 + threadIdx.x) * 4;
    const auto sum = [&](int r) {
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
        if (c >= p.Dh) return x;
#pragma unroll 4
        for (int s = 0; s < p.splits * p.terms_h; ++s) x += *reinterpret_cast<const f32x4*>(p.part + ((int64_t)s * p.M + r) * p.Dh + c);
        if (p.f16) {
            const int scale = p.sc.out[0] - 14 - p.sc.hs[r];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = ldexpf(x[e], scale);
        }
        return x;
    };
    f32x4 x = sum(r0);
    const int row = p.row_idx ? p.row_idx[r0] : r0;
    const bool twice = p.row_idx && __syncthreads_or(threadIdx.x < LMB_ORDER && p.order[threadIdx.x]);
    for (int b = 0; twice && b < M; b += 256) {
        const int r = b + threadIdx.x;
        const uint64_t mine = __ballot(r < M && r != r0 && p.row_idx[r < M ? r : 0] == row);
        __syncthreads();
        if (lane_id() == 0) same[wave] = mine;
        __syncthreads();
        for (int k = 0; k < 4; ++k) {
            for (uint64_t left = same[k]; left; left &= left - 1) {
                const int other = b + 64 * k + __builtin_ctzll(left);
                if (other < r0) return;
                x += sum(other);
            }
        }
    }
    if (c >= p.Dh) return;
    if (p.dh_f32) *reinterpret_cast<f32x4*>((float*)p.d_hidden + row * p.dh_stride + c) = x;
    else *reinterpret_cast<u32x2*>((uint16_t*)p.d_hidden + row * p.dh_stride + c) = u32x2{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
}

// ---- host ---------------------------------------------------------------------------------------------------
constexpr size_t LMB_DZ_BYTES = (size_t)2 << 30;      // dz of a chunk: more rows, fewer columns at a time
// Two bf16 terms or one fp16: a product more for each gradient (2 M V Dh operations, in tiles that take M / 64 steps more one after the other) against a pass over W and three launches
// of 20 us together.  Both gradients, us of two terms / fp16.  V = 126464, Dh = 4096 130 rows 1239 / 1335, 192 1305 / 1350, 256 1473 / 1414, 320 1952 / 1828, 512 2582 / 2057; 64000 x 2048 256
// rows 420 / 444, 384 578 / 558; 151000 x 896 256 rows 522 / 557, 384 715 / 707.  Small products of up to a thousand rows do not pay for the launches: 8000 x 1024 512 rows 67 / 83, 700 99 / 102,
// 1000 115 / 111; 40000 x 256 512 rows 122 / 170; 2000 x 4096 512 rows 85 / 92, 1000 136 / 128; 3500 x 4096 700 rows 198 / 141; 5000 x 256 1000 rows 52 / 66; 1352 x 896 900 rows 47 / 56,
// 1656 94 / 82; 300 x 64 8192 rows 137 / 110.  Where they are alike two terms are: they keep 16 bits.
constexpr int LMB_FEW = 256, LMB_SOME = 1024;
constexpr double LMB_SMALL = 5e12;                    // M^2 V Dh
static int g_lmb_few = 0;                             // dlm_set_option: two terms up to so many rows and for none above (0: by the rule)
static bool lmb_two_terms(int M, int V, int Dh) {
    if (g_lmb_few > 0) return M <= g_lmb_few;
    return M <= LMB_FEW || (M <= LMB_SOME && (double)M * M * V * Dh <= LMB_SMALL);
}
static int g_lmb_columns = 0;                         // dlm_set_option: most columns of a chunk (0: by the bytes)

static int g_lmb_workgroups = 0;                      // dlm_set_option: workgroups of a launch that takes tiles from a list (0: as fit the chip)

int lmb_set_workgroups(int v) {
    if (v < 0 || v % 8) return fail(DLM_ERR_INVALID_ARG, "set_option: lmhead_bwd_workgroups must be a multiple of 8, or 0");
    g_lmb_workgroups = v;
    return DLM_OK;
}
int lmb_set_few(int v) {
    if (v < 0) return fail(DLM_ERR_INVALID_ARG, "set_option: lmhead_bwd_few must not be negative");
    g_lmb_few = v;
    return DLM_OK;
}
int lmb_set_columns(int v) {
    if (v < 0 || v % 256) return fail(DLM_ERR_INVALID_ARG, "set_option: lmhead_bwd_columns must be a multiple of 256, or 0");
    g_lmb_columns = v;
    return DLM_OK;
}

// A shape: its tiles, and the workgroups of it that a CU holds, of the kernels for bf16 gradients and of those for fp32.  Planned for two of 128 x 128 a CU, fp32
// gradients of 500 rows, V = 50000, Dh = 1536 take 1424 us, for one 1126; 64 rows of 32000 x 4096 498 and 421; 1000 rows 3525 either way.
struct LmbTile {
    int i, j, a_cu, a_cu_wide;
};
constexpr LmbTile LMB_TILES[] = {{256, 256, 1, 1}, {256, 128, 1, 1}, {256, 64, 1, 1}, {128, 128, 2, 1}, {64, 64, 4, 4}};
enum { LMB_256, LMB_256x128, LMB_256x64, LMB_128, LMB_64 };
// Workgroups that fit the chip, a multiple of 8
static int device_wgs(const LmbTile& tile, bool wide) {
    if (g_lmb_workgroups > 0) return g_lmb_workgroups;
    const int cus = device_cus();
    return (cus >= 8 ? cus & ~7 : 8) * (wide ? tile.a_cu_wide : tile.a_cu);
}
static int64_t lmb_tiles(int shape, int64_t i, int64_t j) {
    return ((i + LMB_TILES[shape].i - 1) / LMB_TILES[shape].i) * ((j + LMB_TILES[shape].j - 1) / LMB_TILES[shape].j);
}
// The largest square tile of which there are enough for most CUs; fp32 gradients, whose sums take two more registers an entry, have none of 256.
static int lmb_shape(int64_t i, int64_t j, bool wide) {
    if (!wide && lmb_tiles(LMB_256, i, j) >= 160) return LMB_256;
    return lmb_tiles(LMB_128, i, j) >= 160 ? LMB_128 : LMB_64;
}

struct LmbPlan {
    int padded, terms_h, terms_w, terms, f16, chunk, splits;
    int dz, hidden, weight;        // shapes
    size_t rows_at, h_at, tail_at, dz_at, e_at, panel_at, part_at, h16_at, w16_at, ints_at, counters_at, bytes;
};
static size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

static LmbPlan plan_lmb(const dlm_lmhead_bwd_args* a) {
    LmbPlan p = {};
    p.padded = a->M > 0 ? (a->M + 63) & ~63 : 64;
    const bool wide_h = a->d_hidden && a->d_hidden_type == DLM_ROW_F32, wide_w = a->d_w && a->d_w_type == DLM_ROW_F32, wide = wide_h || wide_w;
    p.f16 = !wide && !lmb_two_terms(a->M, a->V, a->Dh);
    p.terms_h = p.f16 ? 1 : wide_h ? 3 : 2;
    p.terms_w = p.f16 ? 1 : wide_w ? 3 : 2;
    p.terms = p.f16 ? 1 : wide ? 3 : 2;
    const int64_t whole = ((int64_t)a->V + 255) & ~(int64_t)255;
    const int held = p.f16 && a->d_hidden && a->d_w ? 2 : p.terms;        // arrays of dz
    int64_t most = (int64_t)(LMB_DZ_BYTES / ((size_t)p.padded * 2 * held)) & ~(int64_t)255;
    if (most < 256) most = 256;
    if (g_lmb_columns > 0 && most > g_lmb_columns) most = g_lmb_columns;
    p.chunk = (int)(whole < most ? whole : most);
    // few rows: tiles no higher than they are
    const int64_t rows = (int64_t)p.padded * p.terms_h, columns = a->V < p.chunk ? a->V : p.chunk;
    p.dz = lmb_shape(columns, p.padded, wide);
    if (p.dz == LMB_256 && p.padded <= 128) p.dz = p.padded <= 64 ? LMB_256x64 : LMB_256x128;
    p.weight = p.hidden = lmb_shape(a->Dh, columns, wide);
    if (p.weight == LMB_256 && rows <= 128 && !p.f16) p.hidden = LMB_256x128;
    // Parts of d_hidden's sum.  In times of a pair of stages (1.8 us of a 256 x 256 tile): the launch takes what all its tiles take together, but no
    // less than d_hidden's rounds of tiles; a part costs its rows written and read again.
    const LmbTile th = LMB_TILES[p.hidden], tw = LMB_TILES[p.weight];
    const int64_t tiles = lmb_tiles(p.hidden, a->Dh, rows), pairs = (columns + 63) / 64, a_cu = wide ? th.a_cu_wide : th.a_cu, wgs = 256 * a_cu;
    const double unit_h = th.i * th.j / 65536.0, unit_w = tw.i * tw.j / 65536.0;
    const double rest = a->d_w ? lmb_tiles(p.weight, a->Dh, columns) * unit_w * (p.padded / 64) * p.terms_w : 0.0;
    const double part = (double)a->M * p.terms_h * a->Dh * 8e-7;
    int best = 1;
    double least = 1e300;
    for (int s = 1; s <= 64 && s * 4 <= pairs; ++s) {
        const double all = (tiles * pairs * unit_h + rest) / 256, rounds = (double)((tiles * s + wgs - 1) / wgs) * pairs / s * unit_h * a_cu, cost = (all > rounds ? all : rounds) + part * s;
        if (cost < least) {
            least = cost;
            best = s;
        }
    }
    p.splits = best;
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        const size_t here = at;
        at += up256(bytes);
        return here;
    };
    p.counters_at = take((3 * LMB_COUNTERS + LMB_ORDER) * sizeof(int));
    p.rows_at = take((size_t)p.padded * sizeof(LmbRow));
    p.h_at = take((size_t)p.padded * a->Dh * 2);
    p.tail_at = take((size_t)64 * a->Dh * 2);
    if (!p.f16 || a->d_hidden) p.dz_at = take((size_t)p.terms * p.padded * p.chunk * 2);
    if (a->d_hidden) p.part_at = take((size_t)p.splits * p.terms_h * a->M * a->Dh * 4);
    if (p.f16) {
        p.h16_at = take((size_t)p.padded * a->Dh * 2);
        if (a->d_hidden) p.w16_at = take((size_t)(a->V & ~63) * a->Dh * 2);
        if (a->d_w) {
            p.e_at = take((size_t)p.padded * p.chunk * 2);
            p.panel_at = take((size_t)(p.padded / 32) * p.chunk);
        }
        p.ints_at = take(((size_t)4 * p.padded + 2 * whole + LMB_STATS * 34 + 2) * 4);
    }
    p.bytes = at;
    return p;
}

static void launch_dz(const LmbPlan& plan, dim3 grid, hipStream_t st, const LmbParams& p) {
#define LMB_DZ(S, TERMS, BLOCK) hipLaunchKernelGGL((lmb_dz_kernel<S, TERMS, BLOCK>), grid, dim3(256), 0, st, p)
    if (plan.terms == 3) {
        if (plan.dz == LMB_128) LMB_DZ(Lmb128, 3, 2);
        else LMB_DZ(Lmb64, 3, 2);
    } else if (plan.f16) {
        if (plan.dz == LMB_256) LMB_DZ(Lmb256, 0, 0);
        else if (plan.dz == LMB_128) LMB_DZ(Lmb128, 0, 0);
        else LMB_DZ(Lmb64, 0, 0);
    } else {
        if (plan.dz == LMB_256) LMB_DZ(Lmb256, 2, 0);
        else if (plan.dz == LMB_256x128) LMB_DZ(Lmb256x128, 2, 0);
        else if (plan.dz == LMB_256x64) LMB_DZ(Lmb256x64, 2, 0);
        else if (plan.dz == LMB_128) LMB_DZ(Lmb128, 2, 0);
        else LMB_DZ(Lmb64, 2, 0);
    }
#undef LMB_DZ
}
static void launch_grad(const LmbPlan& plan, dim3 grid, hipStream_t st, const LmbParams& p) {
#define LMB_GRAD(F16, BLOCK, H, W) hipLaunchKernelGGL((lmb_grad_kernel<F16, BLOCK, H, W>), grid, dim3(256), 0, st, p)
    if (plan.terms == 3) {
        if (plan.weight == LMB_128) LMB_GRAD(false, 4, Lmb128, Lmb128);
        else LMB_GRAD(false, 4, Lmb64, Lmb64);
    } else if (plan.f16) {
        if (plan.weight == LMB_256) LMB_GRAD(true, 0, Lmb256, Lmb256);
        else if (plan.weight == LMB_128) LMB_GRAD(true, 0, Lmb128, Lmb128);
        else LMB_GRAD(true, 0, Lmb64, Lmb64);
    } else {
        if (plan.hidden == LMB_256) LMB_GRAD(false, 0, Lmb256, Lmb256);
        else if (plan.hidden == LMB_256x128) LMB_GRAD(false, 0, Lmb256x128, Lmb256);
        else if (plan.weight == LMB_128) LMB_GRAD(false, 0, Lmb128, Lmb128);
        else LMB_GRAD(false, 0, Lmb64, Lmb64);
    }
#undef LMB_GRAD
}

static int validate_lmb(const dlm_lmhead_bwd_args* a, const char* who) {
    if (!a) return fail(DLM_ERR_INVALID_ARG, "%s: null args", who);
    if (a->struct_size != sizeof(dlm_lmhead_bwd_args))
        return fail(DLM_ERR_INVALID_ARG, "%s: struct_size %u != %zu", who, a->struct_size, sizeof(dlm_lmhead_bwd_args));
    if (a->M < 0 || a->Dh <= 0 || a->V <= 0) return fail(DLM_ERR_INVALID_ARG, "%s: bad sizes M=%d Dh=%d V=%d", who, a->M, a->Dh, a->V);
    if (a->Dh % 64) return fail(DLM_ERR_UNSUPPORTED, "%s: Dh=%d is not a multiple of 64", who, a->Dh);
    if (a->M > 1 << 20 || a->Dh > 1 << 16 || a->V > 1 << 24)
        return fail(DLM_ERR_UNSUPPORTED, "%s: M=%d Dh=%d V=%d (supported: up to 2^20, 2^16, 2^24)", who, a->M, a->Dh, a->V);
    if (a->forbid_token >= a->V) return fail(DLM_ERR_INVALID_ARG, "%s: forbid_token %d >= V", who, a->forbid_token);
    if (!(a->inv_temperature > 0.f) || a->inv_temperature > 3.0e38f) return fail(DLM_ERR_INVALID_ARG, "%s: inv_temperature must be positive and finite", who);
    int rc;
    if (a->d_hidden) {
        if ((rc = validate_row_type(a->d_hidden_type, who, "d_hidden")) != DLM_OK) return rc;
        if ((rc = validate_rows(a->d_hidden, a->d_hidden_stride_row, a->M > 0 ? 2 : 0, a->Dh, row_bytes(a->d_hidden_type), true, who, "d_hidden")) != DLM_OK) return rc;
    }
    if (a->d_w) {
        if ((rc = validate_row_type(a->d_w_type, who, "d_w")) != DLM_OK) return rc;
        if ((rc = validate_rows(a->d_w, a->d_w_stride_row, a->V, a->Dh, row_bytes(a->d_w_type), true, who, "d_w")) != DLM_OK) return rc;
    }
    if (a->M == 0) return DLM_OK;
    if (!a->d_hidden && !a->d_w) return fail(DLM_ERR_INVALID_ARG, "%s: neither d_hidden nor d_w", who);
    if (!a->d_lse && !a->d_ztarget) return fail(DLM_ERR_INVALID_ARG, "%s: neither d_lse nor d_ztarget", who);
    if (a->d_ztarget && !a->target) return fail(DLM_ERR_INVALID_ARG, "%s: d_ztarget needs target", who);
    if (!a->lse) return fail(DLM_ERR_INVALID_ARG, "%s: null lse", who);
    if ((rc = validate_rows(a->hidden, a->hidden_stride_row, 2, a->Dh, 2, false, who, "hidden")) != DLM_OK) return rc;
    if ((rc = validate_rows(a->w, a->w_stride_row, a->V, a->Dh, 2, false, who, "w")) != DLM_OK) return rc;
    if (a->d_w && (a->d_w == a->w || a->d_w == a->d_hidden)) return fail(DLM_ERR_INVALID_ARG, "%s: d_w is w or d_hidden", who);
    if (a->hidden_stride_row < a->Dh || (a->V > 1 && a->w_stride_row < a->Dh)) return fail(DLM_ERR_INVALID_ARG, "%s: row stride < Dh", who);
    if (a->V > 1 && a->w_stride_row >= 1 << 23) return fail(DLM_ERR_UNSUPPORTED, "%s: w_stride_row >= 2^23", who);
    return DLM_OK;
}

}  // namespace dlm

using namespace dlm;

extern "C" size_t dlm_lmhead_bwd_workspace_bytes(const dlm_lmhead_bwd_args* a) {
    if (!a || a->struct_size != sizeof(dlm_lmhead_bwd_args) || a->M < 0 || a->Dh <= 0 || a->V <= 0) return 0;
    return plan_lmb(a).bytes;
}

extern "C" int dlm_lmhead_bwd(const dlm_lmhead_bwd_args* a, void* stream) {
    static const char who[] = "lmhead_bwd";
    int rc;
    if ((rc = validate_lmb(a, who)) != DLM_OK) return rc;
    if (a->M == 0 && (!a->d_w || a->accumulate)) return DLM_OK;
    const LmbPlan plan = plan_lmb(a);
    if (!a->workspace || a->workspace_bytes < plan.bytes) return fail(DLM_ERR_WORKSPACE, "%s: workspace of %zu bytes required", who, plan.bytes);
    if (!aligned16(a->workspace)) return fail(DLM_ERR_WORKSPACE, "%s: workspace not 16-byte aligned", who);
    hipStream_t st = (hipStream_t)stream;
    char* ws = (char*)a->workspace;
    LmbParams p = {};
    p.M = a->M;
    p.Dh = a->Dh;
    p.V = a->V;
    p.m_dev = a->m_dev;
    p.hidden = (const uint16_t*)a->hidden;
    p.h_stride = a->hidden_stride_row;
    p.row_idx = a->row_idx;
    p.w = (const uint16_t*)a->w;
    p.w_stride = a->V > 1 ? a->w_stride_row : a->Dh;
    p.inv_t = a->inv_temperature;
    p.forbid = a->forbid_token < 0 ? -1 : a->forbid_token;
    p.scatter = a->out_scatter;
    p.lse = a->lse;
    p.d_lse = a->d_lse;
    p.d_zt = a->d_ztarget;
    p.target = a->target;
    p.rows = (LmbRow*)(ws + plan.rows_at);
    p.h = (uint16_t*)(ws + plan.h_at);
    p.w_tail = (uint16_t*)(ws + plan.tail_at);
    p.dz = (uint16_t*)(ws + plan.dz_at);
    p.ldz = plan.chunk;
    p.dz_term = (int64_t)plan.padded * plan.chunk;
    p.part = (float*)(ws + plan.part_at);
    p.terms_h = plan.terms_h;
    p.terms_w = plan.terms_w;
    p.f16 = plan.f16;
    if (plan.f16) {
        int* ints = (int*)(ws + plan.ints_at);
        p.sc.row_e = ints;
        p.sc.row_c = ints + plan.padded;
        p.sc.hs = ints + 2 * (int64_t)plan.padded;
        p.sc.ws = ints + 3 * (int64_t)plan.padded;
        p.sc.w_f = ints + 4 * (int64_t)plan.padded;
        p.sc.col = p.sc.w_f + ((int64_t)a->V + 255) / 256 * 256;
        p.sc.row_max = p.sc.col + ((int64_t)a->V + 255) / 256 * 256;
        p.sc.w_some = p.sc.row_max + LMB_STATS;
        p.sc.w_max = p.sc.w_some + LMB_STATS;
        p.sc.out = p.sc.w_max + LMB_STATS * 32;
        p.sc.h16 = (uint16_t*)(ws + plan.h16_at);
        p.sc.w16 = (uint16_t*)(ws + plan.w16_at);
        p.sc.tail16 = p.w_tail;
        p.sc.e = (uint16_t*)(ws + plan.e_at);
        p.sc.panel = (uint8_t*)(ws + plan.panel_at);
    }
    p.last_f = (int)(((int64_t)a->V + 255) / 256 * 256) - 4;
    p.counters = (int*)(ws + plan.counters_at);
    p.order = p.counters + 3 * LMB_COUNTERS;
    p.d_hidden = a->d_hidden;
    p.dh_stride = a->d_hidden_stride_row;
    p.dh_f32 = a->d_hidden_type == DLM_ROW_F32;
    p.d_w = a->d_w;
    p.dw_stride = a->V > 1 ? a->d_w_stride_row : a->Dh;
    p.dw_f32 = a->d_w_type == DLM_ROW_F32;
    p.accumulate = a->accumulate;
    if (a->M > 0) {
        if (plan.f16) {
            hipLaunchKernelGGL(lmb_stat_kernel, dim3(LMB_STATS), dim3(256), 0, st, p);
            if ((rc = check_hip(hipGetLastError(), "lmb_stat_kernel launch")) != DLM_OK) return rc;
        }
        const int more = !plan.f16 ? (a->V % 64 ? 64 : 0) : a->d_hidden ? LMB_STATS * 8 : 0;        // (W's copy is d_hidden's)
        hipLaunchKernelGGL(lmb_gather_kernel, dim3(plan.padded + more), dim3(256), 0, st, p);
        if ((rc = check_hip(hipGetLastError(), "lmb_gather_kernel launch")) != DLM_OK) return rc;
        if (plan.f16) {
            hipLaunchKernelGGL(lmb_scale_kernel, dim3(1), dim3(512), 0, st, p);
            if ((rc = check_hip(hipGetLastError(), "lmb_scale_kernel launch")) != DLM_OK) return rc;
        }
    }
    const bool hidden = a->d_hidden && a->M > 0;
    for (int64_t v0 = 0; v0 < a->V; v0 += plan.chunk) {
        p.v0 = (int)v0;
        p.n = (int)(a->V - v0 < plan.chunk ? a->V - v0 : plan.chunk);
        p.add = v0 > 0;
        const int64_t pairs = (p.n + 63) / 64;
        p.splits = v0 > 0 && pairs < 2 * plan.splits ? 1 : plan.splits;        // (parts that the last chunk has no work for stay as they are)
        const auto up8 = [](int64_t n) { return (n + 7) / 8 * 8; };
        const int64_t n1 = up8(lmb_tiles(plan.dz, p.n, plan.padded)), n3 = a->d_w ? up8(lmb_tiles(plan.weight, a->Dh, p.n)) : 0;
        p.n2 = hidden ? (int)up8(lmb_tiles(plan.hidden, a->Dh, (int64_t)plan.padded * p.terms_h) * p.splits) : 0;
        // A list of tiles where they are more than the workgroups that fit the chip, and long enough to request the next one behind (see LmbLoop)
        if (a->M > 0) {
            const int wgs = device_wgs(LMB_TILES[plan.dz], plan.terms == 3);
            p.queued = n1 > wgs && a->Dh >= 128;
            launch_dz(plan, dim3((unsigned)(p.queued ? wgs : n1)), st, p);
            if ((rc = check_hip(hipGetLastError(), "lmb_dz_kernel launch")) != DLM_OK) return rc;
            const int panel = plan.dz == LMB_256 ? 128 : plan.dz == LMB_128 ? 64 : 32, panels = (plan.padded + panel - 1) / panel;
            if (plan.f16 && a->d_w && panels > 1) {
                hipLaunchKernelGGL(lmb_even_kernel, dim3((unsigned)((p.n + 511) / 512), panels), dim3(256), 0, st, p, panel);
                if ((rc = check_hip(hipGetLastError(), "lmb_even_kernel launch")) != DLM_OK) return rc;
            }
        }
        if (p.n2 + n3 == 0) continue;
        const int wgs = device_wgs(LMB_TILES[plan.weight], plan.terms == 3);
        p.queued = a->M > 0 && p.n2 + n3 > wgs && (!hidden || pairs >= 2 * p.splits);
        launch_grad(plan, dim3((unsigned)(p.queued ? wgs : p.n2 + n3)), st, p);
        if ((rc = check_hip(hipGetLastError(), "lmb_grad_kernel launch")) != DLM_OK) return rc;
    }
    if (!hidden) return DLM_OK;
    p.splits = plan.splits;
    hipLaunchKernelGGL(lmb_join_kernel, dim3(a->M, (a->Dh + 1023) / 1024), dim3(256), 0, st, p);
    return check_hip(hipGetLastError(), "lmb_join_kernel launch");
}
