// dlm_paged_attn: a block of new tokens, or one, against the pages of its sequence.
//
// The g = Hq/Hkv query heads of a KV head and the sequence's query rows are packed into R = g * q_len rows (row = i*g + head), so
// a KV head's keys are read once for 32 of them.  A workgroup owns 32 rows of one (sequence, KV head) and a stretch of its keys; its
// four wavefronts take every fourth 32-key tile, each with LDS of its own, and join through LDS at the end; with a workspace the
// stretches of one sequence go to several workgroups and paged_merge_kernel joins those.
//
// Per tile and wavefront: S^T = K Q^T (a lane then has 16 keys of one row: maximum and sum are in-lane plus one swap of lane
// halves), p rounded to bf16 for the second product (its relative error 2^-9 an entry averages out; the sum uses the unrounded p),
// O^T += V^T P^T with V^T from the transposing LDS read.  Everything else is fp32.
#include "paged.hpp"

namespace dlm {

typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2;

struct PagedAttnParams {
    int B, Lq, Hq, Hkv, g;
    const uint16_t* q;
    int64_t q_sb, q_st, q_sh;
    uint16_t* out;
    int64_t o_sb, o_st, o_sh;
    float* lse;
    const void *k, *v;
    int64_t sp, sh, st;            // strides of a page, a head, a row, in entries
    int n_pages, page_shift;
    const float *k_scale, *v_scale;
    const int32_t* table;
    int64_t table_stride;
    const int32_t* kv_len;
    int max_kv_len;
    const int32_t* q_len;
    int bs;                        // block size of the block-causal mask
    float scale_log2;              // scale * log2(e): the softmax is evaluated with exp2
    // Stretches of `chunk` 32-key tiles: a sequence of T tiles has max(1, ceil(T / chunk)) of them, one workgroup each.
    int chunk, nsplit, row_tiles;
    GridRemap remap;
    float *part_o, *part_ml;       // [nsplit][B * Hq * Lq][d] and [..][2]: sums and (maximum in log2 units, sum) of a stretch
};

__device__ __forceinline__ bf16x8 as_bf16x8(u32x4 v) {
    union { u32x4 u; bf16x8 b; } x;
    x.u = v;
    return x.b;
}
__device__ __forceinline__ int clamped(int v, int hi) { return min(max(v, 0), hi); }

// eight e4m3 entries as bf16 (exact: bf16 has more of both exponent and mantissa)
__device__ __forceinline__ u32x4 widen_e4m3(uint32_t lo, uint32_t hi) {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(lo, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(lo, true);
    const f32x2 c = __builtin_amdgcn_cvt_pk_f32_fp8(hi, false), d = __builtin_amdgcn_cvt_pk_f32_fp8(hi, true);
    return u32x4{pack_bf16x2(a[0], a[1]), pack_bf16x2(b[0], b[1]), pack_bf16x2(c[0], c[1]), pack_bf16x2(d[0], d[1])};
}

// How many keys of the sequence any of the rows before `rows_end` sees
template <bool BC>
__device__ __forceinline__ int visible_keys(const PagedAttnParams& p, int len, int ql, int rows_end) {
    if (!BC) return len;
    const int pos = len - ql + (rows_end - 1) / p.g;
    return pos < 0 ? 0 : min((int64_t)len, ((int64_t)(pos / p.bs) + 1) * p.bs);
}

// NT: non-temporal loads, where one workgroup is the only reader of its keys.
template <int D, bool F8, bool BC, bool NT>
__global__ __launch_bounds__(256, 2) void paged_attn_kernel(PagedAttnParams p) {
    constexpr int NW = 4;
    constexpr int KP = D * 2 + 16;          // pitch of a K row in LDS: 16-byte reads of 16 rows hit distinct banks
    constexpr int VP = D * 2 + 64;          // of a V row: the 4 rows x 64 bytes of a transposing read tile the banks
    constexpr int TILE = 32 * KP + 32 * VP;
    constexpr int ES = F8 ? 1 : 2;          // bytes an entry of the cache
    constexpr int C = D * ES / 16;          // 16-byte pieces a row
    constexpr int RPL = 64 / C;             // rows a load of the wavefront covers
    constexpr int NLD = 32 / RPL;
    constexpr int MP = D + 4;               // pitch of a row of partial sums (floats)
    constexpr int MERGE = NW * 32 * MP * 4;
    __shared__ __attribute__((aligned(16))) unsigned char smem[NW * TILE > MERGE ? NW * TILE : MERGE];

    fetch_args<sizeof(PagedAttnParams)>();
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 31, hi = lane >> 5;
    int grp, rt;
    if (!remap_decode(p.remap, p.B * p.Hkv * p.nsplit, grp, rt)) return;
    const int split = grp % p.nsplit, bh = grp / p.nsplit, kvh = bh % p.Hkv, b = bh / p.Hkv;
    // Pages of the wavefront's next 32 tiles: lane 2j + h holds the one of half h (16 keys, a page is no smaller) of its j-th tile.  One load for 32
    // tiles, requested 32 tiles ahead: a look-up a tile was a trip to memory in front of every fetch.  The first one travels with the
    // sequence's lengths, so it may look at entries behind the sequence's end (but inside the table's row): whatever they hold, a page
    // outside the cache is not read and a key behind the end not seen.
    const int t0 = split * p.chunk, last_entry = (max(p.max_kv_len, 1) - 1) >> p.page_shift;
    const int32_t* table = p.table + b * p.table_stride;
    auto pages_from = [&](int j) { return table[min((int)(((int64_t)(t0 + w + NW * (j + (lane >> 1))) * 32 + 16 * (lane & 1)) >> p.page_shift), last_entry)]; };
    int pages = p.max_kv_len > 0 ? pages_from(0) : 0;
    const int len = clamped(p.kv_len[b], p.max_kv_len), ql = p.q_len ? clamped(p.q_len[b], p.Lq) : p.Lq;
    const int R = ql * p.g, r0 = rt * 32;
    if (r0 >= R) return;
    const int seen = visible_keys<BC>(p, len, ql, min(r0 + 32, R));
    const int T = (seen + 31) >> 5;
    const int Tn = min(T - t0, p.chunk);
    if (split > 0 && Tn <= 0) return;
    const bool alone = T <= p.chunk;        // no other stretch: this workgroup writes the output

    // ---- this lane's query row (B operand: row, 8 consecutive entries) ----
    bf16x8 qf[D / 16];
    const int r = r0 + n, qi = r < R ? r / p.g : 0, qh = r < R ? r - qi * p.g : 0;
    const uint16_t* qp = p.q + b * p.q_sb + qi * p.q_st + (int64_t)(kvh * p.g + qh) * p.q_sh;
#pragma unroll
    for (int c = 0; c < D / 16; ++c) {
        u32x4 v = {0, 0, 0, 0};
        if (r < R) v = *reinterpret_cast<const u32x4*>(qp + 16 * c + 8 * hi);
        qf[c] = as_bf16x8(v);
    }
    const int limit = visible_keys<BC>(p, len, ql, r < R ? (r / p.g + 1) * p.g : min(r0 + 32, R));     // keys this lane's row sees
    const int limit_min = visible_keys<BC>(p, len, ql, r0 + 1);                                         // fewest of any row (the first one's)
    const float scale_log2 = F8 && p.k_scale ? p.scale_log2 * p.k_scale[kvh] : p.scale_log2;

    f32x16 O[D / 32];
    float m_run = -INFINITY, l_run = 0.f;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) O[dt][i] = 0.f;

    unsigned char* Kl = smem + w * TILE;
    unsigned char* Vl = Kl + 32 * KP;
    const int lrow = lane / C, lc = lane % C;
    const unsigned char* kb = (const unsigned char*)p.k + (int64_t)kvh * p.sh * ES;
    const unsigned char* vb = (const unsigned char*)p.v + (int64_t)kvh * p.sh * ES;
    uint32_t off[NLD];                      // of this lane's piece of load q, from the first row of its half tile
#pragma unroll
    for (int q = 0; q < NLD; ++q) off[q] = (uint32_t)(((q * RPL + lrow) & 15) * (int)p.st * ES + lc * 16);

    int pages_next = 0;
    u32x4 kr[NLD], vr[NLD];
    bool there[2];                          // whether the pages of the two halves exist
    auto fetch = [&](int j) {               // requests the wavefront's j-th tile
        const int key = (t0 + w + NW * j) * 32;
        const unsigned char *ks[2], *vs[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int page = __builtin_amdgcn_readlane(pages, 2 * (j & 31) + h);
            there[h] = (unsigned)page < (unsigned)p.n_pages;
            const int64_t base = ((int64_t)(there[h] ? page : 0) * p.sp + (int64_t)((key + 16 * h) & ((1 << p.page_shift) - 1)) * p.st) * ES;
            ks[h] = kb + base;
            vs[h] = vb + base;
        }
#pragma unroll
        for (int q = 0; q < NLD; ++q) {
            const int h = q * RPL / 16;
            kr[q] = NT ? __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(ks[h] + off[q])) : *reinterpret_cast<const u32x4*>(ks[h] + off[q]);
            vr[q] = NT ? __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(vs[h] + off[q])) : *reinterpret_cast<const u32x4*>(vs[h] + off[q]);
        }
    };
    const int J = (Tn - w + NW - 1) / NW;   // tiles of this wavefront
    if (J > 0) {
        if (J > 32) pages_next = pages_from(32);
        fetch(0);
    }
    for (int j = 0; j < J; ++j) {
        const int key0 = (t0 + w + NW * j) * 32;
        const bool here0 = there[0], here1 = there[1];
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // the tile before has been read (one wavefront's LDS operations keep their order)
        const bool whole = key0 + 32 <= seen && here0 && here1;
#pragma unroll
        for (int q = 0; q < NLD; ++q) {
            const int row = q * RPL + lrow;
            const u32x4 z = {0, 0, 0, 0}, kv = kr[q];
            u32x4 vv = vr[q];
            // rows behind the end hold anything, NaN too: as values they have to be zeros (as keys their scores are replaced)
            if (!whole && !(key0 + row < seen && (q * RPL < 16 ? here0 : here1))) vv = z;
            if constexpr (F8) {
                u32x4* kd = reinterpret_cast<u32x4*>(Kl + row * KP + lc * 32);
                u32x4* vd = reinterpret_cast<u32x4*>(Vl + row * VP + lc * 32);
                kd[0] = widen_e4m3(kv[0], kv[1]);
                kd[1] = widen_e4m3(kv[2], kv[3]);
                vd[0] = widen_e4m3(vv[0], vv[1]);
                vd[1] = widen_e4m3(vv[2], vv[3]);
            } else {
                *reinterpret_cast<u32x4*>(Kl + row * KP + lc * 16) = kv;
                *reinterpret_cast<u32x4*>(Vl + row * VP + lc * 16) = vv;
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (j + 1 < J) {
            if (((j + 1) & 31) == 0) {
                pages = pages_next;
                if (j + 33 < J) pages_next = pages_from(j + 33);
            }
            fetch(j + 1);
        }
        f32x16 S;
#pragma unroll
        for (int i = 0; i < 16; ++i) S[i] = 0.f;
#pragma unroll
        for (int c = 0; c < D / 16; ++c)
            S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(Kl + n * KP + (16 * c + 8 * hi) * 2), qf[c], S, 0, 0, 0);
        // entry i is key key0 + 8 (i / 4) + 4 hi + i % 4
        if (key0 + 32 > limit_min || !here0 || !here1) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (key0 + 8 * (i >> 2) + 4 * hi + (i & 3) >= limit || !(i < 8 ? here0 : here1)) S[i] = -INFINITY;
        }
        float mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < 16; i += 2) mx = __builtin_fmaxf(__builtin_fmaxf(mx, S[i]), S[i + 1]);
        const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
        mx = __builtin_fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * scale_log2;
        // The maximum that the exponentials are relative to follows the running one only when that has grown by 2^8 (p stays in range of bf16 and
        // of the sums): the 64 accumulators are rescaled a few times a row instead of at every tile.
        const bool grow = mx > m_run + 8.0f;
        const float m_new = grow ? mx : m_run;
        const float m_use = m_new == -INFINITY ? 0.f : m_new;
        float rs = 0.f;
        uint32_t pk[8];
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            const float p0 = fast_exp2(fmaf(S[i], scale_log2, -m_use)), p1 = fast_exp2(fmaf(S[i + 1], scale_log2, -m_use));
            rs += p0 + p1;
            pk[i >> 1] = pack_bf16x2(p0, p1);
        }
        if (__any(grow)) {
            const float alpha = grow ? fast_exp2(m_run - m_use) : 1.0f;
            l_run *= alpha;
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                for (int i = 0; i < 16; ++i) O[dt][i] *= alpha;
        }
        l_run += rs;
        m_run = m_new;
        const u32x4 plo = {pk[0], pk[1], pk[2], pk[3]}, phi = {pk[4], pk[5], pk[6], pk[7]};
        const bf16x8 pf[2] = {as_bf16x8(plo), as_bf16x8(phi)};
        const int s16 = lane & 15, blk = (lane >> 4) & 1;
        const unsigned char* vbase = Vl + (4 * hi + (s16 >> 2)) * VP + (16 * blk + 4 * (s16 & 3)) * 2;
#pragma unroll
        for (int e = 0; e < 2 * (D / 32); ++e) {
            union { s16x4 h[2]; bf16x8 v; } f;
#pragma unroll
            for (int q = 0; q < 2; ++q)
                f.h[q] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vbase + (16 * (e & 1) + 8 * q) * VP + 32 * (e >> 1) * 2));
            O[e >> 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.v, pf[e & 1], O[e >> 1], 0, 0, 0);
        }
    }

    // ---- join the wavefronts ----
    constexpr float LN2 = 0.6931471805599453f;
    constexpr int C8 = D / 8;
    float* mb = reinterpret_cast<float*>(smem);
    __syncthreads();
    l_run += shfl_xor(l_run, 32);
    float* row = mb + (w * 32 + n) * MP;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4)
            *reinterpret_cast<f32x4*>(row + 32 * dt + 8 * q4 + 4 * hi) = f32x4{O[dt][4 * q4], O[dt][4 * q4 + 1], O[dt][4 * q4 + 2], O[dt][4 * q4 + 3]};
    if (hi == 0) {
        row[D] = m_run;
        row[D + 1] = l_run;
    }
    __syncthreads();
    for (int task = tid; task < 32 * C8; task += 256) {
        const int rr = task / C8, c8 = task - rr * C8;
        if (r0 + rr >= R) continue;
        const int i = (r0 + rr) / p.g, h = kvh * p.g + (r0 + rr) - i * p.g;
        float M = -INFINITY, den = 0.f, wgt[NW], o[8];
#pragma unroll
        for (int k = 0; k < NW; ++k) M = __builtin_fmaxf(M, mb[(k * 32 + rr) * MP + D]);
#pragma unroll
        for (int k = 0; k < NW; ++k) {
            const float mk = mb[(k * 32 + rr) * MP + D];
            wgt[k] = mk == -INFINITY ? 0.f : fast_exp2(mk - M);
            den += wgt[k] * mb[(k * 32 + rr) * MP + D + 1];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = 0.f;
#pragma unroll
        for (int k = 0; k < NW; ++k) {
            const float* src = mb + (k * 32 + rr) * MP + 8 * c8;
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] += wgt[k] * src[e];
        }
        if (!alone) {
            const int64_t at = ((int64_t)split * p.B + b) * p.Hq * p.Lq + (int64_t)h * p.Lq + i;
            *reinterpret_cast<f32x4*>(p.part_o + at * D + 8 * c8) = f32x4{o[0], o[1], o[2], o[3]};
            *reinterpret_cast<f32x4*>(p.part_o + at * D + 8 * c8 + 4) = f32x4{o[4], o[5], o[6], o[7]};
            if (c8 == 0) {
                p.part_ml[at * 2] = M;
                p.part_ml[at * 2 + 1] = den;
            }
            continue;
        }
        const float inv = (den == 0.f ? 0.f : 1.f / den) * (F8 && p.v_scale ? p.v_scale[kvh] : 1.f);
        u32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = pack_bf16x2(o[2 * e] * inv, o[2 * e + 1] * inv);
        *reinterpret_cast<u32x4*>(p.out + b * p.o_sb + i * p.o_st + (int64_t)h * p.o_sh + 8 * c8) = v;
        if (p.lse && c8 == 0) p.lse[((int64_t)b * p.Hq + h) * p.Lq + i] = den == 0.f ? -INFINITY : (M + log2f(den)) * LN2;
    }
}

// Joins the stretches of each (sequence, head, row) that has more than one: M = max m_s, w_s = 2^(m_s - M), out = sum w_s o_s / sum w_s l_s,
// lse = (M + log2 sum w_s l_s) ln 2.  D / 4 threads a row and group of stretches, G groups: group k takes stretches k, k + G, .. in their
// order, four requested at a time, and the groups are added up in theirs.
template <int D, bool F8, bool BC, int G>
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedAttnParams p) {
    constexpr int TPR = D / 4, RPW = 256 / TPR / G;
    __shared__ float part[G > 1 ? 256 / TPR : 1][D + 2];
    const int64_t rows = (int64_t)p.B * p.Hq * p.Lq, row = min((int64_t)blockIdx.x * RPW + threadIdx.x / (TPR * G), rows - 1);
    const int c4 = threadIdx.x % TPR, gi = threadIdx.x / TPR, k = gi % G;
    const int i = (int)(row % p.Lq), bh = (int)(row / p.Lq), h = bh % p.Hq, b = bh / p.Hq;
    const int len = clamped(p.kv_len[b], p.max_kv_len), ql = p.q_len ? clamped(p.q_len[b], p.Lq) : p.Lq;
    const int r0 = (i * p.g + h % p.g) & ~31;
    const int T = i < ql ? (visible_keys<BC>(p, len, ql, min(r0 + 32, ql * p.g)) + 31) >> 5 : 0;
    const int n = T <= p.chunk ? 0 : (T + p.chunk - 1) / p.chunk;          // 0: nothing to join here
    float M = -INFINITY, den = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = k; s0 < n; s0 += 4 * G) {
        float m[4], l[4];
        f32x4 v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t at = min(s0 + u * G, n - 1) * rows + row;        // (past the last one it is loaded again and not used)
            m[u] = p.part_ml[at * 2];
            l[u] = p.part_ml[at * 2 + 1];
            v[u] = *reinterpret_cast<const f32x4*>(p.part_o + at * D + 4 * c4);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (s0 + u * G >= n) continue;
            const float m_new = __builtin_fmaxf(M, m[u]), m_use = m_new == -INFINITY ? 0.f : m_new;
            const float a = fast_exp2(M - m_use), w = fast_exp2(m[u] - m_use);
            M = m_new;
            den = den * a + l[u] * w;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = o[e] * a + v[u][e] * w;
        }
    }
    if constexpr (G > 1) {
        *reinterpret_cast<f32x2*>(&part[gi][4 * c4]) = f32x2{o[0], o[1]};
        *reinterpret_cast<f32x2*>(&part[gi][4 * c4 + 2]) = f32x2{o[2], o[3]};
        if (c4 == 0) {
            part[gi][D] = M;
            part[gi][D + 1] = den;
        }
        __syncthreads();
        if (k > 0) return;
#pragma unroll
        for (int u = 1; u < G; ++u) {
            const float m = part[gi + u][D], m_new = __builtin_fmaxf(M, m), m_use = m_new == -INFINITY ? 0.f : m_new;
            const float a = fast_exp2(M - m_use), w = fast_exp2(m - m_use);
            M = m_new;
            den = den * a + part[gi + u][D + 1] * w;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = o[e] * a + part[gi + u][4 * c4 + e] * w;
        }
    }
    if (n == 0) return;
    const float inv = (den == 0.f ? 0.f : 1.f / den) * (F8 && p.v_scale ? p.v_scale[h / p.g] : 1.f);
    const u32x2 v = {pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv)};
    *reinterpret_cast<u32x2*>(p.out + b * p.o_sb + i * p.o_st + (int64_t)h * p.o_sh + 4 * c4) = v;
    if (p.lse && c4 == 0) p.lse[row] = den == 0.f ? -INFINITY : (M + log2f(den)) * 0.6931471805599453f;
}

// ---- host ---------------------------------------------------------------------------------------------------
static int g_paged_chunk = 0;      // "paged_chunk"

// Tiles of a stretch: as many workgroups as give the chip two each, no stretch under 8 tiles (two a wavefront).
static int plan_chunk(const dlm_paged_attn_args* a) {
    if (g_paged_chunk > 0) return g_paged_chunk;
    const int64_t tiles = ((int64_t)a->max_kv_len + 31) / 32, groups = (int64_t)a->B * a->Hkv * (((int64_t)a->Lq * (a->Hq / a->Hkv) + 31) / 32);
    int64_t n = groups >= 512 ? 1 : 512 / groups;
    const int64_t most = tiles / 8;
    if (n > most) n = most;
    if (n < 1) n = 1;
    const int64_t chunk = (tiles + n - 1) / n;
    return (int)(chunk > 1 ? chunk : 1);
}
static int splits_of(const dlm_paged_attn_args* a, int chunk) {
    const int64_t tiles = ((int64_t)a->max_kv_len + 31) / 32;
    return (int)(tiles > 0 ? (tiles + chunk - 1) / chunk : 1);
}
static size_t paged_workspace_bytes(const dlm_paged_attn_args* a, int nsplit) {
    return nsplit <= 1 ? 0 : (size_t)nsplit * (size_t)a->B * (size_t)a->Hq * (size_t)a->Lq * (size_t)(a->d + 2) * sizeof(float);
}

static int validate_paged_attn(const dlm_paged_attn_args* a) {
    static const char who[] = "paged_attn";
    if (!a) return fail(DLM_ERR_INVALID_ARG, "%s: null args", who);
    if (a->struct_size != sizeof(dlm_paged_attn_args))
        return fail(DLM_ERR_INVALID_ARG, "%s: struct_size %u != %zu", who, a->struct_size, sizeof(dlm_paged_attn_args));
    if (a->B < 0 || a->Lq < 0 || a->Hq <= 0 || a->Hkv <= 0) return fail(DLM_ERR_INVALID_ARG, "%s: bad sizes B=%d Lq=%d Hq=%d Hkv=%d", who, a->B, a->Lq, a->Hq, a->Hkv);
    if (a->Hq % a->Hkv) return fail(DLM_ERR_INVALID_ARG, "%s: Hq=%d is not a multiple of Hkv=%d", who, a->Hq, a->Hkv);
    if (a->d != 64 && a->d != 128) return fail(DLM_ERR_UNSUPPORTED, "%s: head_dim %d (supported: 64, 128)", who, a->d);
    if ((int64_t)a->Lq * (a->Hq / a->Hkv) > (1 << 30)) return fail(DLM_ERR_UNSUPPORTED, "%s: too many rows per KV head", who);
    if (a->mask_mode != DLM_MASK_FULL && a->mask_mode != DLM_MASK_BLOCK_CAUSAL) return fail(DLM_ERR_INVALID_ARG, "%s: unknown mask_mode %d", who, a->mask_mode);
    if (a->mask_mode == DLM_MASK_BLOCK_CAUSAL && a->block_size < 1) return fail(DLM_ERR_INVALID_ARG, "%s: block-causal needs block_size >= 1", who);
    if (!(a->scale == a->scale)) return fail(DLM_ERR_INVALID_ARG, "%s: scale is NaN", who);
    if (a->max_kv_len < 0 || a->max_kv_len > (1 << 30)) return fail(DLM_ERR_INVALID_ARG, "%s: max_kv_len outside [0, 2^30]", who);
    int rc = validate_cache(a->cache, a->Hkv, a->d, who, false);
    if (rc != DLM_OK) return rc;
    if (a->cache.stride_t >= 1 << 26) return fail(DLM_ERR_UNSUPPORTED, "%s: stride_t of the cache is 2^26 or more", who);     // 15 of them in 32 bits
    if (a->table_stride < 0) return fail(DLM_ERR_INVALID_ARG, "%s: table_stride < 0", who);
    // (in pages: no product that could overflow)
    if (((int64_t)a->max_kv_len + a->cache.page_size - 1) / a->cache.page_size > a->table_stride)
        return fail(DLM_ERR_INVALID_ARG, "%s: max_kv_len=%d does not fit a row of the block table", who, a->max_kv_len);
    if (a->B == 0 || a->Lq == 0) return DLM_OK;
    if (!a->q || !a->out || !a->kv_len) return fail(DLM_ERR_INVALID_ARG, "%s: null q/out/kv_len", who);
    if (a->max_kv_len > 0 && !a->block_table) return fail(DLM_ERR_INVALID_ARG, "%s: null block_table", who);
    if (!aligned16(a->q) || !aligned16(a->out)) return fail(DLM_ERR_UNSUPPORTED, "%s: q/out not 16-byte aligned", who);
    const int64_t n[3] = {a->B, a->Lq, a->Hq}, qs[3] = {a->q_stride_b, a->q_stride_t, a->q_stride_h}, os[3] = {a->o_stride_b, a->o_stride_t, a->o_stride_h};
    for (int i = 0; i < 3; ++i)
        if (n[i] > 1 && (qs[i] % 8 || os[i] % 8)) return fail(DLM_ERR_UNSUPPORTED, "%s: q/out strides must be multiples of 8", who);
    if (!apart(n, os, a->d)) return fail(DLM_ERR_INVALID_ARG, "%s: rows of out overlap", who);
    return DLM_OK;
}

template <int D, bool F8, bool BC>
static int launch_paged(const PagedAttnParams& p, unsigned grid, hipStream_t st) {
    if (p.remap.nx == 1) hipLaunchKernelGGL((paged_attn_kernel<D, F8, BC, true>), dim3(grid), dim3(256), 0, st, p);
    else hipLaunchKernelGGL((paged_attn_kernel<D, F8, BC, false>), dim3(grid), dim3(256), 0, st, p);
    int rc = check_hip(hipGetLastError(), "paged_attn_kernel launch");
    if (rc != DLM_OK || p.nsplit <= 1) return rc;
    constexpr int GROUPS = 1024 / D;
    const int64_t rows = (int64_t)p.B * p.Hq * p.Lq;
    if (p.nsplit > 4) hipLaunchKernelGGL((paged_merge_kernel<D, F8, BC, GROUPS>), dim3((unsigned)rows), dim3(256), 0, st, p);
    else hipLaunchKernelGGL((paged_merge_kernel<D, F8, BC, 1>), dim3((unsigned)((rows + GROUPS - 1) / GROUPS)), dim3(256), 0, st, p);
    return check_hip(hipGetLastError(), "paged_merge_kernel launch");
}

int paged_set_chunk(int v) {
    if (v < 0) return fail(DLM_ERR_INVALID_ARG, "set_option: paged_chunk must be >= 0");
    g_paged_chunk = v;
    return DLM_OK;
}

}  // namespace dlm

using namespace dlm;

extern "C" size_t dlm_paged_attn_workspace_bytes(const dlm_paged_attn_args* a) {
    if (!a || a->struct_size != sizeof(dlm_paged_attn_args) || a->B <= 0 || a->Lq <= 0 || a->Hq <= 0 || a->Hkv <= 0 || a->Hq % a->Hkv || a->d <= 0 ||
        a->max_kv_len <= 0)
        return 0;
    return paged_workspace_bytes(a, splits_of(a, plan_chunk(a)));
}

extern "C" int dlm_paged_attn(const dlm_paged_attn_args* a, void* stream) {
    int rc = validate_paged_attn(a);
    if (rc != DLM_OK) return rc;
    if (a->B == 0 || a->Lq == 0) return DLM_OK;
    const dlm_paged_kv& c = a->cache;
    PagedAttnParams p = {};
    p.B = a->B; p.Lq = a->Lq; p.Hq = a->Hq; p.Hkv = a->Hkv; p.g = a->Hq / a->Hkv;
    p.q = (const uint16_t*)a->q; p.q_sb = a->q_stride_b; p.q_st = a->q_stride_t; p.q_sh = a->q_stride_h;
    p.out = (uint16_t*)a->out; p.o_sb = a->o_stride_b; p.o_st = a->o_stride_t; p.o_sh = a->o_stride_h;
    p.lse = a->lse;
    p.k = c.k; p.v = c.v; p.sp = c.stride_page; p.sh = c.stride_h; p.st = c.stride_t;
    p.n_pages = c.n_pages; p.page_shift = log2_of(c.page_size);
    p.k_scale = c.k_scale; p.v_scale = c.v_scale;
    p.table = a->block_table; p.table_stride = a->table_stride;
    p.kv_len = a->kv_len; p.max_kv_len = c.n_pages > 0 ? a->max_kv_len : 0;     // without pages there are no keys
    p.q_len = a->q_len;
    p.bs = a->block_size;
    p.scale_log2 = (a->scale > 0.f ? a->scale : 1.0f / sqrtf((float)a->d)) * 1.4426950408889634f;
    const int64_t tiles = ((int64_t)a->max_kv_len + 31) / 32;
    p.chunk = plan_chunk(a);
    p.nsplit = splits_of(a, p.chunk);
    if (p.nsplit > 1) {
        if (a->workspace && a->workspace_bytes >= paged_workspace_bytes(a, p.nsplit) && aligned16(a->workspace)) {
            p.part_o = (float*)a->workspace;
            p.part_ml = p.part_o + (size_t)p.nsplit * a->B * a->Hq * a->Lq * a->d;
        } else {
            p.nsplit = 1;
            p.chunk = (int)(tiles > 1 ? tiles : 1);
        }
    }
    const int64_t row_tiles = ((int64_t)a->Lq * p.g + 31) / 32, groups = (int64_t)a->B * a->Hkv * p.nsplit;
    if (groups > 0x7fffffff || row_tiles > 0x7fffffff) return fail(DLM_ERR_UNSUPPORTED, "paged_attn: too many workgroups");
    const int64_t grid = set_remap(p.remap, groups, (int)row_tiles, false);
    if (grid == 0) return fail(DLM_ERR_UNSUPPORTED, "paged_attn: too many workgroups");
    if (p.nsplit > 1 && (int64_t)a->B * a->Hq * a->Lq > 0x7fffffff) return fail(DLM_ERR_UNSUPPORTED, "paged_attn: too many rows");
    hipStream_t st = (hipStream_t)stream;
    const bool f8 = c.type == DLM_KV_E4M3, bc = a->mask_mode == DLM_MASK_BLOCK_CAUSAL;
#define PAGED_LAUNCH(D)                                                                                                    \
    (f8 ? (bc ? launch_paged<D, true, true>(p, (unsigned)grid, st) : launch_paged<D, true, false>(p, (unsigned)grid, st))  \
        : (bc ? launch_paged<D, false, true>(p, (unsigned)grid, st) : launch_paged<D, false, false>(p, (unsigned)grid, st)))
    return a->d == 128 ? PAGED_LAUNCH(128) : PAGED_LAUNCH(64);
#undef PAGED_LAUNCH
}
