// dlm_paged_attn: a block of new tokens, or one, against the pages of its sequence.
//
// The g = Hq/Hkv query heads of a KV head and the sequence's query rows are packed into R = g * q_len rows (row = i*g + head), and a workgroup
// takes some of them, a "row group" of one (sequence, KV head).  With a workspace the 32-key tiles of all row groups may be dealt
// out evenly (see Shares), and paged_merge_kernel joins what belongs together.  Three shapes, by R; which, and whether shares, see plan_paged:
//   paged_thin_kernel   16 rows, keys split over the wavefronts (a few short sequences): bound by latency
//   paged_wide_kernel   32 rows, keys split over the wavefronts (single tokens, small blocks): bound by HBM
//   paged_tall_kernel   128 rows, 32 a wavefront, which share the tiles of keys in LDS (blocks with many heads a KV head): bound by the products
//                       and what stands between them
// Per 32-key tile: S^T = K Q^T (a lane then has 8 or 16 keys of one row: maximum and sum are in-lane but for one or two swaps), O^T += V^T P^T with V^T from
// the transposing LDS read.  The second product takes 16-bit operands too, so p is rounded for it (never for the sum): see Weights.  Everything else is fp32.
#include "paged.hpp"

namespace dlm {

typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2;
typedef __attribute__((__vector_size__(8 * sizeof(_Float16)))) _Float16 f16x8;

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
    FastDiv by_g, by_bs, by_shares;
    float scale_log2;              // scale * log2(e): the softmax is evaluated with exp2
    int rows_wg, row_groups;       // rows of a workgroup; row groups that Lq rows make
    int thin_waves;                // wavefronts of a workgroup of 16 rows
    GridRemap remap;               // one workgroup a row group
    // even shares: workgroups, and what they leave to be joined: sums [2 * shares][rows_wg][d] with (maximum in log2 units, sum) [..][2], and for each
    // row group its first workgroup and their number
    int shares;
    float *part_o, *part_ml;
    int32_t* meta;
};

__device__ __forceinline__ bf16x8 as_bf16x8(u32x4 v) {
    union { u32x4 u; bf16x8 b; } x;
    x.u = v;
    return x.b;
}
__device__ __forceinline__ int clamped(int v, int hi) { return min(max(v, 0), hi); }

__device__ __forceinline__ f16x8 as_f16x8(u32x4 v) {
    union { u32x4 u; f16x8 h; } x;
    x.u = v;
    return x.h;
}

// eight e4m3 entries as bf16 or fp16 (exact: both have more exponents, 2^-9 .. 448 are normal numbers, and more mantissa)
template <bool HALF>
__device__ __forceinline__ u32x4 widen_e4m3(uint32_t lo, uint32_t hi) {
    auto pair = [](uint32_t w, bool upper) {
        if constexpr (HALF) {
            union { __attribute__((__vector_size__(2 * sizeof(_Float16)))) _Float16 h; uint32_t u; } x;
            if (upper) x.h = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true);
            else x.h = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false);
            return x.u;
        } else {
            union { __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 b; uint32_t u; } x;
            if (upper) x.b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true);
            else x.b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false);
            return x.u;
        }
    };
    return u32x4{pair(lo, false), pair(lo, true), pair(hi, false), pair(hi, true)};
}

// Keys that query i of a sequence sees
template <bool BC>
__device__ __forceinline__ int visible_keys(const PagedAttnParams& p, int len, int ql, int i) {
    if (!BC) return len;
    const int pos = len - ql + i;
    return pos < 0 ? 0 : (int)min((int64_t)len, ((int64_t)quotient(pos, p.by_bs) + 1) * p.bs);
}

__device__ __forceinline__ int query_of(const PagedAttnParams& p, int r) { return (int)quotient(r, p.by_g); }

// What a workgroup works on: RT rows of one (sequence, KV head) from r0 on, tiles t0 .. t0 + Tn - 1 of 32 keys.
template <int RT, bool BC>
struct Work {
    int b, kvh, r0, len, ql, R, seen, t0, Tn;
    int slot;                               // where its sums go; -1: nobody else has keys of these rows, it writes the output
    // one workgroup a row group
    __device__ __forceinline__ bool place(const PagedAttnParams& p) {
        int grp, rg;
        if (!remap_decode(p.remap, p.B * p.Hkv, grp, rg)) return false;
        kvh = grp % p.Hkv;
        b = grp / p.Hkv;
        r0 = rg * RT;
        t0 = 0;
        slot = -1;
        return true;
    }
    __device__ __forceinline__ void lengths(const PagedAttnParams& p, int len_, int ql_) {
        len = clamped(len_, p.max_kv_len);
        ql = p.q_len ? clamped(ql_, p.Lq) : p.Lq;
        R = ql * p.g;
    }
    // (once r0 is known)
    __device__ __forceinline__ void see(const PagedAttnParams& p) {
        seen = visible_keys<BC>(p, len, ql, query_of(p, min(r0 + RT, R) - 1));
        Tn = (seen + 31) >> 5;
    }
    // keys that row r sees
    __device__ __forceinline__ int limit(const PagedAttnParams& p, int r) const { return visible_keys<BC>(p, len, ql, query_of(p, r)); }
    __device__ __forceinline__ const uint16_t* query(const PagedAttnParams& p, int r) const {
        const int i = query_of(p, r);
        return p.q + b * p.q_sb + i * p.q_st + (int64_t)(kvh * p.g + r - i * p.g) * p.q_sh;
    }
};

constexpr int SMALLEST_SHARE = 8;           // tiles: two a wavefront

// Even shares.  The tiles of all row groups, sequence by sequence, KV head by KV head, make one line of N (a row group has at least one, so that somebody
// writes its zeros; under a block-causal mask each has as many as its sequence's last); with S = max(ceil(N / shares), 8) workgroup w takes tiles
// [w S, (w + 1) S).  So one long sequence among short ones, or too few sequences for the chip, leave no CU idle, and the host need not
// know the lengths.  (What a workgroup keeps of this while it works on a piece is dear: every form with shares spills 34 - 62 scalar registers into vector ones, the
// 32-row one of d = 128, bf16 and a causal mask two vector registers into scratch; without shares 0 - 4 and none.  With equal lengths, 32 sequences of 1000 tokens, 32 rows of
// 28/4 heads: 29 us alone, 40 with shares.)  A share is the end of one row group, some whole ones, the beginning of another: at most two sets of sums, slots 2w (for rows that began
// elsewhere) and 2w + 1.
template <int RT, bool BC>
struct Shares {
    int w, N, S, at, end;                   // its tiles: at .. end - 1
    int b, base, len, ql;                   // the sequence of `at`, its first tile, its lengths as given
    // tiles of each row group of a sequence, and the row groups
    static __device__ __forceinline__ int tiles_of(const PagedAttnParams& p, int len_, int ql_, int& groups) {
        const int len = clamped(len_, p.max_kv_len), ql = p.q_len ? clamped(ql_, p.Lq) : p.Lq;
        groups = p.Hkv * ((ql * p.g + RT - 1) / RT);
        return ql > 0 ? max((visible_keys<BC>(p, len, ql, ql - 1) + 31) >> 5, 1) : 0;
    }
    // false: no share for this workgroup.  smem: 8 ints
    __device__ bool find(const PagedAttnParams& p, int* smem) {
        const int tid = threadIdx.x & 255, lane = lane_id(), wave = tid >> 6;        // (a second 256 threads do the same)
        const int each = (p.B + 255) / 256, from = min(tid * each, p.B), to = min(from + each, p.B);
        int own = 0, groups, l = 0, q = 0;
        for (int i = from; i < to; ++i) {
            l = p.kv_len[i];
            q = p.q_len ? p.q_len[i] : 0;
            own += tiles_of(p, l, q, groups) * groups;
        }
        int sum = own;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int v = __shfl_up(sum, d, 64);
            if (lane >= d) sum += v;
        }
        if (lane == 63) smem[wave] = sum;
        __syncthreads();
        const int s0 = smem[0], s1 = smem[1], s2 = smem[2], s3 = smem[3];
        N = __builtin_amdgcn_readfirstlane(s0 + s1 + s2 + s3);
        if (N == 0) return false;           // nobody asks (and there is no N - 1 to divide)
        S = max((int)quotient(N - 1, p.by_shares) + 1, SMALLEST_SHARE);
        w = blockIdx.x;
        if ((int64_t)w * S >= N) return false;
        at = w * S;
        end = min(N - at, S) + at;
        int first = sum - own + (wave > 0 ? s0 : 0) + (wave > 1 ? s1 : 0) + (wave > 2 ? s2 : 0);
        if (at >= first && at < first + own) {
            int i = from;
            if (each > 1) {                 // (with one sequence a thread l and q are its)
                for (;; ++i) {
                    l = p.kv_len[i];
                    q = p.q_len ? p.q_len[i] : 0;
                    const int u = tiles_of(p, l, q, groups) * groups;
                    if (at < first + u) break;
                    first += u;
                }
            }
            smem[4] = i;
            smem[5] = first;
            smem[6] = l;
            smem[7] = q;
        }
        __syncthreads();
        b = __builtin_amdgcn_readfirstlane(smem[4]);
        base = __builtin_amdgcn_readfirstlane(smem[5]);
        len = __builtin_amdgcn_readfirstlane(smem[6]);
        ql = __builtin_amdgcn_readfirstlane(smem[7]);
        __syncthreads();                    // smem is the tiles' place
        return true;
    }
    // the next piece of the share; false: done
    __device__ __forceinline__ bool next(const PagedAttnParams& p, Work<RT, BC>& wk) {
        if (at >= end) return false;
        int groups, units = tiles_of(p, len, ql, groups);
        while (at >= base + units * groups) {        // (on to the next sequence that has rows; there is one, end being at most N)
            base += units * groups;
            ++b;
            len = p.kv_len[b];
            ql = p.q_len ? p.q_len[b] : 0;
            units = tiles_of(p, len, ql, groups);
        }
        const int grp = __builtin_amdgcn_readfirstlane((at - base) / units), first = base + grp * units;
        wk.b = b;
        wk.lengths(p, len, ql);
        const int rgs = (wk.R + RT - 1) / RT;
        wk.kvh = rgs > 1 ? __builtin_amdgcn_readfirstlane(grp / rgs) : grp;
        wk.r0 = (grp - wk.kvh * rgs) * RT;
        wk.see(p);
        wk.t0 = at - first;
        const int stop = min(end, first + units);
        wk.Tn = max(min(stop - first, wk.Tn) - wk.t0, 0);       // (tiles behind the last one that any of these rows sees are left out)
        const bool whole = wk.t0 == 0 && stop == first + units;
        wk.slot = whole ? -1 : 2 * w + (wk.t0 == 0);
        if (wk.t0 == 0 && threadIdx.x == 0) {
            int32_t* m = p.meta + 2 * (((int64_t)b * p.Hkv + wk.kvh) * p.row_groups + wk.r0 / RT);
            m[0] = w;
            m[1] = (first + units - 1) / S - w + 1;
        }
        at = stop;
        return true;
    }
};

// Where a wavefront's next 32 tiles lie, `step` apart: lane 2j + h holds half h (16 keys, a page is no smaller) of its j-th tile.  One load of page numbers
// for 32 tiles, requested 32 tiles ahead (a look-up a tile was a trip to memory in front of every fetch), and all 64 places are computed at once, one a lane (64-bit
// products a tile were some 50 scalar instructions in the chain of each wavefront: 128 rows, 32 sequences of 1024 tokens in 8 bits 29.8 -> 27.1 us).  The first load travels with the sequence's lengths, so it may look
// at entries behind the sequence's end (but inside the table's row): whatever they hold, a page outside the cache is not read and a key behind the end
// not seen.
template <int ES>
struct Pages {
    const int32_t* table;
    int first, step, last, next;
    uint32_t lo, hi;                        // byte offset in the cache
    uint64_t there;                         // one bit a half: whether there is such a page
    __device__ __forceinline__ int look(const PagedAttnParams& p, int j) const {
        const int lane = lane_id();
        return table[min((int)(((int64_t)(first + step * (j + (lane >> 1))) * 32 + 16 * (lane & 1)) >> p.page_shift), last)];
    }
    __device__ __forceinline__ void settle(const PagedAttnParams& p, int j) {
        const int lane = lane_id();
        const bool in = (unsigned)next < (unsigned)p.n_pages;
        const uint32_t row = ((uint32_t)(first + step * (j + (lane >> 1))) * 32 + 16 * (lane & 1)) & ((1u << p.page_shift) - 1);
        const uint64_t at = ((uint64_t)(in ? (uint32_t)next : 0u) * (uint64_t)p.sp + (uint64_t)row * (uint32_t)p.st) * ES;
        lo = (uint32_t)at;
        hi = (uint32_t)(at >> 32);
        there = __ballot(in);
    }
    __device__ __forceinline__ Pages(const PagedAttnParams& p, int b, int first_tile, int step_) {
        table = p.table + b * p.table_stride;
        first = first_tile;
        step = step_;
        last = (max(p.max_kv_len, 1) - 1) >> p.page_shift;
        next = p.max_kv_len > 0 ? look(p, 0) : 0;
    }
    // before tile 0: `n` tiles in all
    __device__ __forceinline__ void begin(const PagedAttnParams& p, int n) {
        settle(p, 0);
        if (n > 32) next = look(p, 32);
    }
    // before tile j > 0 of n
    __device__ __forceinline__ void advance(const PagedAttnParams& p, int j, int n) {
        if ((j & 31) == 0) {
            settle(p, j);
            if (j + 32 < n) next = look(p, j + 32);
        }
    }
    // byte offset of half h of tile j in the cache; false: there is no such page
    __device__ __forceinline__ bool half(int j, int h, int64_t& base) const {
        const int at = 2 * (j & 31) + h;
        base = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane(hi, at) << 32 | (uint32_t)__builtin_amdgcn_readlane(lo, at));
        return there >> at & 1;
    }
};

// Runs `rows(work, pages)` for what this workgroup has to do; the pages are those of every STEP-th tile from the wavefront's (128 rows: its half of the
// workgroup's) first on.
template <int RT, bool BC, bool EVEN, int ES, int STEP, typename F>
__device__ __forceinline__ void run_rows(const PagedAttnParams& p, unsigned char* smem, const F& rows) {
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> (RT == 128 ? 8 : 6));
    Work<RT, BC> wk;
    if constexpr (EVEN) {
        Shares<RT, BC> sh;
        if (!sh.find(p, reinterpret_cast<int*>(smem))) return;
        while (sh.next(p, wk)) {
            Pages<ES> pages(p, wk.b, wk.t0 + w, STEP);
            rows(wk, pages);
            __syncthreads();                // the LDS is the next piece's
        }
    } else {
        if (!wk.place(p)) return;
        Pages<ES> pages(p, wk.b, w, STEP);  // (in flight together with the lengths)
        wk.lengths(p, p.kv_len[wk.b], p.q_len ? p.q_len[wk.b] : 0);
        if (wk.r0 >= wk.R) return;
        wk.see(p);
        rows(wk, pages);
    }
}

template <bool NT>
__device__ __forceinline__ u32x4 load16(const unsigned char* a) {
    return NT ? __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(a)) : *reinterpret_cast<const u32x4*>(a);
}

// 16 bytes of cache into LDS as bf16 (8-bit values, HALF: as fp16), 16 or 32 bytes from base + off on; an off with bit 4 set: the 16-byte halves of the 32
// change places
template <bool F8, bool HALF>
__device__ __forceinline__ void stage16(unsigned char* base, uint32_t off, u32x4 v) {
    if constexpr (F8) {
        *reinterpret_cast<u32x4*>(base + off) = widen_e4m3<HALF>(v[0], v[1]);
        *reinterpret_cast<u32x4*>(base + (off ^ 16)) = widen_e4m3<HALF>(v[2], v[3]);
    } else *reinterpret_cast<u32x4*>(base + off) = v;
}

// Where byte `off` of a row lies in LDS (32 and 128 rows), 8-bit cache: behind the first 128 bytes the 16-byte halves of every 32 change places.  Else the eight lanes
// that store a row at once, 16 of every 32 bytes, would use half of the banks (128 rows, 32 sequences of 1024 tokens: LDS busy 18000 -> 13500 cycles a CU, 27.2 -> 26.8 us).
template <bool F8>
__device__ __forceinline__ constexpr uint32_t turned(uint32_t off) { return F8 ? off ^ (off >> 3 & 16) : off; }

// The maximum that exponentials are relative to follows the running one only when that has grown by 2^8 (p stays in range of its type and of the
// sums): the accumulators are rescaled a few times a row instead of at every tile.  With an 8-bit cache it lies 2^7 below the largest score, which
// leaves small p more of fp16's range: p is at most 2^15 and loses bits of its 11 below 2^-14, that is 2^-21 times the row's largest.
template <bool F8>
struct Running {
    static constexpr float LIFT = F8 ? 7.0f : 0.0f;
    float m, l;
    // mx: largest score of the tile in log2 units.  Returns the factor for what has been summed up; m_use: what to subtract.
    __device__ __forceinline__ float follow(float mx, float& m_use) {
#pragma clang fp contract(off)
        const bool grow = mx - m > 8.0f + LIFT;          // (a difference: exact where mx and m are so large that m + 8 would be rounded)
        const float m_new = grow ? mx - LIFT : m;
        m_use = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = grow ? fast_exp2(m - m_use) : 1.0f;
        m = m_new;
        return alpha;
    }
};

// exp2(S factor - m_use) is one fused operation an entry, with the product unrounded while m_use is rounded: from 2^30 on they may lie so far apart that the
// row's largest p is 0 or infinite.  From 2^20 on the product is rounded as m_use was, and S becomes the exponent itself.
constexpr float FAR = 0x1p20f;
template <int N, typename V>
__device__ __forceinline__ void far_scores(V& S, float& factor, float& m_use) {
#pragma clang fp contract(off)
    if (__any(__builtin_fabsf(m_use) >= FAR)) {
#pragma unroll
        for (int i = 0; i < N; ++i) S[i] = S[i] * factor - m_use;
        factor = 1.0f;
        m_use = 0.f;
    }
}

// scores of keys that the lane's row does not see; entry i of S is key at + STEP * (i / 4) + i % 4, entries from N/2 on lie in the second half
template <int N, int STEP, typename V>
__device__ __forceinline__ void hide(V& S, int at, int limit, bool here0, bool here1) {
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (at + STEP * (i >> 2) + (i & 3) >= limit || !(i < N / 2 ? here0 : here1)) S[i] = -INFINITY;
}

// One 32-key tile in LDS (K rows KP bytes apart, V rows VP) for the 32 rows of a wavefront, in four parts:
// scores S^T = K Q^T
template <int D, bool F8, int KP>
__device__ __forceinline__ f32x16 scores32(const unsigned char* Kl, const bf16x8 (&qf)[D / 16], int lane) {
    const int n = lane & 31, hi = lane >> 5;
    f32x16 S;
#pragma unroll
    for (int i = 0; i < 16; ++i) S[i] = 0.f;
#pragma unroll
    for (int c = 0; c < D / 16; ++c)
        S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(Kl + n * KP + 32 * c + 16 * (F8 && c >= 4 ? 1 - hi : hi)), qf[c], S, 0, 0, 0);
    return S;
}
// Masks and the running maximum; returns what exponentials are relative to.  factor: from scores to log2 units
template <int D, bool F8>
__device__ __forceinline__ float lead32(f32x16& S, int key0, int limit, int limit_min, bool here0, bool here1, float& factor, Running<F8>& run,
                                        f32x16 (&O)[D / 32], int lane) {
    if (key0 + 32 > limit_min || !here0 || !here1) hide<16, 8>(S, key0 + 4 * (lane >> 5), limit, here0, here1);
    float mx = -INFINITY, m_use;
#pragma unroll
    for (int i = 0; i < 16; i += 2) mx = __builtin_fmaxf(__builtin_fmaxf(mx, S[i]), S[i + 1]);
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
    const float alpha = run.follow(__builtin_fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * factor, m_use);
    if (__any(alpha != 1.0f || __builtin_fabsf(m_use) >= FAR)) {
        run.l *= alpha;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int i = 0; i < 16; ++i) O[dt][i] *= alpha;
        far_scores<16>(S, factor, m_use);
    }
    return m_use;
}
// How probabilities go into the second product, whose operands have 16 bits:
//   FP16  8-bit caches: fp16, in which the values are exact; each p within 2^-11, as many products
//   BOTH  up to 32 rows: the upper half of p's bits and the nearest bf16 of what they leave, twice the products; each p within 2^-15.  Neither is negative and the
//         second is not zero where p is not (2^-23 of p more see to it), so an infinite value stays what it is.
//   BF16  above 32 rows: bf16, each p within 2^-8, as in dlm_block_attn
// The result's error against 64 bits, relative to its norm, is 0.0016 - 0.0017 with FP16 and BOTH, which is its own rounding, and 0.0022 - 0.0023 with BF16.  BOTH
// costs 0 - 2 % where memory bounds, but above 32 rows, where the products do, 8 - 31 % (32 sequences of 1000 tokens, 32 rows of 28/4 heads 28.1 -> 33.3 us; 4 prompts of 4096
// tokens, 32/8 heads 1299 -> 1605; 16384 causal ones of 14/2 heads of 64 609 -> 798).
enum { BF16, BOTH, FP16 };
template <int KIND, int N>
struct Weights {
    uint32_t hi[N / 2], lo[KIND == BOTH ? N / 2 : 1];
    __device__ __forceinline__ void set(int i, float p0, float p1) {        // entries 2i, 2i + 1
        if constexpr (KIND == FP16) {
            union { __attribute__((__vector_size__(2 * sizeof(_Float16)))) _Float16 h; uint32_t u; } x;
            x.h[0] = (_Float16)p0;
            x.h[1] = (_Float16)p1;
            hi[i] = x.u;
        } else if constexpr (KIND == BOTH) {
            auto left = [](float p) { return fmaf(p, 1.0f + 0x1p-23f, -__uint_as_float(__float_as_uint(p) & 0xffff0000u)); };
            hi[i] = __builtin_amdgcn_perm(__float_as_uint(p1), __float_as_uint(p0), 0x07060302u);
            lo[i] = pack_bf16x2(left(p0), left(p1));
        } else hi[i] = pack_bf16x2(p0, p1);
    }
    // entries 8k .. 8k + 7
    __device__ __forceinline__ u32x4 upper(int k) const { return u32x4{hi[4 * k], hi[4 * k + 1], hi[4 * k + 2], hi[4 * k + 3]}; }
    __device__ __forceinline__ u32x4 lower(int k) const { return u32x4{lo[4 * k], lo[4 * k + 1], lo[4 * k + 2], lo[4 * k + 3]}; }
};
// probabilities, and their sum
template <bool F8, int KIND>
__device__ __forceinline__ void weights32(const f32x16& S, float factor, float m_use, Running<F8>& run, Weights<KIND, 16>& pf) {
    float rs = 0.f;
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
        const float p0 = fast_exp2(fmaf(S[i], factor, -m_use)), p1 = fast_exp2(fmaf(S[i + 1], factor, -m_use));
        rs += p0 + p1;
        pf.set(i >> 1, p0, p1);
    }
    run.l += rs;
}
// O^T += V^T P^T
template <int D, int VP, int KIND>
__device__ __forceinline__ void values32(const unsigned char* Vl, const Weights<KIND, 16>& pf, f32x16 (&O)[D / 32], int lane) {
    constexpr bool F8 = KIND == FP16;
    const int hi = lane >> 5, s16 = lane & 15, blk = (lane >> 4) & 1;
    const unsigned char* vbase = Vl + (4 * hi + (s16 >> 2)) * VP + (16 * blk + 4 * (s16 & 3)) * 2;
    const unsigned char* vturned = Vl + (4 * hi + (s16 >> 2)) * VP + ((16 * blk + 4 * (s16 & 3)) * 2 ^ 16);
#pragma unroll
    for (int e = 0; e < 2 * (D / 32); ++e) {
        union { s16x4 h[2]; bf16x8 v; f16x8 f; } f;
#pragma unroll
        for (int q = 0; q < 2; ++q)
            f.h[q] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)((F8 && e >= 4 ? vturned : vbase) + (16 * (e & 1) + 8 * q) * VP + 32 * (e >> 1) * 2));
        if constexpr (KIND == FP16) O[e >> 1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f.f, as_f16x8(pf.upper(e & 1)), O[e >> 1], 0, 0, 0);
        else {
            if constexpr (KIND == BOTH) O[e >> 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.v, as_bf16x8(pf.lower(e & 1)), O[e >> 1], 0, 0, 0);
            O[e >> 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.v, as_bf16x8(pf.upper(e & 1)), O[e >> 1], 0, 0, 0);
        }
    }
}

// What becomes of row r0 + rr: sums to be joined, or the output.  o: 8 entries from c8 * 8 on, relative to M.
template <int D, bool F8, int RT, bool BC>
__device__ __forceinline__ void put_row(const PagedAttnParams& p, const Work<RT, BC>& wk, int rr, int c8, const float (&o)[8], float M, float den) {
    if (wk.slot >= 0) {
        const int64_t at = (int64_t)wk.slot * RT + rr;
        *reinterpret_cast<f32x4*>(p.part_o + at * D + 8 * c8) = f32x4{o[0], o[1], o[2], o[3]};
        *reinterpret_cast<f32x4*>(p.part_o + at * D + 8 * c8 + 4) = f32x4{o[4], o[5], o[6], o[7]};
        if (c8 == 0) {
            p.part_ml[at * 2] = M;
            p.part_ml[at * 2 + 1] = den;
        }
        return;
    }
    const int r = wk.r0 + rr, i = query_of(p, r), h = wk.kvh * p.g + r - i * p.g;
    const float inv = (den == 0.f ? 0.f : 1.f / den) * (F8 && p.v_scale ? p.v_scale[wk.kvh] : 1.f);
    u32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = pack_bf16x2(o[2 * e] * inv, o[2 * e + 1] * inv);
    *reinterpret_cast<u32x4*>(p.out + wk.b * p.o_sb + i * p.o_st + (int64_t)h * p.o_sh + 8 * c8) = v;
    if (p.lse && c8 == 0) p.lse[((int64_t)wk.b * p.Hq + h) * p.Lq + i] = den == 0.f ? -INFINITY : (M + log2f(den)) * 0.6931471805599453f;
}

// Joins NW wavefronts' sums of the same RT rows from LDS: row k * RT + r of `mb` has MP floats, the D entries, the maximum, the sum.
template <int D, bool F8, int RT, int NW, int MP, bool BC>
__device__ __forceinline__ void join_rows(const PagedAttnParams& p, const Work<RT, BC>& wk, const float* mb, int tid) {
    constexpr int C8 = D / 8;
    for (int task = tid; task < RT * C8; task += 64 * NW) {
        const int rr = task / C8, c8 = task - rr * C8;
        if (wk.r0 + rr >= wk.R) continue;
        float M = -INFINITY, den = 0.f, wgt[NW], o[8];
#pragma unroll
        for (int k = 0; k < NW; ++k) M = __builtin_fmaxf(M, mb[(k * RT + rr) * MP + D]);
#pragma unroll
        for (int k = 0; k < NW; ++k) {
            const float mk = mb[(k * RT + rr) * MP + D];
            wgt[k] = mk == -INFINITY ? 0.f : fast_exp2(mk - M);
            den += wgt[k] * mb[(k * RT + rr) * MP + D + 1];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = 0.f;
#pragma unroll
        for (int k = 0; k < NW; ++k) {
            const float* src = mb + (k * RT + rr) * MP + 8 * c8;
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] += wgt[k] * src[e];
        }
        put_row<D, F8>(p, wk, rr, c8, o, M, den);
    }
}

// The thread's index, made anew: what the shapes derive from it is not kept in registers from one row group of a workgroup to the next (the compiler
// hoisted a hundred values out of that loop and spilled them).
__device__ __forceinline__ int fresh_thread() {
    int t = threadIdx.x;
    asm volatile("" : "+v"(t));
    return t;
}

// LDS of the three shapes: values (or keys and values) of a tile a wavefront, which the join's sums replace; two tiles a workgroup
constexpr int larger(int a, int b) { return a > b ? a : b; }
constexpr int thin_smem(int d, int waves) { return waves * larger(32 * (2 * d + 64), 16 * (d + 4) * 4); }
constexpr int wide_smem(int d) { return larger(4 * 32 * (4 * d + 80), 4 * 32 * (d + 4) * 4); }
constexpr int tall_smem(int d) { return 4 * 32 * (4 * d + 80); }

// ---- 16 rows ------------------------------------------------------------------------------------------------
// For short sequences, where latency counts: eight wavefronts split the keys, 16 x 16 x 32 products, and K goes from memory straight into operand
// registers (lane: key l % 16, 16 bytes of its row); V through LDS for the transposing read.  (3 sequences of up to 400 tokens, 14/2 heads
// of 64: four wavefronts of the 32-row shape 6.3 us, of this one 5.8.)
template <int D, bool F8, bool BC, int NW>
__device__ __forceinline__ void paged_thin_rows(const PagedAttnParams& p, const Work<16, BC>& wk, Pages<F8 ? 1 : 2>& pages, unsigned char* smem) {
    constexpr int RT = 16;
    constexpr int VP = D * 2 + 64;
    constexpr int ES = F8 ? 1 : 2;
    constexpr int C = D * ES / 16, RPL = 64 / C, NLD = 32 / RPL;      // V: 16-byte pieces a row, rows a load, loads
    constexpr int NK = D * ES / 64;                                   // K: loads a half tile; 4 lanes have 64 bytes of a row each time
    constexpr int MP = D + 4;

    const int tid = fresh_thread(), lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, q4 = lane >> 4;

    // Query row n (B operand).  Which 8 entries of a row the 4 lane groups multiply in step c only has to be the same for K: with an 8-bit cache 16 bytes
    // of K are two steps' entries.
    bf16x8 qf[D / 32];
    const int r = wk.r0 + n;
    const uint16_t* qp = wk.query(p, r < wk.R ? r : wk.r0);
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
        u32x4 v = *reinterpret_cast<const u32x4*>(qp + (F8 ? 64 * (c >> 1) + 16 * q4 + 8 * (c & 1) : 32 * c + 8 * q4));
        if (r >= wk.R) v = u32x4{0, 0, 0, 0};
        qf[c] = as_bf16x8(v);
    }
    const int limit = wk.limit(p, r < wk.R ? r : wk.R - 1), limit_min = wk.limit(p, wk.r0);
    const float scale_log2 = F8 && p.k_scale ? p.scale_log2 * p.k_scale[wk.kvh] : p.scale_log2;

    f32x4 O[D / 16];
    Running<F8> run = {-INFINITY, 0.f};
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) O[dt] = f32x4{0.f, 0.f, 0.f, 0.f};

    unsigned char* Vl = smem + w * 32 * VP;
    const int lrow = lane / C, lc = lane % C;
    const unsigned char* kb = (const unsigned char*)p.k + (int64_t)wk.kvh * p.sh * ES;
    const unsigned char* vb = (const unsigned char*)p.v + (int64_t)wk.kvh * p.sh * ES;
    uint32_t voff[NLD];
#pragma unroll
    for (int q = 0; q < NLD; ++q) voff[q] = (uint32_t)(((q * RPL + lrow) & 15) * (int)p.st * ES + lc * 16);
    const uint32_t koff = (uint32_t)(n * (int)p.st * ES + q4 * 16);

    u32x4 kr[2][NK], vr[NLD];
    bool there[2];
    auto fetch = [&](int j) {
        const unsigned char *ks[2], *vs[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            int64_t base;
            there[h] = pages.half(j, h, base);
            ks[h] = kb + base;
            vs[h] = vb + base;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int c = 0; c < NK; ++c) kr[h][c] = load16<false>(ks[h] + koff + 64 * c);
#pragma unroll
        for (int q = 0; q < NLD; ++q) vr[q] = load16<false>(vs[q * RPL / 16] + voff[q]);
    };
    const int J = (wk.Tn - w + NW - 1) / NW;        // tiles of this wavefront
    if (J > 0) {
        pages.begin(p, J);
        fetch(0);
    }
    for (int j = 0; j < J; ++j) {
        const int key0 = (wk.t0 + w + NW * j) * 32;
        const bool here0 = there[0], here1 = there[1], whole = key0 + 32 <= wk.seen && here0 && here1;
        f32x4 S0 = {0.f, 0.f, 0.f, 0.f}, S1 = S0;
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
            bf16x8 k0, k1;
            if constexpr (F8) {
                k0 = as_bf16x8(widen_e4m3<false>(kr[0][c >> 1][2 * (c & 1)], kr[0][c >> 1][2 * (c & 1) + 1]));
                k1 = as_bf16x8(widen_e4m3<false>(kr[1][c >> 1][2 * (c & 1)], kr[1][c >> 1][2 * (c & 1) + 1]));
            } else {
                k0 = as_bf16x8(kr[0][c]);
                k1 = as_bf16x8(kr[1][c]);
            }
            S0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, qf[c], S0, 0, 0, 0);
            S1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, qf[c], S1, 0, 0, 0);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // the values before have been read (one wavefront's LDS operations keep their order)
#pragma unroll
        for (int q = 0; q < NLD; ++q) {
            const int row = q * RPL + lrow;
            u32x4 v = vr[q];
            // rows behind the end hold anything, NaN too: as values they have to be zeros (as keys their scores are replaced)
            if (!whole && !(key0 + row < wk.seen && (q * RPL < 16 ? here0 : here1))) v = u32x4{0, 0, 0, 0};
            stage16<F8, true>(Vl + row * VP, lc * 16 * (2 / ES), v);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (j + 1 < J) {
            pages.advance(p, j + 1, J);
            fetch(j + 1);
        }
        // entry i of S0 / S1 is key key0 + 4 q4 + i (+ 16)
        float S[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            S[i] = S0[i];
            S[4 + i] = S1[i];
        }
        if (key0 + 32 > limit_min || !here0 || !here1) hide<8, 16>(S, key0 + 4 * q4, limit, here0, here1);
        float mx = -INFINITY, m_use, rs = 0.f;
#pragma unroll
        for (int i = 0; i < 8; i += 2) mx = __builtin_fmaxf(__builtin_fmaxf(mx, S[i]), S[i + 1]);
        auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
        mx = __builtin_fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
        sw = __builtin_amdgcn_permlane16_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
        const float alpha = run.follow(__builtin_fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * scale_log2, m_use);
        float factor = scale_log2;
        if (__any(alpha != 1.0f || __builtin_fabsf(m_use) >= FAR)) {
            run.l *= alpha;
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt)
#pragma unroll
                for (int i = 0; i < 4; ++i) O[dt][i] *= alpha;
            far_scores<8>(S, factor, m_use);
        }
        Weights<F8 ? FP16 : BOTH, 8> pf;
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const float p0 = fast_exp2(fmaf(S[i], factor, -m_use)), p1 = fast_exp2(fmaf(S[i + 1], factor, -m_use));
            rs += p0 + p1;
            pf.set(i >> 1, p0, p1);
        }
        run.l += rs;
        const unsigned char* vbase = Vl + (4 * q4 + (n >> 2)) * VP + 8 * (n & 3);
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) {
            union { s16x4 h[2]; bf16x8 v; f16x8 f; } f;
#pragma unroll
            for (int q = 0; q < 2; ++q) f.h[q] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vbase + 16 * q * VP + 32 * dt));
            if constexpr (F8) O[dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f.f, as_f16x8(pf.upper(0)), O[dt], 0, 0, 0);
            else {
                O[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.v, as_bf16x8(pf.lower(0)), O[dt], 0, 0, 0);
                O[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.v, as_bf16x8(pf.upper(0)), O[dt], 0, 0, 0);
            }
        }
    }
    float* mb = reinterpret_cast<float*>(smem);
    __syncthreads();
    run.l += shfl_xor(run.l, 16);
    run.l += shfl_xor(run.l, 32);
    float* row = mb + (w * RT + n) * MP;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) *reinterpret_cast<f32x4*>(row + 16 * dt + 4 * q4) = O[dt];
    if (q4 == 0) {
        row[D] = run.m;
        row[D + 1] = run.l;
    }
    __syncthreads();
    join_rows<D, F8, RT, NW, MP>(p, wk, mb, tid);
}

template <int D, bool F8, bool BC, int NW>
__global__ __launch_bounds__(64 * NW, 1) void paged_thin_kernel(PagedAttnParams p) {
    __shared__ __attribute__((aligned(16))) unsigned char smem[thin_smem(D, NW)];
    fetch_args<sizeof(PagedAttnParams)>();
    run_rows<16, BC, false, F8 ? 1 : 2, NW>(p, smem, [&](const Work<16, BC>& wk, Pages<F8 ? 1 : 2>& pages) { paged_thin_rows<D, F8, BC, NW>(p, wk, pages, smem); });
}

// ---- 32 rows ------------------------------------------------------------------------------------------------
// Four wavefronts take every fourth tile, each with a place of its own in LDS (no barriers before the join) and the next tile in flight in registers; two workgroups
// a CU.  Bound by HBM: 64 sequences of 4096 tokens, 32/8 heads of 128: 169 us, 6.3 TB/s (8-bit cache 90, 6.0); one of 65536 with shares 45 + 4.6 for the joins.
// ONE: one row group a sequence and KV head, whose keys nobody else reads
template <int D, bool F8, bool BC, bool ONE>
__device__ __forceinline__ void paged_wide_rows(const PagedAttnParams& p, const Work<32, BC>& wk, Pages<F8 ? 1 : 2>& pages, unsigned char* smem) {
    constexpr int NW = 4, RT = 32;
    constexpr int KP = D * 2 + 16;          // pitch of a K row in LDS: 16-byte reads of 16 rows hit distinct banks
    constexpr int VP = D * 2 + 64;          // of a V row: the 4 rows x 64 bytes of a transposing read tile the banks
    constexpr int TILE = 32 * KP + 32 * VP;
    constexpr int ES = F8 ? 1 : 2;          // bytes an entry of the cache
    constexpr int C = D * ES / 16, RPL = 64 / C, NLD = 32 / RPL;      // 16-byte pieces a row, rows a load, loads
    constexpr int MP = D + 4;               // pitch of a row of sums (floats)

    const int tid = fresh_thread(), lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, hi = lane >> 5;

    bf16x8 qf[D / 16];                      // this lane's query row (B operand: row n, 8 consecutive entries)
    const int r = wk.r0 + n;
    const uint16_t* qp = wk.query(p, r < wk.R ? r : wk.r0);
#pragma unroll
    for (int c = 0; c < D / 16; ++c) {
        u32x4 v = *reinterpret_cast<const u32x4*>(qp + 16 * c + 8 * hi);
        if (r >= wk.R) v = u32x4{0, 0, 0, 0};
        qf[c] = as_bf16x8(v);
    }
    const int limit = wk.limit(p, r < wk.R ? r : wk.R - 1), limit_min = wk.limit(p, wk.r0);
    const float scale_log2 = F8 && p.k_scale ? p.scale_log2 * p.k_scale[wk.kvh] : p.scale_log2;

    f32x16 O[D / 32];
    Running<F8> run = {-INFINITY, 0.f};
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) O[dt][i] = 0.f;

    unsigned char* Kl = smem + w * TILE;
    unsigned char* Vl = Kl + 32 * KP;
    const int lrow = lane / C, lc = lane % C;
    const unsigned char* kb = (const unsigned char*)p.k + (int64_t)wk.kvh * p.sh * ES;
    const unsigned char* vb = (const unsigned char*)p.v + (int64_t)wk.kvh * p.sh * ES;
    uint32_t off[NLD];                      // of this lane's piece of load q, from the first row of its half tile
#pragma unroll
    for (int q = 0; q < NLD; ++q) off[q] = (uint32_t)(((q * RPL + lrow) & 15) * (int)p.st * ES + lc * 16);

    u32x4 kr[NLD], vr[NLD];
    bool there[2];                          // whether the pages of the two halves exist
    auto fetch = [&](int j) {               // requests the wavefront's j-th tile
        const unsigned char *ks[2], *vs[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            int64_t base;
            there[h] = pages.half(j, h, base);
            ks[h] = kb + base;
            vs[h] = vb + base;
        }
#pragma unroll
        for (int q = 0; q < NLD; ++q) {
            kr[q] = load16<ONE>(ks[q * RPL / 16] + off[q]);
            vr[q] = load16<ONE>(vs[q * RPL / 16] + off[q]);
        }
    };
    const int J = (wk.Tn - w + NW - 1) / NW;        // tiles of this wavefront
    if (J > 0) {
        pages.begin(p, J);
        fetch(0);
    }
    for (int j = 0; j < J; ++j) {
        const int key0 = (wk.t0 + w + NW * j) * 32;
        const bool here0 = there[0], here1 = there[1], whole = key0 + 32 <= wk.seen && here0 && here1;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // the tile before has been read (one wavefront's LDS operations keep their order)
#pragma unroll
        for (int q = 0; q < NLD; ++q) {
            const int row = q * RPL + lrow;
            u32x4 v = vr[q];
            // rows behind the end hold anything, NaN too: as values they have to be zeros (as keys their scores are replaced)
            if (!whole && !(key0 + row < wk.seen && (q * RPL < 16 ? here0 : here1))) v = u32x4{0, 0, 0, 0};
            stage16<F8, false>(Kl + row * KP, turned<F8>(lc * 16 * (2 / ES)), kr[q]);
            stage16<F8, true>(Vl + row * VP, turned<F8>(lc * 16 * (2 / ES)), v);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (j + 1 < J) {
            pages.advance(p, j + 1, J);
            fetch(j + 1);
        }
        f32x16 S = scores32<D, F8, KP>(Kl, qf, lane);
        float factor = scale_log2;
        const float m_use = lead32<D, F8>(S, key0, limit, limit_min, here0, here1, factor, run, O, lane);
        Weights<F8 ? FP16 : ONE ? BOTH : BF16, 16> pf;
        weights32(S, factor, m_use, run, pf);
        values32<D, VP>(Vl, pf, O, lane);
    }
    float* mb = reinterpret_cast<float*>(smem);
    __syncthreads();
    run.l += shfl_xor(run.l, 32);
    float* row = mb + (w * RT + n) * MP;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            *reinterpret_cast<f32x4*>(row + 32 * dt + 8 * q + 4 * hi) = f32x4{O[dt][4 * q], O[dt][4 * q + 1], O[dt][4 * q + 2], O[dt][4 * q + 3]};
    if (hi == 0) {
        row[D] = run.m;
        row[D + 1] = run.l;
    }
    __syncthreads();
    join_rows<D, F8, RT, NW, MP>(p, wk, mb, tid);
}

template <int D, bool F8, bool BC, bool ONE, bool EVEN>
__global__ __launch_bounds__(256, 2) void paged_wide_kernel(PagedAttnParams p) {
    __shared__ __attribute__((aligned(16))) unsigned char smem[wide_smem(D)];
    fetch_args<sizeof(PagedAttnParams)>();
    run_rows<32, BC, EVEN, F8 ? 1 : 2, 4>(p, smem, [&](const Work<32, BC>& wk, Pages<F8 ? 1 : 2>& pages) { paged_wide_rows<D, F8, BC, ONE>(p, wk, pages, smem); });
}

template <int N>
struct Const {
    static constexpr int value = N;
};

// ---- 128 rows -----------------------------------------------------------------------------------------------
// Two key groups of four wavefronts take every second tile; wavefront w of a group has rows 32 w .. 32 w + 31.  A group's t-th tile sits in its LDS
// buffer t % 2.  Step t: the scores of tile t + 1 are formed among the exponentials of tile t, then O takes its values; meanwhile K of tile t + 2 and V of
// tile t + 1 go into the places of K of tile t and V of tile t - 1, and K of tile t + 4 and V of tile t + 3 are requested.  One barrier a step.
// One workgroup a CU at d = 128 (235 registers), two at d = 64 (125; with shares 159 - 167, one).  A step of two tiles takes 1.1 us (d = 128), of which the matrix units work 0.43, the vector units
// 0.5 and LDS 0.4: what they overlap is the two wavefronts of a SIMD and the woven products.  4 prompts of 4096 tokens, 32/8 heads, 8-bit cache: 1228 us, 0.9 PFLOP/s.
template <int D, bool F8, bool BC>
__device__ __forceinline__ void paged_tall_rows(const PagedAttnParams& p, const Work<128, BC>& wk, Pages<F8 ? 1 : 2>& pages, unsigned char* smem) {
    constexpr int RT = 128, PF = 2, MP = D + 4;
    constexpr int KP = D * 2 + 16, VP = D * 2 + 64, TILE = 32 * KP + 32 * VP;
    constexpr int ES = F8 ? 1 : 2;
    constexpr int C = D * ES / 16, RPL = 256 / C, NLD = RPL > 32 ? 1 : 32 / RPL;      // rows that one load of the workgroup covers (64 at d = 64, e4m3: every row twice)
    constexpr int OPB = D * 2 + 16;
    static_assert(4 * 32 * OPB <= 4 * TILE && RT * MP * 4 <= 4 * TILE, "sums and results pass through the tiles' place");

    const int thread = fresh_thread(), tid = thread & 255, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, hi = lane >> 5;
    const int wg = __builtin_amdgcn_readfirstlane(thread >> 8);              // key group
    smem += wg * 2 * TILE;

    const int w0 = wk.r0 + 32 * w;          // this wavefront's first row; without one it only helps with the tiles
    const bool mine = w0 < wk.R;
    bf16x8 qf[D / 16];
    const int r = w0 + n;
    const uint16_t* qp = wk.query(p, r < wk.R ? r : wk.r0);
#pragma unroll
    for (int c = 0; c < D / 16; ++c) {
        u32x4 v = *reinterpret_cast<const u32x4*>(qp + 16 * c + 8 * hi);
        if (r >= wk.R) v = u32x4{0, 0, 0, 0};
        qf[c] = as_bf16x8(v);
    }
    const int limit = wk.limit(p, r < wk.R ? r : wk.R - 1), limit_min = wk.limit(p, mine ? w0 : wk.r0);
    const float scale_log2 = F8 && p.k_scale ? p.scale_log2 * p.k_scale[wk.kvh] : p.scale_log2;

    f32x16 O[D / 32];
    Running<F8> run = {-INFINITY, 0.f};
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) O[dt][i] = 0.f;

    const int lrow = tid / C & 31, lc = tid % C;
    const unsigned char* kb = (const unsigned char*)p.k + (int64_t)wk.kvh * p.sh * ES;
    const unsigned char* vb = (const unsigned char*)p.v + (int64_t)wk.kvh * p.sh * ES;
    const uint32_t off = (uint32_t)((lrow & 15) * (int)p.st * ES + lc * 16);      // (a load covers 16 rows or 32)
    u32x4 kr[PF][NLD], vr[PF][NLD];
    int64_t base[2] = {0, 0};               // of the two halves of the newest tile that was looked up
    uint32_t here = 0;                      // whether its pages exist, two bits; those of the tiles before it in the bits above
    auto look = [&](int t) {
        uint32_t both = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) both |= (uint32_t)pages.half(t, h, base[h]) << h;
        here = here << 2 | both;
    };
    auto fetch = [&](u32x4 (&to)[NLD], const unsigned char* from) {
#pragma unroll
        for (int q = 0; q < NLD; ++q) to[q] = load16<false>(from + (NLD == 1 ? (lrow < 16 ? base[0] : base[1]) : base[q]) + off);
    };
    auto store_k = [&](int slot, int buffer) {
#pragma unroll
        for (int q = 0; q < NLD; ++q) stage16<F8, false>(smem + buffer * TILE + (q * RPL + lrow) * KP, turned<F8>(lc * 16 * (2 / ES)), kr[slot][q]);
    };
    auto store_v = [&](int slot, int buffer, int t, uint32_t both) {
        const int key0 = (wk.t0 + 2 * t + wg) * 32;
        const bool whole = key0 + 32 <= wk.seen && both == 3;
#pragma unroll
        for (int q = 0; q < NLD; ++q) {
            const int row = q * RPL + lrow;
            u32x4 v = vr[slot][q];
            if (!whole && !(key0 + row < wk.seen && (both >> (row < 16 ? 0 : 1) & 1))) v = u32x4{0, 0, 0, 0};
            stage16<F8, true>(smem + buffer * TILE + 32 * KP + row * VP, turned<F8>(lc * 16 * (2 / ES)), v);
        }
    };
    const int Tn = (wk.Tn - wg + 1) / 2, steps = (wk.Tn + 1) / 2;     // tiles of this key group, and of the other one if it has more
    f32x16 S;
    if (steps > 0) {
        // What is requested and stored behind the last tile is the last tile again and nobody's: without conditions around them the compiler knows how many
        // loads are in flight and waits for the oldest only.  (A second group without any tile has its first one, behind the end.)
        const int ends = max(Tn, 1) - 1;
        pages.begin(p, Tn);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            if (t == 2) {
                store_k(0, 0);
                store_v(0, 0, 0, here >> 2 & 3);
                store_k(1, 1);
            }
            look(min(t, ends));
            fetch(kr[t & 1], kb);
            asm volatile("" ::: "memory");          // (in this order, as in the steps)
            if (t < 3) fetch(vr[t & 1], vb);
            asm volatile("" ::: "memory");
        }
        __syncthreads();
        S = scores32<D, F8, KP>(smem, qf, lane);
        __syncthreads();
        auto step = [&](int t, auto parity) {
            constexpr int u = decltype(parity)::value;         // t % 2
            store_k(u, u);
            store_v(1 - u, 1 - u, t + 1, here >> 4 & 3);
            fetch(vr[1 - u], vb);
            if (t + 4 < Tn) pages.advance(p, t + 4, Tn);
            look(min(t + 4, ends));
            fetch(kr[u], kb);
            if (mine && t < Tn) {
                float factor = scale_log2;
                const float m_use = lead32<D, F8>(S, (wk.t0 + 2 * t + wg) * 32, limit, limit_min, here >> 8 & 1, here >> 9 & 1, factor, run, O, lane);
                Weights<F8 ? FP16 : BF16, 16> pf;
                if constexpr (D == 128) {
                    const f32x16 next = scores32<D, F8, KP>(smem + (1 - u) * TILE, qf, lane);
                    weights32(S, factor, m_use, run, pf);
                    values32<D, VP>(smem + u * TILE + 32 * KP, pf, O, lane);
                    S = next;
                } else {                        // (four wavefronts a SIMD, of 128 registers each, overlap by themselves; with shares there are two, for which this order has not been chosen)
                    weights32(S, factor, m_use, run, pf);
                    __builtin_amdgcn_sched_barrier(0);
                    values32<D, VP>(smem + u * TILE + 32 * KP, pf, O, lane);
                    S = scores32<D, F8, KP>(smem + (1 - u) * TILE, qf, lane);
                }
            }
            __syncthreads();
        };
        for (int t = 0; t < steps; t += 2) {    // (an odd number of steps: one more with nothing to multiply; an exit between the two would hide what is in flight)
            step(t, Const<0>());
            step(t + 1, Const<1>());
        }
    }
    // the second key group hands its sums to the first, lane for lane
    smem -= wg * 2 * TILE;
    float* row = reinterpret_cast<float*>(smem) + (32 * w + n) * MP;
    if (wg == 1) {
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<f32x4*>(row + 32 * dt + 8 * q + 4 * hi) = f32x4{O[dt][4 * q], O[dt][4 * q + 1], O[dt][4 * q + 2], O[dt][4 * q + 3]};
        if (hi == 0) row[D] = run.m;
        row[D + 1 + hi] = run.l;
    }
    __syncthreads();
    if (wg == 0) {
        const float m1 = row[D], l1 = row[D + 1 + hi], M = __builtin_fmaxf(run.m, m1);
        const float a0 = run.m == -INFINITY ? 0.f : fast_exp2(run.m - M), a1 = m1 == -INFINITY ? 0.f : fast_exp2(m1 - M);
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x4 v = *reinterpret_cast<const f32x4*>(row + 32 * dt + 8 * q + 4 * hi);
#pragma unroll
                for (int e = 0; e < 4; ++e) O[dt][4 * q + e] = a0 * O[dt][4 * q + e] + a1 * v[e];
            }
        run.l = a0 * run.l + a1 * l1;
        run.m = M;
    }
    __syncthreads();                        // (the results pass through the same place)
    if (wg == 1 || !mine) return;
    run.l += shfl_xor(run.l, 32);
    if (wk.slot >= 0) {
        if (r < wk.R) {
            const int64_t at = (int64_t)wk.slot * RT + 32 * w + n;
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *reinterpret_cast<f32x4*>(p.part_o + at * D + 32 * dt + 8 * q + 4 * hi) = f32x4{O[dt][4 * q], O[dt][4 * q + 1], O[dt][4 * q + 2], O[dt][4 * q + 3]};
            if (hi == 0) {
                p.part_ml[at * 2] = run.m;
                p.part_ml[at * 2 + 1] = run.l;
            }
        }
        return;
    }
    // the accumulators have a row a lane: through LDS (a part of its own a wavefront; the tiles are done with) whole rows are written
    const float inv = (run.l == 0.f ? 0.f : 1.f / run.l) * (F8 && p.v_scale ? p.v_scale[wk.kvh] : 1.f);
    unsigned char* ob = smem + w * (32 * OPB);
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            *reinterpret_cast<u32x2*>(ob + n * OPB + (32 * dt + 8 * q + 4 * hi) * 2) =
                u32x2{pack_bf16x2(O[dt][4 * q] * inv, O[dt][4 * q + 1] * inv), pack_bf16x2(O[dt][4 * q + 2] * inv, O[dt][4 * q + 3] * inv)};
    if (p.lse && hi == 0 && r < wk.R) {
        const int i = query_of(p, r), h = wk.kvh * p.g + r - i * p.g;
        p.lse[((int64_t)wk.b * p.Hq + h) * p.Lq + i] = run.l == 0.f ? -INFINITY : (run.m + log2f(run.l)) * 0.6931471805599453f;
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    constexpr int C8 = D / 8;
#pragma unroll
    for (int q = 0; q < 32 * C8 / 64; ++q) {
        const int id = q * 64 + lane, row = id / C8, c8 = id - row * C8;
        if (w0 + row >= wk.R) continue;
        const int i = query_of(p, w0 + row), h = wk.kvh * p.g + (w0 + row) - i * p.g;
        *reinterpret_cast<u32x4*>(p.out + wk.b * p.o_sb + i * p.o_st + (int64_t)h * p.o_sh + 8 * c8) = *reinterpret_cast<const u32x4*>(ob + row * OPB + c8 * 16);
    }
}

template <int D, bool F8, bool BC, bool EVEN>
__global__ __launch_bounds__(512, D == 64 && !EVEN ? 4 : 2) void paged_tall_kernel(PagedAttnParams p) {
    __shared__ __attribute__((aligned(16))) unsigned char smem[tall_smem(D)];
    fetch_args<sizeof(PagedAttnParams)>();
    run_rows<128, BC, EVEN, F8 ? 1 : 2, 2>(p, smem, [&](const Work<128, BC>& wk, Pages<F8 ? 1 : 2>& pages) { paged_tall_rows<D, F8, BC>(p, wk, pages, smem); });
}

// Joins the sums of each (sequence, head, row) whose keys were shared out: M = max m_s, w_s = 2^(m_s - M), out = sum w_s o_s / sum w_s l_s,
// lse = (M + log2 sum w_s l_s) ln 2.  D / 4 threads a row and group of shares, G groups: group k takes shares k, k + G, .. in their order, four
// requested at a time (eight with several groups), and the groups are added up in theirs.
template <int D, bool F8, int G>
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedAttnParams p) {
    constexpr int TPR = D / 4, RPW = 256 / TPR / G, U = G > 1 ? 8 : 4;
    __shared__ float part[G > 1 ? 256 / TPR : 1][D + 2];
    const int64_t rows = (int64_t)p.B * p.Hq * p.Lq, row = min((int64_t)blockIdx.x * RPW + threadIdx.x / (TPR * G), rows - 1);
    const int c4 = threadIdx.x % TPR, gi = threadIdx.x / TPR, k = gi % G;
    const int i = (int)(row % p.Lq), bh = (int)(row / p.Lq), h = bh % p.Hq, b = bh / p.Hq;
    const int ql = p.q_len ? clamped(p.q_len[b], p.Lq) : p.Lq;
    const int r = i * p.g + h % p.g, rr = r % p.rows_wg;
    const int32_t* m = p.meta + 2 * (((int64_t)b * p.Hkv + h / p.g) * p.row_groups + r / p.rows_wg);
    const int w0 = m[0], n = i < ql && m[1] > 1 ? m[1] : 0;                // 0: nothing to join here (rows behind q_len: nobody has written m)
    float M = -INFINITY, den = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = k; s0 < n; s0 += U * G) {
        f32x2 ml[U];
        f32x4 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int s = min(s0 + u * G, n - 1);                          // (past the last one it is loaded again and not used)
            const int64_t at = (int64_t)(2 * (w0 + s) + (s == 0)) * p.rows_wg + rr;
            ml[u] = *reinterpret_cast<const f32x2*>(p.part_ml + at * 2);
            v[u] = *reinterpret_cast<const f32x4*>(p.part_o + at * D + 4 * c4);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (s0 + u * G >= n) continue;
            const float m_new = __builtin_fmaxf(M, ml[u][0]), m_use = m_new == -INFINITY ? 0.f : m_new;
            const float a = fast_exp2(M - m_use), w = fast_exp2(ml[u][0] - m_use);
            M = m_new;
            den = den * a + ml[u][1] * w;
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
static int g_paged_shape = 0;      // "paged_shape"
static int g_paged_shares = 0;     // "paged_shares"

// How a call is laid out.
struct PagedPlan {
    int rows, row_groups;   // rows of a workgroup, row groups of Lq rows
    int thin_waves;         // with 16 rows: wavefronts
    int shares;             // workgroups that share the tiles evenly; 0: one workgroup a row group
    size_t sums, meta;      // of the workspace: floats of sums and (maximum, sum) pairs, ints behind them
    size_t bytes() const { return shares ? sums * sizeof(float) + meta * sizeof(int32_t) : 0; }
};
// T = the longest sequence's tiles; the lengths themselves are not known here, and every sequence is taken to be as long as max_kv_len.  Where they are not that shows: one
// token of 64 sequences, 32/8 heads of 128, one of 8192 tokens and 63 of 100 under a bound of 8192: 85 us alone, which is chosen, 28 with shares; 64 of 100 under a bound of
// 32768: 17 with shares, which are chosen, 9.5 alone.
// Up to 16 rows: two wavefronts for sequences of a few tiles (T <= 4; 64 sequences of up to 120 tokens, 32/32 heads: 23 us, four wavefronts and 32 rows
// 27), eight for few row groups whose keys a CU streams quickly (16 sequences of 1100 tokens, 32/8 heads: 15.3 / 16.3, in 8 bits 10 / 16), else
// 32 rows.  Above 32 rows 32 or 128, one workgroup a row group or even shares, whichever is estimated to take least.  One workgroup a row group costs least
// where the row groups fill the chip (and of one sequence and KV head they run on one XCD, whose L2 they share); it leaves CUs idle where they are few, and one that is
// much longer than the others runs on alone.  Even shares cost a second launch, a scan of the lengths and what is left half done at each border, and their row
// groups do not meet in an L2.  From 256 tiles on always shares, however equal the lengths may be, unless the row groups of one sequence fill the chip by themselves.
// Estimates, in microseconds:
//   up to 32 rows: a CU streams 49 GB/s, the chip 6.6 TB/s; 4.5 for the launch, with shares 11 and at least 17.  64 sequences of 4096 tokens, 32/8 heads: 164 / 168
//                  with shares, of 2048 - 4096 134 / 142, of 100 - 16000 371 / 316; 8 sequences of 500 - 2000, 28/4 heads 22 / 17; one of 65536 579 / 50.
//   above:         a tile of 32 rows takes 0.28 (d = 64: 0.19) in a chain of its own and 0.29 (0.16) of a CU, with shares what its bytes take the chip (8-bit entries
//                  count as 12 bits), one of 128 rows 0.56 (0.44) and 0.78 (0.44), with shares 0.9 (0.53).  Over 998 calls of equal lengths (33 - 896 rows,
//                  1 - 64 sequences of 300 - 12000 tokens) the choice takes 1.2 % longer than the best of the four in the mean, at most 35 %.
//                  32 rows of 28/4 heads, 32 rows / 128 / with shares 32 / 128: 8 sequences of 1000 tokens 17 / 26 / 36 / 27, of 4000 43 / 72 / 84 / 50, of 12000
//                  124 / 198 / 218 / 95; 32 sequences of 1000 43 / 30 / 88 / 40.
//   causal masks:  row groups see half of the new tokens' keys in the middle, which shares do not know (one prompt of 8192 tokens, 28/4 heads, blocks of 32: 640 / with shares 1088).
static PagedPlan plan_paged(const dlm_paged_attn_args* a) {
    static const int shape_rows[5] = {0, 16, 32, 128, 16};
    PagedPlan pl = {};
    const int64_t R = (int64_t)a->Lq * (a->Hq / a->Hkv), T = ((int64_t)a->max_kv_len + 31) / 32, heads = (int64_t)a->B * a->Hkv;
    const int64_t tile = (int64_t)64 * a->d * (a->cache.type == DLM_KV_E4M3 ? 1 : 2);      // bytes
    auto larger = [](double x, double y) { return x > y ? x : y; };
    auto time = [&](int rows, bool shared) {
        const int64_t groups = heads * ((R + rows - 1) / rows);
        const double stream = (double)groups * T * tile / 6.6e6, once = (double)heads * T * tile / 6.4e6;
        const double mean = T - (a->mask_mode == DLM_MASK_BLOCK_CAUSAL ? a->Lq / 64.0 : 0);          // tiles that a row group sees
        const bool d64 = a->d == 64;
        if (rows == 32) {
            if (shared) return larger(R <= 32 ? stream + 11 : stream * (a->cache.type == DLM_KV_E4M3 ? 1.5 : 1) + 13, 17);
            if (R <= 32) return larger((double)T * ((groups + 255) / 256) * tile / 49e3, stream) + 4.5;
            return larger(once, larger(T * (d64 ? 0.19 : 0.28), mean * groups / 256 * (d64 ? 0.16 : 0.29))) + 7;
        }
        if (shared) return (double)T * groups / 256 * (d64 ? 0.53 : 0.9) + 20;
        return larger(once, larger(T * (d64 ? 0.44 : 0.56), groups > 128 ? mean * ((groups + 255) / 256) * (d64 ? 0.44 : 0.78) : 0)) + 9;
    };
    // whether a workgroup a row group is out of the question
    const bool never_alone = T > 256 && (int64_t)a->Hkv * ((R + 127) / 128) < 256;
    auto shares = [&](int rows) { return never_alone || time(rows, true) < time(rows, false); };
    pl.thin_waves = T <= 4 ? 2 : 8;
    if (R <= 16 && (T <= 4 || (heads <= 128 && T * tile <= 560 << 10))) pl.rows = 16;
    else pl.rows = R <= 32 || time(32, shares(32)) <= time(128, shares(128)) ? 32 : 128;
    if (g_paged_shape > 0) {
        pl.rows = shape_rows[g_paged_shape];
        pl.thin_waves = g_paged_shape == 4 ? 2 : 8;
    }
    pl.row_groups = (int)((R + pl.rows - 1) / pl.rows);
    const int64_t groups = heads * pl.row_groups;
    // (the line of tiles is counted in 32 bits, and the joins are one launch)
    if (pl.rows == 16 || groups > 0x7fffffff / (T + 1) || (int64_t)a->B * a->Lq * a->Hq > 1 << 26) return pl;
    pl.shares = g_paged_shares ? (g_paged_shares > 0 ? g_paged_shares : 0) : !shares(pl.rows) ? 0 : pl.rows == 128 ? 256 : 512;
    if (pl.shares > groups * T / SMALLEST_SHARE) pl.shares = (int)(groups * T / SMALLEST_SHARE);
    pl.sums = (size_t)2 * pl.shares * pl.rows * (a->d + 2);
    pl.meta = (size_t)2 * groups;
    return pl;
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
    if (!aligned16(a->workspace)) return fail(DLM_ERR_WORKSPACE, "%s: workspace not 16-byte aligned", who);
    const int64_t n[3] = {a->B, a->Lq, a->Hq}, qs[3] = {a->q_stride_b, a->q_stride_t, a->q_stride_h}, os[3] = {a->o_stride_b, a->o_stride_t, a->o_stride_h};
    for (int i = 0; i < 3; ++i)
        if (n[i] > 1 && (qs[i] % 8 || os[i] % 8)) return fail(DLM_ERR_UNSUPPORTED, "%s: q/out strides must be multiples of 8", who);
    if (!apart(n, os, a->d)) return fail(DLM_ERR_INVALID_ARG, "%s: rows of out overlap", who);
    return DLM_OK;
}

template <int D, bool F8, bool BC, bool EVEN>
static int launch_rows(const PagedAttnParams& p, unsigned grid, hipStream_t st) {
    if (p.rows_wg == 128) hipLaunchKernelGGL((paged_tall_kernel<D, F8, BC, EVEN>), dim3(grid), dim3(512), 0, st, p);
    else if (p.rows_wg == 16) {
        if constexpr (!EVEN) {
            if (p.thin_waves == 2) hipLaunchKernelGGL((paged_thin_kernel<D, F8, BC, 2>), dim3(grid), dim3(128), 0, st, p);
            else hipLaunchKernelGGL((paged_thin_kernel<D, F8, BC, 8>), dim3(grid), dim3(512), 0, st, p);
        }
    } else if (p.row_groups == 1) hipLaunchKernelGGL((paged_wide_kernel<D, F8, BC, true, EVEN>), dim3(grid), dim3(256), 0, st, p);
    else hipLaunchKernelGGL((paged_wide_kernel<D, F8, BC, false, EVEN>), dim3(grid), dim3(256), 0, st, p);
    return check_hip(hipGetLastError(), "paged attention launch");
}

template <int D, bool F8>
static int launch_paged(const PagedAttnParams& p, bool bc, unsigned grid, hipStream_t st) {
    if (!p.shares) return bc ? launch_rows<D, F8, true, false>(p, grid, st) : launch_rows<D, F8, false, false>(p, grid, st);
    int rc = bc ? launch_rows<D, F8, true, true>(p, p.shares, st) : launch_rows<D, F8, false, true>(p, p.shares, st);
    if (rc != DLM_OK) return rc;
    // few row groups: many shares each
    constexpr int GROUPS = 1024 / D;
    const int64_t rows = (int64_t)p.B * p.Hq * p.Lq;
    if ((int64_t)p.B * p.Hkv * p.row_groups * 4 < p.shares) hipLaunchKernelGGL((paged_merge_kernel<D, F8, GROUPS>), dim3((unsigned)rows), dim3(256), 0, st, p);
    else hipLaunchKernelGGL((paged_merge_kernel<D, F8, 1>), dim3((unsigned)((rows + GROUPS - 1) / GROUPS)), dim3(256), 0, st, p);
    return check_hip(hipGetLastError(), "paged_merge_kernel launch");
}

int paged_set_shape(int v) {
    if (v < 0 || v > 4) return fail(DLM_ERR_INVALID_ARG, "set_option: paged_shape must be 0..4");
    g_paged_shape = v;
    return DLM_OK;
}
int paged_set_shares(int v) {
    if (v < -1 || v > 65536) return fail(DLM_ERR_INVALID_ARG, "set_option: paged_shares must be -1..65536");
    g_paged_shares = v;
    return DLM_OK;
}

}  // namespace dlm

using namespace dlm;

extern "C" size_t dlm_paged_attn_workspace_bytes(const dlm_paged_attn_args* a) {
    if (!a || a->struct_size != sizeof(dlm_paged_attn_args) || a->B <= 0 || a->Lq <= 0 || a->Hq <= 0 || a->Hkv <= 0 || a->Hq % a->Hkv || a->d <= 0 ||
        a->max_kv_len <= 0)
        return 0;
    return plan_paged(a).bytes();
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
    p.by_g = fast_div(p.g);
    p.by_bs = fast_div(a->block_size > 0 ? a->block_size : 1);
    p.scale_log2 = (a->scale > 0.f ? a->scale : 1.0f / sqrtf((float)a->d)) * 1.4426950408889634f;
    const PagedPlan pl = plan_paged(a);
    p.rows_wg = pl.rows;
    p.row_groups = pl.row_groups;
    p.thin_waves = pl.thin_waves;
    if (pl.shares && p.max_kv_len > 0 && a->workspace && a->workspace_bytes >= pl.bytes()) {
        p.shares = pl.shares;
        p.by_shares = fast_div(pl.shares);
        p.part_o = (float*)a->workspace;
        p.part_ml = p.part_o + (size_t)2 * pl.shares * pl.rows * a->d;
        p.meta = (int32_t*)(p.part_o + pl.sums);
    }
    const int64_t grid = set_remap(p.remap, (int64_t)a->B * a->Hkv, pl.row_groups, a->mask_mode == DLM_MASK_BLOCK_CAUSAL);      // (longest first)
    const int64_t threads = pl.rows == 128 ? 512 : pl.rows == 16 ? 64 * pl.thin_waves : 256;
    if (grid == 0 || grid * threads > 0xffffffffll || (int64_t)a->B * a->Hkv > 0x7fffffff || (int64_t)a->B * a->Hq * a->Lq > 0x7fffffff) return fail(DLM_ERR_UNSUPPORTED, "paged_attn: too many workgroups");
    hipStream_t st = (hipStream_t)stream;
    const bool f8 = c.type == DLM_KV_E4M3, bc = a->mask_mode == DLM_MASK_BLOCK_CAUSAL;
    if (a->d == 128) return f8 ? launch_paged<128, true>(p, bc, (unsigned)grid, st) : launch_paged<128, false>(p, bc, (unsigned)grid, st);
    return f8 ? launch_paged<64, true>(p, bc, (unsigned)grid, st) : launch_paged<64, false>(p, bc, (unsigned)grid, st);
}
