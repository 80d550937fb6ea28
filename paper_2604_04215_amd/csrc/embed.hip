// dlm_embed and its gradient: rows of the embedding table for a batch of tokens, and rows of equal tokens summed.
//
// The lookup is a copy, bound by what it writes.  The gradient is a sum over rows that lie anywhere: tokens are sorted first (with their positions,
// so that the sum of a token's rows has one order and no atomics are needed), then every row is read once.  In a masked batch one token has half of
// the rows, so the sorted list is cut into chunks of equal length whatever tokens they hold; the sums of a token that goes over the end
// of a chunk are joined by a last launch.
//
// Measured: 65536 rows of 4096 into fp32 214 us, 5.5 TB/s of the 1.17 GB that it cannot do without (a copy: 6.2); 256 rows into bf16 3.9, of which the GPU works 2.7.
// Gradient of 65536 rows of 4096, half of them of one token, added to an fp32 table of 126464: 256 us (sort 9, merge 26, sums 187, of 0.93 GB, join 7);
// of 8192 rows of 3584 into a 16-bit table of 152064, which is cleared: 224 (sort beside 1.09 GB of zeros 190, sums 22, join 5); of 333 rows of 256: 14.7, three launches.
#include "rows.hpp"

namespace dlm {

struct EmbedParams {
    int T, V, Dh;
    const int32_t* tokens;
    const uint16_t* table;
    int64_t table_st;
    float scale;
    void* out;
    int64_t out_st;
};

// TPR threads a row, pieces of 16 bytes of what is written: the stores of a wavefront cover whole lines.  (Eight entries
// of fp32 a thread, two stores of 16 bytes that each fill half of every line: 412 us where this takes 214.)
template <bool F32, int TPR>
__global__ __launch_bounds__(256) void embed_kernel(EmbedParams p) {
    constexpr int ROWS = 256 / TPR, E = Piece<F32>::E;
    const int l = threadIdx.x % TPR;
    const int64_t t = (int64_t)blockIdx.x * ROWS + threadIdx.x / TPR;
    if (t >= p.T) return;
    const int token = p.tokens[t];
    const bool known = (uint32_t)token < (uint32_t)p.V;
    const uint16_t* src = p.table + (int64_t)(known ? token : 0) * p.table_st;
#pragma unroll 4
    for (int c = E * l; c < p.Dh; c += E * TPR) {
        float f[E];
        load_bf16<E>(src + c, f);
#pragma unroll
        for (int e = 0; e < E; ++e) f[e] = known ? f[e] * p.scale : 0.f;
        Piece<F32>::stream_out(p.out, t * p.out_st + c, Piece<F32>::close(f));
    }
}

// ---- gradient: sorting --------------------------------------------------------------------------------------
// Runs of 2^BITS tokens are sorted by themselves, a workgroup each, then up to MERGE runs at a time become one: an entry's place in the merged
// run is its place in its own plus, for every other run, the number of entries there that go before it (a binary search each; equal
// tokens stay in the order of their positions, since earlier runs hold earlier ones).
constexpr int MERGE = 32;
constexpr int EMBED_MAX_V = (1 << 21) - 2;                    // a token (or V: none) and a place in its run share 32 bits: 21 and 11
// 512 entries for a few tokens, which one wavefront sorts without a barrier; 8192, of which there are fewer to merge, where a table is cleared meanwhile, if they
// leave the token its bits.  Where none is, us of the whole call (Dh = 512) in runs of 2048 / 8192: 4096 tokens 33 / 39, 16384 38 / 60, 65536 92 / 101,
// 131072 136 / 134, 300000 268 / 294.
inline int run_bits(int T, int V, bool clears) {
    if (T <= 512) return 9;
    return T <= 2048 || V >= (1 << 19) - 1 || !clears ? 11 : 13;
}

// the value of lane ^ MASK, without a trip through LDS
template <int MASK>
__device__ __forceinline__ uint32_t from_lane_xor(uint32_t v) {
    if constexpr (MASK == 1) return __builtin_amdgcn_mov_dpp(v, 0xB1, 0xf, 0xf, true);
    if constexpr (MASK == 2) return __builtin_amdgcn_mov_dpp(v, 0x4E, 0xf, 0xf, true);
    if constexpr (MASK == 4) return __builtin_amdgcn_mov_dpp(__builtin_amdgcn_mov_dpp(v, 0x141, 0xf, 0xf, true), 0x1B, 0xf, 0xf, true);     // 7 -, then 3 -
    if constexpr (MASK == 8) return __builtin_amdgcn_mov_dpp(v, 0x128, 0xf, 0xf, true);                                                    // rotated by 8 of 16
    if constexpr (MASK == 16) {
        const auto w = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        return lane_id() & 16 ? w[0] : w[1];
    }
    if constexpr (MASK == 32) {
        const auto w = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        return lane_id() & 32 ? w[0] : w[1];
    }
}

struct SortParams {
    int T, V;
    const int32_t* tokens;
    int32_t *token, *pos;          // sorted within each run
    int runs;                      // workgroups behind these clear the table
    // what is cleared: `rows` of `pieces` 16-byte pieces each, `pitch` bytes apart, `total` pieces in all (a table without gaps: rows of 4096 pieces)
    void* table;
    int64_t rows, pitch, total;
    int pieces;
};

// one step of the network: entries whose numbers differ in bit BIT put in order, up or down by bit SIZE; then the steps behind it
template <int BITS, int SIZE, int BIT>
__device__ __forceinline__ void embed_network(uint32_t (&k)[8], uint32_t* lds, int tid) {
    constexpr int THREADS = 1 << (BITS - 3);
    if constexpr (BIT < 3) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (e >> BIT & 1) continue;
            const int o = e | 1 << BIT;
            const bool up = SIZE >= 3 ? SIZE == BITS || !(tid >> (SIZE >= 3 ? SIZE - 3 : 0) & 1) : !(e >> SIZE & 1);
            const uint32_t lo = min(k[e], k[o]), hi = max(k[e], k[o]);
            k[e] = up ? lo : hi;
            k[o] = up ? hi : lo;
        }
    } else {
        constexpr int MASK = 1 << (BIT - 3);
        const bool up = SIZE == BITS || !(tid >> (SIZE - 3) & 1), lower = !(tid & MASK);
        uint32_t other[8];
        if constexpr (MASK < WAVE) {
#pragma unroll
            for (int e = 0; e < 8; ++e) other[e] = from_lane_xor<MASK>(k[e]);
        } else {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; ++e) lds[e * THREADS + tid] = k[e];
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; ++e) other[e] = lds[e * THREADS + (tid ^ MASK)];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) k[e] = up == lower ? min(k[e], other[e]) : max(k[e], other[e]);
    }
    if constexpr (BIT > 0) embed_network<BITS, SIZE, BIT - 1>(k, lds, tid);
    else if constexpr (SIZE < BITS) embed_network<BITS, SIZE + 1, SIZE>(k, lds, tid);
}

template <int BITS>
__global__ __launch_bounds__(1 << (BITS - 3)) void embed_sort_kernel(SortParams p) {
    constexpr int RUN = 1 << BITS, THREADS = RUN / 8;
    __shared__ uint32_t lds[THREADS > WAVE ? RUN : 1];
    const int tid = threadIdx.x;
    if ((int)blockIdx.x >= p.runs) {
        for (int64_t row = blockIdx.x - p.runs; row < p.rows; row += gridDim.x - p.runs) {
            const int n = (int)min((int64_t)p.pieces, p.total - row * p.pieces);
            #pragma unroll 4
            for (int i = tid; i < n; i += THREADS) __builtin_nontemporal_store(u32x4{0, 0, 0, 0}, reinterpret_cast<u32x4*>((char*)p.table + row * p.pitch) + i);
        }
        return;
    }
    const int64_t t0 = (int64_t)blockIdx.x * RUN;
    const int n = (int)min((int64_t)RUN, p.T - t0);
    // key: token, then place; behind the end the largest
    uint32_t k[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int i = 8 * tid + e;
        uint32_t token = 0xffffffffu >> BITS;
        if (i < n) {
            const int32_t x = p.tokens[t0 + i];
            token = (uint32_t)x < (uint32_t)p.V ? x : p.V;
        }
        k[e] = token << BITS | i;
    }
    // Bitonic network over element numbers i = 8 tid + e: partners by the bits of i below 3 are in the thread's own registers, below 9 in the
    // wavefront, above in another one.
    embed_network<BITS, 1, 0>(k, lds, tid);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int i = 8 * tid + e;
        if (i < n) {
            p.token[t0 + i] = k[e] >> BITS;
            p.pos[t0 + i] = (int32_t)t0 + (k[e] & (RUN - 1));
        }
    }
}

// Runs of `len` entries (a power of two, 256 or more), MERGE of them into one.  A workgroup has 256 neighbouring entries of one run, so few tokens of the others lie
// between its first and its last: it looks for these two in every run, takes what stands between them into LDS and searches there.  65536 tokens in 32 runs:
// 26 us, ten of them for the first searches, four for the copy, the rest in LDS; with searches in memory alone, chains of 11 trips, 54.
__global__ __launch_bounds__(256) void embed_merge_kernel(const int32_t* token, const int32_t* pos, int32_t* token_out, int32_t* pos_out, int T, int64_t len) {
    constexpr int ROOM = 16384, SAMPLES = 64, FEW = 32;
    __shared__ int below[4][MERGE];                // entries of a run: below the first token, up to it, below the last, up to it
    __shared__ int32_t between[ROOM];              // (first a sample of each run)
    __shared__ int start[MERGE + 1];               // of each run's tokens in `between`
    const int tid = threadIdx.x;
    const int64_t b0 = (int64_t)blockIdx.x * 256, i = b0 + tid, run = b0 / len, group = run / MERGE * MERGE;
    const auto count = [&](int j) { return (int)max((int64_t)0, min(len, T - (group + j) * len)); };
    // the four searches of every run: among 64 entries of each, then, 32 lanes a search, among 32 at a time of what is left, a trip to memory each
    int64_t seg = len / SAMPLES;
#pragma unroll
    for (int k = 0; k < MERGE * SAMPLES / 256; ++k) {
        const int j = (k * 256 + tid) / SAMPLES;
        const int64_t at = ((k * 256 + tid) % SAMPLES + 1) * seg - 1;
        between[k * 256 + tid] = at < count(j) ? token[(group + j) * len + at] : 0x7fffffff;
    }
    const int first = token[b0], last = token[min(b0 + 255, (int64_t)T - 1)];
    __syncthreads();
    if (tid < 4 * MERGE) {
        const int which = tid / MERGE, j = tid % MERGE, x = (which < 2 ? first : last) + (which & 1);
        int lo = 0;
#pragma unroll
        for (int step = SAMPLES; step > 0; step >>= 1)
            if (lo + step <= SAMPLES && between[j * SAMPLES + lo + step - 1] < x) lo += step;
        below[which][j] = (int)min(lo * seg, (int64_t)count(j));
    }
    while (seg > 1) {
        const int step = (int)max(seg / FEW, (int64_t)1), l = tid % FEW;
        int32_t seen[4 * MERGE * FEW / 256];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 4 * MERGE * FEW / 256; ++k) {
            const int search = (k * 256 + tid) / FEW, j = search % MERGE;
            const int64_t at = below[search / MERGE][j] + (int64_t)(l + 1) * step - 1;
            seen[k] = (l + 1) * (int64_t)step <= seg && at < count(j) ? token[(group + j) * len + at] : 0x7fffffff;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 4 * MERGE * FEW / 256; ++k) {
            const int search = (k * 256 + tid) / FEW, which = search / MERGE;
            const uint64_t under = __ballot(seen[k] < (which < 2 ? first : last) + (which & 1));
            if (l == 0) below[which][search % MERGE] += __popc((uint32_t)(lane_id() < FEW ? under : under >> 32)) * step;
        }
        seg = step;
    }
    __syncthreads();
    if (tid <= MERGE) {
        int at = 0;
#pragma unroll
        for (int j = 0; j < MERGE; ++j) at += j < tid ? max(0, below[2][j] - below[1][j]) : 0;
        start[tid] = at;
    }
    __syncthreads();
    const bool here = start[MERGE] <= ROOM;        // (else every search is in memory: a token that this run lacks fills others)
    if (here) {
        for (int j = tid / WAVE; j < MERGE; j += 256 / WAVE) {
#pragma unroll 4
            for (int k = lane_id(); k < start[j + 1] - start[j]; k += WAVE) between[start[j] + k] = token[(group + j) * len + below[1][j] + k];
        }
        __syncthreads();
    }
    if (i >= T) return;
    const int x = token[i], at = pos[i];
    int64_t to = group * len + (i - run * len);
    for (int j0 = 0; j0 < MERGE && (group + j0) * len < T; j0 += 8) {
        // entries of each run with a token below x, or, in an earlier run, at most x
        int lo[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) lo[j] = below[1][j0 + j];
        if (x == first || x == last) {
#pragma unroll
            for (int j = 0; j < 8; ++j) lo[j] = below[(x == first ? 0 : 2) + (group + j0 + j < run ? 1 : 0)][j0 + j];
        } else if (here) {
            int n[8], s0[8], most = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                s0[j] = start[j0 + j];
                n[j] = start[j0 + j + 1] - s0[j];
                s0[j] -= lo[j];                    // (lo[j] entries lie before those in LDS)
                n[j] += lo[j];
                most = max(most, n[j] - lo[j]);
            }
            for (int step = most > 0 ? 1 << (31 - __builtin_clz(most)) : 0; step > 0; step >>= 1) {
                int seen[8];                       // (all eight asked for before the first is looked at)
#pragma unroll
                for (int j = 0; j < 8; ++j) seen[j] = between[lo[j] + step <= n[j] ? s0[j] + lo[j] + step - 1 : 0];
#pragma unroll
                for (int j = 0; j < 8; ++j) lo[j] += lo[j] + step <= n[j] && seen[j] < x + (group + j0 + j < run ? 1 : 0) ? step : 0;
            }
        } else {
            for (int step = 1 << 28; step > 0; step >>= 1) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (lo[j] + step <= below[2][j0 + j] && token[(group + j0 + j) * len + lo[j] + step - 1] < x + (group + j0 + j < run ? 1 : 0)) lo[j] += step;
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) to += group + j0 + j == run ? 0 : lo[j];
    }
    token_out[to] = x;
    pos_out[to] = at;
}

// ---- gradient: sums -----------------------------------------------------------------------------------------
constexpr int GROUP = 16;          // chunks of a workgroup, one a wavefront
struct EmbedGradParams {
    int T, V, Dh;
    const int32_t *token, *pos;    // sorted
    const void* dy;
    int64_t dy_st;
    float scale;
    void* table;
    int64_t table_st;
    int accumulate;
    int chunk, slices;             // sorted entries a wavefront takes, slices of columns
    int group0;                    // the launch's first group
    float* part;                   // [groups][2][Dh]: the sum of a token that began in an earlier group; of one that goes on in the next
};

// what a table holds of 4 entries
template <bool F32>
__device__ __forceinline__ f32x4 embed_held(const EmbedGradParams& p, int token, int c) {
    const int64_t at = (int64_t)token * p.table_st + c;
    if constexpr (F32) {
        return *reinterpret_cast<const f32x4*>((const float*)p.table + at);
    } else {
        float old[4];
        load_bf16<4>((const uint16_t*)p.table + at, old);
        return f32x4{old[0], old[1], old[2], old[3]};
    }
}
// the sum of a token's rows into the table, on top of `old`
template <bool F32>
__device__ __forceinline__ void embed_store(const EmbedGradParams& p, int token, int c, const f32x4& a, const f32x4& old) {
    const int64_t at = (int64_t)token * p.table_st + c;
    float f[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = a[e] * p.scale;
    if (p.accumulate) {
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] += old[e];
    }
    if constexpr (F32) *reinterpret_cast<f32x4*>((float*)p.table + at) = f32x4{f[0], f[1], f[2], f[3]};
    else *reinterpret_cast<u32x2*>((uint16_t*)p.table + at) = u32x2{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3])};
}

// A wavefront adds the rows of one chunk, 64 pieces of each; at the end of a token it stores the sum.  The sums of a token that lies in several
// chunks of the workgroup meet in LDS and are added in order by the wavefront that has its first row; those of one that lies in several
// groups go to `part`.
//
// Rows come in batches, one ahead; with ACC what the table holds of each row's token comes with it, whether the token ends there or not (then it
// is a line that is at hand already): asked for where a token ends, every such row would wait for all requests before it.
template <bool F32IN, bool F32, bool ACC>
__global__ __launch_bounds__(GROUP * WAVE) void embed_grad_kernel(EmbedGradParams p) {
    using P = Piece<F32IN>;
    constexpr int E = P::E, Q = E / 4, BATCH = ACC ? 4 : 8;
    __shared__ f32x4 lds[GROUP][2][Q][WAVE];       // [0]: of a token that began in an earlier chunk, [1]: of one that goes on in the next
    __shared__ int ends[GROUP + 1][2];             // every chunk's first and last token; the one behind the group
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = lane_id();
    const int nth = blockIdx.x / p.slices, slice = blockIdx.x - nth * p.slices, group = p.group0 + nth;
    const int c0 = (slice * WAVE + lane) * E, c = c0 < p.Dh ? c0 : 0;          // (lanes behind the row read its beginning, and store nothing)
    const bool live = c0 < p.Dh;
    const int64_t first = (int64_t)group * GROUP * p.chunk, i0 = first + (int64_t)wave * p.chunk;
    const int n = (int)max((int64_t)0, min((int64_t)p.chunk, p.T - i0));
    // the chunk's entries, one a lane
    const int at = n > 0 ? min(lane, n - 1) : 0;
    const int tokens = n > 0 ? p.token[i0 + at] : p.V, places = n > 0 ? p.pos[i0 + at] : 0;
    const auto token_of = [&](int i) { return __builtin_amdgcn_readlane(tokens, i); };
    const int x_first = token_of(0);
    int x_last = p.V;                              // the token of the chunk's end, where it began here and goes on
    if (x_first < p.V) {                           // (else the chunk holds no token: V sorts last)
        const int before = i0 > 0 ? p.token[i0 - 1] : -1, behind = i0 + n < p.T ? p.token[i0 + n] : -1;
        typename P::Raw rows[2][BATCH];
        f32x4 old[2][ACC ? BATCH : 1][Q];
        const auto request = [&](int k0, int b) {
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                const int i = min(k0 + k, n - 1);
                rows[b][k] = P::stream(p.dy, (int64_t)__builtin_amdgcn_readlane(places, i) * p.dy_st + c);
                if constexpr (ACC) {
#pragma unroll
                    for (int q = 0; q < Q; ++q) old[b][k][q] = embed_held<F32>(p, token_of(i) < p.V ? token_of(i) : x_first, c + 4 * q);
                }
            }
        };
        f32x4 a[Q];
#pragma unroll
        for (int q = 0; q < Q; ++q) a[q] = f32x4{0.f, 0.f, 0.f, 0.f};
        bool began = x_first != before;            // the token at hand began in this chunk
        const auto add = [&](int k0, int b) {
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                const int i = k0 + k;
                if (i >= n) break;
                float f[E];
                P::open(rows[b][k], f);
#pragma unroll
                for (int e = 0; e < E; ++e) a[e / 4][e % 4] += f[e];
                const int x = token_of(i), next = i + 1 < n ? token_of(i + 1) : behind;
                if (x == next && i + 1 < n) continue;
                const bool goes_on = x == next;    // into the next chunk
                if (goes_on && began) x_last = x;
#pragma unroll
                for (int q = 0; q < Q; ++q) {
                    if (!began || goes_on) lds[wave][began ? 1 : 0][q][lane] = a[q];
                    else if (x < p.V && live) embed_store<F32>(p, x, c + 4 * q, a[q], old[b][ACC ? k : 0][q]);
                    a[q] = f32x4{0.f, 0.f, 0.f, 0.f};
                }
                began = true;
            }
        };
        request(0, 0);
        for (int k0 = 0; k0 < n; k0 += 2 * BATCH) {
            if (k0 + BATCH < n) request(k0 + BATCH, 1);
            add(k0, 0);
            if (k0 + 2 * BATCH < n) request(k0 + 2 * BATCH, 0);
            add(k0 + BATCH, 1);
        }
    }
    if (lane == 0) {
        ends[wave][0] = x_first;
        ends[wave][1] = n > 0 ? token_of(n - 1) : p.V;
        if (wave == GROUP - 1) ends[GROUP][0] = first + (int64_t)GROUP * p.chunk < p.T ? p.token[first + (int64_t)GROUP * p.chunk] : p.V;
    }
    __syncthreads();
    // from this wavefront's chunk on: the token that began in it, and, the first wavefront, one that began in an earlier group
#pragma unroll 1
    for (int which = wave == 0 ? 0 : 1; which < 2; ++which) {
        const int x = which ? x_last : (group > 0 && x_first < p.V && x_first == p.token[first - 1] ? x_first : p.V);
        if (x >= p.V) continue;
        f32x4 sum[Q];
#pragma unroll
        for (int q = 0; q < Q; ++q) sum[q] = lds[wave][which][q][lane];
        int k = wave;                              // the last chunk added
        while (k + 1 < GROUP && ends[k][1] == x && ends[k + 1][0] == x) {
            ++k;
#pragma unroll
            for (int q = 0; q < Q; ++q) sum[q] += lds[k][0][q][lane];
        }
        const bool goes_on = k + 1 == GROUP && ends[k][1] == x && ends[GROUP][0] == x;
        if (!live) continue;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            if (which && !goes_on) embed_store<F32>(p, x, c + 4 * q, sum[q], ACC ? embed_held<F32>(p, x, c + 4 * q) : f32x4{0.f, 0.f, 0.f, 0.f});
            else *reinterpret_cast<f32x4*>(p.part + ((int64_t)group * 2 + which) * p.Dh + c + 4 * q) = sum[q];
        }
    }
}

// For every group whose last token goes on: its sums of that token, one a group, joined in their order.
template <bool F32>
__global__ __launch_bounds__(WAVE) void embed_join_kernel(EmbedGradParams p) {
    const int group = blockIdx.x;
    const int64_t size = (int64_t)GROUP * p.chunk, i0 = group * size, end = i0 + size;      // (the last group is not among them)
    const int x = p.token[end - 1];
    if (x >= p.V || p.token[end] != x) return;
    if (i0 > 0 && p.token[i0] == x && p.token[i0 - 1] == x) return;      // began earlier
    // the group that holds the token's last entry
    int64_t lo = end + 1, hi = p.T;
    while (lo < hi) {
        const int64_t mid = (lo + hi) >> 1;
        if (p.token[mid] == x) lo = mid + 1;
        else hi = mid;
    }
    const int last = (int)((lo - 1) / size);
    const int c = (blockIdx.y * WAVE + lane_id()) * 4;
    if (c >= p.Dh) return;
    f32x4 a = *reinterpret_cast<const f32x4*>(p.part + ((int64_t)group * 2 + 1) * p.Dh + c);
#pragma unroll 8
    for (int k = group + 1; k <= last; ++k) a += *reinterpret_cast<const f32x4*>(p.part + (int64_t)k * 2 * p.Dh + c);
    embed_store<F32>(p, x, c, a, p.accumulate ? embed_held<F32>(p, x, c) : f32x4{0.f, 0.f, 0.f, 0.f});
}

// ---- host ---------------------------------------------------------------------------------------------------
static int validate_embed(int T, int V, int Dh, const int32_t* tokens, float scale, const char* who) {
    if (T < 0 || V <= 0 || Dh <= 0) return fail(DLM_ERR_INVALID_ARG, "%s: bad sizes T=%d V=%d Dh=%d", who, T, V, Dh);
    if (Dh % 8) return fail(DLM_ERR_UNSUPPORTED, "%s: Dh=%d is not a multiple of 8", who, Dh);
    if (!(scale >= -3.0e38f && scale <= 3.0e38f)) return fail(DLM_ERR_INVALID_ARG, "%s: scale must be finite", who);
    if (T > 0 && !tokens) return fail(DLM_ERR_INVALID_ARG, "%s: null tokens", who);
    return DLM_OK;
}

template <bool F32>
static void launch_embed(const EmbedParams& all, hipStream_t st) {
    constexpr int MOST = 1 << 22;                   // rows a launch: its threads stay below 2^32
    for (int64_t t0 = 0; t0 < all.T; t0 += MOST) {
        EmbedParams p = all;
        p.T = (int)(all.T - t0 < MOST ? all.T - t0 : MOST);
        p.tokens = all.tokens + t0;
        p.out = (char*)all.out + t0 * all.out_st * (F32 ? 4 : 2);
        if (p.Dh <= 64) hipLaunchKernelGGL((embed_kernel<F32, 8>), dim3((p.T + 31) / 32), dim3(256), 0, st, p);
        else if (p.Dh <= 512) hipLaunchKernelGGL((embed_kernel<F32, 64>), dim3((p.T + 3) / 4), dim3(256), 0, st, p);
        else hipLaunchKernelGGL((embed_kernel<F32, 256>), dim3(p.T), dim3(256), 0, st, p);
    }
}

// How the gradient is cut up, and where its workspace holds what
struct EmbedPlan {
    int bits, runs, levels, chunk, groups;
    size_t list_bytes, part_at, bytes;              // one list of T; the sums behind the lists
};
static EmbedPlan plan_embed(int T, int V, int Dh, bool clears) {
    EmbedPlan p = {};
    p.bits = run_bits(T, V, clears);
    p.runs = (int)(((int64_t)T + (1 << p.bits) - 1) >> p.bits);
    for (int64_t n = p.runs; n > 1; n = (n + MERGE - 1) / MERGE) ++p.levels;
    // some 8192 wavefronts, of chunks that are neither so short that their borders cost more than their rows nor so long that a few run on alone
    const int64_t slices = (Dh + 511) / 512;
    int64_t chunk = T * slices / 8192;
    chunk = chunk < 8 ? 8 : chunk > WAVE ? WAVE : chunk;
    p.chunk = (int)chunk;
    p.groups = (int)((T + GROUP * chunk - 1) / (GROUP * chunk));
    p.list_bytes = ((size_t)T * 4 + 15) / 16 * 16;
    p.part_at = p.list_bytes * (T > 2048 ? 4 : 2);        // (a second pair of lists to merge into)
    p.bytes = p.part_at + (size_t)p.groups * 2 * Dh * sizeof(float);
    return p;
}

}  // namespace dlm

using namespace dlm;

extern "C" int dlm_embed(const dlm_embed_args* a, void* stream) {
    static const char who[] = "embed";
    if (!a) return fail(DLM_ERR_INVALID_ARG, "%s: null args", who);
    if (a->struct_size != sizeof(dlm_embed_args)) return fail(DLM_ERR_INVALID_ARG, "%s: struct_size %u != %zu", who, a->struct_size, sizeof(dlm_embed_args));
    int rc;
    if ((rc = validate_embed(a->T, a->V, a->Dh, a->tokens, a->scale, who)) != DLM_OK) return rc;
    if ((rc = validate_row_type(a->out_type, who, "out")) != DLM_OK) return rc;
    if (a->T == 0) return DLM_OK;
    if ((rc = validate_rows(a->table, a->table_stride, a->V, a->Dh, 2, false, who, "table")) != DLM_OK) return rc;
    if ((rc = validate_rows(a->out, a->out_stride, a->T, a->Dh, row_bytes(a->out_type), true, who, "out")) != DLM_OK) return rc;
    const EmbedParams p = {a->T, a->V, a->Dh, a->tokens, (const uint16_t*)a->table, a->table_stride, a->scale, a->out, a->out_stride};
    if (a->out_type == DLM_ROW_F32) launch_embed<true>(p, (hipStream_t)stream);
    else launch_embed<false>(p, (hipStream_t)stream);
    return check_hip(hipGetLastError(), "embed_kernel launch");
}

extern "C" size_t dlm_embed_bwd_workspace_bytes(const dlm_embed_bwd_args* a) {
    if (!a || a->struct_size != sizeof(dlm_embed_bwd_args) || a->T <= 0 || a->Dh <= 0) return 0;
    return plan_embed(a->T, a->V, a->Dh, false).bytes;
}

extern "C" int dlm_embed_bwd(const dlm_embed_bwd_args* a, void* stream) {
    static const char who[] = "embed_bwd";
    if (!a) return fail(DLM_ERR_INVALID_ARG, "%s: null args", who);
    if (a->struct_size != sizeof(dlm_embed_bwd_args))
        return fail(DLM_ERR_INVALID_ARG, "%s: struct_size %u != %zu", who, a->struct_size, sizeof(dlm_embed_bwd_args));
    int rc;
    if ((rc = validate_embed(a->T, a->V, a->Dh, a->tokens, a->scale, who)) != DLM_OK) return rc;
    if (a->V > EMBED_MAX_V) return fail(DLM_ERR_UNSUPPORTED, "%s: V=%d (supported: up to %d)", who, a->V, EMBED_MAX_V);
    if (a->T > 1 << 28) return fail(DLM_ERR_UNSUPPORTED, "%s: T=%d (supported: up to 2^28)", who, a->T);
    if (a->Dh > 1 << 16 || (int64_t)a->T * a->Dh > (int64_t)1 << 40) return fail(DLM_ERR_UNSUPPORTED, "%s: T=%d Dh=%d (supported: Dh up to 65536, T Dh up to 2^40)", who, a->T, a->Dh);
    if (a->T > 0 && a->d_table && a->d_table == a->d_out) return fail(DLM_ERR_INVALID_ARG, "%s: d_table is d_out", who);
    if ((rc = validate_row_type(a->d_out_type, who, "d_out")) != DLM_OK) return rc;
    if ((rc = validate_row_type(a->d_table_type, who, "d_table")) != DLM_OK) return rc;
    if ((rc = validate_rows(a->d_out, a->d_out_stride, a->T, a->Dh, row_bytes(a->d_out_type), false, who, "d_out")) != DLM_OK) return rc;
    const int bytes = row_bytes(a->d_table_type);
    if ((rc = validate_rows(a->d_table, a->d_table_stride, a->V, a->Dh, bytes, true, who, "d_table")) != DLM_OK) return rc;
    const size_t need = dlm_embed_bwd_workspace_bytes(a);
    if (need > 0) {
        if (!a->workspace || a->workspace_bytes < need) return fail(DLM_ERR_WORKSPACE, "%s: workspace of %zu bytes required", who, need);
        if (!aligned16(a->workspace)) return fail(DLM_ERR_WORKSPACE, "%s: workspace not 16-byte aligned", who);
    }
    hipStream_t st = (hipStream_t)stream;
    const EmbedPlan plan = plan_embed(a->T, a->V, a->Dh, !a->accumulate);
    char* ws = (char*)a->workspace;
    int32_t* list[4];
    for (int i = 0; i < 4; ++i) list[i] = (int32_t*)(ws + i * plan.list_bytes);
    const int64_t row_bytes_ = (int64_t)a->Dh * bytes, pitch = a->V > 1 ? a->d_table_stride * bytes : row_bytes_;
    SortParams s = {a->T, a->V, a->tokens, list[0], list[1], plan.runs, a->d_table, 0, 0, a->V * row_bytes_ / 16, 0};
    if (!a->accumulate) {
        const bool gaps = pitch != row_bytes_;
        s.pieces = gaps ? (int)(row_bytes_ / 16) : 4096;
        s.pitch = gaps ? pitch : 4096 * 16;
        s.rows = (s.total + s.pieces - 1) / s.pieces;
    }
    const int most = (2048 << 13) >> plan.bits;      // (as many threads whatever the workgroup's size)
    const int clear = (int)(s.rows < most ? s.rows : most);
    if (plan.runs + clear == 0) return DLM_OK;
    if (plan.bits == 9) hipLaunchKernelGGL(embed_sort_kernel<9>, dim3(plan.runs + clear), dim3(64), 0, st, s);
    else if (plan.bits == 11) hipLaunchKernelGGL(embed_sort_kernel<11>, dim3(plan.runs + clear), dim3(256), 0, st, s);
    else hipLaunchKernelGGL(embed_sort_kernel<13>, dim3(plan.runs + clear), dim3(1024), 0, st, s);
    if ((rc = check_hip(hipGetLastError(), "embed_sort_kernel launch")) != DLM_OK) return rc;
    if (a->T == 0) return DLM_OK;
    int from = 0;
    int64_t len = 1 << plan.bits;
    for (int level = 0; level < plan.levels; ++level) {
        const int to = from ^ 2;
        hipLaunchKernelGGL(embed_merge_kernel, dim3((unsigned)(((int64_t)a->T + 255) / 256)), dim3(256), 0, st, list[from], list[from + 1], list[to], list[to + 1], a->T, len);
        if ((rc = check_hip(hipGetLastError(), "embed_merge_kernel launch")) != DLM_OK) return rc;
        from = to;
        len *= MERGE;
    }
    const bool in32 = a->d_out_type == DLM_ROW_F32, out32 = a->d_table_type == DLM_ROW_F32;
    const int per = in32 ? 256 : 512;
    EmbedGradParams p = {a->T, a->V, a->Dh, list[from], list[from + 1], a->d_out, a->d_out_stride, a->scale, a->d_table, a->d_table_stride,
                         a->accumulate, plan.chunk, (a->Dh + per - 1) / per, 0, (float*)(ws + plan.part_at)};
    const dim3 threads(GROUP * WAVE);
    const int most_groups = (1 << 21) / p.slices;    // of a launch: its threads stay below 2^32
#define EMBED_GRAD(IN, OUT)                                                                                \
    {                                                                                                    \
        if (a->accumulate) hipLaunchKernelGGL((embed_grad_kernel<IN, OUT, true>), grid, threads, 0, st, p); \
        else hipLaunchKernelGGL((embed_grad_kernel<IN, OUT, false>), grid, threads, 0, st, p);           \
    }
    for (; p.group0 < plan.groups; p.group0 += most_groups) {
        const dim3 grid((unsigned)((plan.groups - p.group0 < most_groups ? plan.groups - p.group0 : most_groups) * p.slices));
        if (in32 && out32) EMBED_GRAD(true, true)
        else if (in32) EMBED_GRAD(true, false)
        else if (out32) EMBED_GRAD(false, true)
        else EMBED_GRAD(false, false)
        if ((rc = check_hip(hipGetLastError(), "embed_grad_kernel launch")) != DLM_OK) return rc;
    }
#undef EMBED_GRAD
    if (plan.groups < 2) return DLM_OK;
    const dim3 join(plan.groups - 1, (a->Dh + 255) / 256);
    if (out32) hipLaunchKernelGGL((embed_join_kernel<true>), join, dim3(WAVE), 0, st, p);
    else hipLaunchKernelGGL((embed_join_kernel<false>), join, dim3(WAVE), 0, st, p);
    return check_hip(hipGetLastError(), "embed_join_kernel launch");
}
