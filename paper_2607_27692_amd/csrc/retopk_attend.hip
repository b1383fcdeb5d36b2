// retopk_attend.hip -- paged_attention: full attention of single tokens over a paged cache.
//
// The positions of all (token, KV head) groups are cut into equal parts, one a wave
// (retopk_paged_plan.h).  A wave streams its tiles with no barrier: scores, a reference
// maximum, weights and weighted value sums for every query head of the group at once, the next
// tile's rows in flight.  Waves of a block that share a group join their results in shared
// memory, and k_attend_merge joins what is left in parts.  One kernel a page format:
//   k_attend4   4 bits: both products on the matrix cores, codes as exact operands
//   k_attend16  bf16:   both products on the matrix cores, weights in three bf16 parts
//   k_attend    f32:    vector units
// Measured, whole calls, the join's launch of about 5 us in them: 131072 positions, 32 heads on 8,
// d = 128: 35 to 36 us from 4-bit pages (151 MB, 4.2 TB/s), 90 from bf16 pages (537 MB, 5.9 TB/s), 194
// from f32 pages (1.07 GB, 5.5 TB/s); 32 ragged sequences of up to 16K positions, 28 heads on 4, 4 bits:
// 31 us (96 MB, 3.1 TB/s).
#include "retopk.h"
#include "retopk_paged.h"

#include <cfloat>

namespace retopk {
namespace {

constexpr int kAttendThreads = 64 * kAttendWaves;
// Waves that run at once: two on each of the 1024 SIMDs by the registers of most builds, three of the
// 4-bit one of d = 64 (32 ragged sequences: 26.3 us with three, 29.3 with two; the others lose by more).
constexpr int64_t kSimds = 1024;
inline int64_t attend_slots(int format, int d) { return kSimds * (format == RETOPK_PAGES_Q4 && d == 64 ? 3 : 2); }
constexpr float kLn2 = 0.69314718055994530942f;
// A weight is 2^(s * mul - m) in one rounding while the reference m is no larger; past it the rounding
// of m is no longer small (of 2^31 it is 128: a weight of infinity, or all of them 0), and s * mul is
// rounded before the difference as m was.
constexpr float kNearReference = 65536.0f;

struct AttendArgs {
    PagesArgs c;
    const int32_t *seq, *pos;
    const char *q;             // element strides
    int64_t q_ts, q_hs;
    int32_t n_tokens, n_q, group;      // query heads; of a KV head
    int32_t max_len, window;
    int32_t split, waves, chunks;      // AttendPlan
    float scale2;              // log2(e) / sqrt(d): scores are in powers of two
    float *out, *lse;
    int32_t *ends;             // BALANCED: [n_tokens] tiles up to and with a token; a part's tiles; a start's
    float *part_o;             // [parts, group, d]
    float2 *part_ml;           // [parts, group]: maximum (a power of two), sum
};

// The attended positions [first, len) of a token, len = 0 where there are none; its tiles
// begin at base.
struct Span {
    int first, len, base;
    __device__ __forceinline__ int tiles() const { return (len - base + kAttendTile - 1) / kAttendTile; }
};
__device__ __forceinline__ Span span_of(const AttendArgs &a, int32_t s, int32_t p)
{
    Span r = {0, 0, 0};
    if (s < 0 || s >= a.c.n_seqs || p < 0) return r;
    r.len = p < a.max_len ? p + 1 : a.max_len;
    if (a.window > 0 && p >= a.window) r.first = p - a.window + 1;
    if (r.first >= r.len) r.len = r.first = 0;
    r.base = r.first / kAttendTile * kAttendTile;
    return r;
}

// One wave's share of a group: positions [lo, hi) of token t for KV head g, within the token's
// span; the result goes to the output (part < 0) or to that partial result.
struct Share {
    int64_t t;
    int g, seq, lo, hi;
    Span span;
    int64_t part;
    bool joint;                // the block's four waves share the group and join their results
    // row of head j of the group in the output or among the partial results
    __device__ __forceinline__ int64_t row(const AttendArgs &a, int j) const
    {
        return part < 0 ? t * a.n_q + g * a.group + j : part * a.group + j;
    }
};

// Runs f on every share of this wave.
template <typename F>
__device__ __forceinline__ void for_shares(const AttendArgs &a, F f)
{
    constexpr int TPT = kAttendTokens / kAttendThreads;        // tokens a thread
    __shared__ int s_ends[kAttendTokens], s_seq[kAttendTokens], s_pos[kAttendTokens];
    __shared__ uint32_t s_red[kAttendWaves];
    const int hkv = a.c.n_kv_heads, tid = threadIdx.x, lane = tid & 63;
    const int worker = blockIdx.x * kAttendWaves + __builtin_amdgcn_readfirstlane(tid >> 6);
    const bool balanced = a.split == ATTEND_BALANCED;
    int at = 0, last = worker < a.waves ? 1 : 0;
    int empty = 0;                             // tiles before each group's own
    int64_t block_from = 0, block_to = 0;      // the block's tiles
    bool whole_block = false;                  // all of its waves have theirs
    // every token's last tile (of all KV heads), sequence and position, counted by each block for
    // itself, or for up to 64 tokens by each wave, which then has no barrier to wait at
    const bool few = a.n_tokens <= 64;
    const int of = few ? tid & ~63 : 0;
    int *const t_ends = s_ends + of, *const t_seq = s_seq + of, *const t_pos = s_pos + of;
    if (balanced) {
        int sum = 0, ends[TPT];
        const int own = few ? 1 : TPT, t0 = few ? lane : tid * TPT;    // tokens of this thread
#pragma unroll
        for (int i = 0; i < TPT; ++i) {
            ends[i] = sum;
            if (i >= own) continue;
            const int t = t0 + i;
            const int sq = t < a.n_tokens ? a.seq[t] : -1, p = t < a.n_tokens ? a.pos[t] : -1;
            t_seq[t] = sq;
            t_pos[t] = p;
            ends[i] = sum += span_of(a, sq, p).tiles() * hkv;
        }
        uint32_t all;
        int before;
        if (few) {
            const uint32_t incl = wave_incl_scan((uint32_t)sum);
            all = (uint32_t)__builtin_amdgcn_readlane((int)incl, 63);
            before = (int)incl - sum;
        } else {
            before = (int)block_excl_scan<kAttendThreads>((uint32_t)sum, s_red, &all);
        }
        const int per = (int)attend_part(all, (uint32_t)a.waves);
        empty = (int)attend_start(all, (uint32_t)a.waves, (uint32_t)per, (uint32_t)(a.n_tokens * hkv));
        all += (uint32_t)(empty * a.n_tokens * hkv);
        const bool tell = few ? worker == 0 : blockIdx.x == 0;         // the joining kernel
#pragma unroll
        for (int i = 0; i < TPT; ++i) {
            if (i >= own) continue;
            const int t = t0 + i;
            t_ends[t] = before + ends[i] + (t + 1) * empty * hkv;
            if (tell && t < a.n_tokens) a.ends[t] = t_ends[t];
        }
        if (tell && tid == 0) {
            a.ends[a.n_tokens] = per;
            a.ends[a.n_tokens + 1] = empty;
        }
        if (few) wave_lds_fence();
        else __syncthreads();
        const int64_t from = (int64_t)worker * per;
        at = (int)min(from, (int64_t)all);
        last = (int)min(from + per, (int64_t)all);
        block_from = (int64_t)blockIdx.x * kAttendWaves * per;
        block_to = block_from + kAttendWaves * per;
        whole_block = block_to <= (int64_t)all;
    }
    while (at < last) {
        Share w;
        int step = 1;
        if (balanced) {
            // the token that holds tile `at`: as many as end at or before it come first
            int t = 0;
            for (int i = 0; i < a.n_tokens; i += 64)
                t += __popcll(__ballot(i + lane < a.n_tokens && t_ends[i + lane] <= at));
            t = __builtin_amdgcn_readfirstlane(t);
            const int start = t > 0 ? __builtin_amdgcn_readfirstlane(t_ends[t - 1]) : 0;
            const int tiles = (__builtin_amdgcn_readfirstlane(t_ends[t]) - start) / hkv;
            const int first = (at - start) % tiles;
            step = min(tiles - first, last - at);
            w.t = t;
            w.g = (at - start) / tiles;
            w.seq = __builtin_amdgcn_readfirstlane(t_seq[t]);
            w.span = span_of(a, w.seq, __builtin_amdgcn_readfirstlane(t_pos[t]));
            w.lo = w.span.base + max(first - empty, 0) * kAttendTile;
            w.hi = min(w.span.len, w.span.base + (first + step - empty) * kAttendTile);
            const int end = start + (w.g + 1) * tiles, base = end - tiles + empty;     // the group's own tiles
            w.joint = whole_block && block_from >= base && block_to <= end;
            w.part = first <= empty && first + step == tiles ? -1 : (int64_t)(w.joint ? blockIdx.x * kAttendWaves : worker) + (int64_t)t * hkv + w.g;
        } else {
            const bool direct = a.split == ATTEND_DIRECT;
            const int chunk = worker % a.chunks, bg = worker / a.chunks;
            w.t = bg / hkv;
            w.g = bg % hkv;
            w.seq = __builtin_amdgcn_readfirstlane(a.seq[w.t]);
            w.span = span_of(a, w.seq, __builtin_amdgcn_readfirstlane(a.pos[w.t]));
            const int rows = direct ? (w.span.tiles() + kAttendWaves - 1) / kAttendWaves * kAttendTile : kAttendChunk;
            w.lo = w.span.base + chunk * rows;
            w.hi = min(w.span.len, w.lo + rows);
            w.part = direct ? -1 : (int64_t)worker;
            w.joint = direct;
        }
        if (w.lo < w.hi || w.joint) f(w);
        at += step;
    }
}

// Where a wave leaves its result: shared memory for waves that join theirs, else the output or
// a partial result.
template <int D, int GP> struct Joint {
    float o[kAttendWaves][GP][D], m[kAttendWaves][GP], l[kAttendWaves][GP];

    __device__ __forceinline__ float *row(const AttendArgs &a, const Share &w, int j)
    {
        return w.joint ? o[threadIdx.x >> 6][j] : (w.part < 0 ? a.out : a.part_o) + w.row(a, j) * D;
    }
    // the weights' sum and reference of head j, and what the value sums are times
    __device__ __forceinline__ void sum(const AttendArgs &a, const Share &w, int j, float mj, float lj)
    {
        if (w.joint) {
            m[threadIdx.x >> 6][j] = mj;
            l[threadIdx.x >> 6][j] = lj;
        } else if (w.part >= 0) {
            a.part_ml[w.row(a, j)] = make_float2(mj, lj);
        } else if (a.lse) {
            a.lse[w.row(a, j)] = lj > 0.0f ? (mj + log2f(lj)) * kLn2 : -INFINITY;
        }
    }
    static __device__ __forceinline__ float factor(const Share &w, float lj)
    {
        return w.joint || w.part >= 0 ? 1.0f : lj > 0.0f ? 1.0f / lj : 0.0f;
    }
    // at a share's end, by every wave of the block if any joins
    __device__ __forceinline__ void finish(const AttendArgs &a, const Share &w)
    {
        if (!w.joint) return;
        __syncthreads();
        for (int i = threadIdx.x; i < a.group * D; i += kAttendThreads) {
            const int j = i / D, e = i % D;
            float mx = m[0][j], x = 0.0f, lj = 0.0f;
#pragma unroll
            for (int v = 1; v < kAttendWaves; ++v) mx = fmaxf(mx, m[v][j]);
#pragma unroll
            for (int v = 0; v < kAttendWaves; ++v) {
                const float f = __builtin_amdgcn_exp2f(m[v][j] - mx);
                x = fmaf(f, o[v][j][e], x);
                lj = fmaf(f, l[v][j], lj);
            }
            const int64_t to = w.row(a, j);
            if (w.part >= 0) {
                a.part_o[to * D + e] = x;
                if (e == 0) a.part_ml[to] = make_float2(mx, lj);
            } else {
                a.out[to * D + e] = lj > 0.0f ? x / lj : 0.0f;
                if (e == 0 && a.lse) a.lse[to] = lj > 0.0f ? (mx + log2f(lj)) * kLn2 : -INFINITY;
            }
        }
    }
};

// ---------------------------------------------------------------------------
// f32 and bf16 pages
// ---------------------------------------------------------------------------

// Sum over the LPR lanes (8 or 16, a half or a whole DPP row) that share a position.
template <int LPR> __device__ __forceinline__ float lanes_sum(float x)
{
    x += dpp_f32<kQuadXor1>(x);
    x += dpp_f32<kQuadXor2>(x);
    x += dpp_f32<kHalfMirror>(x);
    if constexpr (LPR == 16) x += dpp_f32<0x140>(x);   // row_mirror
    return x;
}

// k_attend (f32 pages): LPR = D / 8 lanes a position, 8 elements of its key and value rows a lane; a wave
// takes 64 / LPR positions at once, U times over in a step, whose rows are loaded a step ahead and
// whose pages are looked up two steps ahead, since any position may be on another page.  All in
// float32 on the vector units: 8 products and 8 value sums a lane, position and head, which
// stay below the time HBM needs for the rows (131072 positions, 4 heads on each of 8: 196 us, 5.5 TB/s of
// the 6.0 that a plain read reaches).  GP >= a.group heads; those past the group repeat
// its first.
template <int D, int GP>
__global__ __launch_bounds__(kAttendThreads, 2) void k_attend(AttendArgs a)
{
    using T = float;
    constexpr int LPR = D / 8, SLOTS = 64 / LPR, U = GP == 8 ? 2 : 4, STEP = SLOTS * U;
    constexpr bool QL = GP == 8;                       // the queries in LDS: registers hold no 8 heads' more
    __shared__ __attribute__((aligned(16))) float s_q[kAttendWaves][QL ? GP : 1][D];
    __shared__ __attribute__((aligned(16))) Joint<D, GP> s_join;
    for_shares(a, [&](const Share &w) {
        const int lane = threadIdx.x & 63, e0 = lane % LPR * 8, slot = lane / LPR;
        const int wave = threadIdx.x >> 6;
        float q[QL ? 1 : GP][8], acc[GP][8], m[GP], l[GP];
#pragma unroll
        for (int j = 0; j < GP; ++j) {
            const int h = w.g * a.group + (j < a.group ? j : 0);
            Oct<T> v;
            float x[8];
            v.load((const T *)a.q + w.t * a.q_ts + h * a.q_hs + e0);
            v.get(x);
            m[j] = -FLT_MAX;
            l[j] = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[i] *= a.scale2;
                if constexpr (!QL) q[j][i] = x[i];
                acc[j][i] = 0.0f;
            }
            if constexpr (QL) Oct<float>::store(&s_q[wave][j][e0], x);     // the same from every slot
        }
        if constexpr (QL) wave_lds_fence();
        const int n_it = (w.hi - w.lo + STEP - 1) / STEP;
        Oct<T> k[U], v[U];
        int32_t r0[U], r1[U];                          // rows of this step and the next, -1: none
        int32_t pages[U];                              // of the step after
        auto look = [&](int it) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int pos = w.lo + it * STEP + u * SLOTS + slot;
                pages[u] = pos >= w.span.first && pos < w.hi ? page_of(a.c, w.seq, pos) : -1;
            }
        };
        auto rows = [&](int it, int32_t (&r)[U]) {
#pragma unroll
            for (int u = 0; u < U; ++u) r[u] = row_on(a.c, pages[u], w.lo + it * STEP + u * SLOTS + slot, w.g);
        };
        auto load = [&](Oct<T> (&x)[U], const char *from, const int32_t (&r)[U]) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                x[u].load_once((const T *)from + (uint64_t)(uint32_t)max(r[u], 0) * D + e0);
        };
        if (n_it > 0) {
            look(0);
            rows(0, r0);
            look(1);
            load(k, a.c.k, r0);
            load(v, a.c.v, r0);
            rows(1, r1);
        }
        for (int it = 0; it < n_it; ++it) {
            look(it + 2);
            float s[U][GP];
#pragma unroll
            for (int j = 0; j < GP; ++j) {
                float y[8];
                if constexpr (QL) {
                    wave_lds_fence();                  // read here, not held in registers over the loop
                    Oct<float> o;
                    o.load(&s_q[wave][j][e0]);
                    o.get(y);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    float x[8];
                    k[u].get(x);
                    s[u][j] = 0.0f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) s[u][j] = fmaf(QL ? y[i] : q[QL ? 0 : j][i], x[i], s[u][j]);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            load(k, a.c.k, r1);                        // past the last step: rows -1, row 0 instead
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int j = 0; j < GP; ++j) s[u][j] = r0[u] >= 0 ? lanes_sum<LPR>(s[u][j]) : -INFINITY;
#pragma unroll
            for (int j = 0; j < GP; ++j) {
                float mn = m[j];
#pragma unroll
                for (int u = 0; u < U; ++u) mn = fmaxf(mn, s[u][j]);
                const float f = __builtin_amdgcn_exp2f(m[j] - mn);
                m[j] = mn;
                float sum = 0.0f;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    s[u][j] = __builtin_amdgcn_exp2f(s[u][j] - mn);
                    sum += s[u][j];
                }
                l[j] = fmaf(l[j], f, sum);
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[j][i] *= f;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float x[8];
                v[u].get(x);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = r0[u] >= 0 ? x[i] : 0.0f;     // whatever lies in row 0
#pragma unroll
                for (int j = 0; j < GP; ++j)
#pragma unroll
                    for (int i = 0; i < 8; ++i) acc[j][i] = fmaf(s[u][j], x[i], acc[j][i]);
            }
            __builtin_amdgcn_sched_barrier(0);
            load(v, a.c.v, r1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < U; ++u) r0[u] = r1[u];
            rows(it + 2, r1);
        }
#pragma unroll
        for (int j = 0; j < GP; ++j) {
#pragma unroll
            for (int o = LPR; o < 64; o <<= 1) {
                const float m2 = __shfl_xor(m[j], o), l2 = __shfl_xor(l[j], o), mn = fmaxf(m[j], m2);
                const float f = __builtin_amdgcn_exp2f(m[j] - mn), f2 = __builtin_amdgcn_exp2f(m2 - mn);
                m[j] = mn;
                l[j] = l[j] * f + l2 * f2;
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[j][i] = acc[j][i] * f + __shfl_xor(acc[j][i], o) * f2;
            }
            if (lane < LPR && j < a.group) {
                const float f = s_join.factor(w, l[j]);
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[j][i] *= f;
                Oct<float>::store(s_join.row(a, w, j) + e0, acc[j]);
                if (lane == 0) s_join.sum(a, w, j, m[j], l[j]);
            }
        }
        s_join.finish(a, w);
        if constexpr (QL) wave_lds_fence();            // the queries of the next share
    });
}

// k_attend16 (bf16 pages): the matrix cores take both products.  A tile is 32 positions; lanes
// 0 .. 31 look up a position's row each, a tile ahead of its loads, and share the row numbers through
// LDS, since any position may be on another page.  Scores: 16 positions x 32 elements x 16 columns,
// lane (col, kq) holding those of positions 4 kq .. + 3 of both halves of the tile for head
// col % GP.  Values: 16 elements x 32 positions x 16 columns, whose positions are in the order in
// which a lane already has its weights; pairs of positions are put side by side with byte permutes.
// A weight is the sum of three bf16 parts (24 bits): column c has part c / GP of head c % GP, for
// GP = 8 the third in a second product.  Products start from zero and are added by the vector units:
// accumulated in the matrix cores the sums lose 2^-24 of the largest product at every step.  Bound by
// HBM: the same positions take 85 to 88 us, 6.1 TB/s and more; 8 sequences of up to 32768 take 66 to 68.
template <int D, int GP>
__global__ __launch_bounds__(kAttendThreads, 2) void k_attend16(AttendArgs a)
{
    constexpr int KS = D / 32, NV = D / 16;
    constexpr int VD = D / 32;                         // dwords of a lane's share of a value row
    __shared__ __attribute__((aligned(16))) uint32_t s_row[kAttendWaves][2][32];
    __shared__ __attribute__((aligned(16))) Joint<D, GP> s_join;
    for_shares(a, [&](const Share &w) {
        const int lane = threadIdx.x & 63, col = lane & 15, kq = lane >> 4;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int hc = col % GP, head = hc < a.group ? hc : 0, part = col / GP;
        const int n_it = (w.hi - w.lo + 31) / 32;

        bf16x8_t qb[KS];
        {
            const u32x4_t *qr = (const u32x4_t *)((const uint16_t *)a.q + w.t * a.q_ts + (w.g * a.group + head) * a.q_hs);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) qb[ks] = __builtin_bit_cast(bf16x8_t, qr[ks * 4 + kq]);
        }
        // page of position lane % 32 of tile `it`, and its row there; -1: not attended or no page
        auto look = [&](int it) {
            const int pos = w.lo + it * 32 + (lane & 31);
            return pos >= w.span.first && pos < w.hi ? page_of(a.c, w.seq, pos) : -1;
        };
        auto row_in = [&](int it, int32_t page) { return row_on(a.c, page, w.lo + it * 32 + (lane & 31), w.g); };
        // publishes a tile's rows (row 0 for none) and returns which there are
        auto publish = [&](int it, int32_t row) {
            if (lane < 32) s_row[wave][it & 1][lane] = (uint32_t)max(row, 0);
            wave_lds_fence();
            return (uint32_t)__ballot(row >= 0);
        };
        u32x4_t kv[2][KS];
        uint32_t vv[8][VD];
        auto load_k = [&](int it) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const u32x4_t *p = (const u32x4_t *)(a.c.k + (uint64_t)s_row[wave][it & 1][16 * u + col] * (2 * D));
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) kv[u][ks] = once(p + ks * 4 + kq);
            }
        };
        auto load_v = [&](int it) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const u32x4_t r = *(const u32x4_t *)&s_row[wave][it & 1][16 * u + 4 * kq];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const char *p = a.c.v + (uint64_t)r[i] * (2 * D) + col * (D / 8);
                    if constexpr (VD == 4) {
                        const u32x4_t x = once((const u32x4_t *)p);
#pragma unroll
                        for (int e = 0; e < 4; ++e) vv[4 * u + i][e] = x[e];
                    } else {
                        const u32x2_t x = once((const u32x2_t *)p);
                        vv[4 * u + i][0] = x[0];
                        vv[4 * u + i][1] = x[1];
                    }
                }
            }
        };
        f32x4_t acc[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) acc[j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        float m = -FLT_MAX, l = 0.0f;
        bool big = false;                              // a reference past kNearReference
        const float after1 = part >= 1 ? 1.0f : 0.0f, after2 = part >= 2 ? 1.0f : 0.0f;

        uint32_t on = 0u, on_next = 0u;
        int32_t ahead = -1;
        if (n_it > 0) {
            const int32_t first = look(0), second = look(1);
            on = publish(0, row_in(0, first));
            load_k(0);
            load_v(0);
            ahead = row_in(1, second);
        }
        for (int it = 0; it < n_it; ++it) {
            const int32_t page = look(it + 2);
            float s[8];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                f32x4_t d[KS];
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
                    d[ks] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kv[u][ks]), qb[ks],
                                                                    f32x4_t{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0);
#pragma unroll
                for (int n = KS / 2; n > 0; n /= 2)
#pragma unroll
                    for (int ks = 0; ks < n; ++ks) d[ks] += d[ks + n];
#pragma unroll
                for (int i = 0; i < 4; ++i) s[4 * u + i] = d[0][i];
            }
            __builtin_amdgcn_sched_barrier(0);
            on_next = publish(it + 1, ahead);          // past the last tile: none, row 0 is loaded
            load_k(it + 1);
            __builtin_amdgcn_sched_barrier(0);
            if (on != 0xFFFFFFFFu) {
                asm volatile("");                      // a branch, not selects in every tile
                const uint32_t mine = on >> (4 * kq);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const bool there = mine >> (16 * (i >> 2) + (i & 3)) & 1u;
                    s[i] = there ? s[i] : -INFINITY;
#pragma unroll
                    for (int e = 0; e < VD; ++e) vv[i][e] = there ? vv[i][e] : 0u;   // whatever lies there
                }
            }
            float tm = -INFINITY;
#pragma unroll
            for (int i = 0; i < 8; ++i) tm = fmaxf(tm, s[i]);
            tm = max_rows_f32(tm) * a.scale2;
            // the reference moves by steps, as in k_attend4
            if (__ballot(tm > m + 1.0f) != 0ull) {
                const float mn = tm > m + 1.0f ? tm + 1.0f : m, f = __builtin_amdgcn_exp2f(m - mn);
                m = mn;
                l *= f;
#pragma unroll
                for (int j = 0; j < NV; ++j) acc[j] *= f;
                big = __ballot(fabsf(m) > kNearReference) != 0ull;
            }
            if (big) {
                asm volatile("");                      // as above
#pragma unroll
                for (int i = 0; i < 8; ++i) s[i] *= a.scale2;
            }
            const float by = big ? 1.0f : a.scale2;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], by, -m));
                l += s[i];
            }
            // this column's part of the weights; the third one too
            u32x4_t pb, pc;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x2_t x = {s[2 * i], s[2 * i + 1]};
                const uint32_t h = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2_t));
                const f32x2_t y = {fmaf(-bf16_lo(h), GP == 4 ? after1 : 1.0f, x[0]), fmaf(-bf16_hi(h), GP == 4 ? after1 : 1.0f, x[1])};
                const uint32_t h2 = __builtin_bit_cast(uint32_t, __builtin_convertvector(y, bf16x2_t));
                if constexpr (GP == 4) {
                    const f32x2_t z = {fmaf(-bf16_lo(h2), after2, y[0]), fmaf(-bf16_hi(h2), after2, y[1])};
                    pb[i] = part < 3 ? __builtin_bit_cast(uint32_t, __builtin_convertvector(z, bf16x2_t)) : 0u;
                } else {
                    const f32x2_t z = {y[0] - bf16_lo(h2), y[1] - bf16_hi(h2)};
                    pb[i] = part == 0 ? h : h2;
                    pc[i] = part == 0 ? __builtin_bit_cast(uint32_t, __builtin_convertvector(z, bf16x2_t)) : 0u;
                }
            }
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                u32x4_t x;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    x[i] = __builtin_amdgcn_perm(vv[2 * i + 1][j / 2], vv[2 * i][j / 2], j & 1 ? 0x07060302u : 0x05040100u);
                f32x4_t d = {0.0f, 0.0f, 0.0f, 0.0f};
                if constexpr (GP == 8)
                    d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, x), __builtin_bit_cast(bf16x8_t, pc), d, 0, 0, 0);
                acc[j] += __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, x), __builtin_bit_cast(bf16x8_t, pb), d, 0, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
            load_v(it + 1);
            __builtin_amdgcn_sched_barrier(0);
            on = on_next;
            ahead = row_in(it + 2, page);
        }
        l = add16_f32(l, l);
        l = add32_f32(l, l);
        if (lane < GP && hc < a.group) s_join.sum(a, w, hc, m, l);
        // rows 4 kq + i of product j are elements (4 kq + i) * NV + j; a head's parts lie GP columns apart
        const float f = s_join.factor(w, l);
        float *out = s_join.row(a, w, hc) + 4 * kq * NV;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j0 = 0; j0 < NV; j0 += 4) {
                f32x4_t o;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    o[j] = acc[j0 + j][i];
                    o[j] += row_ror_f32(o[j], 8);
                    if constexpr (GP == 4) o[j] += row_ror_f32(o[j], 4);
                    o[j] *= f;
                }
                if (col < GP && hc < a.group) *(f32x4_t *)(out + i * NV + j0) = o;
            }
        s_join.finish(a, w);
    });
}

// ---------------------------------------------------------------------------
// 4-bit pages
// ---------------------------------------------------------------------------

typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));

// Codes as operands of the matrix cores: in a half-word (b0 low, b1 high byte) the sign of
// code 0 is bit 15 and its magnitude bits 4 .. 6, which with bit 3 set is the subnormal
// float16 c * 2^-20, exact; code 1 lies four bits lower, codes 2 and 3 the same with the
// bytes swapped.  One and-or a pair of codes, no conversion.
constexpr int kCodeExp = 20;
struct Codes {
    uint32_t mask = 0x80708070u, half = 0x00080008u;
    // held in registers, so that (x & mask) | half is one instruction (literals would make it two)
    __device__ __forceinline__ void hold() { asm volatile("" : "+s"(mask), "+v"(half)); }
    __device__ __forceinline__ uint32_t pair(uint32_t x) const { return (x & mask) | half; }
    __device__ __forceinline__ void quad(uint32_t x, uint32_t (&r)[4]) const
    {
        const uint32_t y = __builtin_amdgcn_perm(x, x, 0x02030001u);
        r[0] = pair(x);
        r[1] = pair(x << 4);
        r[2] = pair(y);
        r[3] = pair(y << 4);
    }
};

// Base rows of the two 16-position halves of a tile: a 4-bit page holds whole halves, so
// that a half has one page, looked up once for the wave.
struct Half {
    int32_t row;               // of its first position; 0 where it has no page
    bool there;
};
__device__ __forceinline__ Half half_of(const PagesArgs &c, const int32_t *table, int32_t pos, int g)
{
    const uint32_t at = divide((uint32_t)pos, c.by_page);
    int32_t page = -1;
    if (at < (uint32_t)c.table_width)
        page = ((const __attribute__((address_space(4))) int32_t *)(uintptr_t)table)[at];
    const bool there = page >= 0 && page < c.n_pages;
    return Half{there ? (page * c.n_kv_heads + g) * c.page_size + (pos - (int32_t)at * c.page_size) : 0, there};
}

// k_attend4: each wave streams its own 32-position tiles.  A matrix column is (half of the
// tile, group of 64 elements, query head), as far as eight columns a half suffice (PACK: d = 64,
// or up to 4 heads of d = 128), else (group, head).  The query is zero outside a column's group, so
// that a product's result is one group's sum of codes times query, to which a lane applies one
// scale and mid: V scores a lane, V = 4 or 8.  The weights times the value scales are the second
// product's other operand, in two float16 parts (24 bits together) of which a common power of
// two, kept above every scale met so far, is taken out; value codes are exact.
//
// What the matrix cores round has a bias (against float64 the outputs of 128K rows were 1.2e-5 off
// with plain accumulation, 2.5e-7 so): products are cut below 2^-24 of the largest, and a sum that
// does not fit 24 bits rounds to one side.  The high parts are therefore whole numbers, whose
// products are multiples of 2^-21 and sum exactly, kFlush tiles long, until the vector units
// add them to acc; the low parts' sums, 2^-12 the size, may be biased.
//
// The vector units bound it, two thirds busy with the codes of both products and the weights' parts, and the
// 6 us until the first tile is there: 131072 positions, 4 heads on each of 8, d = 128 take 33 us (4.6 TB/s);
// without PACK, 32 ragged sequences of 7 heads on each of 4, 29 us (3.3 TB/s); with d = 64, 22.
constexpr int kFlush = 4;
template <typename T, int D, bool PACK>
__global__ __launch_bounds__(kAttendThreads, 2) void k_attend4(AttendArgs a)
{
    constexpr int NG = D / kGroup4;
    constexpr int V = PACK ? 4 : 8;            // positions a lane weighs in a tile
    constexpr int KD = D / 32;                 // code dwords of a lane's share of a key row
    constexpr int NV = D / 16;                 // value products: codes of a lane's share of a row
    constexpr int NQ = sizeof(T) == 4 ? 2 : 1; // float16 parts of the query
    static_assert(PACK || NG == 2, "d = 64 always packs");
    __shared__ __attribute__((aligned(16))) Joint<D, 8> s_join;
    for_shares(a, [&](const Share &w) {
        const int g = w.g, lo = w.lo, hi = w.hi;
        const int lane = threadIdx.x & 63, col = lane & 15, kq = lane >> 4;
        Codes codes;
        codes.hold();
        // group and head of this lane's column; packed columns 4 .. 7 of d = 128 count the heads down,
        // so that a half-row mirror meets the other group of the same head
        const int c8 = col & 7, upper = PACK ? col >> 3 : 0;
        const int gr = NG == 1 ? 0 : PACK ? c8 >> 2 : col >> 3;
        const int hc = PACK && NG == 2 ? (gr ? 7 - c8 : c8) : c8, head = hc < a.group ? hc : 0;
        const int n_it = (hi - lo + 31) / 32;
        const int32_t *table = a.c.table + (int64_t)max(w.seq, 0) * a.c.table_width;

        // the query, scaled by a power of two to [2^14, 2^15): bf16 fits one float16 part, f32 two
        f16x8_t qb[NQ][KD];
        int q_exp;
        float q_sum = 0.0f;
        {
            float x[KD][8], top = 0.0f;
            const T *qr = (const T *)a.q + w.t * a.q_ts + (g * a.group + head) * a.q_hs + kq * (D / 4);
    #pragma unroll
            for (int i = 0; i < KD; ++i) {
                Oct<T> v;
                v.load(qr + 8 * i);
                v.get(x[i]);
    #pragma unroll
                for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[i][e]));
            }
            top = max_rows_f32(top);
            q_exp = top > 0.0f ? __builtin_amdgcn_frexp_expf(top) - 15 : 0;
            const bool mine = NG == 1 || (kq >> 1) == gr;
    #pragma unroll
            for (int i = 0; i < KD; ++i)
    #pragma unroll
                for (int e = 0; e < 8; ++e) {
                    // code order: elements j and j + 4 in register j
                    const float y = mine ? ldexpf(x[i][(e >> 1) + 4 * (e & 1)], -q_exp) : 0.0f;
                    q_sum += y;
                    const _Float16 h = (_Float16)y;
                    qb[0][i][e] = h;
                    if constexpr (NQ == 2) qb[1][i][e] = (_Float16)(y - (float)h);
                }
            q_sum = add16_f32(q_sum, q_sum);
            q_sum = ldexpf(add32_f32(q_sum, q_sum), -kCodeExp);
        }
        // scores in powers of two are the products times this factor; what it cannot hold of the
        // exponent (queries past 2^94 or below 2^-106) is applied apart
        const int s_exp = q_exp + kCodeExp, s_near = min(max(s_exp, -100), 100);
        const float s_mul = ldexpf(a.scale2, s_near);
        const bool far = __ballot(s_exp != s_near) != 0ull;

        u32x4_t kc[2];             // key codes: the row's dwords kq * KD ..
        uint32_t kp[V], vp[V], vc[8];
        Half h0[2], h1[2];         // this tile's halves, the next one's
        auto halves = [&](int it, Half (&h)[2]) {
            const int r = lo + it * 32;
    #pragma unroll
            for (int u = 0; u < 2; ++u) h[u] = half_of(a.c, table, r + 16 * u, g);
        };
        // a half's base is the wave's own, a lane's offset in it the same for every half
        const uint32_t k_off = col * (D / 2) + kq * (D / 8), v_off = 4 * kq * (D / 2) + col * (D / 32);
        auto load_k = [&](const Half (&h)[2]) {
    #pragma unroll
            for (int u = 0; u < 2; ++u) {
                const char *p = a.c.k + (int64_t)h[u].row * (D / 2);
                if constexpr (KD == 4) {
                    kc[u] = once((const u32x4_t *)(p + k_off));
                } else {
                    const u32x2_t x = once((const u32x2_t *)(p + k_off));
                    kc[u][0] = x[0];
                    kc[u][1] = x[1];
                }
            }
        };
        auto load_par = [&](const Half (&h)[2], const uint32_t *par, uint32_t (&w)[V]) {
    #pragma unroll
            for (int u = 0; u < V / 4; ++u) {
                const int32_t row = (PACK ? (upper ? h[1].row : h[0].row) : h[u].row) + 4 * kq;
                const uint32_t *p = par + (int64_t)row * NG + gr;
                if constexpr (NG == 1) {
                    const u32x4_t x = *(const u32x4_t *)p;
    #pragma unroll
                    for (int i = 0; i < 4; ++i) w[4 * u + i] = x[i];
                } else {
    #pragma unroll
                    for (int i = 0; i < 4; ++i) w[4 * u + i] = p[i * NG];
                }
            }
        };
        auto load_v = [&](const Half (&h)[2]) {
    #pragma unroll
            for (int u = 0; u < 2; ++u) {
                const char *p = a.c.v + (int64_t)h[u].row * (D / 2);
    #pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (D == 128) vc[4 * u + i] = once((const uint32_t *)(p + v_off + i * (D / 2)));
                    else vc[4 * u + i] = once((const uint16_t *)(p + v_off + i * (D / 2)));
                }
            }
        };

        // sums of the high parts (exact, and what they were flushed to) and of the low parts
        f32x4_t run[NV], acc[NV], low[NV];
    #pragma unroll
        for (int j = 0; j < NV; ++j) run[j] = acc[j] = low[j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        auto flush = [&]() {
    #pragma unroll
            for (int j = 0; j < NV; ++j) {
                acc[j] += run[j];
                run[j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
            }
        };
        float m = -FLT_MAX, l = 0.0f, z = 0.0f, limit = 0.0f;
        bool big = false;                                    // a reference past kNearReference
        int v_exp = 0;

        auto tile = [&](int it, const Half (&h)[2], const Half (&hn)[2], auto more) {
            float s[V];
            {
                f32x4_t d[2];
    #pragma unroll
                for (int u = 0; u < 2; ++u) {
                    d[u] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    #pragma unroll
                    for (int i = 0; i < KD; ++i) {
                        uint32_t r[4];
                        codes.quad(kc[u][i], r);
                        const f16x8_t x = __builtin_bit_cast(f16x8_t, u32x4_t{r[0], r[1], r[2], r[3]});
    #pragma unroll
                        for (int n = NQ - 1; n >= 0; --n) d[u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, qb[n][i], d[u], 0, 0, 0);
                    }
                }
    #pragma unroll
                for (int i = 0; i < V; ++i) s[i] = PACK ? (upper ? d[1][i & 3] : d[0][i & 3]) : d[i >> 2][i & 3];
            }
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (decltype(more)::value) load_k(hn);
            __builtin_amdgcn_sched_barrier(0);
            const int row = lo + it * 32;
            const bool whole = row >= w.span.first && row + 32 <= hi && h[0].there && h[1].there;
            float tm = -INFINITY;
    #pragma unroll
            for (int i = 0; i < V; ++i) s[i] = fmaf(bf16_lo(kp[i]), s[i], bf16_hi(kp[i]) * q_sum);
            if constexpr (NG == 2) {                                 // the other group of the row
    #pragma unroll
                for (int i = 0; i < V; ++i) s[i] += PACK ? dpp_f32<kHalfMirror>(s[i]) : row_ror_f32(s[i], 8);
            }
            if (far) {
                asm volatile("");                                    // a branch, not selects in every tile
    #pragma unroll
                for (int i = 0; i < V; ++i) s[i] = ldexpf(s[i], s_exp - s_near);
            }
            if (!whole) {
                asm volatile("");
    #pragma unroll
                for (int i = 0; i < V; ++i) {
                    const int u = PACK ? upper : i >> 2, r = row + 16 * u + 4 * kq + (i & 3);
                    const bool on = r >= w.span.first && r < hi && (u ? h[1].there : h[0].there);
                    s[i] = on ? s[i] : -INFINITY;
                    vp[i] = on ? vp[i] : 0u;                         // whatever lies there: weight and value 0
                }
            }
    #pragma unroll
            for (int i = 0; i < V; ++i) tm = fmaxf(tm, s[i]);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (decltype(more)::value) load_par(hn, a.c.k_par, kp);
            __builtin_amdgcn_sched_barrier(0);
            // the reference stays until a score passes it by more than 1, then steps 1 past that score:
            // weights stay below 4 and the sums are rescaled a few times a chunk, not at every new maximum
            if constexpr (PACK) tm = fmaxf(tm, row_ror_f32(tm, 8));
            tm = max_rows_f32(tm) * s_mul;
            if (__ballot(tm > m + 1.0f) != 0ull) {
                const float mn = tm > m + 1.0f ? tm + 1.0f : m, f = __builtin_amdgcn_exp2f(m - mn);
                m = mn;
                l *= f;
                z *= f;
                flush();
    #pragma unroll
                for (int j = 0; j < NV; ++j) {
                    acc[j] *= f;
                    low[j] *= f;
                }
                big = __ballot(fabsf(m) > kNearReference) != 0ull;
            }
            if (big) {
                asm volatile("");
#pragma unroll
                for (int i = 0; i < V; ++i) s[i] *= s_mul;
            }
            const float by = big ? 1.0f : s_mul;
            float top = 0.0f, vs[V];
    #pragma unroll
            for (int i = 0; i < V; ++i) {
                s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], by, -m));
                vs[i] = bf16_lo(vp[i]);
                top = fmaxf(top, vs[i]);
            }
            // a scale past the limit: the power of two moves, with two bits to spare
            if (__ballot(top >= limit) != 0ull && __ballot(top > 0.0f) != 0ull) {
                float w = max_rows_f32(top);
    #pragma unroll
                for (int o = 1; o < 16; o <<= 1) w = fmaxf(w, __shfl_xor(w, o));
                const int e = __builtin_amdgcn_frexp_expf(w) + 2;     // every scale below 2^(e - 2)
                const int n = 14 - e;
                if (limit > 0.0f) {
                    flush();
    #pragma unroll
                    for (int j = 0; j < NV; ++j)
    #pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            acc[j][i] = ldexpf(acc[j][i], n - v_exp);
                            low[j][i] = ldexpf(low[j][i], n - v_exp);
                        }
                }
                v_exp = n;
                limit = ldexpf(1.0f, e);
            }
            uint32_t ph[V / 2], pl[V / 2];
    #pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                const float x = s[2 * i] * ldexpf(vs[2 * i], v_exp), y = s[2 * i + 1] * ldexpf(vs[2 * i + 1], v_exp);
                const f16x2_t hx = __builtin_bit_cast(f16x2_t, __builtin_amdgcn_cvt_pkrtz(rintf(x), rintf(y)));
                const f32x2_t r = {fmaf(-1.0f, (float)hx[0], x), fmaf(-1.0f, (float)hx[1], y)};
                ph[i] = __builtin_bit_cast(uint32_t, hx);
                pl[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(r, f16x2_t));
            }
    #pragma unroll
            for (int i = 0; i < V; ++i) {
                z = fmaf(s[i], bf16_hi(vp[i]), z);
                l += s[i];
            }
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (decltype(more)::value) load_par(hn, a.c.v_par, vp);
            __builtin_amdgcn_sched_barrier(0);
            // positions 0 .. 3 of the operand are the lower half's, 4 .. 7 the upper half's
            u32x4_t bh, bl;
    #pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool mine = !PACK || (i >> 1) == upper;
                bh[i] = mine ? ph[i % (V / 2)] : 0u;
                bl[i] = mine ? pl[i % (V / 2)] : 0u;
            }
    #pragma unroll
            for (int w = 0; w < NV / 4; ++w) {
                uint32_t r[4][4];                                    // [code][pair of positions]
    #pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t x = __builtin_amdgcn_perm(vc[2 * i + 1], vc[2 * i], w ? 0x07060302u : 0x05040100u);
                    const uint32_t y = __builtin_amdgcn_perm(vc[2 * i + 1], vc[2 * i], w ? 0x06070203u : 0x04050001u);
                    r[0][i] = codes.pair(x);
                    r[1][i] = codes.pair(x << 4);
                    r[2][i] = codes.pair(y);
                    r[3][i] = codes.pair(y << 4);
                }
    #pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const f16x8_t x = __builtin_bit_cast(f16x8_t, u32x4_t{r[j][0], r[j][1], r[j][2], r[j][3]});
                    low[4 * w + j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, __builtin_bit_cast(f16x8_t, bl), low[4 * w + j], 0, 0, 0);
                    run[4 * w + j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, __builtin_bit_cast(f16x8_t, bh), run[4 * w + j], 0, 0, 0);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (decltype(more)::value) load_v(hn);
            __builtin_amdgcn_sched_barrier(0);
            if (it % kFlush == kFlush - 1) flush();
        };
        if (n_it > 0) {
            halves(0, h0);
            load_k(h0);
            load_par(h0, a.c.k_par, kp);
            load_par(h0, a.c.v_par, vp);
            load_v(h0);
            for (int it = 0; it + 1 < n_it; ++it) {
                halves(it + 1, h1);
                tile(it, h0, h1, std::true_type{});
                h0[0] = h1[0];
                h0[1] = h1[1];
            }
            tile(n_it - 1, h0, h0, std::false_type{});
            flush();
        }
        if constexpr (PACK) {
            l += row_ror_f32(l, 8);
            z += row_ror_f32(z, 8);
        }
        l = add16_f32(l, l);
        l = add32_f32(l, l);
        z = add16_f32(z, z);
        z = add32_f32(z, z);
        if (lane < 8 && gr == 0 && hc < a.group) s_join.sum(a, w, hc, m, l);
        // rows 4 kq + i of product j are elements (4 kq + i) * (D / 16) + j, right in the columns of
        // their own group
        const float f = s_join.factor(w, l);
        float *out = s_join.row(a, w, hc) + 4 * kq * (D / 16);
        const bool mine = !(PACK && col >= 8) && (NG == 1 || (kq >> 1) == gr) && hc < a.group;
    #pragma unroll
        for (int i = 0; i < 4; ++i)
    #pragma unroll
            for (int j0 = 0; j0 < NV; j0 += 4) {
                f32x4_t o;
    #pragma unroll
                for (int j = 0; j < 4; ++j) {
                    o[j] = ldexpf(acc[j0 + j][i] + low[j0 + j][i], kCodeExp - v_exp);
                    if constexpr (PACK) o[j] += row_ror_f32(o[j], 8);
                    o[j] = (o[j] + z) * f;
                }
                if (mine) *(f32x4_t *)(out + i * (D / 16) + j0) = o;
            }
        s_join.finish(a, w);
    });
}

// Joins the parts of a group: block = (token, query head), whose waves fold kMergeUnroll parts at
// a time, all of them read in one round trip, and are then joined themselves.  Bound by its launch and
// three dependent reads: 32 heads of 64 parts take 5.3 us, 896 of a few each 5.2.
constexpr int kMergeWaves = 16, kMergeUnroll = 16;
template <int D>
__global__ __launch_bounds__(kMergeWaves * 64) void k_attend_merge(AttendArgs a)
{
    constexpr int E = D / 64, U = kMergeUnroll;
    __shared__ float s_o[kMergeWaves][D];
    __shared__ float2 s_ml[kMergeWaves];
    const int64_t row = blockIdx.x, t = row / a.n_q;
    const int h = (int)(row % a.n_q), g = h / a.group;
    int64_t part;
    int nch;
    // parts `lead` .. lead + joints - 1 are blocks', every kAttendWaves-th number, the others waves'
    int lead = 0, joints = 0;
    if (a.split == ATTEND_BALANCED) {
        const int per = a.ends[a.n_tokens], empty = a.ends[a.n_tokens + 1], start = t > 0 ? a.ends[t - 1] : 0;
        const int tiles = (a.ends[t] - start) / a.c.n_kv_heads, from = start + g * tiles;
        const AttendParts p = attend_parts(from + empty, from + tiles, per);
        if (p.count == 1 && p.joints == 0) return;     // all in one wave, which wrote the output
        nch = p.count;
        lead = p.lead;
        joints = p.joints;
        part = p.first + t * a.c.n_kv_heads + g;
    } else {
        nch = (span_of(a, a.seq[t], a.pos[t]).tiles() + kAttendChunk / kAttendTile - 1) / (kAttendChunk / kAttendTile);
        part = (t * a.c.n_kv_heads + g) * a.chunks;
    }
    const int j = h - g * a.group;
    auto place = [&](int c) {
        const int extra = c < lead ? 0 : c < lead + joints ? c - lead : joints;
        return (part + c + extra * (kAttendWaves - 1)) * a.group + j;
    };
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, waves = blockDim.x >> 6;
    float m = -FLT_MAX, l = 0.0f, o[E] = {};
    for (int c0 = wave * U; c0 < nch; c0 += waves * U) {
        float2 x[U];
        float v[U][E];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = min(c0 + u, nch - 1);
            const int64_t at = place(c);
            x[u] = a.part_ml[at];
#pragma unroll
            for (int e = 0; e < E; ++e) v[u][e] = a.part_o[at * D + lane * E + e];
        }
        float mn = m;
#pragma unroll
        for (int u = 0; u < U; ++u) mn = fmaxf(mn, x[u].x);
        const float f = __builtin_amdgcn_exp2f(m - mn);
        m = mn;
        l *= f;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] *= f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float w = c0 + u < nch ? __builtin_amdgcn_exp2f(x[u].x - mn) : 0.0f;
            l = fmaf(w, x[u].y, l);
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = fmaf(w, v[u][e], o[e]);
        }
    }
#pragma unroll
    for (int e = 0; e < E; ++e) s_o[wave][lane * E + e] = o[e];
    if (lane == 0) s_ml[wave] = make_float2(m, l);
    __syncthreads();
    if (tid >= 64) return;
    for (int w = 0; w < waves; ++w) m = fmaxf(m, s_ml[w].x);
    l = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = 0.0f;
    for (int w = 0; w < waves; ++w) {
        const float f = __builtin_amdgcn_exp2f(s_ml[w].x - m);
        l = fmaf(f, s_ml[w].y, l);
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = fmaf(f, s_o[w][lane * E + e], o[e]);
    }
#pragma unroll
    for (int e = 0; e < E; ++e) a.out[row * D + lane * E + e] = l > 0.0f ? o[e] / l : 0.0f;
    if (lane == 0 && a.lse) a.lse[row] = l > 0.0f ? (m + log2f(l)) * kLn2 : -INFINITY;
}

template <int D> const void *attend_f32_kernel(int group)
{
    return group <= 1 ? (const void *)&k_attend<D, 1> : group <= 2 ? (const void *)&k_attend<D, 2>
           : group <= 4 ? (const void *)&k_attend<D, 4> : (const void *)&k_attend<D, 8>;
}
template <typename T> const void *attend4_kernel(int d, int group)
{
    if (d == 64) return (const void *)&k_attend4<T, 64, true>;
    return group <= 4 ? (const void *)&k_attend4<T, 128, true> : (const void *)&k_attend4<T, 128, false>;
}
template <int D> const void *attend_kernel(int format, int dtype, int group)
{
    if (format == RETOPK_PAGES_BF16)
        return group <= 4 ? (const void *)&k_attend16<D, 4> : (const void *)&k_attend16<D, 8>;
    if (format == RETOPK_PAGES_F32) return attend_f32_kernel<D>(group);
    return dtype == RETOPK_BF16 ? attend4_kernel<uint16_t>(D, group) : attend4_kernel<float>(D, group);
}

// Checks the arguments the workspace depends on and makes the plan.
retopk_status plan_of(const retopk_pages &c, int64_t n_tokens, int32_t n_q_heads, int64_t max_len, int64_t window,
                      AttendPlan *out)
{
    if (n_tokens < 0 || n_q_heads < 1 || max_len < 1 || window < 0) return RETOPK_ERR_ARG;
    if (n_q_heads % c.n_kv_heads != 0) return RETOPK_ERR_ARG;
    if (n_q_heads / c.n_kv_heads > 8) return RETOPK_ERR_UNSUPPORTED;
    const int64_t limit = (int64_t)1 << 31, rows = (int64_t)c.page_size * c.table_width;
    if (n_tokens >= limit || n_tokens * n_q_heads >= limit) return RETOPK_ERR_UNSUPPORTED;
    if (max_len > rows) max_len = rows;
    if (window > rows) window = 0;
    *out = attend_plan(n_tokens, n_q_heads, c.n_kv_heads, c.head_dim, max_len, window,
                       attend_slots(c.format, c.head_dim), c.format == RETOPK_PAGES_F32 ? kAttendDirectF32 : kAttendDirect);
    return out->waves < limit ? RETOPK_OK : RETOPK_ERR_UNSUPPORTED;
}

}  // namespace
}  // namespace retopk

using namespace retopk;

extern "C" {

int64_t paged_attention_workspace(const retopk_pages *c, int64_t n_tokens, int32_t n_q_heads, int64_t max_len,
                                  int64_t window)
{
    retopk_status st = check_pages(c, c && c->format == RETOPK_PAGES_F32 ? RETOPK_F32 : RETOPK_BF16);
    AttendPlan p;
    if (st == RETOPK_OK) st = plan_of(*c, n_tokens, n_q_heads, max_len, window, &p);
    return st == RETOPK_OK ? p.workspace : (int64_t)st;
}

retopk_status paged_attention(const retopk_pages *c, int32_t dtype, int64_t n_tokens, int32_t n_q_heads,
                              const int32_t *seq, const int32_t *pos, retopk_rows q, int64_t max_len, int64_t window,
                              float *out, float *lse, void *workspace, int64_t workspace_bytes, void *stream)
{
    retopk_status st = check_pages(c, dtype);
    if (st != RETOPK_OK) return st;
    AttendPlan p;
    if ((st = plan_of(*c, n_tokens, n_q_heads, max_len, window, &p)) != RETOPK_OK) return st;
    if (n_tokens == 0) return RETOPK_OK;
    const int d = c->head_dim;
    if (!seq || !pos || ((uintptr_t)seq & 3u) || ((uintptr_t)pos & 3u) || !out || !aligned16(out) ||
        (lse && ((uintptr_t)lse & 3u)))
        return RETOPK_ERR_ARG;
    if (!rows_ok(q, n_tokens, n_q_heads, d, dtype == RETOPK_BF16 ? 2 : 4, false)) return RETOPK_ERR_ARG;
    if (p.workspace > 0) {
        if (workspace_bytes < p.workspace) return RETOPK_ERR_TOO_LARGE;
        if (!workspace || !aligned16(workspace)) return RETOPK_ERR_ARG;
    }
    const int64_t rows = (int64_t)c->page_size * c->table_width;
    AttendArgs a = {};
    a.n_tokens = (int32_t)n_tokens;
    a.split = p.split;
    a.waves = (int32_t)p.waves;
    a.c = pages_args(*c);
    a.seq = seq;
    a.pos = pos;
    a.q = (const char *)q.p;
    a.q_ts = q.token_stride;
    a.q_hs = q.head_stride;
    a.n_q = n_q_heads;
    a.group = n_q_heads / c->n_kv_heads;
    a.max_len = (int32_t)(max_len < rows ? max_len : rows);
    a.window = window <= rows ? (int32_t)window : 0;
    a.chunks = p.split == ATTEND_DIRECT ? kAttendWaves : (int32_t)p.chunks;
    a.scale2 = (float)(1.44269504088896340736 / __builtin_sqrt((double)d));
    a.out = out;
    a.lse = lse;
    a.ends = (int32_t *)workspace;
    a.part_o = (float *)((char *)workspace + p.ends_bytes);
    a.part_ml = (float2 *)(a.part_o + p.parts * a.group * d);
    hipStream_t s = (hipStream_t)stream;
    void *args[1] = {&a};
    const void *f = d == 64 ? attend_kernel<64>(c->format, dtype, a.group) : attend_kernel<128>(c->format, dtype, a.group);
    if (hipLaunchKernel(f, dim3((unsigned)ceil_div(p.waves, kAttendWaves)), dim3(kAttendThreads), args, 0, s) != hipSuccess)
        return RETOPK_ERR_HIP;
    if (p.split != ATTEND_DIRECT) {
        f = d == 64 ? (const void *)&k_attend_merge<64> : (const void *)&k_attend_merge<128>;
        // waves for the parts of a group that is almost all there is, or of twice the mean one: more
        // would be idle in most blocks (32 sequences, 28 heads: 10.7 us with 9 waves a block)
        int64_t most = p.chunks;
        if (p.split == ATTEND_BALANCED) {
            most = ceil_div(p.waves, kAttendWaves * c->n_kv_heads) + 2 * kAttendWaves;
            const int64_t twice = 2 * ceil_div(p.waves, n_tokens * c->n_kv_heads) + 2 * kAttendWaves;
            most = most < twice ? most : twice;
        }
        const int64_t need = ceil_div(most, kMergeUnroll);
        const int64_t waves = need < kMergeWaves ? need : kMergeWaves;
        if (hipLaunchKernel(f, dim3((unsigned)(n_tokens * n_q_heads)), dim3((unsigned)(64 * waves)), args, 0, s) != hipSuccess)
            return RETOPK_ERR_HIP;
    }
    return RETOPK_OK;
}

}  // extern "C"
