// retopk_attend.hip -- paged_attention: full attention of single tokens over a paged cache.
//
// Block (chunk, KV head, token) folds its positions into a running maximum, sum and
// weighted value sum for every query head of the group; with more than one chunk a token,
// k_attend_merge joins the partial results.
#include "retopk.h"
#include "retopk_paged.h"

#include <cfloat>

namespace retopk {
namespace {

constexpr int kAttendThreads = 256;

struct AttendArgs {
    PagesArgs c;
    const int32_t *seq, *pos;
    const char *q;             // element strides
    int64_t q_ts, q_hs;
    int32_t n_q, group;        // query heads; of a KV head
    int32_t max_len, window;
    int32_t chunk_rows, chunks;
    float inv_sqrt_d;
    float *out, *lse;          // chunks == 1
    float *part_o;             // else [tokens * n_q, chunks, d]
    float2 *part_ml;           // [tokens * n_q, chunks]: maximum, sum
};

// The attended positions [first, len) of a token, len = 0 where there are none; chunk c
// begins at first rounded down to a tile, + c * chunk_rows.
struct Span {
    int first, len, base;
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

// Writes the result of a token's head, or of one of its chunks.
__device__ __forceinline__ void write_result(const AttendArgs &a, int64_t row, int chunk, int d, int e, float o,
                                             float m, float l)
{
    if (a.chunks == 1) {
        a.out[row * d + e] = l > 0.0f ? o / l : 0.0f;
        if (e == 0 && a.lse) a.lse[row] = l > 0.0f ? m + logf(l) : -INFINITY;
    } else {
        a.part_o[(row * a.chunks + chunk) * d + e] = o;
        if (e == 0) a.part_ml[row * a.chunks + chunk] = make_float2(m, l);
    }
}

// The plain kernel: D / 8 lanes a row, every position's scores, maximum and weights in
// turn.  GP >= a.group heads; those past the group repeat its first.
template <typename T, int D, int GP, int FMT>
__global__ __launch_bounds__(kAttendThreads) void k_attend(AttendArgs a)
{
    constexpr int LPR = D / 8, SLOTS = kAttendThreads / LPR, NW = kAttendThreads / 64;
    __shared__ float s_m[NW][GP], s_l[NW][GP], s_o[NW][GP][D];
    const int chunk = blockIdx.x % a.chunks, bg = blockIdx.x / a.chunks;
    const int g = bg % a.c.n_kv_heads;
    const int64_t t = bg / a.c.n_kv_heads;
    const int32_t sq = a.seq[t];
    const Span sp = span_of(a, sq, a.pos[t]);
    const int lo = sp.base + chunk * a.chunk_rows, hi = min(sp.len, lo + a.chunk_rows);
    if (lo >= hi && !(chunk == 0 && a.chunks == 1)) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, e0 = tid % LPR * 8;

    float q[GP][8], acc[GP][8], m[GP], l[GP];
#pragma unroll
    for (int j = 0; j < GP; ++j) {
        const int h = g * a.group + (j < a.group ? j : 0);
        Oct<T> v;
        v.load((const T *)a.q + t * a.q_ts + h * a.q_hs + e0);
        v.get(q[j]);
        m[j] = -FLT_MAX;
        l[j] = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[j][i] = 0.0f;
    }
    for (int r = max(lo, sp.first) + tid / LPR; r < hi; r += SLOTS) {
        const int64_t row = row_of(a.c, sq, r, g);
        if (row < 0) continue;
        float k[8], v[8];
        if constexpr (FMT == RETOPK_PAGES_Q4) {
            const int64_t w = row * (D / 8) + e0 / 8, par = row * (D / kGroup4) + e0 / kGroup4;
            values4(((const uint32_t *)a.c.k)[w], a.c.k_par[par], k);
            values4(((const uint32_t *)a.c.v)[w], a.c.v_par[par], v);
        } else {
            Oct<T> x, y;
            x.load((const T *)a.c.k + row * D + e0);
            y.load((const T *)a.c.v + row * D + e0);
            x.get(k);
            y.get(v);
        }
#pragma unroll
        for (int j = 0; j < GP; ++j) {
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) s = fmaf(q[j][i], k[i], s);
#pragma unroll
            for (int o = LPR / 2; o > 0; o >>= 1) s += __shfl_xor(s, o);
            s *= a.inv_sqrt_d;
            const float mn = fmaxf(m[j], s), f = expf(m[j] - mn), p = expf(s - mn);
            m[j] = mn;
            l[j] = l[j] * f + p;
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[j][i] = fmaf(p, v[i], acc[j][i] * f);
        }
    }
    // the wave's slots, then the waves
#pragma unroll
    for (int j = 0; j < GP; ++j) {
#pragma unroll
        for (int o = LPR; o < 64; o <<= 1) {
            const float m2 = __shfl_xor(m[j], o), l2 = __shfl_xor(l[j], o), mn = fmaxf(m[j], m2);
            const float f = expf(m[j] - mn), f2 = expf(m2 - mn);
            m[j] = mn;
            l[j] = l[j] * f + l2 * f2;
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[j][i] = acc[j][i] * f + __shfl_xor(acc[j][i], o) * f2;
        }
        if (lane < LPR) {
#pragma unroll
            for (int i = 0; i < 8; ++i) s_o[wave][j][e0 + i] = acc[j][i];
            s_m[wave][j] = m[j];
            s_l[wave][j] = l[j];
        }
    }
    __syncthreads();
    for (int i = tid; i < a.group * D; i += kAttendThreads) {
        const int j = i / D, e = i % D;
        float mx = s_m[0][j], o = 0.0f, ls = 0.0f;
#pragma unroll
        for (int w = 1; w < NW; ++w) mx = fmaxf(mx, s_m[w][j]);
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float f = expf(s_m[w][j] - mx);
            o += f * s_o[w][j][e];
            ls += f * s_l[w][j];
        }
        write_result(a, t * a.n_q + g * a.group + j, chunk, D, e, o, mx, ls);
    }
}

// Joins a token's chunks: block = (token, query head).
template <int D>
__global__ __launch_bounds__(kAttendThreads) void k_attend_merge(AttendArgs a)
{
    constexpr int P = kAttendThreads / D, NW = kAttendThreads / 64;
    __shared__ float s_red[NW], s_o[P][D], s_l[P];
    const int64_t row = blockIdx.x, t = row / a.n_q;
    const Span sp = span_of(a, a.seq[t], a.pos[t]);
    const int nch = (sp.len - sp.base + a.chunk_rows - 1) / a.chunk_rows;
    const int tid = threadIdx.x, e = tid % D, part = tid / D;
    const float2 *ml = a.part_ml + row * a.chunks;
    float m = -FLT_MAX;
    for (int c = tid; c < nch; c += kAttendThreads) m = fmaxf(m, ml[c].x);
    m = block_reduce<kAttendThreads>(m, s_red, [](float x, float y) { return fmaxf(x, y); });
    float o = 0.0f, l = 0.0f;
    for (int c = part; c < nch; c += P) {
        const float2 x = ml[c];
        const float f = expf(x.x - m);
        l = fmaf(f, x.y, l);
        o = fmaf(f, a.part_o[(row * a.chunks + c) * D + e], o);
    }
    s_o[part][e] = o;
    if (e == 0) s_l[part] = l;
    __syncthreads();
    if (part == 0) {
#pragma unroll
        for (int p = 1; p < P; ++p) {
            o += s_o[p][e];
            l += s_l[p];
        }
        a.out[row * D + e] = l > 0.0f ? o / l : 0.0f;
        if (e == 0 && a.lse) a.lse[row] = l > 0.0f ? m + logf(l) : -INFINITY;
    }
}

template <typename T, int D, int FMT> const void *attend_kernel(int group)
{
    return group <= 1 ? (const void *)&k_attend<T, D, 1, FMT> : group <= 2 ? (const void *)&k_attend<T, D, 2, FMT>
           : group <= 4 ? (const void *)&k_attend<T, D, 4, FMT> : (const void *)&k_attend<T, D, 8, FMT>;
}
template <int D> const void *attend_kernel(int format, int dtype, int group)
{
    if (format == RETOPK_PAGES_BF16) return attend_kernel<uint16_t, D, RETOPK_PAGES_BF16>(group);
    if (format == RETOPK_PAGES_F32) return attend_kernel<float, D, RETOPK_PAGES_F32>(group);
    return dtype == RETOPK_BF16 ? attend_kernel<uint16_t, D, RETOPK_PAGES_Q4>(group)
                                : attend_kernel<float, D, RETOPK_PAGES_Q4>(group);
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
    *out = attend_plan(n_tokens, n_q_heads, c.n_kv_heads, c.head_dim, max_len, window);
    return out->blocks < limit ? RETOPK_OK : RETOPK_ERR_UNSUPPORTED;
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
    a.chunk_rows = (int32_t)p.chunk_rows;
    a.chunks = (int32_t)p.chunks;
    a.inv_sqrt_d = (float)(1.0 / __builtin_sqrt((double)d));
    a.out = out;
    a.lse = lse;
    a.part_o = (float *)workspace;
    a.part_ml = (float2 *)((float *)workspace + n_tokens * n_q_heads * p.chunks * d);
    hipStream_t s = (hipStream_t)stream;
    void *args[1] = {&a};
    const void *f = d == 64 ? attend_kernel<64>(c->format, dtype, a.group) : attend_kernel<128>(c->format, dtype, a.group);
    if (hipLaunchKernel(f, dim3((unsigned)p.blocks), dim3(kAttendThreads), args, 0, s) != hipSuccess)
        return RETOPK_ERR_HIP;
    if (p.chunks > 1) {
        f = d == 64 ? (const void *)&k_attend_merge<64> : (const void *)&k_attend_merge<128>;
        if (hipLaunchKernel(f, dim3((unsigned)(n_tokens * n_q_heads)), dim3(kAttendThreads), args, 0, s) != hipSuccess)
            return RETOPK_ERR_HIP;
    }
    return RETOPK_OK;
}

}  // extern "C"
