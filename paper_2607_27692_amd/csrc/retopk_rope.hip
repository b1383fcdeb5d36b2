// retopk_rope.hip -- rotary positions, and rows into and out of the paged cache:
// retopk_rope_init, rotary_embed, paged_append, paged_gather, and the argument checks of
// the paged calls.
//
// All three kernels stream: 8 elements of a row to a lane (16 bytes of bf16), D / 8 lanes
// to a row, 256 / (D / 8) tokens to a block, which walks over some of the heads with its
// tokens' cosines and sines in registers.  Consecutive tokens of one head lie side by side
// in a page, so a block's writes of 4-bit rows are whole lines.  Bound by HBM, where a copy reaches
// 4.7 TB/s: 8K tokens of 40 heads of 128 rotate in 39 us (168 MB, 4.3 TB/s); 16K tokens of 32 query and
// 8 KV heads go to 4-bit pages in 84 (355 MB, 4.2); 64K rows of 8 heads are read back in 53 (344 MB,
// most of it written, 6.5).  One token takes 4 to 5, 5.6 and 2.9 us.
#include "retopk.h"
#include "retopk_paged.h"

#include <cmath>

namespace retopk {

retopk_status check_pages(const retopk_pages *c, int32_t dtype)
{
    if (!c) return RETOPK_ERR_ARG;
    if (dtype != RETOPK_F32 && dtype != RETOPK_BF16) return RETOPK_ERR_ARG;
    if (c->format != RETOPK_PAGES_F32 && c->format != RETOPK_PAGES_BF16 && c->format != RETOPK_PAGES_Q4)
        return RETOPK_ERR_ARG;
    if (c->n_kv_heads < 1 || c->head_dim < 1 || c->page_size < 1 || c->n_pages < 1 || c->n_seqs < 1 ||
        c->table_width < 1)
        return RETOPK_ERR_ARG;
    if (!c->k || !c->v || !c->table || !aligned16(c->k) || !aligned16(c->v) || ((uintptr_t)c->table & 3u))
        return RETOPK_ERR_ARG;
    if (c->format == RETOPK_PAGES_Q4 &&
        (!c->k_par || !c->v_par || !aligned16(c->k_par) || !aligned16(c->v_par)))
        return RETOPK_ERR_ARG;
    if (c->head_dim != 64 && c->head_dim != 128) return RETOPK_ERR_UNSUPPORTED;
    if (c->format == RETOPK_PAGES_F32 && dtype != RETOPK_F32) return RETOPK_ERR_UNSUPPORTED;
    if (c->format == RETOPK_PAGES_BF16 && dtype != RETOPK_BF16) return RETOPK_ERR_UNSUPPORTED;
    if (c->format == RETOPK_PAGES_Q4 && c->page_size % 16 != 0) return RETOPK_ERR_UNSUPPORTED;
    const int64_t limit = (int64_t)1 << 31, heads = (int64_t)c->n_kv_heads * c->page_size;
    if (heads >= limit || heads * c->n_pages >= limit) return RETOPK_ERR_UNSUPPORTED;
    if ((int64_t)c->page_size * c->table_width >= limit) return RETOPK_ERR_UNSUPPORTED;
    return RETOPK_OK;
}

PagesArgs pages_args(const retopk_pages &c)
{
    PagesArgs a = {};
    a.k = (char *)c.k;
    a.v = (char *)c.v;
    a.k_par = c.k_par;
    a.v_par = c.v_par;
    a.table = c.table;
    a.n_kv_heads = c.n_kv_heads;
    a.page_size = c.page_size;
    a.n_pages = c.n_pages;
    a.n_seqs = c.n_seqs;
    a.table_width = c.table_width;
    a.by_page = divisor_of(c.page_size);
    return a;
}

bool rows_ok(const retopk_rows &x, int64_t tokens, int64_t heads, int d, int es, bool written)
{
    if (!x.p || !aligned16(x.p) || x.token_stride < 0 || x.head_stride < 0) return false;
    const int64_t per = 16 / es;
    if (x.token_stride % per || x.head_stride % per) return false;
    if (!written) return true;
    if (heads > 1 && x.head_stride < d) return false;
    if (tokens > 1 && x.token_stride < d) return false;
    // one dimension's rows lie between those of the other, or after all of them
    return tokens <= 1 || heads <= 1 || x.token_stride >= (heads - 1) * x.head_stride + d ||
           x.head_stride >= (tokens - 1) * x.token_stride + d;
}

namespace {

constexpr int kRowThreads = 256;
// Blocks that run at once on 256 CUs, four on each by the registers, five of those that put bf16 rows
// into bf16 pages.  A few more than that cost a second round: 4099 tokens of 16 heads of 64, f32, rotate in
// 9.7 us in 774 blocks and in 10.9 in 1032; 5 prompts in bf16 are appended in 21.4 us in 1280, in 22.5 in 960.
constexpr int64_t kRowBlocks = 1024, kRowBlocksBf16 = 1280;
constexpr int64_t kMaxGrid = ((int64_t)1 << 31) - 1;

bool rope_ok(const retopk_rope *r, int d)
{
    if (r->rot_dim < 2 || r->rot_dim > d || r->rot_dim % 2 || (r->interleaved != 0 && r->interleaved != 1) ||
        !std::isfinite(r->factor))
        return false;
    for (int i = 0; i < r->rot_dim / 2; ++i)
        if (!std::isfinite(r->freq[i])) return false;
    return true;
}

// Strided rows of T on the device.
template <typename T> struct Rows {
    T *p;
    int64_t ts, hs;
    __device__ __forceinline__ T *at(int64_t t, int h) const { return p + t * ts + h * hs; }
};
template <typename T> Rows<T> rows_of(const retopk_rows &x) { return Rows<T>{(T *)x.p, x.token_stride, x.head_stride}; }

// ---------------------------------------------------------------------------
// The rotation of one lane's 8 elements
// ---------------------------------------------------------------------------

// sin and cos of x in float64: x less a multiple n of pi/2 (its nearest double and the rest of
// it, each times n in one rounding), then the Taylor series about 0, whose first terms left out
// are below 2^-58 for |r| <= pi/4; the quadrant n mod 4 says which of the two is which.  Past
// 2^28, where n times the rest of pi/2 would no longer be small, the library's.
__device__ __forceinline__ void angle(double x, double &s, double &c)
{
    if (!(fabs(x) < 268435456.0)) {
        sincos(x, &s, &c);
        return;
    }
    const double n = rint(x * 0.63661977236758134308);
    double r = fma(-n, 1.5707963267948965580, x);
    r = fma(-n, 6.1232339957367658861e-17, r);
    const double z = r * r;
    double p = 1.0 / 355687428096000.0;                        // 1 / 17!
    p = fma(p, z, -1.0 / 1307674368000.0);
    p = fma(p, z, 1.0 / 6227020800.0);
    p = fma(p, z, -1.0 / 39916800.0);
    p = fma(p, z, 1.0 / 362880.0);
    p = fma(p, z, -1.0 / 5040.0);
    p = fma(p, z, 1.0 / 120.0);
    p = fma(p, z, -1.0 / 6.0);
    const double sr = fma(p * z, r, r);
    double q = 1.0 / 20922789888000.0;                         // 1 / 16!
    q = fma(q, z, -1.0 / 87178291200.0);
    q = fma(q, z, 1.0 / 479001600.0);
    q = fma(q, z, -1.0 / 3628800.0);
    q = fma(q, z, 1.0 / 40320.0);
    q = fma(q, z, -1.0 / 720.0);
    q = fma(q, z, 1.0 / 24.0);
    q = fma(q, z, -0.5);
    const double cr = fma(q, z, 1.0);
    const int k = (int)n;
    s = k & 1 ? cr : sr;
    c = k & 1 ? sr : cr;
    if (k & 2) s = -s;
    if ((k + 1) & 2) c = -c;
}

// Cosines and sines of a block's tokens, a few angles a thread: pos * freq in float64, which
// keeps every bit that float32 results show at any position.  The positions are read apart, before
// the first rows: loads return in order, and the angles would wait for the rows.
template <int D> struct Angles {
    static constexpr int TT = kRowThreads * 8 / D, N = TT * (D / 2) / kRowThreads;
    int32_t p[N];

    static __device__ __forceinline__ int token(int k) { return (threadIdx.x + k * kRowThreads) / (D / 2); }
    __device__ __forceinline__ void read(const int32_t *pos, int64_t t0, int64_t n)
    {
#pragma unroll
        for (int k = 0; k < N; ++k) p[k] = pos[min(t0 + token(k), n - 1)];
        __builtin_amdgcn_sched_barrier(0);
    }
    __device__ __forceinline__ void make(const retopk_rope &r, bool inverse, double2 *s_cs) const
    {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int i = threadIdx.x + k * kRowThreads, pair = i % (D / 2);
            if (pair < r.rot_dim / 2) {
                double s, c;
                angle((double)p[k] * r.freq[pair], s, c);
                s_cs[i] = make_double2(c * r.factor, (inverse ? -s : s) * r.factor);
            }
        }
    }
};

// A lane's elements e0 .. e0 + 7 of rows of one token: element i becomes
// x[i] * c[i] + partner * s[i], the partner being the other element of its pair.
template <typename T, int D> struct Turn {
    double c[8], s[8];
    int e0, half, rot, other;  // other: where the partners of a whole lane begin
    bool inside, lanes;        // partners in the lane itself; or all in one other lane

    __device__ __forceinline__ void place(const retopk_rope &r, int lane_e0)
    {
        e0 = lane_e0;
        rot = r.rot_dim;
        half = rot / 2;
        inside = r.interleaved != 0;
        lanes = !inside && half % 8 == 0;
        other = e0 < half ? e0 + half : e0 < rot ? e0 - half : e0;
    }
    __device__ __forceinline__ void angles(const double2 *cs)
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = e0 + i;
            c[i] = 1.0;
            s[i] = 0.0;
            if (e < rot) {
                const int pair = inside ? e / 2 : (e < half ? e : e - half);
                const bool first = inside ? (e % 2 == 0) : e < half;
                const double2 v = cs[pair];
                c[i] = v.x;
                s[i] = first ? -v.y : v.y;
            }
        }
    }
    __device__ __forceinline__ void turn(const T *row, const Oct<T> &partner, float (&x)[8]) const
    {
        float y[8];
        if (inside) {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = x[i ^ 1];
        } else if (lanes) {
            partner.get(y);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int e = e0 + i;
                y[i] = Oct<T>::one(row + (e < half ? e + half : e < rot ? e - half : e));
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float z = (float)fma((double)x[i], c[i], (double)y[i] * s[i]);
            x[i] = e0 + i < rot ? z : x[i];
        }
    }
};

// Walks a token's rows first .. last - 1, from `begin` on and round to it, kAhead of them loaded
// ahead of their use, the first ones by start(), before the angles are there: at(h) is row h, and f(h, x)
// takes its elements, turned if h < n_rot.  In place: a row's lanes are in one wave, and its loads,
// partners included, have all returned before its stores.
constexpr int kAhead = 2;
template <typename T, int D, typename At> struct Walk {
    Turn<T, D> turn;
    int e0, first, last, begin, n_rot;
    At at;
    Oct<T> own[kAhead], partner[kAhead];

    __device__ __forceinline__ int nth(int i) const
    {
        const int count = last - first, h = begin + min(i, count - 1);
        return h < last ? h : h - count;
    }
    __device__ __forceinline__ void load(int i, int u)
    {
        const int h = nth(i);
        const T *row = at(h);
        own[u].load(row + e0);
        if (h < n_rot && turn.lanes) partner[u].load(row + turn.other);
    }
    __device__ __forceinline__ void start(const retopk_rope &r)
    {
        turn.place(r, e0);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) load(u, u);
    }
    template <typename F> __device__ __forceinline__ void run(F f)
    {
        const int count = last - first;
        for (int i0 = 0; i0 < count; i0 += kAhead) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int h = nth(i0 + u);
                if (i0 + u < count) {
                    float x[8];
                    own[u].get(x);
                    if (h < n_rot) turn.turn(at(h), partner[u], x);
                    __builtin_amdgcn_sched_barrier(0);
                    load(i0 + u + kAhead, u);
                    __builtin_amdgcn_sched_barrier(0);
                    f(h, x);
                }
            }
        }
    }
};
template <typename T, int D, typename At>
__device__ __forceinline__ Walk<T, D, At> walk_of(int e0, int first, int last, int begin, int n_rot, At at)
{
    return Walk<T, D, At>{{}, e0, first, last, begin, n_rot, at, {}, {}};
}

// rotary_embed.  Block (x, y): tokens x * TT .., heads y * per_block ..
template <typename T, int D>
__global__ __launch_bounds__(kRowThreads) void k_rotary(retopk_rope r, Rows<T> x, Rows<T> out, const int32_t *pos,
                                                        int64_t n, int heads, int per_block, int inverse)
{
    constexpr int LPR = D / 8, TT = kRowThreads / LPR;
    __shared__ double2 s_cs[TT][D / 2];
    const int64_t t0 = (int64_t)blockIdx.x * TT;
    const int tok = threadIdx.x / LPR, e0 = threadIdx.x % LPR * 8;
    const int64_t t = min(t0 + tok, n - 1);            // lanes past the last token only read
    const int h0 = blockIdx.y * per_block, h1 = min(heads, h0 + per_block);
    auto walk = walk_of<T, D>(e0, h0, h1, h0, heads, [&](int h) { return (const T *)x.at(t, h); });
    Angles<D> angles;
    angles.read(pos, t0, n);
    walk.start(r);
    angles.make(r, inverse != 0, &s_cs[0][0]);
    __syncthreads();
    if (t0 + tok >= n) return;
    walk.turn.angles(s_cs[tok]);
    walk.run([&](int h, const float (&v)[8]) { Oct<T>::store(out.at(t, h) + e0, v); });
}

// ---------------------------------------------------------------------------
// Rows into the cache
// ---------------------------------------------------------------------------

// A lane's 8 elements as codes of its group (8 lanes side by side); the parameter word is
// the same in every lane of the group.  mid and scale are rounded to bf16, the nearest
// steps at half the bytes of float32.  With a = |x - mid| / scale the magnitude is the whole part
// of a, and for x below mid the largest whole number below a, so that the levels are half open:
// a is taken 2^-48 too small there and 2^-48 too large above, more than its roundings and less
// than the distance of a quotient of these types from a whole number it does not equal.
__device__ __forceinline__ void quantise4(const float (&x)[8], uint32_t &codes, uint32_t &par)
{
    float top = x[0], low = x[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) {
        top = fmaxf(top, x[i]);
        low = fminf(low, x[i]);
    }
    top = fmaxf(top, dpp_f32<kQuadXor1>(top));
    low = fminf(low, dpp_f32<kQuadXor1>(low));
    top = fmaxf(top, dpp_f32<kQuadXor2>(top));
    low = fminf(low, dpp_f32<kQuadXor2>(low));
    top = fmaxf(top, dpp_f32<kHalfMirror>(top));
    low = fminf(low, dpp_f32<kHalfMirror>(low));
    const uint32_t mid_b = bf16_bits((float)(((double)top + (double)low) * 0.5));
    const double mid = (double)__uint_as_float(mid_b << 16);
    const double up = (double)top - mid, down = mid - (double)low;
    const uint32_t scale_b = bf16_bits((float)((up > down ? up : down) * (1.0 / 7.5)));
    const double scale = (double)__uint_as_float(scale_b << 16);
    par = scale_b | (mid_b << 16);
    // 1 / scale by two Newton steps, 2^-48 too small; scale 0: 0, any code stands for mid
    double inv = scale > 0.0 ? __builtin_amdgcn_rcp(scale) : 0.0;
    inv = fma(fma(-scale, inv, 1.0), inv, inv);
    inv = fma(fma(-scale, inv, 1.0), inv, inv) * (1.0 - 0x1p-48);
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const double d = (double)x[i] - mid;
        const bool below = d < 0.0;
        const double a = fabs(d) * inv * (below ? 1.0 : 1.0 + 0x1p-47);
        const uint32_t m = min((uint32_t)a, 7u);
        // elements 0 .. 3 of a half-word: magnitude and sign bit places
        const int mp[4] = {4, 0, 12, 8}, sp[4] = {15, 11, 7, 3};
        w[i >> 2] |= (m << mp[i & 3]) | (below ? 1u << sp[i & 3] : 0u);
    }
    codes = w[0] | (w[1] << 16);
}

template <int FMT, int D, bool STREAM>
__device__ __forceinline__ void store_row(const PagesArgs &c, bool key, int32_t row, int e0, const float (&x)[8])
{
    if constexpr (FMT == RETOPK_PAGES_Q4) {
        uint32_t codes, par;
        quantise4(x, codes, par);
        if (row < 0) return;
        char *base = key ? c.k : c.v;
        uint32_t *pars = key ? c.k_par : c.v_par;
        put<STREAM>((uint32_t *)(base + (int64_t)row * (D / 2) + e0 / 2), codes);
        if (e0 % kGroup4 == 0) pars[(int64_t)row * (D / kGroup4) + e0 / kGroup4] = par;
    } else if constexpr (FMT == RETOPK_PAGES_BF16) {
        if (row >= 0) Oct<uint16_t>::store<STREAM>((uint16_t *)(key ? c.k : c.v) + (int64_t)row * D + e0, x);
    } else {
        if (row >= 0) Oct<float>::store<STREAM>((float *)(key ? c.k : c.v) + (int64_t)row * D + e0, x);
    }
}

// paged_append.  The heads a block walks over: queries, then keys, then values.
template <typename T, int D, int FMT, bool STREAM>
__global__ __launch_bounds__(kRowThreads) void k_append(PagesArgs c, retopk_rope r, int rotate, Rows<T> k, Rows<T> v,
                                                        Rows<T> q, Rows<T> q_out, const int32_t *seq,
                                                        const int32_t *pos, int64_t n, int n_q, int per_block)
{
    constexpr int LPR = D / 8, TT = kRowThreads / LPR;
    __shared__ double2 s_cs[TT][D / 2];
    const int64_t t0 = (int64_t)blockIdx.x * TT;
    const int heads = n_q + 2 * c.n_kv_heads, h0 = blockIdx.y * per_block;
    const int h1 = min(heads, h0 + per_block), n_rot = rotate ? n_q + c.n_kv_heads : 0;
    const int tok = threadIdx.x / LPR, e0 = threadIdx.x % LPR * 8;
    const int64_t t = min(t0 + tok, n - 1);            // lanes past the last token only read
    // blocks begin a quarter of their heads apart, so that some write queries while others are
    // busy with codes
    auto walk = walk_of<T, D>(e0, h0, h1, h0 + (int)(blockIdx.x & 3) * (h1 - h0) / 4, n_rot, [&](int h) {
        return (const T *)(h < n_q ? q.at(t, h) : h < n_q + c.n_kv_heads ? k.at(t, h - n_q) : v.at(t, h - n_q - c.n_kv_heads));
    });
    const int32_t s = seq[t], p = pos[t];
    Angles<D> angles;
    if (h0 < n_rot) angles.read(pos, t0, n);
    walk.start(r);
    if (h0 < n_rot) angles.make(r, false, &s_cs[0][0]);
    const int32_t row0 = row_of(c, s, p, 0);
    __syncthreads();
    if (t0 + tok >= n || s < 0 || s >= c.n_seqs) return;
    if (h0 < n_rot) walk.turn.angles(s_cs[tok]);
    walk.run([&](int h, const float (&x)[8]) {
        if (h < n_q) {
            Oct<T>::store(q_out.at(t, h) + e0, x);
        } else {
            const bool key = h < n_q + c.n_kv_heads;
            const int g = h - n_q - (key ? 0 : c.n_kv_heads);
            store_row<FMT, D, STREAM>(c, key, row0 < 0 ? -1 : row0 + g * c.page_size, e0, x);
        }
    });
}

// paged_gather.
template <typename T, int D, int FMT, bool STREAM>
__global__ __launch_bounds__(kRowThreads) void k_gather(PagesArgs c, Rows<T> k, Rows<T> v, const int32_t *seq,
                                                        const int32_t *pos, int64_t n, int per_block)
{
    constexpr int LPR = D / 8, TT = kRowThreads / LPR;
    const int64_t t = (int64_t)blockIdx.x * TT + threadIdx.x / LPR;
    const int e0 = threadIdx.x % LPR * 8;
    if (t >= n) return;
    const int32_t row0 = row_of(c, seq[t], pos[t], 0);
    if (row0 < 0) return;
    const int h0 = blockIdx.y * per_block, h1 = min(2 * c.n_kv_heads, h0 + per_block);
    for (int h = h0; h < h1; ++h) {
        const bool key = h < c.n_kv_heads;
        const int g = key ? h : h - c.n_kv_heads;
        const Rows<T> &to = key ? k : v;
        if (!to.p) continue;
        const int64_t row = row0 + (int64_t)g * c.page_size;
        float x[8];
        if constexpr (FMT == RETOPK_PAGES_Q4) {
            const uint32_t codes = *(const uint32_t *)((key ? c.k : c.v) + row * (D / 2) + e0 / 2);
            values4(codes, (key ? c.k_par : c.v_par)[row * (D / kGroup4) + e0 / kGroup4], x);
        } else if constexpr (FMT == RETOPK_PAGES_BF16) {
            Oct<uint16_t> o;
            o.load((const uint16_t *)(key ? c.k : c.v) + row * D + e0);
            o.get(x);
        } else {
            Oct<float> o;
            o.load((const float *)(key ? c.k : c.v) + row * D + e0);
            o.get(x);
        }
        Oct<T>::template store<STREAM>(to.at(t, g) + e0, x);
    }
}

// Grid of `heads` heads of n tokens, TT tokens to a block: the heads are shared out evenly over
// grid.y, as far as all blocks run at once, or to one a head.
struct RowGrid {
    dim3 grid;
    int per_block;
};
bool row_grid(int64_t n, int d, int64_t heads, int64_t blocks, RowGrid *out)
{
    const int64_t tiles = ceil_div(n, kRowThreads * 8 / d);
    if (tiles > kMaxGrid || heads > 65535) return false;
    int64_t shares = blocks / tiles;
    shares = shares < 1 ? 1 : shares > heads ? heads : shares;
    const int64_t per = ceil_div(heads, shares);
    out->per_block = (int)per;
    out->grid = dim3((unsigned)tiles, (unsigned)ceil_div(heads, per));
    return true;
}

// Rows that later steps read, not the next kernel, go past the caches once they are more than
// the L2s hold together.  What the next kernel reads does not (rotated queries, where a reader
// right after takes 1 to 4 % longer in all than with plain stores).
constexpr int64_t kStreamBytes = (int64_t)32 << 20;

retopk_status launched() { return hipGetLastError() == hipSuccess ? RETOPK_OK : RETOPK_ERR_HIP; }

template <typename T, int D>
void launch_append(int format, bool stream, const RowGrid &g, hipStream_t s, const PagesArgs &c, const retopk_rope &r, int rotate,
                   const retopk_rows &k, const retopk_rows &v, const retopk_rows &q, const retopk_rows &q_out,
                   const int32_t *seq, const int32_t *pos, int64_t n, int n_q)
{
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, g.grid, dim3(kRowThreads), 0, s, c, r, rotate, rows_of<T>(k), rows_of<T>(v),
                           rows_of<T>(q), rows_of<T>(q_out), seq, pos, n, n_q, g.per_block);
    };
    constexpr int own = sizeof(T) == 2 ? RETOPK_PAGES_BF16 : RETOPK_PAGES_F32;
    if (format == RETOPK_PAGES_Q4) stream ? go(k_append<T, D, RETOPK_PAGES_Q4, true>) : go(k_append<T, D, RETOPK_PAGES_Q4, false>);
    else stream ? go(k_append<T, D, own, true>) : go(k_append<T, D, own, false>);
}

template <typename T, int D>
void launch_gather(int format, bool stream, const RowGrid &g, hipStream_t s, const PagesArgs &c, const retopk_rows &k,
                   const retopk_rows &v, const int32_t *seq, const int32_t *pos, int64_t n)
{
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, g.grid, dim3(kRowThreads), 0, s, c, rows_of<T>(k), rows_of<T>(v), seq, pos, n,
                           g.per_block);
    };
    constexpr int own = sizeof(T) == 2 ? RETOPK_PAGES_BF16 : RETOPK_PAGES_F32;
    if (format == RETOPK_PAGES_Q4) stream ? go(k_gather<T, D, RETOPK_PAGES_Q4, true>) : go(k_gather<T, D, RETOPK_PAGES_Q4, false>);
    else stream ? go(k_gather<T, D, own, true>) : go(k_gather<T, D, own, false>);
}

// Runs f with the element type of dtype and the head dimension as types.
template <typename F> void by_type(int dtype, int d, F f)
{
    if (dtype == RETOPK_BF16) {
        if (d == 64) f((uint16_t)0, std::integral_constant<int, 64>{});
        else f((uint16_t)0, std::integral_constant<int, 128>{});
    } else {
        if (d == 64) f(0.0f, std::integral_constant<int, 64>{});
        else f(0.0f, std::integral_constant<int, 128>{});
    }
}

}  // namespace
}  // namespace retopk

using namespace retopk;

extern "C" {

retopk_status retopk_rope_init(retopk_rope *r, int32_t rot_dim, int32_t interleaved, double theta,
                               const retopk_rope_scaling *scaling)
{
    if (!r || rot_dim < 2 || rot_dim > 128 || rot_dim % 2 || (interleaved != 0 && interleaved != 1))
        return RETOPK_ERR_ARG;
    if (!std::isfinite(theta) || !(theta > 1.0)) return RETOPK_ERR_ARG;
    const int kind = scaling ? scaling->kind : (int)RETOPK_ROPE_PLAIN;
    if (kind < RETOPK_ROPE_PLAIN || kind > RETOPK_ROPE_RAMP) return RETOPK_ERR_ARG;
    const double two_pi = 6.283185307179586476925286766559;
    double f = 1.0, n0 = 0.0, low = 0.0, high = 0.0;
    if (kind != RETOPK_ROPE_PLAIN) {
        f = scaling->factor;
        if (!std::isfinite(f) || !(f >= 1.0)) return RETOPK_ERR_ARG;
    }
    if (kind == RETOPK_ROPE_NTK) {
        if (rot_dim <= 2) return RETOPK_ERR_ARG;
        theta = theta * std::pow(f, (double)rot_dim / (rot_dim - 2));
        if (!std::isfinite(theta)) return RETOPK_ERR_ARG;
    }
    double first = 0.0, last = 0.0, size = 1.0;
    if (kind == RETOPK_ROPE_BANDS || kind == RETOPK_ROPE_RAMP) {
        n0 = scaling->original_len;
        low = scaling->low;
        high = scaling->high;
        if (!std::isfinite(n0) || !(n0 > 0.0) || !std::isfinite(high) || !(low > 0.0) || !(high > low))
            return RETOPK_ERR_ARG;
    }
    if (kind == RETOPK_ROPE_RAMP) {
        // the pair that makes `turns` turns over the trained context, as a real index
        auto index = [&](double turns) { return rot_dim * std::log(n0 / (turns * two_pi)) / (2.0 * std::log(theta)); };
        first = std::fmax(0.0, std::floor(index(high)));
        last = std::fmin((double)(rot_dim - 1), std::ceil(index(low)));
        size = 0.1 * std::log(f) + 1.0;
    }
    retopk_rope got = {};
    got.rot_dim = rot_dim;
    got.interleaved = interleaved;
    got.factor = size;
    for (int i = 0; i < rot_dim / 2; ++i) {
        double w = std::pow(theta, -2.0 * i / rot_dim);
        double keep = 1.0;
        if (kind == RETOPK_ROPE_LINEAR) keep = 0.0;
        if (kind == RETOPK_ROPE_BANDS) keep = (n0 * w / two_pi - low) / (high - low);
        if (kind == RETOPK_ROPE_RAMP) keep = 1.0 - (i - first) / std::fmax(last - first, 0.001);
        keep = std::fmin(1.0, std::fmax(0.0, keep));
        got.freq[i] = keep == 1.0 ? w : keep == 0.0 ? w / f : w * (keep + (1.0 - keep) / f);
    }
    *r = got;
    return RETOPK_OK;
}

retopk_status rotary_embed(const retopk_rope *r, int32_t dtype, int32_t head_dim, int32_t n_heads, int64_t n_tokens,
                           const int32_t *pos, retopk_rows x, retopk_rows out, int32_t inverse, void *stream)
{
    if (!r || (dtype != RETOPK_F32 && dtype != RETOPK_BF16) || head_dim < 1 || n_heads < 1 || n_tokens < 0)
        return RETOPK_ERR_ARG;
    if (inverse != 0 && inverse != 1) return RETOPK_ERR_ARG;
    if (head_dim != 64 && head_dim != 128) return RETOPK_ERR_UNSUPPORTED;
    if (!rope_ok(r, head_dim)) return RETOPK_ERR_ARG;
    if (n_tokens == 0) return RETOPK_OK;
    const int es = dtype == RETOPK_BF16 ? 2 : 4;
    if (!pos || ((uintptr_t)pos & 3u) || !rows_ok(x, n_tokens, n_heads, head_dim, es, x.p == out.p) ||
        !rows_ok(out, n_tokens, n_heads, head_dim, es, true))
        return RETOPK_ERR_ARG;
    if (x.p == out.p && (x.token_stride != out.token_stride || x.head_stride != out.head_stride))
        return RETOPK_ERR_ARG;
    RowGrid g;
    if (!row_grid(n_tokens, head_dim, n_heads, kRowBlocks, &g)) return RETOPK_ERR_UNSUPPORTED;
    by_type(dtype, head_dim, [&](auto zero, auto d) {
        using T = decltype(zero);
        hipLaunchKernelGGL((k_rotary<T, decltype(d)::value>), g.grid, dim3(kRowThreads), 0, (hipStream_t)stream, *r,
                           rows_of<T>(x), rows_of<T>(out), pos, n_tokens, n_heads, g.per_block, inverse);
    });
    return launched();
}

retopk_status paged_append(const retopk_pages *c, const retopk_rope *r, int32_t dtype, int64_t n_tokens,
                           const int32_t *seq, const int32_t *pos, retopk_rows k, retopk_rows v, int32_t n_q_heads,
                           retopk_rows q, retopk_rows q_out, void *stream)
{
    const retopk_status st = check_pages(c, dtype);
    if (st != RETOPK_OK) return st;
    if (n_tokens < 0 || n_q_heads < 0 || (n_q_heads > 0 && !r)) return RETOPK_ERR_ARG;
    if (r && !rope_ok(r, c->head_dim)) return RETOPK_ERR_ARG;
    if (n_tokens == 0) return RETOPK_OK;
    const int es = dtype == RETOPK_BF16 ? 2 : 4, d = c->head_dim;
    if (!seq || !pos || ((uintptr_t)seq & 3u) || ((uintptr_t)pos & 3u)) return RETOPK_ERR_ARG;
    if (!rows_ok(k, n_tokens, c->n_kv_heads, d, es, false) || !rows_ok(v, n_tokens, c->n_kv_heads, d, es, false))
        return RETOPK_ERR_ARG;
    if (n_q_heads > 0) {
        if (!rows_ok(q, n_tokens, n_q_heads, d, es, q.p == q_out.p) ||
            !rows_ok(q_out, n_tokens, n_q_heads, d, es, true))
            return RETOPK_ERR_ARG;
        if (q.p == q_out.p && (q.token_stride != q_out.token_stride || q.head_stride != q_out.head_stride))
            return RETOPK_ERR_ARG;
    }
    RowGrid g;
    if (!row_grid(n_tokens, d, (int64_t)n_q_heads + 2 * (int64_t)c->n_kv_heads,
                  c->format == RETOPK_PAGES_BF16 ? kRowBlocksBf16 : kRowBlocks, &g))
        return RETOPK_ERR_UNSUPPORTED;
    const int64_t row = c->format == RETOPK_PAGES_Q4 ? d / 2 : d * es;
    const bool past = 2 * n_tokens * c->n_kv_heads * row > kStreamBytes;
    const PagesArgs a = pages_args(*c);
    const retopk_rope none = {}, &rope = r ? *r : none;
    by_type(dtype, d, [&](auto zero, auto dim) {
        launch_append<decltype(zero), decltype(dim)::value>(c->format, past, g, (hipStream_t)stream, a, rope, r ? 1 : 0, k,
                                                            v, q, q_out, seq, pos, n_tokens, n_q_heads);
    });
    return launched();
}

retopk_status paged_gather(const retopk_pages *c, int32_t dtype, int64_t n_tokens, const int32_t *seq,
                           const int32_t *pos, retopk_rows k, retopk_rows v, void *stream)
{
    const retopk_status st = check_pages(c, dtype);
    if (st != RETOPK_OK) return st;
    if (n_tokens < 0) return RETOPK_ERR_ARG;
    if (n_tokens == 0 || (!k.p && !v.p)) return RETOPK_OK;
    const int es = dtype == RETOPK_BF16 ? 2 : 4, d = c->head_dim;
    if (!seq || !pos || ((uintptr_t)seq & 3u) || ((uintptr_t)pos & 3u)) return RETOPK_ERR_ARG;
    if ((k.p && !rows_ok(k, n_tokens, c->n_kv_heads, d, es, true)) ||
        (v.p && !rows_ok(v, n_tokens, c->n_kv_heads, d, es, true)))
        return RETOPK_ERR_ARG;
    RowGrid g;
    if (!row_grid(n_tokens, d, 2 * (int64_t)c->n_kv_heads, kRowBlocks, &g)) return RETOPK_ERR_UNSUPPORTED;
    const bool past = 2 * n_tokens * c->n_kv_heads * d * es > kStreamBytes;
    const PagesArgs a = pages_args(*c);
    by_type(dtype, d, [&](auto zero, auto dim) {
        launch_gather<decltype(zero), decltype(dim)::value>(c->format, past, g, (hipStream_t)stream, a, k, v, seq, pos,
                                                            n_tokens);
    });
    return launched();
}

}  // extern "C"
