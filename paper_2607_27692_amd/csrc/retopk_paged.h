// retopk_paged.h -- shared by the paged-cache entry points (retopk_rope.hip,
// retopk_attend.hip): their argument checks on the host, and on the device the place of
// a position in the pages and the 4-bit format.  Not part of the public C ABI.
#pragma once

#include "retopk_device.h"
#include "retopk_internal.h"
#include "retopk_paged_plan.h"

namespace retopk {

constexpr int kGroup4 = 64;           // elements of a 4-bit row that share a scale and a mid

// The pages as a kernel takes them.  A row's number is (page * Hkv + head) * page_size +
// slot; check_pages keeps all of them below 2^31, so that only byte offsets need 64 bits.
struct PagesArgs {
    char *k, *v;
    uint32_t *k_par, *v_par;
    const int32_t *table;
    int32_t n_kv_heads, page_size, n_pages, n_seqs, table_width;
    Divisor by_page;
};

// Host checks (retopk_rope.hip), before any HIP call.
retopk_status check_pages(const retopk_pages *c, int32_t dtype);
PagesArgs pages_args(const retopk_pages &c);
// Rows of `heads` heads of d elements of es bytes: pointer and strides 16-byte aligned,
// strides not negative; for a tensor that is written, no two rows on each other.
bool rows_ok(const retopk_rows &x, int64_t tokens, int64_t heads, int d, int es, bool written);

// The page of position p of sequence s, -1 for none; and the number of the row that holds it on
// that page for KV head g, or -1.
__device__ __forceinline__ int32_t page_of(const PagesArgs &c, int32_t s, int32_t p)
{
    if (s < 0 || s >= c.n_seqs || p < 0) return -1;
    const uint32_t at = divide((uint32_t)p, c.by_page);
    return at < (uint32_t)c.table_width ? c.table[(int64_t)s * c.table_width + at] : -1;
}
__device__ __forceinline__ int32_t row_on(const PagesArgs &c, int32_t page, int32_t p, int g)
{
    if (page < 0 || page >= c.n_pages) return -1;
    const uint32_t at = divide((uint32_t)p, c.by_page);
    return (page * c.n_kv_heads + g) * c.page_size + (p - (int32_t)at * c.page_size);
}
__device__ __forceinline__ int32_t row_of(const PagesArgs &c, int32_t s, int32_t p, int g)
{
    return row_on(c, page_of(c, s, p), p, g);
}

typedef float f32x2_t __attribute__((ext_vector_type(2)));

// bf16 bits of x, and of two values side by side, rounded to nearest even.
__device__ __forceinline__ uint32_t bf16_pair(float x, float y)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{x, y}), bf16x2_t));
}
__device__ __forceinline__ uint32_t bf16_bits(float x) { return bf16_pair(x, 0.0f); }

// A load of rows that are read once a step: kept out of the caches' way, which the next layer's
// rows would need anyway.  With plain loads the 4-bit 128K layer took 40.3 us from HBM (35.9 so),
// eight bf16 sequences of up to 32K rows 79.3 (73.0).
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
template <typename V> __device__ __forceinline__ V once(const V *p) { return __builtin_nontemporal_load(p); }

// A store; STREAM: past the caches.
template <bool STREAM, typename V> __device__ __forceinline__ void put(V *p, V v)
{
    if constexpr (STREAM) __builtin_nontemporal_store(v, p);
    else *p = v;
}

// Elements of type T (float, or uint16_t for bf16) as 8 floats, and back.
template <typename T> struct Oct;
template <> struct Oct<float> {
    u32x4_t a, b;
    __device__ __forceinline__ void load(const float *p)
    {
        a = ((const u32x4_t *)p)[0];
        b = ((const u32x4_t *)p)[1];
    }
    __device__ __forceinline__ void load_once(const float *p)
    {
        a = once((const u32x4_t *)p);
        b = once((const u32x4_t *)p + 1);
    }
    __device__ __forceinline__ void get(float (&x)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = __uint_as_float(a[i]);
            x[i + 4] = __uint_as_float(b[i]);
        }
    }
    template <bool STREAM = false> static __device__ __forceinline__ void store(float *p, const float (&x)[8])
    {
        u32x4_t u, v;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            u[i] = __float_as_uint(x[i]);
            v[i] = __float_as_uint(x[i + 4]);
        }
        put<STREAM>((u32x4_t *)p, u);
        put<STREAM>((u32x4_t *)p + 1, v);
    }
    static __device__ __forceinline__ float one(const float *p) { return *p; }
};
template <> struct Oct<uint16_t> {
    u32x4_t a;
    __device__ __forceinline__ void load(const uint16_t *p) { a = *(const u32x4_t *)p; }
    __device__ __forceinline__ void get(float (&x)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = bf16_lo(a[i]);
            x[2 * i + 1] = bf16_hi(a[i]);
        }
    }
    template <bool STREAM = false> static __device__ __forceinline__ void store(uint16_t *p, const float (&x)[8])
    {
        u32x4_t u;
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = bf16_pair(x[2 * i], x[2 * i + 1]);
        put<STREAM>((u32x4_t *)p, u);
    }
    static __device__ __forceinline__ float one(const uint16_t *p) { return __uint_as_float((uint32_t)*p << 16); }
};

// The 8 values of a dword of 4-bit codes (elements 8 i .. 8 i + 7 of a row) of a group
// with this parameter word.  c * scale is exact (4 and 8 bits), so the sum rounds once.
__device__ __forceinline__ void values4(uint32_t codes, uint32_t par, float (&x)[8])
{
    const float scale = bf16_lo(par), mid = bf16_hi(par);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t w = codes >> (16 * h);
        const uint32_t m[4] = {(w >> 4) & 7u, w & 7u, (w >> 12) & 7u, (w >> 8) & 7u};
        const uint32_t s[4] = {(w >> 15) & 1u, (w >> 11) & 1u, (w >> 7) & 1u, (w >> 3) & 1u};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float c = (float)m[j] + 0.5f;
            x[4 * h + j] = fmaf(scale, s[j] ? -c : c, mid);
        }
    }
}

}  // namespace retopk
