// Shared by the sources of the 4-bit cache (cache.hip, cache_attention*.hip): how a page is laid out, and its numbers one by one.
#pragma once
#include "spmi_internal.h"

constexpr int kCacheBlock = 32;          // numbers that share a scale
constexpr int kCacheTile = 16;           // tokens of a record
constexpr int kCacheMinExp = -100, kCacheMaxExp = 125;      // 0.5 * 2^-100 and 6 * 2^125 are normal numbers of bf16 and f32
constexpr uint32_t kCacheNaN = 255;      // the scale of a block with a number that is not finite; others: exponent + 127

// A page holds, head after head, records of 16 tokens: codes of K, codes of V, scales of K, scales of V.  With nb = blocks of a head:
//   K codes   word (t * 4 + g) * nb + s: numbers 32 s + 8 g .. + 7 of token t, the first in the lowest bits
//   V codes   byte t % 4 of word ((t / 4) * 16 + n) * nb + s: number 32 s + n of token t in the low half, 32 s + 16 + n in the high one
//   scales    byte t * sb + s, sb = nb rounded up to a power of two
// so that 16 bytes of a lane are what it feeds to the matrix cores for tiles of 16 tokens: of K all it needs of a token (t = lane % 16, a
// quarter g = lane / 16 of every block), of V four tokens of two numbers of every block; and one token can be written without reading
// (a byte never holds two tokens).
struct cache_layout {
    int nb, sb;
    __host__ __device__ int v_codes() const { return 256 * nb; }
    __host__ __device__ int k_scales() const { return 512 * nb; }
    __host__ __device__ int v_scales() const { return 512 * nb + 16 * sb; }
    __host__ __device__ int record() const { return 512 * nb + 32 * sb; }
};
static inline __host__ __device__ cache_layout cache_layout_of(int D)
{
    const int nb = (D + kCacheBlock - 1) / kCacheBlock;
    return {nb, nb <= 2 ? nb : nb <= 4 ? 4 : 8};
}

// The cache as kernels take it.
struct cache_view {
    uint8_t *data;
    int64_t pages;
    int P, G, D;                         // tokens of a page, heads, head size
    cache_layout lay;
    __device__ __forceinline__ uint8_t *record(int64_t page, int g, int token) const
    {
        return data + ((page * G + g) * (P / kCacheTile) + token / kCacheTile) * lay.record();
    }
};

// NULL of c, SHAPE, TOO_LARGE; the memory may be missing.
static inline sp_status cache_check(const sp_cache *c, cache_view *v)
{
    if (!c) return SP_ERR_NULL;
    if (c->pages < 0 || c->pageTokens < kCacheTile || c->pageTokens % kCacheTile || c->kvHeads < 1 || c->kvHeads > 65535 || c->headDim < 1 || c->headDim > 256) return SP_ERR_SHAPE;
    if (c->pages >= ceil_div((int64_t)1 << 31, c->pageTokens)) return SP_ERR_TOO_LARGE;
    *v = {(uint8_t *)c->data, c->pages, c->pageTokens, c->kvHeads, c->headDim, cache_layout_of(c->headDim)};
    return SP_OK;
}
// Is the memory of a cache with pages there, where it may be?
static inline bool cache_has_memory(const cache_view &v) { return v.pages == 0 || v.data; }

// Eight numbers of a row, which rows aligned to 16 bytes are read and written in.
template <typename T> struct cache_eight_of { typedef T type __attribute__((ext_vector_type(8), aligned(16))); };
template <typename T> using cache_row8 = typename cache_eight_of<T>::type;
static_assert(alignof(cache_row8<float>) == 16, "");

typedef __bf16 cache_bf16;
typedef _Float16 cache_f16;

template <int BYTE>
__device__ __forceinline__ uint32_t cache_convert(uint32_t word, float scale)       // two codes -> two numbers
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, BYTE));
}

// What a code and a scale stand for.
__device__ __forceinline__ float cache_number(uint32_t code, uint32_t scale)
{
    const uint32_t m = code & 7;
    const float size = m < 2 ? 0.5f * (float)m : __uint_as_float(((m >> 1) + 126u) << 23 | (m & 1) << 22);     // two bits of exponent, one of fraction
    const float x = scale == kCacheNaN ? NAN : size * __uint_as_float(scale << 23);
    return code & 8 ? -x : x;
}
__device__ __forceinline__ float cache_key(const cache_view &c, const uint8_t *record, int t, int d)
{
    const int s = d >> 5, g = (d >> 3) & 3;
    const uint32_t w = ((const uint32_t *)record)[(t * 4 + g) * c.lay.nb + s];
    return cache_number((w >> (4 * (d & 7))) & 15, record[c.lay.k_scales() + t * c.lay.sb + s]);
}
__device__ __forceinline__ float cache_value(const cache_view &c, const uint8_t *record, int t, int d)
{
    const int s = d >> 5;
    const uint32_t b = record[c.lay.v_codes() + (((t >> 2) * 16 + (d & 15)) * c.lay.nb + s) * 4 + (t & 3)];
    return cache_number(d & 16 ? b >> 4 : b & 15, record[c.lay.v_scales() + t * c.lay.sb + s]);
}
