// Attention over the 4-bit cache: the kernels (cache_attention_*.hip instantiate them, cache_attention.hip calls them).
//
// Scores are computed transposed, S^T = K Q^T, in 16 x 16 tiles of the matrix cores (v_mfma_f32_16x16x32_bf16): a column is a query and
// head, a row a token.  Lane l of a wave has column l % 16 and rows 4 (l / 16) .. + 3 of a tile, so a column's weights are, as they lie,
// the second operand of O^T = V^T P^T over the 32 tokens of two tiles.  The cache's layout is that of the first operands: a lane turns the
// words that it loads into bf16 (v_cvt_scalef32_pk_bf16_fp4, which multiplies by the block's power of two), and keys and values go
// from memory to the matrix cores without passing the LDS.
#pragma once
#include "cache.h"
#include <math.h>

constexpr float kCacheLog2e = 1.4426950408889634f, kCacheLn2 = 0.6931471805599453f;

struct cache_attn_args {
    cache_view c;
    const void *Q;
    void *O;
    float *lse;
    const int32_t *table, *length, *start;
    int64_t ldq, hdq, ldo, hdo, ldt, width, requests, tokens;
    int H, R, causal;                    // R = H / G heads share a head of the cache
    float sign, step;                    // scale log2(e) = sign step; sign = -1, 0, 1 goes into Q, step > 0
    int vec;                             // rows of Q and O are aligned to 8 numbers
    spmi_divisor32 records;              // of a page: P / 16
    float *part;                         // workspace: [slot][head of the cache][column][32 nb] sums
    float2 *stat;                        //            [slot][head of the cache][column]: running maximum (in units of log 2; minus infinity: no weight) and total
    uint32_t slots;                      // slots there is room for
    uint32_t *plan;                      // see cache_plan_kernel; null: workgroups do without
};

// ---- work ------------------------------------------------------------------------------------------------------------------
// The columns of a request (its queries times the heads that share a head of the cache) are cut into tiles, its tokens into chunks, and an
// item is a tile, a chunk and a head of the cache.  Lengths are known on the GPU alone, so every workgroup finds its item by a scan over
// the requests: 64 at a time, of which a plan says the right ones where there are more.  The heads of one item are neighbours: workgroups go
// to the eight XCDs in turn, so that with 8 heads (or 4, 16, ..) what one L2 holds of the pages serves all tiles of a request.
// Chunks are as long as makes about kCacheTarget items of all work, at least kCacheLeast tokens.  Where the table has room for kCacheWhole tokens
// or fewer, nothing is cut and one launch does: 4 requests of up to 1000 tokens (f32) 12.0 us instead of 15 to 17 with chunks of 256 or 512 and a join, 2 prompts of
// 200 behind 1000 33 instead of 41; beyond, chunks are worth their join: one request of 2000 15.9 us with chunks of 256 (512: 17.5, 1024: 17.0), of 8192 14.9 (16.6, 17.3).
constexpr int kCacheTarget = 512, kCacheLeast = 256, kCacheWhole = 1024;

struct cache_request { uint32_t n, columns, tiles, tokens, row0; int32_t last; uint32_t r; };      // row0: its first row; last: position of its last query, -1 or more; r: its number
struct cache_item {
    int64_t r, row0;                     // the request and its first row
    cache_request q;
    uint32_t tile, chunk, chunks, slot;  // slot: of the tile's first chunk; the next one's is q.tiles further on
};

static inline __host__ __device__ int64_t cache_limit(int64_t x, int64_t lo, int64_t hi) { return x < lo ? lo : x > hi ? hi : x; }

// Columns of a request's tiles in a launch of tiles of `cols`: a quarter where few fill at most half of one (see cache_many_kernel).
__device__ __forceinline__ uint32_t cache_width(uint32_t columns, uint32_t cols) { return cols > 16 && columns * 2 <= cols ? cols / 4 : cols; }

__device__ __forceinline__ cache_request cache_request_of(const cache_attn_args &a, int64_t r, uint32_t cols)
{
    cache_request q = {0, 0, 0, 0, 0, -1, (uint32_t)r};
    if (r >= a.requests) return q;
    const int64_t s0 = cache_limit(a.start[r], 0, a.tokens), s1 = cache_limit(a.start[r + 1], 0, a.tokens), len = a.length[r];
    if (s1 <= s0) return q;
    q.n = (uint32_t)((int64_t)a.start[r + 1] - a.start[r]);              // rows behind the last one of Q are queries, too
    q.columns = (uint32_t)(s1 - s0) * (uint32_t)a.R;
    const uint32_t width = cache_width(q.columns, cols);
    q.tiles = (q.columns + width - 1) / width;
    q.tokens = (uint32_t)cache_limit(len, 0, a.width * a.c.P);
    q.row0 = (uint32_t)s0;
    q.last = (int32_t)(len < 0 ? 0 : len) - 1;
    return q;
}

__device__ __forceinline__ uint32_t cache_wave_scan(uint32_t v, int lane)           // sum of lanes 0 .. lane
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) { const uint32_t o = __shfl_up(v, d, 64); v += lane >= d ? o : 0; }
    return v;
}
template <typename V>
__device__ __forceinline__ V cache_wave_total(V v)
{
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d, 64);
    return v;
}

// Tokens of a chunk; work = sum over the requests of tiles * tokens, of which T items of a head get equal shares.  Chunks are no shorter than that,
// so those of requests that have several (less than 2 tokens / length) are fewer than 2 T.
constexpr uint32_t kCacheUncut = 1u << 31;           // no request has as many
__host__ __device__ __forceinline__ uint32_t cache_share(const cache_attn_args &a) { return ((uint32_t)kCacheTarget + a.c.G - 1) / (uint32_t)a.c.G; }
__host__ __device__ __forceinline__ uint32_t cache_chunk_tokens(const cache_attn_args &a, uint64_t work)
{
    const uint64_t T = cache_share(a), c = (work + T - 1) / T;
    return c < kCacheLeast ? kCacheLeast : c > kCacheUncut ? kCacheUncut : ((uint32_t)c + 127) & ~127u;
}
// `times` quarters longer
__host__ __device__ __forceinline__ uint32_t cache_grown(uint32_t length, int times)
{
    const uint64_t c = length + (uint64_t)((length / 4 + 63) & ~63u) * times;
    return c > kCacheUncut ? kCacheUncut : (uint32_t)c;
}
static inline int64_t cache_slots(int G) { return 2 * ceil_div(kCacheTarget, G); }

struct cache_counts { uint32_t chunks, items, slots, joins; };           // of a request; joins: tiles with more than one chunk
__host__ __device__ __forceinline__ cache_counts cache_counts_of(const cache_request &q, uint32_t length)
{
    const uint32_t chunks = q.tokens <= length ? 1 : (q.tokens + length - 1) / length, items = q.tiles * chunks;
    return {chunks, items, chunks > 1 ? items : 0, chunks > 1 ? q.tiles : 0};
}

// The plan of a step of prompts, or of more than 64 requests, by one workgroup: the length of chunks, the number of joins, then for every 64
// requests the items, the slots and the joins before them.  (A scan over all requests in every workgroup took 230 of the 320 us of a step of 1024
// requests of up to 512 tokens.)
// Prompts: a workgroup that comes after all places are taken has them wait for it, so chunks grow by quarters, up to twice, until there is a place
// for every item.  (Single tokens leave room for half as many workgroups again, and more chunks finish closer together.)
__global__ __launch_bounds__(1024) static void cache_plan_kernel(cache_attn_args a, uint32_t cols)
{
    __shared__ uint64_t sums[16];
    __shared__ uint32_t counts[16];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const uint32_t blocks = (uint32_t)((a.requests + 63) / 64);
    uint32_t length = kCacheUncut;
    if (a.slots) {
        uint64_t work = 0;
        for (int64_t r = threadIdx.x; r < a.requests; r += blockDim.x) {
            const cache_request q = cache_request_of(a, r, cols);
            work += (uint64_t)q.tiles * q.tokens;
        }
        work = cache_wave_total(work);
        if (lane == 0) sums[w] = work;
        __syncthreads();
        work = 0;
        for (int k = 0; k < waves; ++k) work += sums[k];
        length = cache_chunk_tokens(a, work);
        if (cols > 16) {
            for (int tries = 0; tries < 5; ++tries) {
                uint32_t items = 0;
                for (int64_t r = threadIdx.x; r < a.requests; r += blockDim.x) items += cache_counts_of(cache_request_of(a, r, cols), cache_grown(length, tries)).items;
                items = cache_wave_total(items);
                __syncthreads();
                if (lane == 0) counts[w] = items;
                __syncthreads();
                items = 0;
                for (int k = 0; k < waves; ++k) items += counts[k];
                if (items <= cache_share(a)) { length = cache_grown(length, tries); break; }
                if (tries == 0 && items > 2 * cache_share(a)) break;      // tiles enough as they are
            }
        }
    }
    uint32_t *items = a.plan + 2, *slots = items + blocks, *joins = slots + blocks;
    for (uint32_t b = w; b < blocks; b += waves) {
        const cache_counts c = cache_counts_of(cache_request_of(a, (int64_t)b * 64 + lane, cols), length);
        const uint32_t x = cache_wave_total(c.items), y = cache_wave_total(c.slots), z = cache_wave_total(c.joins);
        if (lane == 0) { items[b] = x; slots[b] = y; joins[b] = z; }
    }
    __syncthreads();
    for (int which = w; which < 3; which += waves) {
        uint32_t *of = which == 0 ? items : which == 1 ? slots : joins, before = 0;
        for (uint32_t b = 0; b < blocks; b += 64) {
            const uint32_t v = b + lane < blocks ? of[b + lane] : 0, upto = before + cache_wave_scan(v, lane);
            if (b + lane < blocks) of[b + lane] = upto - v;
            before = __builtin_amdgcn_readlane(upto, 63);
        }
        if (which == 2 && lane == 0) { a.plan[0] = length; a.plan[1] = before; }
    }
}

// The lanes' requests in the order of their tokens, the longest first, so that a launch does not end with the longest alone.
__device__ __forceinline__ void cache_longest_first(cache_request *q, int lane)
{
    uint32_t rank = 0;
    for (int k = 0; k < 64; ++k) {
        const uint32_t other = __builtin_amdgcn_readlane(q->tokens, k);
        rank += other > q->tokens || (other == q->tokens && k < lane) ? 1 : 0;
    }
    auto move = [rank](uint32_t x) { return (uint32_t)__builtin_amdgcn_ds_permute((int)rank * 4, (int)x); };
    *q = {move(q->n), move(q->columns), move(q->tiles), move(q->tokens), move(q->row0), (int32_t)move((uint32_t)q->last), move(q->r)};
}

// Item `index` of all (joined = false), or tile `index` of those that have more than one chunk.  For a whole wave; false: there is none.
__device__ __forceinline__ bool cache_find(const cache_attn_args &a, uint32_t cols, uint32_t index, bool joined, int lane, cache_item *item)
{
    cache_request q;
    uint32_t length = kCacheUncut, items = 0, slots = 0;
    if (!a.plan) {
        q = cache_request_of(a, lane, cols);
        if (a.slots) length = cache_chunk_tokens(a, cache_wave_total((uint64_t)q.tiles * q.tokens));
    } else {
        if (joined && index >= a.plan[1]) return false;
        const uint32_t blocks = (uint32_t)((a.requests + 63) / 64), *before = a.plan + 2 + (joined ? 2 * blocks : 0);
        uint32_t block = 0;                              // the last one that begins at the index or before
        if (blocks > 1)
            for (uint32_t b = 0; b < blocks; b += 64) {
                const uint64_t some = __builtin_amdgcn_ballot_w64(b + lane < blocks && before[b + lane < blocks ? b + lane : 0] <= index);
                if (!some) break;
                block = b + 63 - __builtin_clzll(some);
            }
        length = a.plan[0];
        items = before[block];
        slots = a.plan[2 + blocks + block];
        q = cache_request_of(a, (int64_t)block * 64 + lane, cols);
    }
    length = __builtin_amdgcn_readfirstlane(length);
    if (joined && !__builtin_amdgcn_ballot_w64(q.tokens > length && q.tiles)) return false;         // no chunks to join here
    if (cols > 16) cache_longest_first(&q, lane);
    const cache_counts c = cache_counts_of(q, length);
    const uint32_t mine = joined ? c.joins : c.items, upto = items + cache_wave_scan(mine, lane), slot = slots + cache_wave_scan(c.slots, lane);
    const uint64_t behind = __builtin_amdgcn_ballot_w64(upto > index);
    if (!behind) return false;
    const int k = __builtin_ctzll(behind);
    auto of = [k](uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane((int)x, k); };
    const uint32_t rest = index - (of(upto) - of(mine));
    item->r = of(q.r);
    item->row0 = of(q.row0);
    item->q = {of(q.n), of(q.columns), of(q.tiles), of(q.tokens), of(q.row0), (int32_t)of((uint32_t)q.last), of(q.r)};
    item->chunks = of(c.chunks);
    item->tile = rest % item->q.tiles;
    item->chunk = rest / item->q.tiles;
    item->slot = of(slot) - of(c.slots) + item->tile;
    return item->tile < item->q.tiles && item->chunk < item->chunks;
}

__device__ __forceinline__ uint32_t cache_page_of(const cache_attn_args &a, uint32_t record) { return spmi_div_by32(record, a.records); }

// ---- one column by itself ---------------------------------------------------------------------------------------------------

constexpr int kCachePer = 4;             // numbers of a lane: head sizes up to 256

__device__ __forceinline__ float cache_wave_sum(float v)
{
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d, 64);
    return v;
}

// For the tokens [t0, t1) of request r, one row and head: top, the maximum of the scores s in units of log 2, and total and acc, the sums of
// 2^(s - top - far) and of that times V; a wave, lanes across the head's numbers.  Every token is looked at alone, so that nothing that the row does
// not attend to can reach it: the tiles fall back on it where a sum is not finite, as a token that other columns attend to is multiplied
// with zero there, which infinities and NaN survive, or as sums of large values leave the range of f32.  Here they do not: a weight is half at
// most (far >= 1), and the sums are halved whenever the total gets past a half, so that acc stays below the largest value.
template <typename T>
__device__ __forceinline__ void cache_row(const cache_attn_args &a, int64_t r, int64_t i, int h, uint32_t t0, uint32_t t1, int lane,
                                       float &top, int &far, float &total, float (&acc)[kCachePer])
{
    const int g = h / a.R, D = a.c.D;
    const T *row = (const T *)a.Q + i * a.ldq + h * a.hdq;
    const float step = a.sign * a.step;
    float q[kCachePer];
#pragma unroll
    for (int k = 0; k < kCachePer; ++k) { q[k] = lane + 64 * k < D ? (float)row[lane + 64 * k] : 0.f; acc[k] = 0; }
    top = -INFINITY; total = 0; far = 1;
#pragma unroll 1
    for (uint32_t t = t0; t < t1; ++t) {
        const int64_t page = a.table[r * a.ldt + t / (uint32_t)a.c.P];
        if (page < 0 || page >= a.c.pages) continue;
        const int u = (int)(t % (uint32_t)a.c.P);
        const uint8_t *rec = a.c.record(page, g, u);
        float s = 0;
#pragma unroll
        for (int k = 0; k < kCachePer; ++k) if (lane + 64 * k < D) s += q[k] * cache_key(a.c, rec, u % kCacheTile, lane + 64 * k);
        s = cache_wave_sum(s) * step;
        if (s == -INFINITY) continue;                    // weight 0
        const float up = s > top ? s : top;              // not a number: stays with the old maximum, the weight carries it
        const float old = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - up), w = ldexpf(__builtin_amdgcn_exp2f(s - (up == -INFINITY ? 0.f : up)), -far);
        top = up;
        total = total * old + w;
#pragma unroll
        for (int k = 0; k < kCachePer; ++k) if (lane + 64 * k < D) acc[k] = acc[k] * old + w * cache_value(a.c, rec, u % kCacheTile, lane + 64 * k);
        if (total > 0.5f) {
            total *= 0.5f; ++far;
#pragma unroll
            for (int k = 0; k < kCachePer; ++k) acc[k] *= 0.5f;
        }
    }
}

// ---- tiles ------------------------------------------------------------------------------------------------------------------

typedef float cache_f4 __attribute__((ext_vector_type(4)));
typedef __bf16 cache_b8 __attribute__((ext_vector_type(8)));
typedef __bf16 cache_b2 __attribute__((ext_vector_type(2)));
typedef uint32_t cache_u4 __attribute__((ext_vector_type(4)));

// Q and weights as sums of bf16 numbers: 8 bits each, so that three hold all of f32.
template <typename T> struct cache_parts { static constexpr int n = sizeof(T) == 4 ? 3 : 2; };
template <> struct cache_parts<cache_bf16> { static constexpr int n = 1; };

template <int N>
__device__ __forceinline__ void cache_words(const uint8_t *p, uint32_t (&w)[N])     // 4-byte aligned
{
    typedef uint32_t v4 __attribute__((ext_vector_type(4), aligned(4)));
    typedef uint32_t v2 __attribute__((ext_vector_type(2), aligned(4)));
    const uint32_t *x = (const uint32_t *)p;
    int k = 0;
#pragma unroll
    for (; k + 4 <= N; k += 4) { const v4 v = *(const v4 *)(x + k); w[k] = v[0]; w[k + 1] = v[1]; w[k + 2] = v[2]; w[k + 3] = v[3]; }
    if constexpr (N % 4 >= 2) { const v2 v = *(const v2 *)(x + k); w[k] = v[0]; w[k + 1] = v[1]; k += 2; }
    if constexpr (N % 2) w[k] = x[k];
}
__device__ __forceinline__ uint32_t cache_pair(float x, float y)                    // rounded to bf16
{
    typedef float f2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f2){x, y}, cache_b2));
}

// What a lane holds of a record, 16 tokens: its words of K and V and their scales.
template <int NB>
struct cache_record {
    static constexpr int SB = NB <= 2 ? NB : NB <= 4 ? 4 : 8, KS = (SB + 3) / 4, bytes = 512 * NB + 32 * SB;
    uint32_t k[NB], v[NB], ks[KS], vs[SB];
    __device__ __forceinline__ void load(const uint8_t *rec, int lane)
    {
        constexpr int scales = 512 * NB;
        const int t = lane & 15, g = lane >> 4;
        cache_words(rec + (t * 4 + g) * (NB * 4), k);
        if constexpr (SB == 1) ks[0] = rec[scales + t];
        else if constexpr (SB == 2) ks[0] = *(const uint16_t *)(rec + scales + t * 2);
        else cache_words(rec + scales + t * SB, ks);
        cache_words(rec + 256 * NB + (g * 16 + t) * (NB * 4), v);
        cache_words(rec + scales + 16 * SB + g * 4 * SB, vs);
    }
    // A scale as the conversion takes it, which looks at the exponent (bits 23 to 30) alone: the byte is moved there, whatever lies beside it.
    static __device__ __forceinline__ float scale(uint32_t w, int b) { return __uint_as_float(b == 3 ? w >> 1 : w << (23 - 8 * b)); }
    __device__ __forceinline__ cache_b8 key(int b) const                // the operand of block b of K
    {
        const float f = scale(ks[b / 4], b % 4);
        return __builtin_bit_cast(cache_b8, (cache_u4){cache_convert<0>(k[b], f), cache_convert<1>(k[b], f), cache_convert<2>(k[b], f), cache_convert<3>(k[b], f)});
    }
    __device__ __forceinline__ float v_scale(int token, int b) const { return scale(vs[(token * SB + b) / 4], (token * SB + b) % 4); }
    // half of the operands of block b of V: numbers 0 .. 15 and 16 .. 31 of four tokens
    __device__ __forceinline__ void values(int b, uint32_t (&lo)[2], uint32_t (&hi)[2]) const
    {
        const uint32_t c0 = cache_convert<0>(v[b], v_scale(0, b)), c1 = cache_convert<1>(v[b], v_scale(1, b));
        const uint32_t c2 = cache_convert<2>(v[b], v_scale(2, b)), c3 = cache_convert<3>(v[b], v_scale(3, b));
        lo[0] = __builtin_amdgcn_perm(c1, c0, 0x05040100);
        lo[1] = __builtin_amdgcn_perm(c3, c2, 0x05040100);
        hi[0] = __builtin_amdgcn_perm(c1, c0, 0x07060302);
        hi[1] = __builtin_amdgcn_perm(c3, c2, 0x07060302);
    }
    __device__ __forceinline__ void blank(int token)                   // the token's values are zeros
    {
#pragma unroll
        for (int b = 0; b < NB; ++b) v[b] &= ~(255u << (8 * token));
        if constexpr (SB >= 4) {
#pragma unroll
            for (int b = 0; b < SB / 4; ++b) vs[token * (SB / 4) + b] = 0x7f7f7f7f;
        } else {
            constexpr uint32_t ones = SB == 2 ? 0xffff : 0xff;
            uint32_t &w = vs[token * SB / 4];
            const int at = 8 * (token * SB % 4);
            w = (w & ~(ones << at)) | ((0x7f7f & ones) << at);
        }
    }
};

// 32 tokens in registers.
template <int NB>
struct cache_tokens {
    cache_record<NB> half[2];
    __device__ __forceinline__ void values(int b, cache_b8 &lo, cache_b8 &hi) const
    {
        uint32_t l[2][2], h[2][2];
        half[0].values(b, l[0], h[0]);
        half[1].values(b, l[1], h[1]);
        lo = __builtin_bit_cast(cache_b8, (cache_u4){l[0][0], l[0][1], l[1][0], l[1][1]});
        hi = __builtin_bit_cast(cache_b8, (cache_u4){h[0][0], h[0][1], h[1][0], h[1][1]});
    }
};

// A number that all lanes share, in a vector register.
__device__ __forceinline__ float cache_spread(float x) { asm volatile("" : "+v"(x)); return x; }

// 16 NQ columns of one tile over some of its tokens, by one wave.
template <typename T, int NB, int NQ>
struct cache_wave {
    static constexpr int parts = cache_parts<T>::n;
    cache_b8 q[NQ][parts][NB];
    cache_f4 o[NQ][2 * NB];
    float top[NQ], mu[NQ], most[NQ];     // running maximum (the same in the four lanes of a column); what is taken off; sum of weights that moves it
    float total[NQ];                     // a lane's own share of the total
    uint32_t end[NQ];                    // the column attends to tokens before this one

    // Q's column: 8 numbers of every block
    __device__ __forceinline__ void load_q(const cache_attn_args &a, const cache_item &it, uint32_t first, int g, int lane)
    {
        const int D = a.c.D;
#pragma unroll
        for (int k = 0; k < NQ; ++k) {
            const uint32_t col = first + 16 * k + (lane & 15);
            const bool there = col < it.q.columns;
            const uint32_t i = there ? col / (uint32_t)a.R : 0, hh = there ? col % (uint32_t)a.R : 0;
            const T *row = (const T *)a.Q + (it.row0 + i) * a.ldq + (int64_t)(g * a.R + hh) * a.hdq;
            const int64_t e = a.causal ? (int64_t)it.q.last - it.q.n + 2 + i : (int64_t)it.q.tokens;
            end[k] = there ? (uint32_t)cache_limit(e, 0, it.q.tokens) : it.q.tokens;
            top[k] = -INFINITY; mu[k] = 0; most[k] = -1; total[k] = 0;
#pragma unroll
            for (int s = 0; s < 2 * NB; ++s) o[k][s] = (cache_f4)(0.f);
#pragma unroll
            for (int s = 0; s < NB; ++s) {
                const int d0 = 32 * s + 8 * (lane >> 4);
                float x[8];
                if (a.vec) {
                    cache_row8<T> v = {};
                    if (there && d0 < D) v = *(const cache_row8<T> *)(row + d0);
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[j] = (float)v[j];
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[j] = there && d0 + j < D ? (float)row[d0 + j] : 0.f;
                }
                // cut off (not rounded) to 8 bits, part after part: nothing is lost and nothing overflows
                uint32_t w[parts][4] = {};
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    float y = x[j] * a.sign;
                    const bool finite = y - y == 0;
#pragma unroll
                    for (int p = 0; p < parts; ++p) {
                        uint32_t u = __float_as_uint(y);
                        if (p == 0 && !finite) u = y == y ? u : 0x7fc00000u;
                        if (p > 0 && !finite) u = 0;
                        w[p][j / 2] |= j % 2 ? u & 0xffff0000u : u >> 16;
                        y -= __uint_as_float(u & 0xffff0000u);
                    }
                }
#pragma unroll
                for (int p = 0; p < parts; ++p) q[k][p][s] = __builtin_bit_cast(cache_b8, (cache_u4){w[p][0], w[p][1], w[p][2], w[p][3]});
            }
        }
    }

    // S^T of 32 tokens; key(half, b): the operands of K
    template <typename F>
    __device__ __forceinline__ void scores(cache_f4 (&s)[NQ][2], F key) const
    {
#pragma unroll
        for (int k = 0; k < NQ; ++k) s[k][0] = s[k][1] = (cache_f4)(0.f);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const cache_b8 x[2] = {key(0, b), key(1, b)};
#pragma unroll
            for (int p = 0; p < parts; ++p)
#pragma unroll
                for (int k = 0; k < NQ; ++k)
#pragma unroll
                    for (int half = 0; half < 2; ++half)         // sums that do not wait for each other
                        s[k][half] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[half], q[k][p][b], s[k][half], 0, 0, 0);
        }
    }
    // Where some column attends to some of the 32 tokens from t on only; there: which halves' pages exist
    __device__ __forceinline__ void leave_out(cache_f4 (&s)[NQ][2], uint32_t t, uint32_t there, int lane) const
    {
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t at = t + 16 * half + 4 * (lane >> 4) + j;
#pragma unroll
                for (int k = 0; k < NQ; ++k) s[k][half][j] = ((there >> half) & 1) && at < end[k] ? s[k][half][j] : -INFINITY;
            }
    }
    // The weights as operands, and their sums.
    __device__ __forceinline__ void weights(const cache_f4 (&s)[NQ][2], float step, cache_b8 (&w)[NQ][parts])
    {
#pragma unroll
        for (int k = 0; k < NQ; ++k) {
            // The maximum that is taken off lags behind by up to 8 (a factor of 256), which the sum of the weights says: moving it costs a pass
            // over the sums, and it moves in the first tokens of a chunk, hardly later.
            float y[8], sum;
            auto exponentials = [&]() {
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[k][j / 4][j % 4], step, -mu[k]));
                sum = ((y[0] + y[1]) + (y[2] + y[3])) + ((y[4] + y[5]) + (y[6] + y[7]));
            };
            exponentials();
            if (__builtin_amdgcn_ballot_w64(sum > most[k])) {
                float up = fmaxf(fmaxf(fmaxf(s[k][0][0], s[k][0][1]), fmaxf(s[k][0][2], s[k][0][3])), fmaxf(fmaxf(s[k][1][0], s[k][1][1]), fmaxf(s[k][1][2], s[k][1][3])));
                up = fmaxf(up, __shfl_xor(up, 16, 64));
                up = fmaxf(top[k], fmaxf(up, __shfl_xor(up, 32, 64)) * step);
                const float now = up == -INFINITY ? 0.f : up, f = top[k] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mu[k] - now);
                top[k] = up; mu[k] = now;
                most[k] = up == -INFINITY ? -1.f : 256.f;        // the first score that is not minus infinity moves it
                total[k] *= f;
#pragma unroll
                for (int b = 0; b < 2 * NB; ++b) o[k][b] *= f;
                exponentials();
            }
            total[k] += sum;
#pragma unroll
            for (int p = 0; p < parts; ++p) {
                cache_u4 u;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    u[j] = cache_pair(y[2 * j], y[2 * j + 1]);
                    y[2 * j] -= __uint_as_float(u[j] << 16);
                    y[2 * j + 1] -= __uint_as_float(u[j] & 0xffff0000u);
                }
                w[k][p] = __builtin_bit_cast(cache_b8, u);
            }
        }
    }
    // O^T += V^T P^T for numbers 16 b .. 16 b + 15
    __device__ __forceinline__ void sums(int b, cache_b8 value, const cache_b8 (&w)[NQ][parts])
    {
#pragma unroll
        for (int k = 0; k < NQ; ++k)
#pragma unroll
            for (int p = 0; p < parts; ++p) o[k][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(value, w[k][p], o[k][b], 0, 0, 0);
    }

    // 32 tokens from t on, in registers.  partial: some column attends to some of them only; tokens: the request's.
    // One path for both, as two would be merged by the compiler into one that keeps everything of both at once.
    __device__ __forceinline__ void tokens32(cache_tokens<NB> &x, float step, uint32_t t, uint32_t tokens, uint32_t there, bool partial, int lane)
    {
        cache_f4 s[NQ][2];
        scores(s, [&](int half, int b) { return x.half[half].key(b); });
        if (partial) {
            leave_out(s, t, there, lane);
#pragma unroll
            for (int half = 0; half < 2; ++half)         // behind the request's tokens anything may be there
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (!((there >> half) & 1) || t + 16 * half + 4 * (lane >> 4) + j >= tokens) x.half[half].blank(j);
        }
        cache_b8 w[NQ][parts];
        weights(s, step, w);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            cache_b8 lo, hi;
            x.values(b, lo, hi);
            sums(2 * b, lo, w);
            sums(2 * b + 1, hi, w);
        }
    }

    // The tokens from t on, 32 at a time every `stride`, up to `to`; `whole`: all columns attend to all tokens before it.
    __device__ __forceinline__ void run(const cache_attn_args &a, const cache_item &it, int g, uint32_t t, uint32_t stride, uint32_t to, uint32_t whole, int lane)
    {
        if (t >= to) return;
        const int32_t *table = a.table + it.r * a.ldt;
        const uint32_t per = (uint32_t)a.c.P / kCacheTile, count = (uint32_t)a.c.pages;
        const int64_t page_bytes = (int64_t)per * a.c.G * cache_record<NB>::bytes;
        const uint8_t *data = a.c.data + g * (int64_t)per * cache_record<NB>::bytes;
        auto page_of = [&](uint32_t record) { return cache_page_of(a, record); };
        // Tokens before `to` have a page in the table; the second 16 of 32 may lie behind the table's end, and are behind the request's then.
        auto pages = [&](uint32_t at, int32_t (&p)[2]) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const uint32_t n = page_of(at / kCacheTile + half);
                p[half] = table[n < a.width ? n : a.width - 1];
            }
        };
        auto fetch = [&](uint32_t at, const int32_t (&p)[2], cache_tokens<NB> &x) {
            uint32_t there = 0;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const uint32_t record = at / kCacheTile + half, in = record - page_of(record) * per;
                const bool ok = (uint32_t)p[half] < count;
                there |= ok ? 1u << half : 0;
                x.half[half].load(data + ((ok ? (uint32_t)p[half] : 0u) * page_bytes + in * (int64_t)cache_record<NB>::bytes), lane);
            }
            return there;
        };
        // Two places, one filled while the other is worked on; pages a step ahead of that.  At the end the last tokens are loaded again: no
        // branches in between.
        const uint32_t last = t + (to - 1 - t) / stride * stride;
        int32_t p[2];
        cache_tokens<NB> x[2];
        uint32_t next = t < last ? t + stride : last, there[2];
        pages(t, p);
        there[0] = fetch(t, p, x[0]);
        pages(next, p);
        while (true) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                there[1 - k] = fetch(next, p, x[1 - k]);
                const uint32_t then = next < last ? next + stride : last;
                pages(then, p);
                tokens32(x[k], a.step, t, it.q.tokens, there[k], t + 32 > whole || there[k] != 3, lane);
                if (t == last) return;
                t = next;
                next = then;
            }
        }
    }
};

// The tokens of an item and of them those that its columns, `first` and `count - 1` more, attend to.
struct cache_span { uint32_t from, to, whole; };
__device__ __forceinline__ cache_span cache_span_of(const cache_attn_args &a, const cache_item &it, uint32_t first, uint32_t count)
{
    const uint32_t each = it.chunks == 1 ? it.q.tokens : ((it.q.tokens + it.chunks - 1) / it.chunks + 63) & ~63u;      // whole steps
    cache_span s;
    const uint64_t from = (uint64_t)it.chunk * each, to = from + each;
    s.from = (uint32_t)(from < it.q.tokens ? from : it.q.tokens);
    s.to = (uint32_t)(to < it.q.tokens ? to : it.q.tokens);
    s.whole = it.q.tokens;
    if (a.causal) {
        const int64_t before = (int64_t)it.q.last - it.q.n + 2;   // what the request's first query attends to, at least
        const uint32_t end = (uint32_t)cache_limit(before + (first + count - 1) / (uint32_t)a.R, 0, it.q.tokens);
        s.whole = (uint32_t)cache_limit(before + first / (uint32_t)a.R, 0, it.q.tokens);
        if (end < s.to) s.to = end;
    }
    return s;
}

// A column's result: O and lse, or a part of them for the join.
template <typename T, int NB>
struct cache_column {
    T *out;
    float *lse, *part;
    float2 *stat;
    __device__ __forceinline__ cache_column(const cache_attn_args &a, const cache_item &it, int g, uint32_t col, uint32_t cols)
    {
        const uint32_t i = col / (uint32_t)a.R, h = g * a.R + col % (uint32_t)a.R;
        out = (T *)a.O + (it.row0 + i) * a.ldo + (int64_t)h * a.hdo;
        lse = a.lse ? a.lse + (int64_t)h * a.tokens + it.row0 + i : nullptr;
        const int64_t at = ((it.slot + (int64_t)it.chunk * it.q.tiles) * a.c.G + g) * cols + col % cols;
        part = it.chunks > 1 ? a.part + at * (32 * NB) : nullptr;
        stat = a.stat + at;
    }
    __device__ __forceinline__ void numbers(const cache_attn_args &a, int d, cache_f4 x, float total) const       // d a multiple of 4
    {
        if (part) { *(cache_f4 *)(part + d) = x; return; }
        const float f = total == 0 ? 0.f : 1 / total;
        typedef T v4 __attribute__((ext_vector_type(4)));
        if (a.vec) { if (d < a.c.D) *(v4 *)(out + d) = (v4){(T)(x[0] * f), (T)(x[1] * f), (T)(x[2] * f), (T)(x[3] * f)}; }
        else
#pragma unroll
            for (int j = 0; j < 4; ++j) if (d + j < a.c.D) out[d + j] = (T)(x[j] * f);
    }
    // top: minus infinity where nothing weighs, so that the join's maximum is that of the chunks that do
    __device__ __forceinline__ void total(float top, float sum) const
    {
        if (part) *stat = {top, sum};
        else if (lse) *lse = sum == 0 ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kCacheLn2;
    }
};

// A column whose sums are not finite although its total is, made again.
template <typename T, int NB>
__device__ __forceinline__ void cache_again(const cache_attn_args &a, const cache_item &it, int g, uint32_t col, uint32_t cols, uint32_t from, uint32_t to, int lane)
{
    const uint32_t i = col / (uint32_t)a.R;
    const cache_span s = cache_span_of(a, it, col, 1);
    float top, total, acc[kCachePer];
    int far;
    cache_row<T>(a, it.r, it.row0 + i, g * a.R + col % (uint32_t)a.R, from, to < s.to ? to : s.to, lane, top, far, total, acc);
    const cache_column<T, NB> c(a, it, g, col, cols);
#pragma unroll
    for (int k = 0; k < kCachePer; ++k) {
        const int d = lane + 64 * k;
        if (c.part) { if (d < 32 * NB) c.part[d] = d < a.c.D ? acc[k] : 0.f; }
        else if (d < a.c.D) c.out[d] = (T)(total == 0 ? 0.f : acc[k] / total);
    }
    // a part's sums go with its total as they are; what was taken off them counts as maximum
    if (lane == 0) c.total(c.part ? top + (float)far : top, c.part ? total : ldexpf(total, far));
}

// The kernel's arguments (its first ones), to be loaded where they are used: kept from the kernel's beginning on they would not fit the scalar registers.
__device__ __forceinline__ const cache_attn_args &cache_late()
{
    typedef const __attribute__((address_space(4))) cache_attn_args *pointer;
    pointer p = (pointer)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *(const cache_attn_args *)p;
}
// Groups of 16 columns of a wave, and waves on a SIMD, so that nothing is kept in scratch memory.
template <typename T> constexpr int cache_nq(int nb) { return nb <= (cache_parts<T>::n == 3 ? 3 : 4) ? 2 : 1; }
template <typename T> constexpr int cache_few_waves(int nb) { return nb <= (cache_parts<T>::n == 3 ? 3 : 4) ? 3 : nb <= (cache_parts<T>::n == 1 ? 8 : 9 - cache_parts<T>::n) ? 2 : 1; }
template <typename T> constexpr int cache_many_waves(int nb) { return nb <= (cache_parts<T>::n == 1 ? 8 : 9 - cache_parts<T>::n) ? 2 : 1; }

// 16 NQ columns or fewer: the four waves of a workgroup take 32 tokens in turn, and they meet in the LDS.
template <typename T, int NB, int NQ>
struct cache_meeting { float sums[4][16 * NQ][32 * NB + 4]; float2 stats[4][16 * NQ]; };

template <typename T, int NB, int NQ>
__device__ __forceinline__ void cache_few(const cache_attn_args &a, const cache_item &it, int g, uint32_t cols, int w, int lane, cache_meeting<T, NB, NQ> &m)
{
    const uint32_t width = cache_width(it.q.columns, cols), first = it.tile * width, count = it.q.columns - first < width ? it.q.columns - first : width;
    const cache_span span = cache_span_of(a, it, first, count);
    const int q = lane & 15;
    {
        cache_wave<T, NB, NQ> x;
        x.load_q(a, it, first, g, lane);
        x.run(a, it, g, span.from + 32 * w, 128, span.to, span.whole, lane);
#pragma unroll
        for (int k = 0; k < NQ; ++k) {
            float total = x.total[k];
            total += __shfl_xor(total, 16, 64);
            total += __shfl_xor(total, 32, 64);
            if (lane < 16) m.stats[w][16 * k + q] = {x.top[k], total};
#pragma unroll
            for (int b = 0; b < 2 * NB; ++b) *(cache_f4 *)&m.sums[w][16 * k + q][16 * b + 4 * (lane >> 4)] = x.o[k][b];
        }
    }
    __syncthreads();
    const cache_attn_args &late = cache_late();
    for (uint32_t group = 0; group < count; group += 16) {
        const uint32_t c = group + (threadIdx.x >> 4);   // a column for every 16 threads
        float top = -INFINITY, total = 0, f[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) top = fmaxf(top, m.stats[k][c].x);
        bool some[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 s = m.stats[k][c];
            some[k] = !(s.y == 0);                       // sums without weight may hold anything
            f[k] = __builtin_amdgcn_exp2f(s.x - top);
            total += some[k] ? s.y * f[k] : 0.f;
        }
        const bool there = c < count;
        constexpr int each = (8 * NB + 15) / 16;
        cache_f4 y[each];
        bool fine = true;
#pragma unroll
        for (int j = 0; j < each; ++j) {
            const int d = 4 * (q + 16 * j);
            y[j] = (cache_f4)(0.f);
            if (d < 32 * NB) {
#pragma unroll
                for (int k = 0; k < 4; ++k) if (some[k]) y[j] += *(const cache_f4 *)&m.sums[k][c][d] * f[k];
                fine = fine && y[j][0] - y[j][0] == 0 && y[j][1] - y[j][1] == 0 && y[j][2] - y[j][2] == 0 && y[j][3] - y[j][3] == 0;
            }
        }
        const uint64_t spoilt = __builtin_amdgcn_ballot_w64(there && !fine && total == total);
        if (there && !((spoilt >> (lane & 48)) & 0xffff)) {
            const cache_column<T, NB> out(late, it, g, first + c, cols);
#pragma unroll
            for (int j = 0; j < each; ++j) {
                const int d = 4 * (q + 16 * j);
                if (d < 32 * NB) out.numbers(late, d, y[j], total);
            }
            if (q == 0) out.total(top, total);
        }
#pragma unroll 1
        for (int k = 0; k < 4; ++k)
            if ((spoilt >> (16 * k)) & 0xffff) cache_again<T, NB>(late, it, g, first + group + 4 * w + k, cols, span.from, span.to, lane);
    }
}

// Single tokens of requests (and other steps of few columns a request).  The pages' bytes bound it: 64 requests of up to 8192 tokens, 8 heads of 128,
// 4 columns each, take 65 us, 4.9 TB/s; the instructions of 16 columns (300 a step of 32 tokens) would allow 10.  Two places for tokens in registers and three
// waves a SIMD keep 50 KB a compute unit on their way.
template <typename T, int NB>
__global__ __launch_bounds__(256, cache_few_waves<T>(NB)) void cache_few_kernel(cache_attn_args a)
{
    __shared__ cache_meeting<T, NB, 1> meeting;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    cache_item it;
    const uint32_t index = blockIdx.x / (uint32_t)a.c.G, g = blockIdx.x - index * a.c.G;
    if (!cache_find(a, 16, index, false, lane, &it)) return;
    if (it.chunks > 1 && it.slot + (uint64_t)it.chunk * it.q.tiles >= a.slots) return;       // (rows of requests that overlap)
    cache_few<T, NB, 1>(a, it, (int)g, 16, w, lane, meeting);
}

// Prompts: the four waves of a workgroup take 16 NQ columns each and all tokens of the chunk, 64 at a time.  A wave turns 16 of the 64 into
// operands, which the four share in LDS: in registers of their own the conversions would take as long as the exponentials.  Two places: one
// is filled while the other is worked on.  (NB > 4: one place, there is no room for two workgroups otherwise.)  Requests whose columns would
// leave two waves or more without any are dealt with as single tokens are, 16 NQ columns (or 16) a workgroup.
// What two waves a SIMD issue bounds it: of 64 tokens and 32 columns 64 products (1024 cycles of the matrix cores), 64 exponentials and about 230 other vector
// instructions.  8 requests of 512 to 1024 queries behind 2048 to 8192 tokens, 32 heads of 128 on 8, take 0.51 ms, 902 TFLOP/s.
template <typename T, int NB, int NQ>
__global__ __launch_bounds__(256, cache_many_waves<T>(NB)) void cache_many_kernel(cache_attn_args a)
{
    constexpr uint32_t cols = 64 * NQ;
    constexpr int places = NB <= 4 ? 2 : 1, kv = 4 * NB * 1024, stage = 2 * kv;      // kv: bytes of the operands of K (and of V) of 64 tokens
    __shared__ union __align__(16) {
        cache_meeting<T, NB, 1> meeting;
        cache_meeting<T, NB, NQ> wide;
        struct { char at[places][stage]; uint32_t there[places][4]; } staged;
    } lds;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t index = blockIdx.x / (uint32_t)a.c.G;
    const int g = (int)(blockIdx.x - index * a.c.G);
    cache_item it;
    if (!cache_find(a, cols, index, false, lane, &it)) return;
    if (it.chunks > 1 && it.slot + (uint64_t)it.chunk * it.q.tiles >= a.slots) return;       // (rows of requests that overlap)
    if (it.q.columns <= 16) { cache_few<T, NB, 1>(a, it, g, cols, w, lane, lds.meeting); return; }
    if (cache_width(it.q.columns, cols) < cols) { cache_few<T, NB, NQ>(a, it, g, cols, w, lane, lds.wide); return; }
    const uint32_t tile0 = it.tile * cols, tile_count = it.q.columns - tile0 < cols ? it.q.columns - tile0 : cols;
    const cache_span all = cache_span_of(a, it, tile0, tile_count);
    const uint32_t first = tile0 + 16 * NQ * w, mine = tile_count > 16 * NQ * w ? tile_count - 16 * NQ * w : 0, count = mine < 16 * NQ ? mine : 16 * NQ;
    const cache_span span = cache_span_of(a, it, count ? first : tile0, count ? count : 1);
    cache_wave<T, NB, NQ> x;
    x.load_q(a, it, first, g, lane);
    const float step = cache_spread(a.step);

    const int32_t *table = a.table + it.r * a.ldt;
    const uint32_t per = (uint32_t)a.c.P / kCacheTile, count_pages = (uint32_t)a.c.pages;
    const int64_t page_bytes = (int64_t)per * a.c.G * cache_record<NB>::bytes;
    const uint8_t *data = a.c.data + g * (int64_t)per * cache_record<NB>::bytes;
    // a wave's 16 of the 64 tokens from t on; behind the table's end the request has none
    auto page = [&](uint32_t t) {
        const uint32_t n = cache_page_of(a, t / kCacheTile + w);
        return table[n < a.width ? n : a.width - 1];
    };
    cache_record<NB> rec;
    auto fetch = [&](uint32_t t, int32_t p) {
        const uint32_t record = t / kCacheTile + w, in = record - cache_page_of(a, record) * per;
        const bool ok = (uint32_t)p < count_pages;
        rec.load(data + ((ok ? (uint32_t)p : 0u) * page_bytes + in * (int64_t)cache_record<NB>::bytes), lane);
        return ok;
    };
    auto put = [&](int place, uint32_t t, bool ok) {
        char *to = lds.staged.at[place];
        if (!ok || t + 16 * w + 16 > it.q.tokens)
#pragma unroll
            for (int j = 0; j < 4; ++j) if (!ok || t + 16 * w + 4 * (lane >> 4) + j >= it.q.tokens) rec.blank(j);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            *(cache_b8 *)(to + (w * NB + b) * 1024 + lane * 16) = rec.key(b);
            uint32_t lo[2], hi[2];
            rec.values(b, lo, hi);
            char *v = to + kv + ((w >> 1) * NB + b) * 2048 + lane * 16 + (w & 1) * 8;
            *(uint2 *)v = {lo[0], lo[1]};
            *(uint2 *)(v + 1024) = {hi[0], hi[1]};
        }
        if (lane == 0) lds.staged.there[place][w] = ok;
    };
    // Operands are asked for a product ahead of their use: of V before the exponentials, of the next K before the product with V.
    auto work = [&](int place, uint32_t t) {
        const char *at = lds.staged.at[place] + lane * 16;
        const uint4 f = *(const uint4 *)lds.staged.there[place];
        cache_b8 key[2 * NB], value[2 * NB], w[NQ][cache_parts<T>::n];
        cache_f4 s[NQ][2];
#pragma unroll
        for (int b = 0; b < 2 * NB; ++b) key[b] = *(const cache_b8 *)(at + b * 1024);
        const uint32_t there = __builtin_amdgcn_readfirstlane(f.x | f.y << 1 | f.z << 2 | f.w << 3);
#pragma unroll
        for (int pair = 0; pair < 2; ++pair) {
            x.scores(s, [&](int half, int b) { return key[half * NB + b]; });
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int b = 0; b < 2 * NB; ++b) value[b] = *(const cache_b8 *)(at + kv + (pair * 2 * NB + b) * 1024);
            const uint32_t both = (there >> (2 * pair)) & 3;
            if (t + 32 * pair + 32 > span.whole || both != 3) x.leave_out(s, t + 32 * pair, both, lane);
            x.weights(s, step, w);
            __builtin_amdgcn_sched_barrier(0);
            if (pair == 0)
#pragma unroll
                for (int b = 0; b < 2 * NB; ++b) key[b] = *(const cache_b8 *)(at + (2 * NB + b) * 1024);
#pragma unroll
            for (int b = 0; b < 2 * NB; ++b) x.sums(b, value[b], w);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    if (all.from < all.to) {
        const uint32_t last = all.from + (all.to - 1 - all.from) / 64 * 64;
        uint32_t t = all.from, next = t < last ? t + 64 : last;
        bool ok = fetch(t, page(t));
        put(0, t, ok);
        int32_t p = page(next);
        ok = fetch(next, p);
        __syncthreads();
        if constexpr (places == 2) {
            for (int place = 0;; place ^= 1) {
                if (t != last) {
                    const uint32_t then = next < last ? next + 64 : last;
                    p = page(then);
                    put(place ^ 1, next, ok);
                    ok = fetch(then, p);
                }
                work(place, t);
                if (t == last) break;
                __syncthreads();
                t = next;
                next = next < last ? next + 64 : last;
            }
        } else {
            while (true) {
                work(0, t);
                if (t == last) break;
                __syncthreads();
                put(0, next, ok);
                t = next;
                next = next < last ? next + 64 : last;
                ok = fetch(next, page(next));
                __syncthreads();
            }
        }
    }
    const cache_attn_args &late = cache_late();
    uint64_t spoilt = 0;                                 // a bit a column
#pragma unroll
    for (int k = 0; k < NQ; ++k) {
        float total = x.total[k];
        total += __shfl_xor(total, 16, 64);
        total += __shfl_xor(total, 32, 64);
        bool fine = true;
#pragma unroll
        for (int b = 0; b < 2 * NB; ++b)
#pragma unroll
            for (int j = 0; j < 4; ++j) fine = fine && x.o[k][b][j] - x.o[k][b][j] == 0;
        const uint32_t col = 16 * k + (lane & 15);
        const bool there = col < count;
        const uint64_t bad = __builtin_amdgcn_ballot_w64(there && !fine && total == total);
        const uint32_t these = (uint32_t)(bad | bad >> 16 | bad >> 32 | bad >> 48) & 0xffff;
        spoilt |= (uint64_t)these << (16 * k);
        if (there && !((these >> (lane & 15)) & 1)) {
            const cache_column<T, NB> out(late, it, g, first + col, cols);
#pragma unroll
            for (int b = 0; b < 2 * NB; ++b) out.numbers(late, 16 * b + 4 * (lane >> 4), x.o[k][b], total);
            if (lane < 16) out.total(x.top[k], total);
        }
    }
#pragma unroll 1
    for (; spoilt; spoilt &= spoilt - 1) cache_again<T, NB>(late, it, g, first + __builtin_ctzll(spoilt), cols, all.from, all.to, lane);
}

// A launch and loads that depend on each other bound it: 6.7 us beside the 65 of 64 single tokens over 8192.
// Joins the chunks of the tiles that have several: of up to 16 chunks a wave for each column, of more a workgroup (or some columns in turn).  The chunks' factors first, then the
// sums, a quarter of the chunks a wave: loads that do not wait for each other.
template <typename T, int NB>
__global__ __launch_bounds__(256) void cache_join_kernel(cache_attn_args a, int cols)
{
    constexpr int pad = 32 * NB, per = (pad + 63) / 64;
    __shared__ float factor[2 * kCacheTarget], sums[4][pad];
    __shared__ float stats[2][4];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t index = blockIdx.x / (uint32_t)a.c.G;
    const int g = (int)(blockIdx.x - index * a.c.G);
    cache_item it;
    if (!cache_find(a, cols, index, true, lane, &it)) return;
    if (it.slot + (uint64_t)(it.chunks - 1) * it.q.tiles >= a.slots) return;       // so there are at most 2 kCacheTarget chunks
    const int64_t step = (int64_t)it.q.tiles * a.c.G * cols;
    const uint32_t width = cache_width(it.q.columns, cols), most = it.q.columns - it.tile * width, columns = most < width ? most : width;
    if (it.chunks <= 16) {                               // a wave for each column
        for (uint32_t column = blockIdx.y + w * gridDim.y; column < columns; column += 4 * gridDim.y) {
            const uint32_t col = it.tile * width + column;
            const int64_t base = ((int64_t)it.slot * a.c.G + g) * cols + col % (uint32_t)cols;
            const float2 s = (uint32_t)lane < it.chunks ? a.stat[base + lane * step] : make_float2(-INFINITY, 0);
            float top = s.x;
#pragma unroll
            for (int d = 8; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
            const float f = s.y == 0 ? 0.f : __builtin_amdgcn_exp2f(s.x - top);      // (sums without weight are zeros)
            float total = s.y == 0 ? 0.f : s.y * f, acc[per] = {};
#pragma unroll
            for (int d = 8; d >= 1; d >>= 1) total += __shfl_xor(total, d, 64);
            total = __shfl(total, 0, 64); top = __shfl(top, 0, 64);
            const float share = total == 0 ? 0.f : f / total;            // before the sums, which are no larger than the values then
            for (uint32_t k0 = 0; k0 < it.chunks; k0 += 4) {             // four at a time; behind the last one that one again, without weight
                float x[4][per];
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k) {
                    const float *part = a.part + (base + (k0 + k < it.chunks ? k0 + k : it.chunks - 1) * step) * pad;
#pragma unroll
                    for (int j = 0; j < per; ++j) x[k][j] = pad % 64 == 0 || lane + 64 * j < pad ? part[lane + 64 * j] : 0.f;
                }
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k) {
                    const float fk = __shfl(share, (int)(k0 + k), 64);
#pragma unroll
                    for (int j = 0; j < per; ++j) acc[j] += x[k][j] * fk;
                }
            }
            const uint32_t i = col / (uint32_t)a.R, h = g * a.R + col % (uint32_t)a.R;
            T *out = (T *)a.O + (it.row0 + i) * a.ldo + (int64_t)h * a.hdo;
#pragma unroll
            for (int j = 0; j < per; ++j) if (lane + 64 * j < a.c.D) out[lane + 64 * j] = (T)acc[j];
            if (a.lse && lane == 0) a.lse[(int64_t)h * a.tokens + it.row0 + i] = total == 0 ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * kCacheLn2;
        }
        return;
    }
    for (uint32_t column = blockIdx.y; column < columns; column += gridDim.y) {
        const uint32_t col = it.tile * width + column;
        const int64_t base = ((int64_t)it.slot * a.c.G + g) * cols + col % (uint32_t)cols;
        float top = -INFINITY, total = 0;
        for (uint32_t k = threadIdx.x; k < it.chunks; k += 256) top = fmaxf(top, a.stat[base + k * step].x);
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
        if (lane == 0) stats[0][w] = top;
        __syncthreads();
        top = fmaxf(fmaxf(stats[0][0], stats[0][1]), fmaxf(stats[0][2], stats[0][3]));
        for (uint32_t k = threadIdx.x; k < it.chunks; k += 256) {
            const float2 s = a.stat[base + k * step];
            const float f = s.y == 0 ? 0.f : __builtin_amdgcn_exp2f(s.x - top);      // (sums without weight are zeros)
            factor[k] = f;
            total += s.y == 0 ? 0.f : s.y * f;
        }
        total = cache_wave_sum(total);
        if (lane == 0) stats[1][w] = total;
        __syncthreads();
        total = (stats[1][0] + stats[1][1]) + (stats[1][2] + stats[1][3]);
        const float inverse = total == 0 ? 0.f : 1 / total;              // before the sums, as above
        float acc[per] = {};
#pragma unroll 8
        for (uint32_t k = w; k < it.chunks; k += 4) {
            const float *part = a.part + (base + k * step) * pad;
#pragma unroll
            for (int j = 0; j < per; ++j) if (pad % 64 == 0 || lane + 64 * j < pad) acc[j] += part[lane + 64 * j] * (factor[k] * inverse);
        }
#pragma unroll
        for (int j = 0; j < per; ++j) if (pad % 64 == 0 || lane + 64 * j < pad) sums[w][lane + 64 * j] = acc[j];
        __syncthreads();
        const uint32_t i = col / (uint32_t)a.R, h = g * a.R + col % (uint32_t)a.R;
        T *out = (T *)a.O + (it.row0 + i) * a.ldo + (int64_t)h * a.hdo;
        if ((int)threadIdx.x < a.c.D) {
            const int d = threadIdx.x;
            out[d] = (T)((sums[0][d] + sums[1][d]) + (sums[2][d] + sums[3][d]));
        }
        if (a.lse && threadIdx.x == 0) a.lse[(int64_t)h * a.tokens + it.row0 + i] = total == 0 ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * kCacheLn2;
        __syncthreads();
    }
}

// ---- launch -----------------------------------------------------------------------------------------------------------------

// What a call launches; by sizes that the host knows.
struct cache_choice {
    bool few;                            // tiles of 16 columns, or of 64 NQ
    int cols;
    int64_t items, slots;                // upper bounds; slots = 0: no request can have more than one chunk
    int64_t joins;                       // tiles of requests with more than one chunk, at most
    size_t part, stat, plan;             // bytes
    size_t bytes() const { return part + stat + plan; }
};


template <typename T>
cache_choice cache_choose(const cache_attn_args &a)
{
    cache_choice c;
    const int64_t requests = a.requests < a.tokens ? a.requests : a.tokens, columns = a.tokens * a.R;
    c.few = columns <= 16 * requests;
    c.cols = c.few ? 16 : 64 * cache_nq<T>(a.c.lay.nb);
    c.slots = a.width * a.c.P <= kCacheWhole ? 0 : cache_slots(a.c.G);
    const int64_t tiles = columns / c.cols + (c.few ? 1 : 2) * requests;
    c.joins = tiles < c.slots / 2 ? tiles : c.slots / 2;
    c.items = tiles + (c.slots ? ceil_div(kCacheTarget, a.c.G) : 0);
    const size_t rows = (size_t)c.slots * a.c.G * c.cols;
    c.part = rows * 32 * a.c.lay.nb * sizeof(float);
    c.stat = (rows * sizeof(float2) + 255) & ~(size_t)255;
    c.plan = a.requests > 64 || (!c.few && c.slots) ? ((2 + 3 * (((size_t)a.requests + 63) / 64)) * sizeof(uint32_t) + 255) & ~(size_t)255 : 0;
    return c;
}

template <typename T, int NB>
void cache_launch(const cache_attn_args &a, const cache_choice &c, hipStream_t st)
{
    constexpr int NQ = cache_nq<T>(NB);
    if (c.plan) cache_plan_kernel<<<1, a.requests <= 64 ? 64 : 1024, 0, st>>>(a, c.cols);
    if (c.few) cache_few_kernel<T, NB><<<(unsigned)(c.items * a.c.G), 256, 0, st>>>(a);
    else cache_many_kernel<T, NB, NQ><<<(unsigned)(c.items * a.c.G), 256, 0, st>>>(a);
    if (c.slots) cache_join_kernel<T, NB><<<dim3((unsigned)(c.joins * a.c.G), c.few ? (c.joins * a.c.G <= 256 ? 16 : 4) : c.cols / 8), 256, 0, st>>>(a, c.cols);
}

template <typename T> sp_status cache_attention(const cache_attn_args &a, const cache_choice &c, hipStream_t st);
template <typename T> cache_choice cache_choice_of(const cache_attn_args &a);

#define CACHE_ATTENTION_OF(T)                                                                        \
    template <> sp_status cache_attention<T>(const cache_attn_args &a, const cache_choice &c, hipStream_t st) \
    {                                                                                                \
        switch (a.c.lay.nb) {                                                                        \
        case 1: cache_launch<T, 1>(a, c, st); break;                                                 \
        case 2: cache_launch<T, 2>(a, c, st); break;                                                 \
        case 3: cache_launch<T, 3>(a, c, st); break;                                                 \
        case 4: cache_launch<T, 4>(a, c, st); break;                                                 \
        case 5: cache_launch<T, 5>(a, c, st); break;                                                 \
        case 6: cache_launch<T, 6>(a, c, st); break;                                                 \
        case 7: cache_launch<T, 7>(a, c, st); break;                                                 \
        default: cache_launch<T, 8>(a, c, st);                                                       \
        }                                                                                            \
        SP_HIP(hipGetLastError());                                                                   \
        return SP_OK;                                                                                \
    }                                                                                                \
    template <> cache_choice cache_choice_of<T>(const cache_attn_args &a) { return cache_choose<T>(a); }
