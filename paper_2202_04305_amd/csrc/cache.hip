// The 4-bit cache: its size, the pages and slots of a step, rows into the pages and back.
#include "cache.h"

extern "C" sp_status sp_cache_bytes(const sp_cache *c, size_t *bytes)
{
    if (!bytes) return SP_ERR_NULL;
    *bytes = 0;
    cache_view v;
    SP_TRY(cache_check(c, &v));
    *bytes = (size_t)v.pages * v.G * (v.P / kCacheTile) * v.lay.record();
    return SP_OK;
}

// ---- pages and slots --------------------------------------------------------------------------------------------------------

namespace {

__device__ __forceinline__ int64_t at_least_0(int32_t x) { return x < 0 ? 0 : x; }
__device__ __forceinline__ int32_t saturated(int64_t x) { return x > INT32_MAX ? INT32_MAX : x < INT32_MIN ? INT32_MIN : (int32_t)x; }

constexpr int kMapGroup = 64;            // requests of a workgroup: a wave scans them

__device__ __forceinline__ int64_t map_scan(int64_t v, int lane)             // sum of lanes 0 .. lane
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) { const int64_t o = __shfl_up(v, d, 64); v += lane >= d ? o : 0; }
    return v;
}

// One launch: workgroup (b, y) sums up the requests before its 64, scans its own, and writes slice y of their pages and tokens.  No
// workgroup reads what another writes: a token in a new page takes the page from the list, as whoever writes the table does.
// A launch's latency bounds it (four loads that depend on each other): 8 requests of one token 2.7 us, 509 requests of 250000 tokens 8.4.
__global__ __launch_bounds__(256) void map_kernel(sp_cache_step s, spmi_divisor32 by_page)
{
    __shared__ int64_t before[2][4];
    __shared__ int64_t first_token[kMapGroup + 1], first_page[kMapGroup + 1];
    __shared__ uint32_t length[kMapGroup];
    const int64_t r0 = (int64_t)blockIdx.x * kMapGroup;
    const uint32_t P = s.pageTokens;
    const int count = (int)(s.requests - r0 < kMapGroup ? s.requests - r0 : kMapGroup), tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    // pages of `tokens` < 2^32 tokens
    auto pages_of = [&](int64_t tokens) { return tokens <= INT32_MAX - (int64_t)P ? (int64_t)spmi_div_by32((uint32_t)tokens + P - 1, by_page) : (tokens + P - 1) / P; };
    auto needed = [&](int64_t len, int64_t add) { return pages_of(len + add) - pages_of(len); };
    int64_t tokens = 0, pages = 0;
    for (int64_t r = tid; r < r0; r += 256) {
        const int64_t len = at_least_0(s.length[r]), add = at_least_0(s.added[r]);
        tokens += add;
        pages += needed(len, add);
    }
    const int64_t taken = *s.taken;
    int64_t len = 0, add = 0;
    if (w == 0 && lane < count) { len = at_least_0(s.length[r0 + lane]); add = at_least_0(s.added[r0 + lane]); }
    if (r0) {
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) { tokens += __shfl_xor(tokens, d, 64); pages += __shfl_xor(pages, d, 64); }
        if (lane == 0) { before[0][w] = tokens; before[1][w] = pages; }
        __syncthreads();
        tokens = (before[0][0] + before[0][1]) + (before[0][2] + before[0][3]);
        pages = (before[1][0] + before[1][1]) + (before[1][2] + before[1][3]);
    }
    if (w == 0) {
        const int64_t more = needed(len, add);
        const int64_t t = tokens + map_scan(add, lane), p = pages + map_scan(more, lane);
        first_token[lane] = t - add; first_page[lane] = p - more;
        length[lane] = (uint32_t)len;
        if (lane == 63) { first_token[64] = t; first_page[64] = p; }
    }
    __syncthreads();
    const int64_t all_tokens = first_token[64], all_pages = first_page[64];          // requests beyond `count` have neither
    auto free_page = [&](int64_t k) -> int64_t {
        k += taken;
        const int64_t page = k >= 0 && k < s.freeCount ? s.freePages[k] : -1;
        return page >= 0 && page < s.pages ? page : -1;
    };
    auto request_of = [&](const int64_t *first, int64_t x) {             // the last one that begins at x or before
        int k = 0;
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) k += k + d < count && first[k + d] <= x ? d : 0;
        return k;
    };
    const int64_t step = (int64_t)gridDim.y * 256, me = (int64_t)blockIdx.y * 256 + tid;
    for (int64_t x = first_page[0] + me; x < all_pages; x += step) {
        const int k = request_of(first_page, x);
        const int64_t at = pages_of(length[k]) + x - first_page[k];
        if (at < s.width) s.table[(r0 + k) * s.ldt + at] = (int32_t)free_page(x);
    }
    const int64_t end = all_tokens < s.tokens ? all_tokens : s.tokens;
    for (int64_t x = first_token[0] + me; x < end; x += step) {
        const int k = request_of(first_token, x);
        const int64_t position = length[k] + x - first_token[k], held = pages_of(length[k]);
        int64_t slot = -1;
        if (position <= INT32_MAX) {
            const uint32_t at = spmi_div_by32((uint32_t)position, by_page);
            int64_t page = -1;
            if (at < s.width) page = at >= held ? free_page(first_page[k] + at - held) : s.table[(r0 + k) * s.ldt + at];
            if (page >= 0 && page < s.pages) slot = page * P + (uint32_t)position - at * P;
        }
        s.position[x] = saturated(position);
        s.slot[x] = (int32_t)slot;
    }
    const bool last = r0 + count == s.requests;
    if (last) for (int64_t x = end + me; x < s.tokens; x += step) s.position[x] = s.slot[x] = -1;
    if (blockIdx.y == 0) {
        if (w == 0 && lane < count) {
            s.start[r0 + lane] = saturated(first_token[lane]);
            s.lengthOut[r0 + lane] = saturated(len + add);
        }
        if (last && tid == 0) {
            s.start[s.requests] = saturated(all_tokens);
            *s.takenOut = saturated(taken + all_pages);
        }
    }
}

}  // namespace

extern "C" sp_status sp_cache_map(const sp_cache_step *s, void *stream)
{
    if (!s) return SP_ERR_NULL;
    if (s->requests < 0 || s->tokens < 0 || s->pages < 0 || s->freeCount < 0 || s->width < 0 || s->ldt < s->width || s->pageTokens < kCacheTile ||
        s->pageTokens % kCacheTile) return SP_ERR_SHAPE;
    const int64_t top = (int64_t)1 << 31;
    if (s->pages >= ceil_div(top, s->pageTokens) || s->requests >= top || s->tokens >= top) return SP_ERR_TOO_LARGE;
    if (!s->taken || !s->takenOut || !s->start || (s->requests && (!s->length || !s->added || !s->lengthOut || (s->width && !s->table))) ||
        (s->freeCount && !s->freePages) || (s->tokens && (!s->position || !s->slot))) return SP_ERR_NULL;
    // a workgroup for each 64 requests (one where there are none), cut into slices of 1024 tokens of what the step has room for
    const int64_t groups = s->requests ? ceil_div(s->requests, kMapGroup) : 1;
    int64_t slices = ceil_div(ceil_div(s->tokens, groups), 1024);
    slices = slices < 1 ? 1 : slices > 256 ? 256 : slices;
    if (groups >= (int64_t)1 << 24) return SP_ERR_TOO_LARGE;
    map_kernel<<<dim3((unsigned)groups, (unsigned)slices), 256, 0, (hipStream_t)stream>>>(*s, spmi_make_divisor32(s->pageTokens));
    SP_HIP(hipGetLastError());
    return SP_OK;
}

// ---- rows into the pages and back -------------------------------------------------------------------------------------------

namespace {

struct cache_rows {
    cache_view c;
    const int32_t *slot;
    int64_t tokens;
    const void *K, *V;
    void *Kout, *Vout;
    int64_t ldk, hdk, ldv, hdv;
};

// The least e with top <= 7 * 2^e, within the range.
__device__ __forceinline__ int cache_exponent(float top)
{
    int e;
    const float m = frexpf(top, &e);                     // top = m 2^e, m in [0.5, 1): 7 * 2^(e - 3) = 0.875 * 2^e
    e -= m > 0.875f ? 2 : 3;
    return e < kCacheMinExp ? kCacheMinExp : e > kCacheMaxExp ? kCacheMaxExp : e;
}

constexpr int kStoreTokens = 32;         // of a workgroup, which takes one head of them

// Eight numbers of a row, zeros behind its end.
template <typename T>
__device__ __forceinline__ cache_row8<T> load8(const T *row, int d0, int D, bool vec)
{
    cache_row8<T> v = {};
    if (vec) { if (d0 < D) v = *(const cache_row8<T> *)(row + d0); }
    else
#pragma unroll
        for (int j = 0; j < 8; ++j) if (d0 + j < D) v[j] = row[d0 + j];
    return v;
}

// Rows into the pages.  Four neighbouring lanes have a block of 32 numbers, 8 each, which are a word of K as they lie.  A token's values are
// every fourth byte of 64 NB, so the tokens of a workgroup meet in the LDS: neighbours that share the words of four tokens there are a group, which
// goes out as words if it has all four, as bytes otherwise.  The rows' bytes and the instructions (400 a wave) bound it alike: 32768 bf16 rows of 8
// heads of 128 take 38 us, 4.5 TB/s of 170 MB (50 with the places worked out for each word).
template <typename T, int NB>
__global__ __launch_bounds__(256) void store_kernel(cache_rows a, int vec)
{
    constexpr int words = 4 * NB, row = 16 * NB;         // lanes of a token; words of four tokens' values
    __shared__ uint32_t values[kStoreTokens][row];       // [group]
    __shared__ uint8_t *record[kStoreTokens], *to[kStoreTokens];         // of a token (null: not stored); of a group
    __shared__ uint32_t place[kStoreTokens], mask[kStoreTokens];         // of a token: its number in the record + 16 * its group; of a group
    const cache_view &c = a.c;
    const uint32_t window = blockIdx.x / (uint32_t)c.G, head = blockIdx.x - window * (uint32_t)c.G;
    const int64_t i0 = (int64_t)window * kStoreTokens;
    const int tokens = (int)(a.tokens - i0 < kStoreTokens ? a.tokens - i0 : kStoreTokens), g = (int)head;
    const int lane = threadIdx.x & 63;
    int64_t slot = -1;
    if ((int)threadIdx.x < tokens) slot = a.slot[i0 + threadIdx.x];
    // all rows are asked for at once, before it is known where they go
    constexpr int each = (kStoreTokens * words + 255) / 256;
    cache_row8<T> in[each][2];
#pragma unroll
    for (int k = 0; k < each; ++k) {
        const int x = threadIdx.x + 256 * k, i = x / words, d0 = x % words * 8;
        if (i >= tokens) continue;
        in[k][0] = load8<T>((const T *)a.K + (i0 + i) * a.ldk + g * a.hdk, d0, c.D, vec);
        in[k][1] = load8<T>((const T *)a.V + (i0 + i) * a.ldv + g * a.hdv, d0, c.D, vec);
    }
    if (threadIdx.x < 64) {
        if (slot >= c.pages * c.P) slot = -1;
        if (lane < kStoreTokens) mask[lane] = 0;
        const int four = slot < 0 ? -1 : (int)(slot >> 2), before = __shfl_up(four, 1, 64);
        const bool first = lane == 0 || four < 0 || four != before;
        const int group = __popcll(__builtin_amdgcn_ballot_w64(first) & (~0ull >> (63 - lane))) - 1;
        if (lane < tokens) {
            const uint32_t t = slot < 0 ? 0 : (uint32_t)slot % (uint32_t)c.P, u = t % kCacheTile;
            uint8_t *rec = slot < 0 ? nullptr : c.record((uint32_t)slot / (uint32_t)c.P, g, (int)t);
            record[lane] = rec;
            place[lane] = u + 16 * group;
            if (first && rec) to[group] = rec + c.lay.v_codes() + (u >> 2) * (row * 4);
            if (rec) atomicOr(&mask[group], 1u << (u & 3));
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < each; ++k) {                     // the four lanes of a block stay together
        const int x = threadIdx.x + 256 * k, i = x / words, s = (x % words) / 4, q = x & 3;
        if (i >= tokens) continue;
        uint8_t *rec = record[i];
        if (!rec) continue;
        const int u = place[i] & 15, group = place[i] >> 4;
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            float v[8], top = 0, none = 0;               // none: 0, or not a number
#pragma unroll
            for (int j = 0; j < 8; ++j) { v[j] = (float)in[k][which][j]; top = fmaxf(top, fabsf(v[j])); none += v[j] - v[j]; }
            top = fmaxf(top, __shfl_xor(top, 1, 64)); none += __shfl_xor(none, 1, 64);
            top = fmaxf(top, __shfl_xor(top, 2, 64)); none += __shfl_xor(none, 2, 64);
            const bool finite = none == 0;
            const int e = cache_exponent(finite ? top : 0.f);
            const float scale = __uint_as_float((uint32_t)(e + 127) << 23);
            uint32_t code = 0;
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[0], v[1], scale, 0);
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[2], v[3], scale, 1);
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[4], v[5], scale, 2);
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[6], v[7], scale, 3);
            if (q == 0) rec[(which ? c.lay.v_scales() : c.lay.k_scales()) + u * c.lay.sb + s] = finite ? (uint8_t)(e + 127) : (uint8_t)kCacheNaN;
            if (!which) ((uint32_t *)rec)[(u * 4 + q) * NB + s] = code;
            else {
                // numbers 32 s + n and 32 s + 16 + n share a byte: lanes q and q + 2, of which each writes four, n = 8 (q & 1) + 4 (q >> 1) + 0 .. 3
                const uint32_t other = __shfl_xor(code, 2, 64), lo = q < 2 ? code & 0xffff : other >> 16, hi = q < 2 ? other & 0xffff : code >> 16;
                uint8_t *at = (uint8_t *)&values[group][(8 * (q & 1) + 4 * (q >> 1)) * NB + s] + (u & 3);
#pragma unroll
                for (int j = 0; j < 4; ++j) at[j * NB * 4] = (uint8_t)(((lo >> (4 * j)) & 15) | ((hi >> (4 * j)) & 15) << 4);
            }
        }
    }
    __syncthreads();
#pragma unroll 1
    for (int x = threadIdx.x; x < tokens * row; x += 256) {
        const int group = x / row, k = x % row;
        const uint32_t some = mask[group];
        if (!some) continue;                             // there are fewer groups than tokens, or its token is not stored
        uint8_t *at = to[group] + k * 4;
        const uint32_t word = values[group][k];
        if (some == 15) *(uint32_t *)at = word;
        else
#pragma unroll
            for (int j = 0; j < 4; ++j) if ((some >> j) & 1) at[j] = (uint8_t)(word >> (8 * j));
    }
}

// Eight codes, to pairs of bf16.
__device__ __forceinline__ void cache_eight(uint32_t word, float scale, uint32_t (&x)[4])
{
    x[0] = cache_convert<0>(word, scale); x[1] = cache_convert<1>(word, scale); x[2] = cache_convert<2>(word, scale); x[3] = cache_convert<3>(word, scale);
}
template <typename T>
__device__ __forceinline__ void store8(T *row, int d0, int D, bool vec, const uint32_t (&x)[4])
{
    cache_row8<T> v;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (T)__uint_as_float(j % 2 ? x[j / 2] & 0xffff0000u : x[j / 2] << 16);
    if (vec) { if (d0 < D) *(cache_row8<T> *)(row + d0) = v; }
    else
#pragma unroll
        for (int j = 0; j < 8; ++j) if (d0 + j < D) row[d0 + j] = v[j];
}

// Rows out of the pages: a lane for 8 numbers of K and of V.  Their bytes bound it: 32768 bf16 rows of 8 heads of 128 take 37 us, 4.6 TB/s of 170 MB,
// though V's bytes are loaded one by one (a token's lie in two lines).
template <typename T, int NB>
__global__ __launch_bounds__(256) void load_kernel(cache_rows a, int vec)
{
    constexpr int words = 4 * NB;
    const cache_view &c = a.c;
    const int64_t n = a.tokens * c.G * words;
    for (int64_t x = blockIdx.x * (int64_t)256 + threadIdx.x; x < n; x += (int64_t)gridDim.x * 256) {
        const int64_t r = x / words, i = n <= INT32_MAX ? (uint32_t)r / (uint32_t)c.G : r / c.G;
        const int g = (int)(r - i * c.G), s = (int)(x % words) / 4, q = (int)(x & 3), d0 = 32 * s + 8 * q;
        const int64_t slot = a.slot[i];
        uint32_t k[4] = {}, v[4] = {};                   // as pairs of bf16
        if (slot >= 0 && slot < c.pages * c.P) {
            const int t = (int)((uint32_t)slot % (uint32_t)c.P), u = t % kCacheTile;
            const uint8_t *rec = c.record((uint32_t)slot / (uint32_t)c.P, g, t);
            const uint32_t kw = ((const uint32_t *)rec)[(u * 4 + q) * NB + s];
            const uint8_t *b = rec + c.lay.v_codes() + (((u >> 2) * 16 + 8 * (q & 1)) * NB + s) * 4 + (u & 3);
            uint32_t vw = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) vw |= (((uint32_t)b[j * NB * 4] >> (q & 2 ? 4 : 0)) & 15) << (4 * j);
            const float ks = __uint_as_float((uint32_t)rec[c.lay.k_scales() + u * c.lay.sb + s] << 23), vs = __uint_as_float((uint32_t)rec[c.lay.v_scales() + u * c.lay.sb + s] << 23);
            cache_eight(kw, ks, k);
            cache_eight(vw, vs, v);
        }
        store8<T>((T *)a.Kout + i * a.ldk + g * a.hdk, d0, c.D, vec, k);
        store8<T>((T *)a.Vout + i * a.ldv + g * a.hdv, d0, c.D, vec, v);
    }
}

sp_status check_rows(const sp_cache *c, int dtype, int64_t tokens, bool out, cache_rows *a)
{
    SP_TRY(c ? SP_OK : SP_ERR_NULL);
    if (dtype != (int)SP_F32 && dtype != (int)SP_F16 && dtype != (int)SP_BF16) return SP_ERR_DTYPE;
    if (tokens < 0) return SP_ERR_SHAPE;
    const int64_t least = out ? c->headDim : 0;
    if (out ? (tokens > 1 && (a->ldk < least || a->ldv < least)) || (c->kvHeads > 1 && (a->hdk < least || a->hdv < least))
            : a->ldk < 0 || a->ldv < 0 || a->hdk < 0 || a->hdv < 0) return SP_ERR_SHAPE;
    SP_TRY(cache_check(c, &a->c));
    if (tokens >= (int64_t)1 << 31 || ceil_div(tokens, kStoreTokens) * c->kvHeads >= (int64_t)1 << 24) return SP_ERR_TOO_LARGE;        // 2^32 threads of a launch
    a->tokens = tokens;
    if (tokens && (!a->slot || !cache_has_memory(a->c) || (out ? !a->Kout || !a->Vout : !a->K || !a->V))) return SP_ERR_NULL;
    return SP_OK;
}

// Can rows be read and written 8 numbers at a time?
bool aligned(const cache_rows &a, int size)
{
    const int64_t stray = (uintptr_t)a.K | (uintptr_t)a.V | (uintptr_t)a.Kout | (uintptr_t)a.Vout | (uintptr_t)(size * (a.ldk | a.hdk | a.ldv | a.hdv));
    return a.c.D % 8 == 0 && stray % 16 == 0;
}

template <typename T, int NB>
void launch_rows(const cache_rows &a, bool store, hipStream_t st)
{
    const int vec = aligned(a, sizeof(T));
    if (store) store_kernel<T, NB><<<(unsigned)(ceil_div(a.tokens, kStoreTokens) * a.c.G), 256, 0, st>>>(a, vec);
    else {
        const int64_t blocks = ceil_div(a.tokens * a.c.G * 4 * NB, 256);
        load_kernel<T, NB><<<(unsigned)(blocks < 65536 ? blocks : 65536), 256, 0, st>>>(a, vec);
    }
}

template <typename T>
void launch_rows_of(const cache_rows &a, bool store, hipStream_t st)
{
    switch (a.c.lay.nb) {
    case 1: return launch_rows<T, 1>(a, store, st);
    case 2: return launch_rows<T, 2>(a, store, st);
    case 3: return launch_rows<T, 3>(a, store, st);
    case 4: return launch_rows<T, 4>(a, store, st);
    case 5: return launch_rows<T, 5>(a, store, st);
    case 6: return launch_rows<T, 6>(a, store, st);
    case 7: return launch_rows<T, 7>(a, store, st);
    default: return launch_rows<T, 8>(a, store, st);
    }
}

sp_status run_rows(const cache_rows &a, int dtype, bool store, hipStream_t st)
{
    if (dtype == SP_F32) launch_rows_of<float>(a, store, st);
    else if (dtype == SP_F16) launch_rows_of<cache_f16>(a, store, st);
    else launch_rows_of<cache_bf16>(a, store, st);
    SP_HIP(hipGetLastError());
    return SP_OK;
}

}  // namespace

extern "C" sp_status sp_cache_store(const sp_cache *c, int dtype, int64_t tokens, const int32_t *slot, const void *K, int64_t ldk, int64_t hdk,
                                    const void *V, int64_t ldv, int64_t hdv, void *stream)
{
    cache_rows a = {{}, slot, 0, K, V, nullptr, nullptr, ldk, hdk, ldv, hdv};
    SP_TRY(check_rows(c, dtype, tokens, false, &a));
    if (tokens == 0 || a.c.pages == 0) return SP_OK;
    return run_rows(a, dtype, true, (hipStream_t)stream);
}

extern "C" sp_status sp_cache_load(const sp_cache *c, int dtype, int64_t tokens, const int32_t *slot, void *K, int64_t ldk, int64_t hdk,
                                   void *V, int64_t ldv, int64_t hdv, void *stream)
{
    cache_rows a = {{}, slot, 0, nullptr, nullptr, K, V, ldk, hdk, ldv, hdv};
    SP_TRY(check_rows(c, dtype, tokens, true, &a));
    if (tokens == 0) return SP_OK;
    return run_rows(a, dtype, false, (hipStream_t)stream);
}
