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
__device__ __forceinline__ int32_t saturated(int64_t x) { return x > INT32_MAX ? INT32_MAX : (int32_t)x; }

constexpr int kMapGroup = 64;            // requests of a workgroup

// One launch: workgroup (b, y) sums up the requests before its 64, scans its own, and writes slice y of their pages and tokens.  No
// workgroup reads what another writes: a token in a new page takes the page from the list, as whoever writes the table does.
__global__ __launch_bounds__(256) void map_kernel(sp_cache_step s)
{
    __shared__ int64_t sum[2][256];
    __shared__ int64_t first_token[kMapGroup + 1], first_page[kMapGroup + 1], length[kMapGroup];
    const int64_t r0 = (int64_t)blockIdx.x * kMapGroup, P = s.pageTokens;
    const int count = (int)(s.requests - r0 < kMapGroup ? s.requests - r0 : kMapGroup), tid = threadIdx.x;
    int64_t tokens = 0, pages = 0;
    for (int64_t r = tid; r < r0; r += 256) {
        const int64_t len = at_least_0(s.length[r]), add = at_least_0(s.added[r]);
        tokens += add;
        pages += (len + add + P - 1) / P - (len + P - 1) / P;
    }
    sum[0][tid] = tokens; sum[1][tid] = pages;
    __syncthreads();
    for (int d = 128; d >= 1; d >>= 1) {
        if (tid < d) { sum[0][tid] += sum[0][tid + d]; sum[1][tid] += sum[1][tid + d]; }
        __syncthreads();
    }
    if (tid == 0) {
        int64_t t = sum[0][0], p = sum[1][0];
        for (int k = 0; k < count; ++k) {
            const int64_t len = at_least_0(s.length[r0 + k]), add = at_least_0(s.added[r0 + k]);
            first_token[k] = t; first_page[k] = p; length[k] = len;
            t += add;
            p += (len + add + P - 1) / P - (len + P - 1) / P;
        }
        first_token[count] = t; first_page[count] = p;
    }
    __syncthreads();
    const int64_t taken = *s.taken;
    auto free_page = [&](int64_t k) -> int64_t {
        k += taken;
        const int64_t page = k >= 0 && k < s.freeCount ? s.freePages[k] : -1;
        return page >= 0 && page < s.pages ? page : -1;
    };
    auto request_of = [&](const int64_t *first, int64_t x) {             // the last one that begins at x or before
        int lo = 0, hi = count;
        while (hi - lo > 1) { const int mid = (lo + hi) / 2; if (first[mid] <= x) lo = mid; else hi = mid; }
        return lo;
    };
    const int64_t step = (int64_t)gridDim.y * 256, me = (int64_t)blockIdx.y * 256 + tid;
    for (int64_t x = first_page[0] + me; x < first_page[count]; x += step) {
        const int k = request_of(first_page, x);
        const int64_t at = (length[k] + P - 1) / P + x - first_page[k];
        if (at < s.width) s.table[(r0 + k) * s.ldt + at] = (int32_t)free_page(x);
    }
    const int64_t end = first_token[count] < s.tokens ? first_token[count] : s.tokens;
    for (int64_t x = first_token[0] + me; x < end; x += step) {
        const int k = request_of(first_token, x);
        const int64_t position = length[k] + x - first_token[k], at = position / P, held = (length[k] + P - 1) / P;
        int64_t page = -1;
        if (at < s.width) page = at >= held ? free_page(first_page[k] + at - held) : s.table[(r0 + k) * s.ldt + at];
        s.position[x] = saturated(position);
        s.slot[x] = page >= 0 && page < s.pages ? (int32_t)(page * P + position % P) : -1;
    }
    const bool last = r0 + count == s.requests;
    if (last) for (int64_t x = end + me; x < s.tokens; x += step) s.position[x] = s.slot[x] = -1;
    if (blockIdx.y == 0) {
        if (tid < count) {
            s.start[r0 + tid] = saturated(first_token[tid]);
            s.lengthOut[r0 + tid] = saturated(length[tid] + at_least_0(s.added[r0 + tid]));
        }
        if (last && tid == 0) {
            s.start[s.requests] = saturated(first_token[count]);
            *s.takenOut = saturated(taken + first_page[count]);
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
    // a workgroup for each 64 requests (one where there are none), cut into slices of 2048 tokens of what the step has room for
    const int64_t groups = s->requests ? ceil_div(s->requests, kMapGroup) : 1;
    int64_t slices = ceil_div(ceil_div(s->tokens, groups), 2048);
    slices = slices < 1 ? 1 : slices > 256 ? 256 : slices;
    map_kernel<<<dim3((unsigned)groups, (unsigned)slices), 256, 0, (hipStream_t)stream>>>(*s);
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

// A thread for each block of 32 numbers of K or V.
template <typename T>
__global__ __launch_bounds__(256) void store_kernel(cache_rows a)
{
    const cache_view &c = a.c;
    const int nb = c.lay.nb;
    const int64_t n = a.tokens * c.G * 2 * nb;
    for (int64_t x = blockIdx.x * (int64_t)256 + threadIdx.x; x < n; x += (int64_t)gridDim.x * 256) {
        const int s = (int)(x % nb), which = (int)(x / nb % 2), g = (int)(x / (2 * nb) % c.G);
        const int64_t i = x / (2 * nb) / c.G;
        const int64_t slot = a.slot[i];
        if (slot < 0 || slot >= c.pages * c.P) continue;
        const T *in = which ? (const T *)a.V + i * a.ldv + g * a.hdv : (const T *)a.K + i * a.ldk + g * a.hdk;
        float v[kCacheBlock], top = 0;
        bool finite = true;
        for (int d = 0; d < kCacheBlock; ++d) {
            v[d] = 32 * s + d < c.D ? (float)in[32 * s + d] : 0.f;
            top = fmaxf(top, fabsf(v[d]));
            finite = finite && v[d] - v[d] == 0;
        }
        const int e = cache_exponent(finite ? top : 0.f);
        const float scale = __uint_as_float((uint32_t)(e + 127) << 23);
        uint32_t code[4];
        for (int w = 0; w < 4; ++w) {
            uint32_t q = 0;
            q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[8 * w], v[8 * w + 1], scale, 0);
            q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[8 * w + 2], v[8 * w + 3], scale, 1);
            q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[8 * w + 4], v[8 * w + 5], scale, 2);
            q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[8 * w + 6], v[8 * w + 7], scale, 3);
            code[w] = q;
        }
        const int t = (int)(slot % c.P);
        uint8_t *rec = c.record(slot / c.P, g, t);
        const int u = t % kCacheTile;
        rec[(which ? c.lay.v_scales() : c.lay.k_scales()) + u * c.lay.sb + s] = finite ? (uint8_t)(e + 127) : (uint8_t)kCacheNaN;
        if (!which) for (int w = 0; w < 4; ++w) ((uint32_t *)rec)[(u * 4 + w) * nb + s] = code[w];
        else for (int k = 0; k < 16; ++k) {
            const uint32_t lo = (code[k / 8] >> (4 * (k % 8))) & 15, hi = (code[2 + k / 8] >> (4 * (k % 8))) & 15;
            rec[c.lay.v_codes() + (((u >> 2) * 16 + k) * nb + s) * 4 + (u & 3)] = (uint8_t)(lo | hi << 4);
        }
    }
}

// A thread for each number of K and of V.
template <typename T>
__global__ __launch_bounds__(256) void load_kernel(cache_rows a)
{
    const cache_view &c = a.c;
    const int64_t n = a.tokens * c.G * c.D;
    for (int64_t x = blockIdx.x * (int64_t)256 + threadIdx.x; x < n; x += (int64_t)gridDim.x * 256) {
        const int d = (int)(x % c.D), g = (int)(x / c.D % c.G);
        const int64_t i = x / c.D / c.G;
        const int64_t slot = a.slot[i];
        float k = 0, v = 0;
        if (slot >= 0 && slot < c.pages * c.P) {
            const int t = (int)(slot % c.P);
            const uint8_t *rec = c.record(slot / c.P, g, t);
            k = cache_key(c, rec, t % kCacheTile, d);
            v = cache_value(c, rec, t % kCacheTile, d);
        }
        ((T *)a.Kout)[i * a.ldk + g * a.hdk + d] = (T)k;
        ((T *)a.Vout)[i * a.ldv + g * a.hdv + d] = (T)v;
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
    if (tokens >= (int64_t)1 << 31) return SP_ERR_TOO_LARGE;
    a->tokens = tokens;
    if (tokens && (!a->slot || !cache_has_memory(a->c) || (out ? !a->Kout || !a->Vout : !a->K || !a->V))) return SP_ERR_NULL;
    return SP_OK;
}

int grid(int64_t threads) { const int64_t b = ceil_div(threads, 256); return (int)(b < 65536 ? b : 65536); }

}  // namespace

extern "C" sp_status sp_cache_store(const sp_cache *c, int dtype, int64_t tokens, const int32_t *slot, const void *K, int64_t ldk, int64_t hdk,
                                    const void *V, int64_t ldv, int64_t hdv, void *stream)
{
    cache_rows a = {{}, slot, 0, K, V, nullptr, nullptr, ldk, hdk, ldv, hdv};
    SP_TRY(check_rows(c, dtype, tokens, false, &a));
    if (tokens == 0 || a.c.pages == 0) return SP_OK;
    const int n = grid(tokens * a.c.G * 2 * a.c.lay.nb);
    hipStream_t st = (hipStream_t)stream;
    if (dtype == SP_F32) store_kernel<float><<<n, 256, 0, st>>>(a);
    else if (dtype == SP_F16) store_kernel<cache_f16><<<n, 256, 0, st>>>(a);
    else store_kernel<cache_bf16><<<n, 256, 0, st>>>(a);
    SP_HIP(hipGetLastError());
    return SP_OK;
}

extern "C" sp_status sp_cache_load(const sp_cache *c, int dtype, int64_t tokens, const int32_t *slot, void *K, int64_t ldk, int64_t hdk,
                                   void *V, int64_t ldv, int64_t hdv, void *stream)
{
    cache_rows a = {{}, slot, 0, nullptr, nullptr, K, V, ldk, hdk, ldv, hdv};
    SP_TRY(check_rows(c, dtype, tokens, true, &a));
    if (tokens == 0) return SP_OK;
    const int n = grid(tokens * a.c.G * a.c.D);
    hipStream_t st = (hipStream_t)stream;
    if (dtype == SP_F32) load_kernel<float><<<n, 256, 0, st>>>(a);
    else if (dtype == SP_F16) load_kernel<cache_f16><<<n, 256, 0, st>>>(a);
    else load_kernel<cache_bf16><<<n, 256, 0, st>>>(a);
    SP_HIP(hipGetLastError());
    return SP_OK;
}
