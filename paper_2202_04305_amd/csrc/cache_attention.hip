// Attention over the 4-bit cache: the entry points and their checks.  A wave for each row and head.
#include "cache.h"

namespace {

struct cache_attn_args {
    cache_view c;
    const void *Q;
    void *O;
    float *lse;
    const int32_t *table, *length, *start;
    int64_t ldq, hdq, ldo, hdo, ldt, width, requests, tokens;
    int H, R, causal;                    // R = H / G heads share a head of the cache
    float scale;
};

constexpr int kCachePer = 4;             // numbers of a lane: head sizes up to 256

__device__ __forceinline__ float cache_wave_sum(float v)
{
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d, 64);
    return v;
}

// top (running maximum), total and acc = sum of e^(s - top) V over the tokens [t0, t1) of request r, for one row and head; a wave, lanes
// across the head's numbers.  Every token is looked at alone, so that nothing that the row does not attend to can reach it.
template <typename T>
__device__ __forceinline__ void cache_row(const cache_attn_args &a, int64_t r, int64_t i, int h, int64_t t0, int64_t t1, int lane,
                                          float &top, float &total, float (&acc)[kCachePer])
{
    const int g = h / a.R, D = a.c.D;
    const T *row = (const T *)a.Q + i * a.ldq + h * a.hdq;
    float q[kCachePer];
#pragma unroll
    for (int k = 0; k < kCachePer; ++k) { q[k] = lane + 64 * k < D ? (float)row[lane + 64 * k] : 0.f; acc[k] = 0; }
    top = -INFINITY; total = 0;
    for (int64_t t = t0; t < t1; ++t) {
        const int64_t page = a.table[r * a.ldt + t / a.c.P];
        if (page < 0 || page >= a.c.pages) continue;
        const int u = (int)(t % a.c.P);
        const uint8_t *rec = a.c.record(page, g, u);
        float s = 0;
#pragma unroll
        for (int k = 0; k < kCachePer; ++k) if (lane + 64 * k < D) s += q[k] * cache_key(a.c, rec, u % kCacheTile, lane + 64 * k);
        s = cache_wave_sum(s) * a.scale;
        if (s == -INFINITY) continue;                    // weight 0
        const float up = s > top ? s : top;              // not a number: stays with the old maximum, the weight carries it
        const float old = top == -INFINITY ? 0.f : __expf(top - up), w = __expf(s - (up == -INFINITY ? 0.f : up));
        top = up;
        total = total * old + w;
#pragma unroll
        for (int k = 0; k < kCachePer; ++k) if (lane + 64 * k < D) acc[k] = acc[k] * old + w * cache_value(a.c, rec, u % kCacheTile, lane + 64 * k);
    }
}

template <typename T>
__global__ __launch_bounds__(256) void row_kernel(cache_attn_args a)
{
    const int64_t x = (int64_t)blockIdx.x * 4 + threadIdx.x / 64, i = x / a.H;
    const int h = (int)(x % a.H), lane = threadIdx.x % 64;
    if (i >= a.tokens || i < a.start[0] || i >= a.start[a.requests]) return;
    int64_t lo = 0, hi = a.requests;                     // the last request that begins at row i or before
    while (hi - lo > 1) { const int64_t mid = (lo + hi) / 2; if (a.start[mid] <= i) lo = mid; else hi = mid; }
    const int64_t len = a.length[lo], n = a.start[lo + 1] - a.start[lo];
    int64_t end = len < a.width * a.c.P ? len : a.width * a.c.P;
    if (a.causal && len - n + i - a.start[lo] + 1 < end) end = len - n + i - a.start[lo] + 1;
    float top, total, acc[kCachePer];
    cache_row<T>(a, lo, i, h, 0, end, lane, top, total, acc);
    T *out = (T *)a.O + i * a.ldo + h * a.hdo;
#pragma unroll
    for (int k = 0; k < kCachePer; ++k) if (lane + 64 * k < a.c.D) out[lane + 64 * k] = (T)(total == 0 ? 0.f : acc[k] / total);
    if (a.lse && lane == 0) a.lse[h * a.tokens + i] = total == 0 ? -INFINITY : top + logf(total);
}

sp_status check_problem(const sp_cache *c, const sp_cache_problem *p, cache_attn_args *a)
{
    if (!c || !p) return SP_ERR_NULL;
    if (p->dtype != (int)SP_F32 && p->dtype != (int)SP_F16 && p->dtype != (int)SP_BF16) return SP_ERR_DTYPE;
    const sp_status st = cache_check(c, &a->c);
    if (st == SP_ERR_SHAPE) return st;
    if (p->heads < 1 || p->heads > 65535 || p->heads % c->kvHeads || p->requests < 0 || p->tokens < 0 || p->width < 0 || p->ldt < p->width ||
        p->ldq < 0 || p->hdq < 0) return SP_ERR_SHAPE;
    const float s = (float)(p->scale * 1.4426950408889634);
    if (!(s - s == 0)) return SP_ERR_SHAPE;              // the kernels hold it in 32 bits: not finite there
    if (p->causal != 0 && p->causal != 1) return SP_ERR_UNSUPPORTED;
    SP_TRY(st);
    const int64_t top = (int64_t)1 << 31;
    if (p->requests >= top || p->tokens >= top) return SP_ERR_TOO_LARGE;
    if (ceil_div(p->tokens * p->heads, 4) >= (int64_t)1 << 24) return SP_ERR_TOO_LARGE;
    a->Q = p->Q; a->table = p->table; a->length = p->length; a->start = p->start;
    a->ldq = p->ldq; a->hdq = p->hdq; a->ldt = p->ldt; a->width = p->width; a->requests = p->requests; a->tokens = p->tokens;
    a->H = p->heads; a->R = p->heads / c->kvHeads; a->causal = p->causal; a->scale = (float)p->scale;
    return SP_OK;
}

}  // namespace

extern "C" sp_status sp_cache_attention_workspace(const sp_cache *c, const sp_cache_problem *p, size_t *bytes)
{
    if (!bytes) return SP_ERR_NULL;
    *bytes = 0;
    cache_attn_args a;
    return check_problem(c, p, &a);
}

extern "C" sp_status sp_cache_attention(const sp_cache *c, const sp_cache_problem *p, void *O, int64_t ldo, int64_t hdo, float *lse,
                                        void *workspace, size_t workspaceBytes, void *stream)
{
    cache_attn_args a;
    memset(&a, 0, sizeof(a));
    SP_TRY(check_problem(c, p, &a));
    if ((a.tokens > 1 && ldo < a.c.D) || (a.H > 1 && hdo < a.c.D)) return SP_ERR_SHAPE;
    if (a.tokens == 0 || a.requests == 0) return SP_OK;
    if (!O || !a.Q || !a.length || !a.start || (a.width && !a.table) || !cache_has_memory(a.c)) return SP_ERR_NULL;
    (void)workspace; (void)workspaceBytes;
    a.O = O; a.ldo = ldo; a.hdo = hdo; a.lse = lse;
    const int n = (int)ceil_div(a.tokens * a.H, 4);
    hipStream_t st = (hipStream_t)stream;
    if (p->dtype == SP_F32) row_kernel<float><<<n, 256, 0, st>>>(a);
    else if (p->dtype == SP_F16) row_kernel<cache_f16><<<n, 256, 0, st>>>(a);
    else row_kernel<cache_bf16><<<n, 256, 0, st>>>(a);
    SP_HIP(hipGetLastError());
    return SP_OK;
}
