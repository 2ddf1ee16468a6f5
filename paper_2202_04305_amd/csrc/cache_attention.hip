// Attention over the 4-bit cache: the entry points and their checks.
#include "cache_attention.h"

template <> cache_choice cache_choice_of<float>(const cache_attn_args &a);
template <> cache_choice cache_choice_of<cache_f16>(const cache_attn_args &a);
template <> cache_choice cache_choice_of<cache_bf16>(const cache_attn_args &a);
template <> sp_status cache_attention<float>(const cache_attn_args &a, const cache_choice &c, hipStream_t st);
template <> sp_status cache_attention<cache_f16>(const cache_attn_args &a, const cache_choice &c, hipStream_t st);
template <> sp_status cache_attention<cache_bf16>(const cache_attn_args &a, const cache_choice &c, hipStream_t st);

namespace {

sp_status check_problem(const sp_cache *c, const sp_cache_problem *p, cache_attn_args *a, cache_choice *choice)
{
    if (!c || !p) return SP_ERR_NULL;
    if (p->dtype != (int)SP_F32 && p->dtype != (int)SP_F16 && p->dtype != (int)SP_BF16) return SP_ERR_DTYPE;
    memset(a, 0, sizeof(*a));
    const sp_status st = cache_check(c, &a->c);
    if (st == SP_ERR_SHAPE) return st;
    if (p->heads < 1 || p->heads > 65535 || p->heads % c->kvHeads || p->requests < 0 || p->tokens < 0 || p->width < 0 || p->ldt < p->width ||
        p->ldq < 0 || p->hdq < 0) return SP_ERR_SHAPE;
    const float step = (float)(p->scale * 1.4426950408889634);
    if (!(step - step == 0)) return SP_ERR_SHAPE;        // the kernels hold it in 32 bits: not finite there
    if (p->causal != 0 && p->causal != 1) return SP_ERR_UNSUPPORTED;
    SP_TRY(st);
    const int64_t top = (int64_t)1 << 31;
    if (p->requests >= top || p->tokens >= top || p->width >= ceil_div(top, c->pageTokens)) return SP_ERR_TOO_LARGE;
    a->Q = p->Q; a->table = p->table; a->length = p->length; a->start = p->start;
    a->ldq = p->ldq; a->hdq = p->hdq; a->ldt = p->ldt; a->width = c->pages ? p->width : 0; a->requests = p->requests; a->tokens = p->tokens;
    a->H = p->heads; a->R = p->heads / c->kvHeads; a->causal = p->causal; a->sign = step < 0 ? -1.f : step > 0 ? 1.f : 0.f; a->step = step == 0 ? 1.f : fabsf(step);
    a->records = spmi_make_divisor32(c->pageTokens / kCacheTile);
    *choice = p->dtype == SP_F32 ? cache_choice_of<float>(*a) : p->dtype == SP_F16 ? cache_choice_of<cache_f16>(*a) : cache_choice_of<cache_bf16>(*a);
    if (a->tokens * a->R >= top || choice->items * a->c.G >= (int64_t)1 << 24) return SP_ERR_TOO_LARGE;        // 2^32 threads of a launch
    return SP_OK;
}

}  // namespace

extern "C" sp_status sp_cache_attention_workspace(const sp_cache *c, const sp_cache_problem *p, size_t *bytes)
{
    if (!bytes) return SP_ERR_NULL;
    *bytes = 0;
    cache_attn_args a;
    cache_choice choice;
    SP_TRY(check_problem(c, p, &a, &choice));
    *bytes = choice.bytes();
    return SP_OK;
}

extern "C" sp_status sp_cache_attention(const sp_cache *c, const sp_cache_problem *p, void *O, int64_t ldo, int64_t hdo, float *lse,
                                        void *workspace, size_t workspaceBytes, void *stream)
{
    cache_attn_args a;
    cache_choice choice;
    SP_TRY(check_problem(c, p, &a, &choice));
    if ((a.tokens > 1 && ldo < a.c.D) || (a.H > 1 && hdo < a.c.D)) return SP_ERR_SHAPE;
    if (a.tokens == 0 || a.requests == 0) return SP_OK;
    if (!O || !a.Q || !a.length || !a.start || (a.width && !a.table) || !cache_has_memory(a.c)) return SP_ERR_NULL;
    const size_t need = choice.bytes();
    if (need > 0 && !workspace) return SP_ERR_NULL;
    if (need > workspaceBytes || ((uintptr_t)workspace & 255)) return SP_ERR_SHAPE;
    a.O = O; a.ldo = ldo; a.hdo = hdo; a.lse = lse;
    a.stat = (float2 *)workspace;
    if (choice.plan) a.plan = (uint32_t *)((char *)workspace + choice.stat);
    a.part = (float *)((char *)workspace + choice.stat + choice.plan);
    a.slots = (uint32_t)choice.slots;
    const int size = p->dtype == SP_F32 ? 4 : 2;
    const int64_t stray = (uintptr_t)a.Q | (uintptr_t)O | (uintptr_t)(size * (a.ldq | a.hdq | ldo | hdo));
    a.vec = a.c.D % 8 == 0 && stray % 16 == 0;
    hipStream_t st = (hipStream_t)stream;
    if (p->dtype == SP_F32) return cache_attention<float>(a, choice, st);
    if (p->dtype == SP_F16) return cache_attention<cache_f16>(a, choice, st);
    return cache_attention<cache_bf16>(a, choice, st);
}
