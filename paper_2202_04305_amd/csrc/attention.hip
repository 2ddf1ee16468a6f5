// Attention over a stored pattern, forward: argument checks, the kernels that make O and lse, the join of rows that were cut.
#include "attention.h"
#include <math.h>

namespace {

constexpr int kThreads = 256;

template <typename T>
__global__ __launch_bounds__(kThreads) void forward_rows_kernel(attn_args a, attn_plan_view p, T *__restrict__ O, int64_t ldo, int64_t hdo,
                                                                float *__restrict__ lse)
{
    const int lane = threadIdx.x & 63;
    const int64_t x = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
    if (x >= a.m * a.H) return;
    const int64_t i = x / a.H;
    const int h = (int)(x % a.H);
    float top, total, acc[kAttnPer];
    const int64_t b = i / p.br;
    attn_row_forward<T>(a, p, b, (int)(i % p.br), p.chunk0[b], p.chunk0[b + 1], i, h, lane, top, total, acc);
    const float inv = total == 0 ? 0.f : 1.f / total;
#pragma unroll
    for (int k = 0; k < kAttnPer; ++k)
        if (lane + 64 * k < a.D) O[i * ldo + h * hdo + lane + 64 * k] = (T)(acc[k] * inv);
    if (lse && lane == 0) lse[h * a.m + i] = total == 0 ? -INFINITY : top + __builtin_amdgcn_logf(total) * kLn2;
}

}  // namespace

// The bias's far buckets begin at the smallest whole distances d >= e (M / e)^(k / (N - e)).  A power that is a whole number comes out
// of the floating point as one give or take a few ulp, and is taken as one; one that is not does not come that close.
static void make_borders(const sp_attention_problem *p, attn_args *a)
{
    a->side = p->bidirectional ? p->buckets / 2 : p->buckets;
    a->exact = a->side / 2;
    const int far = a->side - a->exact;
    a->borders = far - 1;
    a->last = a->exact;
    for (int k = 1; k < far; ++k) {
        const long double x = (long double)a->exact * powl((long double)p->maxDistance / a->exact, (long double)k / far);
        const long double near = roundl(x);
        a->border[k - 1] = (int16_t)(fabsl(x - near) < 1e-12L * x ? near : ceill(x));
        a->last = a->border[k - 1];
    }
}

sp_status spmi_attention_check(const sp_tensor *S, const sp_attention_problem *p, int grad, attn_args *a)
{
    if (!S || !p) return SP_ERR_NULL;
    if (S->enc.rank != 2) return SP_ERR_RANK;
    if (p->dtype != (int)SP_F32 && p->dtype != (int)SP_F16 && p->dtype != (int)SP_BF16) return SP_ERR_DTYPE;
    if (p->heads < 1 || p->kvHeads < 1 || p->heads % p->kvHeads || p->headDim < 1 || p->headDim > 256 || p->heads > 65535) return SP_ERR_SHAPE;
    if ((p->causal != 0 && p->causal != 1) || (p->bidirectional != 0 && p->bidirectional != 1)) return SP_ERR_UNSUPPORTED;
    if (p->buckets < 0 || p->buckets > 64) return SP_ERR_SHAPE;
    if (p->buckets) {
        const int side = p->bidirectional ? p->buckets / 2 : p->buckets;
        if (side < 2 || (p->bidirectional && p->buckets % 2) || p->maxDistance <= side / 2 || p->maxDistance > 4096 || p->ldt < p->heads) return SP_ERR_SHAPE;
    }
    for (int64_t s : {p->ldq, p->hdq, p->ldk, p->hdk, p->ldv, p->hdv}) if (s < 0) return SP_ERR_SHAPE;
    if (!(p->scale - p->scale == 0)) return SP_ERR_SHAPE;            // not finite
    if (S->enc.perm[0] != 0 || S->enc.lt[1] != SP_COMPRESSED || !S->attention[0] || (grad && !S->attention[1])) return SP_ERR_UNSUPPORTED;
    memset(a, 0, sizeof(*a));
    a->Q = p->Q; a->K = p->K; a->V = p->V; a->table = p->table;
    a->ldq = p->ldq; a->hdq = p->hdq; a->ldk = p->ldk; a->hdk = p->hdk; a->ldv = p->ldv; a->hdv = p->hdv; a->ldt = p->ldt;
    a->qpos = p->qpos; a->kpos = p->kpos;
    a->m = S->shape[0]; a->n = S->shape[1];
    a->D = p->headDim; a->H = p->heads; a->Hk = p->kvHeads; a->G = p->heads / p->kvHeads;
    a->scale = (float)p->scale; a->c = (float)(p->scale * 1.4426950408889634);
    a->buckets = p->buckets; a->bidirectional = p->bidirectional; a->causal = p->causal;
    if (p->buckets) make_borders(p, a);
    return SP_OK;
}

extern "C" sp_status sp_attention_workspace(const sp_tensor *S, const sp_attention_problem *p, int grad, size_t *bytes)
{
    if (!bytes) return SP_ERR_NULL;
    *bytes = 0;
    attn_args a;
    SP_TRY(spmi_attention_check(S, p, grad, &a));
    *bytes = grad ? (size_t)a.m * a.H * 4 : 0;
    return SP_OK;
}

template <typename T>
static sp_status forward_t(const sp_tensor *S, const attn_args &a, T *O, int64_t ldo, int64_t hdo, float *lse, hipStream_t st)
{
    const sp_attn_plan *plan = S->attention[0];
    hipLaunchKernelGGL(forward_rows_kernel<T>, dim3((unsigned)ceil_div(a.m * a.H, 4)), dim3(kThreads), 0, st, a, attn_view(plan, 0), O, ldo, hdo, lse);
    SP_HIP(hipGetLastError());
    return SP_OK;
}

extern "C" sp_status sp_attention(const sp_tensor *S, const sp_attention_problem *p, void *O, int64_t ldo, int64_t hdo, float *lse,
                                  void *workspace, size_t workspaceBytes, void *stream)
{
    attn_args a;
    SP_TRY(spmi_attention_check(S, p, 0, &a));
    if ((a.m > 1 && ldo < a.D) || (a.H > 1 && hdo < a.D)) return SP_ERR_SHAPE;
    if (a.m == 0) return SP_OK;
    const bool pairs = S->nvalues > 0;
    if (!O || (pairs && (!a.Q || !a.K || !a.V || ((a.buckets || a.causal) && (!a.qpos || !a.kpos)) || (a.buckets && !a.table)))) return SP_ERR_NULL;
    size_t need = 0;
    SP_TRY(sp_attention_workspace(S, p, 0, &need));
    if (need > 0 && !workspace) return SP_ERR_NULL;
    if (need > workspaceBytes || ((uintptr_t)workspace & 255)) return SP_ERR_SHAPE;
    hipStream_t st = (hipStream_t)stream;
    if (p->dtype == SP_F32) return forward_t<float>(S, a, (float *)O, ldo, hdo, lse, st);
    if (p->dtype == SP_F16) return forward_t<attn_f16>(S, a, (attn_f16 *)O, ldo, hdo, lse, st);
    return forward_t<attn_bf16>(S, a, (attn_bf16 *)O, ldo, hdo, lse, st);
}
