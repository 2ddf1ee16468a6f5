// Attention over a stored pattern, backward.
#include "attention.h"

namespace {

constexpr int kThreads = 256;

// D[h,i] = sum_d dO[i,h,d] * O[i,h,d]
template <typename T>
__global__ __launch_bounds__(kThreads) void delta_kernel(attn_args a, const T *__restrict__ O, int64_t ldo, int64_t hdo, const T *__restrict__ dO,
                                                         int64_t lddo, int64_t hddo, float *__restrict__ delta)
{
    const int lane = threadIdx.x & 63;
    const int64_t x = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
    if (x >= a.m * a.H) return;
    const int64_t i = x / a.H;
    const int h = (int)(x % a.H);
    float u[kAttnPer], v[kAttnPer];
    attn_load_row(O + i * ldo + h * hdo, a.D, lane, u);
    attn_load_row(dO + i * lddo + h * hddo, a.D, lane, v);
    const float s = attn_dot(u, v);
    if (lane == 0) delta[h * a.m + i] = s;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void dq_rows_kernel(attn_args a, attn_plan_view p, sp_attention_grads g, const float *__restrict__ delta)
{
    const int lane = threadIdx.x & 63;
    const int64_t x = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
    if (x >= a.m * a.H) return;
    const int64_t i = x / a.H, b = i / p.br;
    const int h = (int)(x % a.H);
    float acc[kAttnPer];
    attn_row_dq<T>(a, p, b, (int)(i % p.br), p.chunk0[b], p.chunk0[b + 1], i, h, lane, (const T *)g.dO + i * g.lddo + h * g.hddo, g.lse[h * a.m + i],
                   delta[h * a.m + i], acc, [](int64_t, float) {});
#pragma unroll
    for (int k = 0; k < kAttnPer; ++k)
        if (lane + 64 * k < a.D) ((T *)g.dQ)[i * g.lddq + h * g.hddq + lane + 64 * k] = (T)(acc[k] * a.scale);
}

// one wave for a bucket and a head: every pair of the pattern is looked at
template <typename T>
__global__ __launch_bounds__(64) void dtable_kernel(attn_args a, attn_plan_view p, sp_attention_grads g, const float *__restrict__ delta)
{
    const int lane = threadIdx.x, bucket = blockIdx.x / a.H, h = blockIdx.x % a.H;
    float sum = 0, acc[kAttnPer];
    for (int64_t i = 0; i < a.m; ++i) {
        const int64_t b = i / p.br;
        attn_row_dq<T>(a, p, b, (int)(i % p.br), p.chunk0[b], p.chunk0[b + 1], i, h, lane, (const T *)g.dO + i * g.lddo + h * g.hddo, g.lse[h * a.m + i],
                       delta[h * a.m + i], acc, [&](int64_t j, float ds) { if (attn_bucket(a, attn_distance(a.kpos[j], a.qpos[i])) == bucket) sum += ds; });
    }
    if (lane == 0) ((T *)g.dTable)[bucket * g.lddt + h] = (T)sum;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void dkv_rows_kernel(attn_args a, attn_plan_view p, sp_attention_grads g, const float *__restrict__ delta)
{
    const int lane = threadIdx.x & 63;
    const int64_t x = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
    if (x >= a.n * a.Hk) return;
    const int64_t j = x / a.Hk, b = j / p.br;
    const int kv = (int)(x % a.Hk);
    float dk[kAttnPer] = {0}, dv[kAttnPer] = {0};
    for (int h = kv * a.G; h < (kv + 1) * a.G; ++h)
        attn_row_dkv<T>(a, p, b, (int)(j % p.br), p.chunk0[b], p.chunk0[b + 1], j, h, lane, (const T *)g.dO, g.lddo, g.hddo, g.lse, delta, dk, dv);
#pragma unroll
    for (int k = 0; k < kAttnPer; ++k)
        if (lane + 64 * k < a.D) {
            ((T *)g.dK)[j * g.lddk + kv * g.hddk + lane + 64 * k] = (T)(dk[k] * a.scale);
            ((T *)g.dV)[j * g.lddv + kv * g.hddv + lane + 64 * k] = (T)dv[k];
        }
}

template <typename T>
sp_status grad_t(const sp_tensor *S, const attn_args &a, const sp_attention_grads &g, float *delta, hipStream_t st)
{
    const attn_plan_view rows = attn_view(S->attention[0], 0), keys = attn_view(S->attention[1], 0);
    if (a.m > 0) {
        hipLaunchKernelGGL(delta_kernel<T>, dim3((unsigned)ceil_div(a.m * a.H, 4)), dim3(kThreads), 0, st, a, (const T *)g.O, g.ldo, g.hdo, (const T *)g.dO,
                           g.lddo, g.hddo, delta);
        hipLaunchKernelGGL(dq_rows_kernel<T>, dim3((unsigned)ceil_div(a.m * a.H, 4)), dim3(kThreads), 0, st, a, rows, g, delta);
    }
    if (a.n > 0) hipLaunchKernelGGL(dkv_rows_kernel<T>, dim3((unsigned)ceil_div(a.n * a.Hk, 4)), dim3(kThreads), 0, st, a, keys, g, delta);
    if (a.buckets && g.dTable) hipLaunchKernelGGL(dtable_kernel<T>, dim3((unsigned)(a.buckets * a.H)), dim3(64), 0, st, a, rows, g, delta);
    SP_HIP(hipGetLastError());
    return SP_OK;
}

}  // namespace

extern "C" sp_status sp_attention_grad(const sp_tensor *S, const sp_attention_problem *p, const sp_attention_grads *g,
                                       void *workspace, size_t workspaceBytes, void *stream)
{
    attn_args a;
    SP_TRY(spmi_attention_check(S, p, 1, &a));
    if (!g) return SP_ERR_NULL;
    for (int64_t s : {g->ldo, g->hdo, g->lddo, g->hddo}) if (s < 0) return SP_ERR_SHAPE;
    if ((a.H > 1 && g->hddq < a.D) || (a.m > 1 && g->lddq < a.D)) return SP_ERR_SHAPE;
    if ((a.Hk > 1 && (g->hddk < a.D || g->hddv < a.D)) || (a.n > 1 && (g->lddk < a.D || g->lddv < a.D))) return SP_ERR_SHAPE;
    if (a.buckets && g->dTable && g->lddt < a.H) return SP_ERR_SHAPE;
    const bool pairs = S->nvalues > 0;
    if (pairs && (!a.Q || !a.K || !a.V || ((a.buckets || a.causal) && (!a.qpos || !a.kpos)) || (a.buckets && !a.table))) return SP_ERR_NULL;
    if (a.m > 0 && (!g->O || !g->lse || !g->dO || !g->dQ)) return SP_ERR_NULL;
    if (a.n > 0 && (!g->dK || !g->dV)) return SP_ERR_NULL;
    size_t need = 0;
    SP_TRY(sp_attention_workspace(S, p, 1, &need));
    if (need > 0 && !workspace) return SP_ERR_NULL;
    if (need > workspaceBytes || ((uintptr_t)workspace & 255)) return SP_ERR_SHAPE;
    hipStream_t st = (hipStream_t)stream;
    if (p->dtype == SP_F32) return grad_t<float>(S, a, *g, (float *)workspace, st);
    if (p->dtype == SP_F16) return grad_t<attn_f16>(S, a, *g, (float *)workspace, st);
    return grad_t<attn_bf16>(S, a, *g, (float *)workspace, st);
}
