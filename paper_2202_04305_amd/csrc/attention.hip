// Attention over a stored pattern: the entry points, their checks, and what a call launches (a rule on the plan and the heads, the same
// for the workspace's size and for the call).
#include "attention_tiles.h"
#include <math.h>

namespace {

int padded(int D) { return (D + 3) & ~3; }

forward_choice choose(const sp_attn_plan *plan, const attn_args &a, int size)
{
    forward_choice c;
    (attn_mapping &)c = attn_map(plan, a, size, 2);
    const size_t rows = c.cut ? (size_t)plan->items[c.level] * a.H * plan->br : 0;
    c.part = (rows * padded(a.D) * 4 + 255) & ~(size_t)255;
    c.part_stat = (rows * 8 + 255) & ~(size_t)255;
    return c;
}

grad_choice choose(const sp_tensor *S, const attn_args &a, int size, bool table)
{
    const sp_attn_plan *rows = S->attention[0], *keys = S->attention[1];
    grad_choice c;
    c.rows = attn_map(rows, a, size, 3);
    // short 16-bit rows stay whole (see kAttnTwice)
    if (size == 2 && S->nvalues <= kAttnTwicePairs * a.m && c.rows.level < kAttnTwiceLevel) c.rows.level = rows->levels - 1 < kAttnTwiceLevel ? rows->levels - 1 : kAttnTwiceLevel;
    c.rows.cut = rows->cut[c.rows.level] > 0;
    // the bias's gradient from sums that need a row's whole D: rows are not cut then, unless a few long ones would hold up the rest for
    // longer than the whole pass takes, and the sums have to fit the LDS
    const int row = (a.D <= 32 ? 32 : a.D <= 64 ? 64 : a.D <= 128 ? 128 : 256) * size;
    c.exact = table && size == 2 && c.rows.whole_us <= 2 * c.rows.us + 20 && attn_dq_lds(a, c.rows, row, true, true, true) <= kAttnLds;
    if (c.exact) { c.rows.level = rows->levels - 1; c.rows.cut = false; }
    c.keys_level = attn_pick_level(keys, a.Hk, attn_chunk_us(a.D, size, 4) * a.G * (keys->br == 128 ? 1 : 0.7), 3, 8.0 * a.D * a.Hk);
    c.keys_cut = keys->cut[c.keys_level] > 0;
    const size_t p1 = c.rows.cut ? (size_t)rows->items[c.rows.level] * a.H * rows->br * padded(a.D) * 4 : 0;
    const size_t p2 = c.keys_cut ? (size_t)keys->items[c.keys_level] * a.Hk * keys->br * 2 * padded(a.D) * 4 : 0;
    auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
    c.delta = up((size_t)a.m * a.H * 4);
    c.log_sum = a.buckets ? c.delta : 0;
    c.part = up(p1 > p2 ? p1 : p2);
    c.table = up(table ? (size_t)rows->items[c.rows.level] * a.H * a.buckets * 4 : 0);
    return c;
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

static sp_status check_problem(const sp_tensor *S, const sp_attention_problem *p, int grad, attn_args *a)
{
    if (!S || !p) return SP_ERR_NULL;
    if (S->enc.rank != 2) return SP_ERR_RANK;
    if (p->dtype != (int)SP_F32 && p->dtype != (int)SP_F16 && p->dtype != (int)SP_BF16) return SP_ERR_DTYPE;
    if (p->heads < 1 || p->kvHeads < 1 || p->heads % p->kvHeads || p->headDim < 1 || p->heads > 65535) return SP_ERR_SHAPE;
    if (p->headDim > (p->dtype == (int)SP_F32 ? 128 : 256)) return SP_ERR_SHAPE;
    if ((p->causal != 0 && p->causal != 1) || (p->bidirectional != 0 && p->bidirectional != 1)) return SP_ERR_UNSUPPORTED;
    if (p->buckets < 0 || p->buckets > 64) return SP_ERR_SHAPE;
    if (p->buckets) {
        const int side = p->bidirectional ? p->buckets / 2 : p->buckets;
        if (side < 2 || (p->bidirectional && p->buckets % 2) || p->maxDistance <= side / 2 || p->maxDistance > 4096 || p->ldt < p->heads) return SP_ERR_SHAPE;
    }
    for (int64_t s : {p->ldq, p->hdq, p->ldk, p->hdk, p->ldv, p->hdv}) if (s < 0) return SP_ERR_SHAPE;
    const float c = (float)(p->scale * 1.4426950408889634);
    if (!(c - c == 0)) return SP_ERR_SHAPE;                          // the kernels hold it in 32 bits: not finite there
    if (S->enc.perm[0] != 0 || S->enc.lt[1] != SP_COMPRESSED || !S->attention[0] || (grad && !S->attention[1])) return SP_ERR_UNSUPPORTED;
    memset(a, 0, sizeof(*a));
    a->Q = p->Q; a->K = p->K; a->V = p->V; a->table = p->table;
    a->ldq = p->ldq; a->hdq = p->hdq; a->ldk = p->ldk; a->hdk = p->hdk; a->ldv = p->ldv; a->hdv = p->hdv; a->ldt = p->ldt;
    a->qpos = p->qpos; a->kpos = p->kpos;
    a->m = S->shape[0]; a->n = S->shape[1];
    a->D = p->headDim; a->H = p->heads; a->Hk = p->kvHeads; a->G = p->heads / p->kvHeads;
    a->scale = (float)p->scale; a->c = c;
    a->buckets = p->buckets; a->bidirectional = p->bidirectional; a->causal = p->causal;
    if (p->buckets) make_borders(p, a);
    return SP_OK;
}

extern "C" sp_status sp_attention_workspace(const sp_tensor *S, const sp_attention_problem *p, int grad, size_t *bytes)
{
    if (!bytes) return SP_ERR_NULL;
    *bytes = 0;
    attn_args a;
    SP_TRY(check_problem(S, p, grad, &a));
    if (grad) {
        for (int table = 0; table <= (a.buckets > 0); ++table) {         // with and without the table's gradient
            const grad_choice c = choose(S, a, p->dtype == SP_F32 ? 4 : 2, table != 0);
            const size_t need = c.bytes();
            if (need > *bytes) *bytes = need;
        }
    } else {
        const forward_choice c = choose(S->attention[0], a, p->dtype == SP_F32 ? 4 : 2);
        *bytes = c.part + c.part_stat;
    }
    return SP_OK;
}

extern "C" sp_status sp_attention(const sp_tensor *S, const sp_attention_problem *p, void *O, int64_t ldo, int64_t hdo, float *lse,
                                  void *workspace, size_t workspaceBytes, void *stream)
{
    forward_args f;
    memset(&f, 0, sizeof(f));
    attn_args &a = f.a;
    SP_TRY(check_problem(S, p, 0, &a));
    if ((a.m > 1 && ldo < a.D) || (a.H > 1 && hdo < a.D)) return SP_ERR_SHAPE;
    if (a.m == 0) return SP_OK;
    const bool pairs = S->nvalues > 0;
    if (!O || (pairs && (!a.Q || !a.K || !a.V || ((a.buckets || a.causal) && (!a.qpos || !a.kpos)) || (a.buckets && !a.table)))) return SP_ERR_NULL;
    if (!pairs) a.buckets = a.causal = 0;                // nothing is read
    if (!a.buckets && !a.causal) a.qpos = a.kpos = nullptr;
    const sp_attn_plan *plan = S->attention[0];
    const int size = p->dtype == SP_F32 ? 4 : 2;
    const forward_choice c = choose(plan, a, size);
    const size_t need = c.part + c.part_stat;
    if (need > 0 && !workspace) return SP_ERR_NULL;
    if (need > workspaceBytes || ((uintptr_t)workspace & 255)) return SP_ERR_SHAPE;
    f.p = attn_view(plan, c.level);
    f.O = O; f.ldo = ldo; f.hdo = hdo; f.lse = lse;
    f.part = (float *)workspace;
    f.part_stat = (float *)((char *)workspace + c.part);
    f.groups = c.groups; f.mode = c.mode; f.pd = padded(a.D);
    attn_alignment rows(a.D, size);
    rows.with(a.Q, a.ldq, a.hdq); rows.with(a.K, a.ldk, a.hdk); rows.with(a.V, a.ldv, a.hdv); rows.with(O, ldo, hdo);
    f.vec = rows.vec;
    if (!attn_launches(ceil_div(plan->cut[c.level] * plan->br * a.H, 4), 256)) return SP_ERR_TOO_LARGE;     // the join
    hipStream_t st = (hipStream_t)stream;
    if (p->dtype == SP_F32) return attn_forward<float>(plan, f, c, st);
    if (p->dtype == SP_F16) return attn_forward<attn_f16>(plan, f, c, st);
    return attn_forward<attn_bf16>(plan, f, c, st);
}

extern "C" sp_status sp_attention_grad(const sp_tensor *S, const sp_attention_problem *p, const sp_attention_grads *g,
                                       void *workspace, size_t workspaceBytes, void *stream)
{
    grad_args f;
    memset(&f, 0, sizeof(f));
    attn_args &a = f.a;
    SP_TRY(check_problem(S, p, 1, &a));
    if (!g) return SP_ERR_NULL;
    for (int64_t s : {g->ldo, g->hdo, g->lddo, g->hddo}) if (s < 0) return SP_ERR_SHAPE;
    if ((a.H > 1 && g->hddq < a.D) || (a.m > 1 && g->lddq < a.D)) return SP_ERR_SHAPE;
    if ((a.Hk > 1 && (g->hddk < a.D || g->hddv < a.D)) || (a.n > 1 && (g->lddk < a.D || g->lddv < a.D))) return SP_ERR_SHAPE;
    if (a.buckets && g->dTable && g->lddt < a.H) return SP_ERR_SHAPE;
    const bool pairs = S->nvalues > 0;
    if (pairs && (!a.Q || !a.K || !a.V || ((a.buckets || a.causal) && (!a.qpos || !a.kpos)) || (a.buckets && !a.table))) return SP_ERR_NULL;
    if (a.m > 0 && (!g->O || !g->lse || !g->dO || !g->dQ)) return SP_ERR_NULL;
    if (a.n > 0 && (!g->dK || !g->dV)) return SP_ERR_NULL;
    const int size = p->dtype == SP_F32 ? 4 : 2;
    const grad_choice c = choose(S, a, size, a.buckets && g->dTable);
    const size_t need = c.bytes();
    if (need > 0 && !workspace) return SP_ERR_NULL;
    if (need > workspaceBytes || ((uintptr_t)workspace & 255)) return SP_ERR_SHAPE;
    f.g = *g;
    f.pd = padded(a.D); f.exact = c.exact;
    f.delta = (float *)workspace;
    if (a.buckets) f.log_sum = (float *)((char *)workspace + c.delta);
    f.part = (float *)((char *)workspace + c.delta + c.log_sum);
    if (a.buckets && g->dTable) f.part_table = (float *)((char *)f.part + c.part);
    attn_alignment rows(a.D, size);
    rows.with(a.Q, a.ldq, a.hdq); rows.with(a.K, a.ldk, a.hdk); rows.with(a.V, a.ldv, a.hdv);
    rows.with(g->O, g->ldo, g->hdo); rows.with(g->dO, g->lddo, g->hddo);
    rows.with(g->dQ, g->lddq, g->hddq); rows.with(g->dK, g->lddk, g->hddk); rows.with(g->dV, g->lddv, g->hddv);
    f.vec = rows.vec;
    const sp_attn_plan *rows_plan = S->attention[0], *keys_plan = S->attention[1];
    if ((c.rows.cut && !attn_launches(ceil_div(rows_plan->cut[c.rows.level] * rows_plan->br * a.H, 4), 256)) ||
        (c.keys_cut && !attn_launches(ceil_div(keys_plan->cut[c.keys_level] * keys_plan->br * a.Hk, 4), 256))) return SP_ERR_TOO_LARGE;     // the joins
    hipStream_t st = (hipStream_t)stream;
    if (p->dtype == SP_F32) return attn_backward<float>(S, f, c, st);
    if (p->dtype == SP_F16) return attn_backward<attn_f16>(S, f, c, st);
    return attn_backward<attn_bf16>(S, f, c, st);
}
