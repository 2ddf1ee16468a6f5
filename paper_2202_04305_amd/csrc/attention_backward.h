// Attention over a stored pattern, backward.  With D = sum dO * O for every row and head, the pairs' ds = p (dO V^T - D) come from a
// row's stored lse alone, so two kernels make them, each where it needs them: one over the rows of the pattern (dQ and the
// bias's gradient), one over its columns, by the transposed plan (dK and dV).  Seven products instead of five, but every result is
// summed by one workgroup in one order: no atomics on memory, the same bits on every call.
// Compiled once for each type (attention_backward_*.hip).
#pragma once
#include "attention_tiles.h"

namespace {

constexpr int kThreads = 256;

// D[h,i] = sum_d dO[i,h,d] * O[i,h,d]: LPR lanes for a row, 16 bytes of it each
template <typename T, int LPR>
__global__ __launch_bounds__(kThreads) void delta_kernel(grad_args f, float *__restrict__ delta)
{
    constexpr int V = 16 / (int)sizeof(T);
    typedef typename attn_mma<T>::frag frag;
    const attn_args &a = f.a;
    const int l = threadIdx.x % LPR;
    const int64_t x = (int64_t)blockIdx.x * (kThreads / LPR) + threadIdx.x / LPR;
    float s = 0;
    const int64_t i = x / a.H;
    const int h = (int)(x % a.H);
    if (x < a.m * a.H) {
        const T *u = (const T *)f.g.O + i * f.g.ldo + h * f.g.hdo, *v = (const T *)f.g.dO + i * f.g.lddo + h * f.g.hddo;
        const frag p = attn_tile<T, 32>::granule(u, l * V, a.D, f.vec, true), q = attn_tile<T, 32>::granule(v, l * V, a.D, f.vec, true);
#pragma unroll
        for (int k = 0; k < V; ++k) s += (float)p[k] * (float)q[k];
    }
#pragma unroll
    for (int d = LPR / 2; d >= 1; d >>= 1) s += __shfl_xor(s, d, 64);
    if (l == 0 && x < a.m * a.H) delta[h * a.m + i] = s;
}

// dQ: the forward kernel's frame (items, gathered columns through LDS, tiles of 32 rows), with dO beside Q and V read as K is.
// With a bias its gradient as well: every lane adds its pairs' ds to a place of its own for each bucket in LDS, so that no two
// lanes ever add to one number; the lanes' sums are added in order at the end.
template <typename T, int DT, int WM, int WN, int KW, bool POS>
__global__ __launch_bounds__(64 * WM * WN, DT * sizeof(T) <= 256 ? 2 : 1) void dq_kernel(grad_args f)
{
    typedef attn_tile<T, DT> tile;
    typedef typename tile::frag frag;
    constexpr int NT = 64 * WM * WN, KT = KW * WN, TILES = KW / 32;
    constexpr int PIECES = KT * tile::kGranules / NT, ROWSTEP = NT / tile::kGranules;
    constexpr int STEP = KT > kAttnChunk ? KT / kAttnChunk : 1, SUB = KT < kAttnChunk ? kAttnChunk / KT : 1;
    extern __shared__ __align__(16) char lds[];
    attn_lds *sK = (attn_lds *)lds, *sV = sK + KT * tile::kRow;
    int *s_kpos = (int *)(lds + 2 * KT * tile::kRow);
    const attn_args &a = f.a;
    const attn_plan_view &p = f.p;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wn = WN > 1 ? wave : 0;
    const int64_t item_no = blockIdx.x / f.groups;
    const int group = blockIdx.x % f.groups;
    const attn_item item(p, item_no);
    const attn_lane me(a, p.br, item.block, f.mode, group, lane, wave, WM);
    const int r = me.r;
    const bool busy = __builtin_amdgcn_ballot_w64(me.valid) != 0, some = me.valid && item.c1 > item.c0;
    const float cc = POS ? kLog2e : fabsf(a.c);

    frag q[tile::kSteps], go[tile::kSteps];
    tile::load_lane((const T *)a.Q + me.row * a.ldq + me.head * a.hdq, a.D, f.vec, some, POS ? 1.f : a.c, q, lane);
    tile::load_lane((const T *)f.g.dO + me.row * f.g.lddo + me.head * f.g.hddo, a.D, f.vec, some, 1.f, go, lane);
    float off = f.g.lse[me.head * a.m + me.row];
    if (off == -INFINITY) off = INFINITY;                // no weight left
    if (!POS) off *= kLog2e;
    const float delta = f.delta[me.head * a.m + me.row];
    int qp = 0;
    attn_bias bias = {nullptr, nullptr, 0, 1, 0};
    float *hist = nullptr;
    if (POS) {
        if (a.qpos) qp = a.qpos[me.row];
        if (a.buckets) {
            bias = attn_lane_bias<T>(a, lds + 2 * KT * tile::kRow + KT * 4, f.mode, group, lane, wave, WM);
            if (f.part_table) {
                hist = (float *)(bias.table + a.buckets * bias.slots) + wave * a.buckets * 64;
                for (int b = 0; b < a.buckets; ++b) hist[b * 64 + lane] = 0;
            }
        }
    }
    attn_f32x16 acc[tile::kBlocks];
#pragma unroll
    for (int x = 0; x < tile::kBlocks; ++x) acc[x] = (attn_f32x16)(0.f);

    const T *Kh = (const T *)a.K + (int64_t)me.kv * a.hdk, *Vh = (const T *)a.V + (int64_t)me.kv * a.hdv;
    const int my_row = tid / tile::kGranules, my_g = tid % tile::kGranules;
    const int64_t first = (int64_t)(item.c0 - item.chunk0) * kAttnChunk, steps = (int64_t)(item.c1 - item.c0 + STEP - 1) / STEP * SUB;
    int32_t at[PIECES], pos_at = 0;
    frag kf[PIECES], vf[PIECES];
    int kp_next = 0;
    auto fetch_columns = [&](int64_t step) {
        const int64_t x = first + step * KT;
#pragma unroll
        for (int k = 0; k < PIECES; ++k) at[k] = item.cols.get(x + my_row + k * ROWSTEP);
        if (POS && tid < KT) pos_at = item.cols.get(x + tid);
    };
    auto fetch_rows = [&]() {
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            kf[k] = tile::granule(Kh + (int64_t)at[k] * a.ldk, my_g * tile::kPer, a.D, f.vec, true);
            vf[k] = tile::granule(Vh + (int64_t)at[k] * a.ldv, my_g * tile::kPer, a.D, f.vec, true);
        }
        if (POS && a.kpos && tid < KT) kp_next = a.kpos[pos_at];
    };
    if (steps > 0) {
        fetch_columns(0);
        fetch_rows();
        if (steps > 1) fetch_columns(1);
    }
    for (int64_t step = 0; step < steps; ++step) {
        __syncthreads();
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            tile::put(sK, my_row + k * ROWSTEP, my_g, kf[k]);
            tile::put(sV, my_row + k * ROWSTEP, my_g, vf[k]);
        }
        if (POS && tid < KT) s_kpos[tid] = kp_next;
        __syncthreads();
        if (step + 1 < steps) {
            fetch_rows();
            if (step + 2 < steps) fetch_columns(step + 2);
        }
        const int col0 = (int)(step % SUB) * KT + wn * KW;
        const int chunk = item.c0 + (int)(step / SUB) * STEP + col0 / kAttnChunk;
        if (!busy || chunk >= item.c1) continue;
        const int state = __builtin_amdgcn_readfirstlane(item.state(p, chunk, r));
        if (state == 0) continue;
        const uint64_t word = item.word(p, chunk, r) >> (col0 % kAttnChunk);
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            attn_f32x16 s = tile::scores(sK, wn * KW + 32 * t, q, lane);
            const attn_f32x16 dp = tile::scores(sV, wn * KW + 32 * t, go, lane);
            // what is not stored, and rows that do not exist, add nothing
            const uint32_t bits = (me.valid ? (uint32_t)(word >> (32 * t)) : 0u) >> (4 * (lane >> 5));
#pragma unroll
            for (int x = 0; x < 16; ++x) {
                bool there = bits >> (8 * (x >> 2) + (x & 3)) & 1;
                float v = s[x];
                int bucket = 0;
                if (POS) {
                    const int kp = s_kpos[wn * KW + 32 * t + 8 * (x >> 2) + 4 * (lane >> 5) + (x & 3)];
                    v *= a.scale;
                    if (a.buckets) { bucket = bias.bucket(kp, qp); v += bias.at(bucket); }
                    if (a.causal && kp > qp) there = false;
                    there = there && v != -INFINITY;     // weight 0, whatever dp is
                    v = (v - off) * cc;
                } else v = __builtin_fmaf(v, cc, -off);
                v = there ? __builtin_amdgcn_exp2f(v) * (dp[x] - delta) : 0.f;
                if (POS && hist && there) atomicAdd(&hist[bucket * 64 + lane], v);      // a place of this lane's own: one order
                s[x] = v;
            }
            tile::add_rows(acc, sK, wn * KW + 32 * t, s, lane);
        }
    }
    float odd = 0;
#pragma unroll
    for (int x = 0; x < tile::kBlocks; ++x)
#pragma unroll
        for (int k = 0; k < 16; ++k) odd += acc[x][k] * 0.f;
    uint64_t again = __builtin_amdgcn_ballot_w64(me.valid && !(odd == 0.f));

    if (POS && hist) {
        // a lane for a bucket (and, where lanes are heads, a head): places added in order
        __syncthreads();
        const float *all = (const float *)(bias.table + a.buckets * bias.slots);
        float *out = f.part_table + item.part * a.H * a.buckets;
        if (f.mode == kHeadsTogether) {
            for (int x = tid; x < a.buckets * 32; x += NT) {
                const int b = x >> 5, h = x & 31, per = 32, parts = (a.G + per - 1) / per, y = (group % parts) * per + h;
                if (y >= a.G) continue;
                float sum = 0;
                for (int w = 0; w < WM * WN; ++w) sum += all[(w * a.buckets + b) * 64 + h] + all[(w * a.buckets + b) * 64 + 32 + h];
                out[((group / parts) * a.G + y) * a.buckets + b] = sum;
            }
        } else {
            const int waves = f.mode == kHeadsOfRows ? 1 : WM * WN;      // that share a head
            for (int x = wave; x < a.buckets * (WM * WN / waves); x += WM * WN) {
                const int b = x % a.buckets, w0 = x / a.buckets * waves;
                int h = group;
                if (f.mode == kHeadsOfRows) {
                    const int parts = (a.G + WM - 1) / WM, y = (group % parts) * WM + w0;
                    if (y >= a.G) continue;
                    h = (group / parts) * a.G + y;
                }
                float sum = 0;
                for (int w = w0; w < w0 + waves; ++w) sum += all[(w * a.buckets + b) * 64 + lane];
                sum = attn_wave_sum(sum);
                if (lane == 0) out[h * a.buckets + b] = sum;
            }
        }
    }

    const int64_t place = (item.part * a.H + me.head) * p.br + r;
    T *out = (T *)f.g.dQ + me.row * f.g.lddq + me.head * f.g.hddq;
    if (WN == 1) {
        again |= again >> 32;
        if (me.valid && !(again >> (lane & 31) & 1)) {
#pragma unroll
            for (int x = 0; x < tile::kBlocks; ++x)
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const int d = 32 * x + 8 * b + 4 * (lane >> 5);
                    const attn_f32x4 v = {acc[x][4 * b], acc[x][4 * b + 1], acc[x][4 * b + 2], acc[x][4 * b + 3]};
                    if (item.whole) attn_store4(out, d, a.D, f.vec, v * a.scale);
                    else attn_store4(f.part + place * f.pd, d, f.pd, true, v);
                }
        }
    } else {
        __syncthreads();
        float *sums = (float *)lds, *bad = (float *)lds + WN * 32 * DT;
#pragma unroll
        for (int x = 0; x < tile::kBlocks; ++x)
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const int g = (8 * x + 2 * b + (lane >> 5)) ^ (lane & 7);
                *(attn_f32x4 *)(sums + (wn * 32 + (lane & 31)) * DT + 4 * g) = (attn_f32x4){acc[x][4 * b], acc[x][4 * b + 1], acc[x][4 * b + 2], acc[x][4 * b + 3]};
            }
        if (lane < 32) bad[wn * 32 + lane] = (again | again >> 32) >> lane & 1 ? 1.f : 0.f;
        __syncthreads();
        constexpr int LANES = NT / 32, EACH = DT / LANES;
        const int mine = tid / LANES, part = tid % LANES;
        float any = 0;
#pragma unroll
        for (int x = 0; x < WN; ++x) any += bad[x * 32 + mine];
        const int64_t row2 = ((int64_t)__shfl((int)(me.row >> 32), mine, 64) << 32) | (uint32_t)__shfl((int)me.row, mine, 64);
        const int head2 = __shfl(me.head, mine, 64), r2 = __shfl(r, mine, 64);
        const bool valid2 = __shfl((int)me.valid, mine, 64) != 0;
        const int64_t place2 = (item.part * a.H + head2) * p.br + r2;
        if (valid2 && any == 0) {
#pragma unroll
            for (int k = 0; k < EACH; k += 4) {
                const int d = part * EACH + k;
                attn_f32x4 v = (attn_f32x4)(0.f);
#pragma unroll
                for (int x = 0; x < WN; ++x) v += *(attn_f32x4 *)(sums + (x * 32 + mine) * DT + 4 * ((d >> 2) ^ (mine & 7)));
                if (item.whole) attn_store4((T *)f.g.dQ + row2 * f.g.lddq + head2 * f.g.hddq, d, a.D, f.vec, v * a.scale);
                else attn_store4(f.part + place2 * f.pd, d, f.pd, true, v);
            }
        }
        again = 0;
        for (int x = 0; x < 32; ++x) {
            float y = 0;
            for (int w = 0; w < WN; ++w) y += bad[w * 32 + x];
            if (y != 0 && x % WN == wn) again |= (uint64_t)1 << x;
        }
    }
    for (again &= 0xffffffffu; again; again &= again - 1) {
        const int x = __builtin_ctzll(again);
        const int64_t i = ((int64_t)__builtin_amdgcn_readlane((int)(me.row >> 32), x) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)me.row, x);
        const int h = __builtin_amdgcn_readlane(me.head, x), rr = __builtin_amdgcn_readlane(r, x);
        float one[kAttnPer];
        attn_row_dq<T>(a, p, item.block, rr, item.c0, item.c1, i, h, lane, (const T *)f.g.dO + i * f.g.lddo + h * f.g.hddo, f.g.lse[h * a.m + i],
                       f.delta[h * a.m + i], one);
        const int64_t at1 = (item.part * a.H + h) * p.br + rr;
#pragma unroll
        for (int k = 0; k < kAttnPer; ++k) {
            const int d = lane + 64 * k;
            if (d >= a.D) continue;
            if (item.whole) ((T *)f.g.dQ)[i * f.g.lddq + h * f.g.hddq + d] = (T)(one[k] * a.scale);
            else f.part[at1 * f.pd + d] = one[k];
        }
    }
}

// dK and dV: blocks of keys (lanes) over the queries that attend to them, head by head of the keys' group.  Q and dO come through
// LDS, K and V stay in registers; the scores are those of the forward kernel with the roles exchanged, so weights and ds are again
// operands as they lie.  WM waves take 32 keys each.
template <typename T, int DT, int WM, int KW, bool POS>
__global__ __launch_bounds__(64 * WM, DT * sizeof(T) <= 256 ? 2 : 1) void dkv_kernel(grad_args f)
{
    typedef attn_tile<T, DT> tile;
    typedef typename tile::frag frag;
    constexpr int NT = 64 * WM, KT = KW, TILES = KW / 32;
    constexpr int PIECES = KT * tile::kGranules / NT, ROWSTEP = NT / tile::kGranules;
    constexpr int SUB = kAttnChunk / KT;
    static_assert(KT <= NT && KT <= kAttnChunk, "a thread for each query of a step");
    extern __shared__ __align__(16) char lds[];
    attn_lds *sQ = (attn_lds *)lds, *sO = sQ + KT * tile::kRow;
    float *s_lse = (float *)(lds + 2 * KT * tile::kRow), *s_delta = s_lse + KT;
    int *s_qpos = (int *)(s_delta + KT);
    const attn_args &a = f.a;
    const attn_plan_view &p = f.p;                       // of the transposed pattern: rows are keys
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t item_no = blockIdx.x / a.Hk;
    const int kv = blockIdx.x % a.Hk;
    const attn_item item(p, item_no);
    const int r = 32 * wave + (lane & 31);
    int64_t key = item.block * p.br + r;
    const bool valid = key < a.n;
    if (!valid) key = a.n - 1;
    const bool busy = __builtin_amdgcn_ballot_w64(valid) != 0, some = valid && item.c1 > item.c0;
    const float cc = POS ? kLog2e : fabsf(a.c);
    frag kx[tile::kSteps], vx[tile::kSteps];
    tile::load_lane((const T *)a.K + key * a.ldk + kv * a.hdk, a.D, f.vec, some, POS ? 1.f : a.c, kx, lane);
    tile::load_lane((const T *)a.V + key * a.ldv + kv * a.hdv, a.D, f.vec, some, 1.f, vx, lane);
    int kp = 0;
    attn_bias bias = {nullptr, nullptr, 0, 1, 0};
    float *table = nullptr;
    if (POS) {
        if (a.kpos) kp = a.kpos[key];
        if (a.buckets) {
            bias = attn_make_bias<T>(a, (char *)(s_qpos + KT), 1, [&](int) { return kv * a.G; });
            table = const_cast<float *>(bias.table);
        }
    }
    attn_f32x16 dk[tile::kBlocks], dv[tile::kBlocks];
#pragma unroll
    for (int x = 0; x < tile::kBlocks; ++x) dk[x] = dv[x] = (attn_f32x16)(0.f);

    const int my_row = tid / tile::kGranules, my_g = tid % tile::kGranules;
    const int64_t first = (int64_t)(item.c0 - item.chunk0) * kAttnChunk;
    const int64_t per_head = (int64_t)(item.c1 - item.c0) * SUB, steps = per_head * a.G;
    int32_t at[PIECES], one_at = 0;
    frag qf[PIECES], of[PIECES];
    float lse_next = 0, delta_next = 0;
    int qp_next = 0;
    auto fetch_columns = [&](int64_t within) {           // step of a head
        const int64_t x = first + within * KT;
#pragma unroll
        for (int k = 0; k < PIECES; ++k) at[k] = item.cols.get(x + my_row + k * ROWSTEP);
        if (tid < KT) one_at = item.cols.get(x + tid);
    };
    auto fetch_rows = [&](int h) {
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            qf[k] = tile::granule((const T *)a.Q + (int64_t)at[k] * a.ldq + h * a.hdq, my_g * tile::kPer, a.D, f.vec, true);
            of[k] = tile::granule((const T *)f.g.dO + (int64_t)at[k] * f.g.lddo + h * f.g.hddo, my_g * tile::kPer, a.D, f.vec, true);
        }
        if (tid < KT) {
            const float l = f.g.lse[h * a.m + one_at];
            lse_next = l == -INFINITY ? INFINITY : POS ? l : l * kLog2e;
            delta_next = f.delta[h * a.m + one_at];
            if (POS && a.qpos) qp_next = a.qpos[one_at];
        }
    };
    int64_t within = 0, within2 = 0;                     // of the step at hand, of the columns fetched last
    int h = kv * a.G, h1 = h;                            // head of the step at hand, of the rows fetched last
    auto advance = [&](int64_t &w) { if (++w == per_head) w = 0; return w == 0; };
    if (steps > 0) {
        fetch_columns(0);
        fetch_rows(h);
        advance(within2);
        if (steps > 1) fetch_columns(within2);
    }
    for (int64_t step = 0; step < steps; ++step) {
        __syncthreads();
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            tile::put(sQ, my_row + k * ROWSTEP, my_g, qf[k]);
            tile::put(sO, my_row + k * ROWSTEP, my_g, of[k]);
        }
        if (tid < KT) {
            s_lse[tid] = lse_next;
            s_delta[tid] = delta_next;
            if (POS) s_qpos[tid] = qp_next;
        }
        if (POS && a.buckets && within == 0)
            for (int b = tid; b < a.buckets; b += NT) table[b] = (float)((const T *)a.table)[(int64_t)b * a.ldt + h];
        __syncthreads();
        if (step + 1 < steps) {
            if (within2 == 0) ++h1;
            fetch_rows(h1);
            advance(within2);
            if (step + 2 < steps) fetch_columns(within2);
        }
        const int col0 = (int)(within % SUB) * KT, chunk = item.c0 + (int)(within / SUB);
        if (advance(within)) ++h;
        if (!busy) continue;
        const int state = __builtin_amdgcn_readfirstlane(item.state(p, chunk, r));
        if (state == 0) continue;
        const uint64_t word = item.word(p, chunk, r) >> col0;
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            attn_f32x16 s = tile::scores(sQ, 32 * t, kx, lane);
            attn_f32x16 dp = tile::scores(sO, 32 * t, vx, lane);
            const uint32_t bits = (valid ? (uint32_t)(word >> (32 * t)) : 0u) >> (4 * (lane >> 5));
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const int q0 = 32 * t + 8 * b + 4 * (lane >> 5);
                const attn_f32x4 lse = *(const attn_f32x4 *)(s_lse + q0), delta = *(const attn_f32x4 *)(s_delta + q0);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const int x = 4 * b + c;
                    bool there = bits >> (8 * b + c) & 1;
                    float v = s[x];
                    if (POS) {
                        const int qp = s_qpos[q0 + c];
                        v *= a.scale;
                        if (a.buckets) v += bias.at(bias.bucket(kp, qp));
                        if (a.causal && kp > qp) there = false;
                        there = there && v != -INFINITY;
                        v = (v - lse[c]) * cc;
                    } else v = __builtin_fmaf(v, cc, -lse[c]);
                    v = there ? __builtin_amdgcn_exp2f(v) : 0.f;
                    s[x] = v;
                    dp[x] = there ? v * (dp[x] - delta[c]) : 0.f;
                }
            }
            tile::add_rows(dv, sO, 32 * t, s, lane);
            tile::add_rows(dk, sQ, 32 * t, dp, lane);
        }
    }
    float odd = 0;
#pragma unroll
    for (int x = 0; x < tile::kBlocks; ++x)
#pragma unroll
        for (int k = 0; k < 16; ++k) odd += dk[x][k] * 0.f + dv[x][k] * 0.f;
    uint64_t again = __builtin_amdgcn_ballot_w64(valid && !(odd == 0.f));
    again |= again >> 32;
    if (valid && !(again >> (lane & 31) & 1)) {
        float *part = f.part + ((item.part * a.Hk + kv) * p.br + r) * 2 * f.pd;
#pragma unroll
        for (int x = 0; x < tile::kBlocks; ++x)
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const int d = 32 * x + 8 * b + 4 * (lane >> 5);
                const attn_f32x4 k4 = {dk[x][4 * b], dk[x][4 * b + 1], dk[x][4 * b + 2], dk[x][4 * b + 3]};
                const attn_f32x4 v4 = {dv[x][4 * b], dv[x][4 * b + 1], dv[x][4 * b + 2], dv[x][4 * b + 3]};
                if (item.whole) {
                    attn_store4((T *)f.g.dK + key * f.g.lddk + kv * f.g.hddk, d, a.D, f.vec, k4 * a.scale);
                    attn_store4((T *)f.g.dV + key * f.g.lddv + kv * f.g.hddv, d, a.D, f.vec, v4);
                } else {
                    attn_store4(part, d, f.pd, true, k4);
                    attn_store4(part + f.pd, d, f.pd, true, v4);
                }
            }
    }
    for (again &= 0xffffffffu; again; again &= again - 1) {
        const int x = __builtin_ctzll(again);
        const int64_t j = ((int64_t)__builtin_amdgcn_readlane((int)(key >> 32), x) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)key, x);
        const int rr = __builtin_amdgcn_readlane(r, x);
        float k1[kAttnPer] = {0}, v1[kAttnPer] = {0};
        for (int g = kv * a.G; g < (kv + 1) * a.G; ++g)
            attn_row_dkv<T>(a, p, item.block, rr, item.c0, item.c1, j, g, lane, (const T *)f.g.dO, f.g.lddo, f.g.hddo, f.g.lse, f.delta, k1, v1);
        float *part = f.part + ((item.part * a.Hk + kv) * p.br + rr) * 2 * f.pd;
#pragma unroll
        for (int k = 0; k < kAttnPer; ++k) {
            const int d = lane + 64 * k;
            if (d >= a.D) continue;
            if (item.whole) {
                ((T *)f.g.dK)[j * f.g.lddk + kv * f.g.hddk + d] = (T)(k1[k] * a.scale);
                ((T *)f.g.dV)[j * f.g.lddv + kv * f.g.hddv + d] = (T)v1[k];
            } else {
                part[d] = k1[k];
                part[f.pd + d] = v1[k];
            }
        }
    }
}

// Rows (dq: of a head; dkv: keys of a kv head) that were cut into several items: their parts added in a fixed order.  PER: vectors of D
// numbers for a row (dq 1: dQ; dkv 2: dK, dV), of which the first is scaled.
template <typename T, int LP, int PER>
__global__ __launch_bounds__(kThreads) void join_kernel(grad_args f, int64_t rows, int heads)
{
    const attn_plan_view &p = f.p;
    const int lane = threadIdx.x & 63, D = f.a.D;
    const int64_t x = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
    if (x >= rows * heads) return;
    const int64_t i = x / heads, b = i / p.br;
    const int h = (int)(x % heads), first = p.item0[b], parts = p.item0[b + 1] - first;
    if (parts == 1) return;
#pragma unroll
    for (int v = 0; v < PER; ++v) {
        T *out = PER == 1 ? (T *)f.g.dQ + i * f.g.lddq + h * f.g.hddq
                          : v == 0 ? (T *)f.g.dK + i * f.g.lddk + h * f.g.hddk : (T *)f.g.dV + i * f.g.lddv + h * f.g.hddv;
        const attn_f32x4 sum = attn_add_parts<LP>(parts, f.pd, lane, [&](int k) {
            return f.part + ((((int64_t)(first + k) * heads + h) * p.br + i % p.br) * PER + v) * f.pd;
        }, [](int) { return 1.f; });
        if (lane < LP) attn_store4(out, 4 * lane, D, f.vec, v == 0 ? sum * f.a.scale : sum);
    }
}

// dTable[b,h] = the items' sums, a workgroup for a bucket and head, in a fixed order
template <typename T>
__global__ __launch_bounds__(kThreads) void table_kernel(grad_args f, int64_t items)
{
    __shared__ float s_sum[kThreads / 64];
    const attn_args &a = f.a;
    const int b = blockIdx.x % a.buckets, h = blockIdx.x / a.buckets;
    float sum = 0;
    for (int64_t x = threadIdx.x; x < items; x += kThreads) sum += f.part_table[(x * a.H + h) * a.buckets + b];
    sum = attn_wave_sum(sum);
    if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) ((T *)f.g.dTable)[(int64_t)b * f.g.lddt + h] = (T)(s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3]);
}

template <typename K>
sp_status launch(K kernel, const grad_args &f, int64_t groups, int threads, size_t lds, hipStream_t st)
{
    if (groups >= ((int64_t)1 << 31)) return SP_ERR_TOO_LARGE;
    if (lds > 65536) SP_HIP(hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
    hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(threads), lds, st, f);
    SP_HIP(hipGetLastError());
    return SP_OK;
}

template <typename T, int DT, int WM, int WN, int KW, bool POS>
sp_status launch_dq(const grad_args &f, const attn_mapping &c, int64_t items, hipStream_t st)
{
    constexpr int KT = KW * WN;
    size_t lds = 2 * (size_t)KT * DT * sizeof(T) + (POS ? KT * 4 + attn_bias_bytes(f.a, c.slots()) : 0) + (POS && f.part_table ? (size_t)WM * WN * f.a.buckets * 256 : 0);
    const size_t join = WN > 1 ? (size_t)WN * 32 * (DT + 1) * 4 : 0;
    return launch(dq_kernel<T, DT, WM, WN, KW, POS>, f, items * c.groups, 64 * WM * WN, lds > join ? lds : join, st);
}
template <typename T, int DT, bool POS>
sp_status launch_dq_mode(const grad_args &f, const attn_mapping &c, int64_t items, hipStream_t st)
{
    // K and V of a step and the bias's sums have to fit the LDS together
    constexpr int kRow = DT * (int)sizeof(T), WN = kRow >= 1024 ? (POS ? 1 : 2) : kRow == 512 && POS ? 2 : 4;
    if (c.wn > 1) return launch_dq<T, DT, 1, WN, 32, POS>(f, c, items, st);
    return launch_dq<T, DT, 4, 1, (kRow == 64 ? 64 : 32), POS>(f, c, items, st);
}
template <typename T, int DT, bool POS>
sp_status launch_dkv_mode(const grad_args &f, int br, int64_t items, hipStream_t st)
{
    constexpr int KW = DT * (int)sizeof(T) == 64 ? 64 : 32;
    const size_t lds = 2 * (size_t)KW * DT * sizeof(T) + KW * 12 + (POS ? attn_bias_bytes(f.a, 1) : 0);
    if (br == 128) return launch(dkv_kernel<T, DT, 4, KW, POS>, f, items * f.a.Hk, 256, lds, st);
    return launch(dkv_kernel<T, DT, 1, KW, POS>, f, items * f.a.Hk, 64, lds, st);
}

template <typename T, int DT>
sp_status grad_d(const sp_tensor *S, grad_args &f, const grad_choice &c, hipStream_t st)
{
    attn_args &a = f.a;
    const sp_attn_plan *rows = S->attention[0], *keys = S->attention[1];
    if (S->nvalues == 0) {                               // no pairs: zeros, and nothing of the problem is read
        if (f.part_table) hipLaunchKernelGGL(table_kernel<T>, dim3((unsigned)(a.buckets * a.H)), dim3(kThreads), 0, st, f, (int64_t)0);
        f.part_table = nullptr;
        a.buckets = a.causal = 0;
    }
    if (!a.buckets && !a.causal) a.qpos = a.kpos = nullptr;
    const bool pos = a.buckets || a.causal || a.scale == 0;
    if (a.m > 0) {
        constexpr int LPR = DT * (int)sizeof(T) / 16;
        hipLaunchKernelGGL((delta_kernel<T, LPR>), dim3((unsigned)ceil_div(a.m * a.H, kThreads / LPR)), dim3(kThreads), 0, st, f, (float *)f.delta);
        SP_HIP(hipGetLastError());
        f.p = attn_view(rows, c.rows.level);
        f.groups = c.rows.groups; f.mode = c.rows.mode;
        const int64_t items = rows->items[c.rows.level];
        if (pos) SP_TRY((launch_dq_mode<T, DT, true>(f, c.rows, items, st)));
        else SP_TRY((launch_dq_mode<T, DT, false>(f, c.rows, items, st)));
        if (c.rows.cut) hipLaunchKernelGGL((join_kernel<T, DT / 4, 1>), dim3((unsigned)ceil_div(a.m * a.H, 4)), dim3(kThreads), 0, st, f, a.m, a.H);
        if (f.part_table) hipLaunchKernelGGL(table_kernel<T>, dim3((unsigned)(a.buckets * a.H)), dim3(kThreads), 0, st, f, items);
        SP_HIP(hipGetLastError());
    }
    if (a.n > 0) {
        f.p = attn_view(keys, c.keys_level);
        const int64_t items = keys->items[c.keys_level];
        if (pos) SP_TRY((launch_dkv_mode<T, DT, true>(f, keys->br, items, st)));
        else SP_TRY((launch_dkv_mode<T, DT, false>(f, keys->br, items, st)));
        if (c.keys_cut) hipLaunchKernelGGL((join_kernel<T, DT / 4, 2>), dim3((unsigned)ceil_div(a.n * a.Hk, 4)), dim3(kThreads), 0, st, f, a.n, a.Hk);
        SP_HIP(hipGetLastError());
    }
    return SP_OK;
}

}  // namespace

template <typename T>
sp_status attn_backward(const sp_tensor *S, grad_args &f, const grad_choice &c, hipStream_t st)
{
    if (f.a.D <= 32) return grad_d<T, 32>(S, f, c, st);
    if (f.a.D <= 64) return grad_d<T, 64>(S, f, c, st);
    if (f.a.D <= 128) return grad_d<T, 128>(S, f, c, st);
    return grad_d<T, 256>(S, f, c, st);
}
