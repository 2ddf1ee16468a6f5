// Attention over a stored pattern, backward.  With D = sum dO * O for every row and head, the pairs' ds = p (dO V^T - D) come from a
// row's stored lse alone, so two kernels make them, each where it needs them: one over the rows of the pattern (dQ and the
// bias's gradient), one over its columns, by the transposed plan (dK and dV).  Seven products instead of five, but every result is
// summed by one workgroup in one order: no atomics on memory, the same bits on every call.
// Compiled once for each type (attention_backward_*.hip).
#pragma once
#include "attention_tiles.h"

namespace {

constexpr int kThreads = 256;

// v where bit k of `bits` is set, otherwise 0, whatever v is.
__device__ __forceinline__ float attn_where(uint32_t bits, int k, float v) { return __uint_as_float(__float_as_uint(v) & (uint32_t)__builtin_amdgcn_sbfe((int)bits, k, 1)); }

// Adds a lane's 16 pairs to its sums by bucket: hist[(bucket * 64 + lane) * N ...].  Two pairs are read, added and written back at a
// time; where they share a bucket, the second one goes on from the first one's sum, and the last write stays.  (Four at a time save half
// of the waiting and cost three times the comparing.)
template <int N>
__device__ __forceinline__ void attn_add_by_bucket(attn_lds_f32 *hist, int lane, const int (&bucket)[16], const float (&x)[16], const float (&y)[16])
{
    typedef float sums __attribute__((ext_vector_type(2)));
    typedef __attribute__((address_space(3))) sums lds_sums;
#pragma unroll
    for (int g = 0; g < 16; g += 2) {
        attn_lds_f32 *at[2];
        float u[2], v[2] = {0, 0};
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            at[c] = hist + (bucket[g + c] * 64 + lane) * N;
            if (N == 2) {
                const sums r = *(lds_sums *)at[c];
                u[c] = r.x; v[c] = r.y;
            } else u[c] = *at[c];
        }
        const bool same = bucket[g] == bucket[g + 1];
        u[0] += x[g]; v[0] += y[g];
        u[1] = (same ? u[0] : u[1]) + x[g + 1];
        v[1] = (same ? v[0] : v[1]) + y[g + 1];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            if (N == 2) {
                sums r;
                r.x = u[c]; r.y = v[c];
                *(lds_sums *)at[c] = r;
            } else *at[c] = u[c];
        }
    }
}

// log2 of what the weights e^(s - lse) of a lane's whole row sum to.  lse = top + log(total) is rounded to 32 bits, and far from zero that
// takes the logarithm from it: of n scores of -3.4e38 (a bias of a type's lowest value) every weight would be 1, not 1 / n.  Up to kAttnNearLse
// the rounding changes a weight by less than 2^-14 and is left alone (0); for tiles with a row beyond, the row's scores are made once more
// here, by the same instructions in the same order as in the kernels' tiles, so the same bits.  (Where the steps of a score are 64 wide, one
// that rounds to another step weighs e^64.)  Rows of K come straight from memory, a lane's as it needs them: such tiles are few.  (All of them,
// by a bias 2048 higher, and the steps take 2.6 times as long: 16 sequences of 200 to 512, 12 heads of 64: 197 and 499 us.)
constexpr float kAttnNearLse = 1024;
template <typename T, int DT>
__device__ __forceinline__ float attn_log_sum(const grad_args &f, const attn_item &item, const attn_lane &me, const typename attn_tile<T, DT>::frag (&q)[attn_tile<T, DT>::kSteps],
                                              int qp, float lse, int lane)
{
    typedef attn_tile<T, DT> tile;
    const attn_args &a = f.a;
    const attn_plan_view &p = f.p;
    const T *Kh = (const T *)a.K + (int64_t)me.kv * a.hdk;
    float sum = 0;
    for (int chunk = item.chunk0; chunk < p.chunk0[item.block + 1]; ++chunk) {
        const uint64_t word = item.word(p, chunk, me.r);
        for (int t = 0; t < 2; ++t) {
            const int64_t x0 = (int64_t)(chunk - item.chunk0) * kAttnChunk + 32 * t;
            const T *row = Kh + item.cols.get(x0 + (lane & 31)) * a.ldk;
            attn_f32x16 s = (attn_f32x16)(0.f);
#pragma unroll
            for (int k = 0; k < tile::kSteps; ++k) s = attn_mma<T>::mul(tile::granule(row, (2 * k + (lane >> 5)) * tile::kPer, a.D, f.vec, true), q[k], s);
            const uint32_t bits = (uint32_t)(word >> (32 * t)) >> (4 * (lane >> 5));
#pragma unroll
            for (int x = 0; x < 16; ++x) {
                const int kp = a.kpos[item.cols.get(x0 + 8 * (x >> 2) + 4 * (lane >> 5) + (x & 3))];
                const float of = (float)((const T *)a.table)[(int64_t)attn_bucket(a, attn_distance(kp, qp)) * a.ldt + me.head];
                const bool there = bits >> (8 * (x >> 2) + (x & 3)) & 1 && !(a.causal && kp > qp);
                sum += there ? attn_weight(__builtin_fmaf(s[x], a.scale, of), lse) : 0.f;
            }
        }
    }
    sum = attn_pair_sum(sum);
    return me.valid && fabsf(lse) >= kAttnNearLse && sum > 0 ? __builtin_amdgcn_logf(sum) : 0.f;
}

// dQ: the forward kernel's frame (items, gathered columns through LDS, tiles of 32 rows), with dO beside Q and V read as K is.
//
// 16 sequences of 256 to 512 queries over 512 to 1024 keys, 12 heads of 64, bf16: 47 us, 460 TFLOP/s for three products; bound by the
// vector work of a pair (an exponential and six operations) beside 24 of the matrix cores' cycles.
//
// With a bias its gradient as well: every lane adds its pairs' terms to a place of its own for each bucket in LDS, so that no two
// lanes ever add to one number, and the lanes' sums are added in order at the end; tiles that share a bucket are summed in registers.
// (Atomic adds to LDS take a cycle a lane, 64 for an instruction: 273 us for 16 sequences of 512, 12 heads, instead of 94.)
// `exact`: the terms are p dP and p, and ds = p (dP - D) is made of the sums with each row's D = sum p dP.  A bucket's ds almost
// cancel, and D from an O that was rounded to 16 bits would be most of their error (2.4e-3 of the gradient instead of 1.7e-3, the
// rounding of the result).  Not exact: the terms are ds.  That is f32, whose O is not rounded, and 16-bit types where rows are cut or the
// sums do not fit the LDS: D takes O's rounding there.  Either way the order of the sums is fixed.
template <typename T, int DT, int WM, int WN, int KW, bool POS>
__global__ __launch_bounds__(64 * WM * WN, DT * sizeof(T) <= 256 ? 2 : 1) void dq_kernel(grad_args f)
{
    typedef attn_tile<T, DT> tile;
    typedef typename tile::frag frag;
    constexpr int NT = 64 * WM * WN, KT = KW * WN, TILES = KW / 32;
    constexpr int STEP = KT > kAttnChunk ? KT / kAttnChunk : 1, SUB = KT < kAttnChunk ? kAttnChunk / KT : 1;
    extern __shared__ __align__(1024) char lds[];
    constexpr int FT = WN > 1 ? 64 : NT, FC = WN > 1 ? KW : KT;
    const attn_args &a = f.a;
    const attn_plan_view &p = f.p;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wn = WN > 1 ? wave : 0;
    const int ftid = WN > 1 ? lane : tid;
    constexpr int kShare = WN > 1 ? WN * 128 : 0;        // behind K and V
    attn_lds_i32 *s_kpos = (attn_lds_i32 *)((attn_lds *)lds + 4 * KT * tile::kRow + kShare) + wn * 2 * FC;
    const int64_t item_no = blockIdx.x / f.groups;
    const int group = blockIdx.x % f.groups;
    const attn_item item(p, item_no);
    const attn_lane me(a, item, f.mode, group, lane, wave, WM);
    const int r = me.r;
    const bool busy = __builtin_amdgcn_ballot_w64(me.valid) != 0, some = me.valid && item.c1 > item.c0;
    const float cc = POS ? kLog2e : fabsf(a.c);

    frag q[tile::kSteps], go[tile::kSteps];
    tile::load_lane((const T *)a.Q + me.row * a.ldq + me.head * a.hdq, a.D, f.vec, some, POS ? 1.f : a.c, q, lane);
    tile::load_lane((const T *)f.g.dO + me.row * f.g.lddo + me.head * f.g.hddo, a.D, f.vec, me.valid, 1.f, go, lane);
    float off = f.g.lse[me.head * a.m + me.row];
    if (off == -INFINITY) off = INFINITY;                // no weight left
    if (!POS) off *= kLog2e;
    // D = sum dO * O of the lane's row
    float delta = 0;
    {
        const T *o = (const T *)f.g.O + me.row * f.g.ldo + me.head * f.g.hdo;
#pragma unroll
        for (int s = 0; s < tile::kSteps; ++s) {
            const frag u = tile::granule(o, (2 * s + (lane >> 5)) * tile::kPer, a.D, f.vec, me.valid);
#pragma unroll
            for (int k = 0; k < tile::kPer; ++k) delta += (float)u[k] * (float)go[s][k];
        }
        delta = attn_pair_sum(delta);
    }
    float rest = 0, log_sum = 0;                         // sum of ds over the row's pairs; log2 of that of its weights
    int qp = 0, q_lo = 0, q_hi = 0;
    attn_bias bias = {};
    attn_lds_f32 *hist = nullptr;                             // [buckets][64] of ds; exact: of p dP and p
    const int places = attn_places(a), hist_size = places * 64 * (f.exact ? 2 : 1);
    float far_x[2] = {0, 0}, far_p[2] = {0, 0};          // the far buckets behind and ahead
    if (POS) {
        if (a.qpos) { qp = a.qpos[me.row]; q_lo = attn_wave_min(qp); q_hi = attn_wave_max(qp); }
        if (a.buckets) {
            if (__builtin_amdgcn_ballot_w64(me.valid && fabsf(off) >= kAttnNearLse && off - off == 0) != 0)
                log_sum = attn_log_sum<T, DT>(f, item, me, q, qp, off, lane);
            bias = attn_lane_bias<T>(a, (attn_lds *)lds + 4 * KT * tile::kRow + kShare + 2 * KT * 4, f.mode, group, lane, wave, WM);
            if (f.part_table) {
                hist = bias.table + (((places << bias.shift) + 3) & ~3) + wave * hist_size;
                for (int b = lane; b < hist_size; b += 64) hist[b] = 0;
            }
        }
    }
    attn_f32x16 acc[tile::kBlocks];
#pragma unroll
    for (int x = 0; x < tile::kBlocks; ++x) acc[x] = (attn_f32x16)(0.f);

    const int64_t steps = (int64_t)(item.c1 - item.c0 + STEP - 1) / STEP * SUB;
    attn_ring<T, DT, FT, FC, POS> ring;
    ring.lds = (attn_lds *)lds + wn * 4 * FC * tile::kRow;
    ring.ldx = a.ldk; ring.ldy = a.ldv;
    ring.cols = item.cols; ring.x0 = (int64_t)(item.c0 - item.chunk0) * kAttnChunk + wn * FC; ring.step = KT; ring.tid = ftid;
    ring.pos = a.kpos; ring.sign = POS ? a.causal : 0; ring.limit = q_hi;
    ring.D = a.D; ring.vec = f.vec;
    const T *Kh = (const T *)a.K + (int64_t)me.kv * a.hdk, *Vh = (const T *)a.V + (int64_t)me.kv * a.hdv;
    if (a.D != DT || ring.sign) ring.zero();
    if (POS && a.causal && WM > 1) {
        if (lane == 0) s_kpos[wave] = q_hi;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WM; ++w) ring.limit = s_kpos[w] > ring.limit ? s_kpos[w] : ring.limit;
    }
    if (POS || a.D != DT) __syncthreads();
    auto my_chunk = [&](int64_t step, int &col0) {
        col0 = (int)(step % SUB) * KT + wn * KW;
        const int chunk = item.c0 + (int)(step / SUB) * STEP + col0 / kAttnChunk;
        return busy && chunk < item.c1 ? chunk : -1;
    };
    uint64_t word = 0, word_next = 0;
    int state = 0, state_next = 0;
    auto fetch_pairs = [&](int64_t step) {
        int col0;
        const int chunk = my_chunk(step, col0);
        state_next = 0;
        if (chunk >= 0) { state_next = item.state(p, chunk, r); word_next = item.word(p, chunk, r); }
    };
    auto walk = [&](auto early) {
        constexpr bool EARLY = decltype(early)::value;
        if (steps > 0) {
            ring.begin(steps, [](int64_t s) { return s; });
            fetch_pairs(0);
            ring.rows(0, Kh, Vh);
        }
        for (int64_t step = 0; step < steps; ++step) {
            ring.arrive();
            if (POS && ftid < FC) s_kpos[(step & 1) * FC + ftid] = ring.kp_one;
            if (WN == 1) __syncthreads();
            else {
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_wave_barrier();
            }
            word = word_next; state = state_next;
            const attn_lds *sK = ring.x_of(step), *sV = ring.y_of(step);
            if (step + 1 < steps) {
                ring.advance();
                if (step + ring.kAhead < steps) ring.columns(step + ring.kAhead);
                fetch_pairs(step + 1);
                ring.rows(step + 1, Kh, Vh);
            }
            int col0;
            if (my_chunk(step, col0) < 0) continue;
            state = __builtin_amdgcn_readfirstlane(state);
            if (state == 0) continue;
            word >>= col0 % kAttnChunk;
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                const attn_lds_i32 *kp = s_kpos + (step & 1) * FC + 32 * t;
                attn_near near = {false, false, false, 0};
                if (POS) {
                    const int col = kp[lane & 31];
                    near = attn_look(a, attn_distance(col, q_hi), attn_distance(col, q_lo));
                    if (near.nothing) continue;
                }
                attn_f32x16 s = tile::scores(sK, 32 * t, q, a.D, lane);
                attn_f32x16 dp = tile::scores(sV, 32 * t, go, a.D, lane);
                // what is not stored, and rows that do not exist, add nothing
                const uint32_t bits = (me.valid ? (uint32_t)(word >> (32 * t)) : 0u) >> (4 * (lane >> 5));
                if (!POS) {
#pragma unroll
                    for (int x = 0; x < 16; ++x) s[x] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[x], cc, -off)) * (dp[x] - delta);
                    if (state != 2) {                        // a lane of no row keeps its own nonsense to itself
#pragma unroll
                        for (int x = 0; x < 16; ++x) s[x] = attn_where(bits, 8 * (x >> 2) + (x & 3), s[x]);
                    }
                } else {
                    // Loops of one kind of work each, without branches inside, so that the LDS's answers overlap.  A score of minus
                    // infinity has weight 0, whatever dP is.
                    const bool one = !a.buckets || near.far;
                    uint32_t there = 0;
#pragma unroll
                    for (int b = 0; b < 4; ++b) there |= (bits >> 8 * b & 15) << 4 * b;
                    if (near.ask) {
#pragma unroll
                        for (int x = 0; x < 16; ++x) there &= ~((uint32_t)(kp[8 * (x >> 2) + 4 * (lane >> 5) + (x & 3)] > qp) << x);
                    }
                    if (one) {
                        const float all_of = a.buckets ? bias.at(near.place) : 0.f;
#pragma unroll
                        for (int x = 0; x < 16; ++x) s[x] = __builtin_fmaf(s[x], a.scale, all_of);
                    } else
                        attn_add_bias(bias, s, a.scale, [&](int x) { return kp[8 * (x >> 2) + 4 * (lane >> 5) + (x & 3)]; }, [&](int) { return qp; });
                    if (attn_any_lowest(s)) {
#pragma unroll
                        for (int x = 0; x < 16; ++x) there &= ~((uint32_t)(s[x] == -INFINITY) << x);
                    }
                    float sum_x = 0, sum_p = 0, term[16], weight[16];
#pragma unroll
                    for (int x = 0; x < 16; ++x) {
                        weight[x] = attn_where(there, x, __builtin_amdgcn_exp2f(__builtin_fmaf(s[x] - off, cc, -log_sum)));
                        s[x] = attn_where(there, x, weight[x] * (dp[x] - delta));
                        term[x] = attn_where(there, x, weight[x] * (dp[x] - (f.exact ? 0.f : delta)));
                        sum_x += term[x]; sum_p += weight[x];
                    }
                    if (!EARLY && hist && !one) {
                        int place[16];
#pragma unroll
                        for (int x = 0; x < 16; ++x) place[x] = bias.lut[bias.index(kp[8 * (x >> 2) + 4 * (lane >> 5) + (x & 3)], qp)];
                        if (f.exact) attn_add_by_bucket<2>(hist, lane, place, term, weight);
                        else attn_add_by_bucket<1>(hist, lane, place, term, weight);
                    }
                    if (!EARLY && hist && one) {
                        const bool behind = near.place == a.side - 1;
                        far_x[0] += behind ? sum_x : 0.f; far_p[0] += behind ? sum_p : 0.f;
                        far_x[1] += behind ? 0.f : sum_x; far_p[1] += behind ? 0.f : sum_p;
                    }
                }
                if (sizeof(T) == 2) {
#pragma unroll
                    for (int x = 0; x < 16; ++x) rest += s[x];
                }
                if (!EARLY) tile::add_rows(acc, sK, 32 * t, s, a.D, lane);
            }
        }
    };
    // Short rows go through their steps twice, and the first time their ds only add up to what D misses.
    if (sizeof(T) == 2 && item.whole && item.c1 - item.c0 <= kAttnTwice && p.rowptr[item.row0 + item.rows] - p.rowptr[item.row0] <= kAttnTwicePairs * item.rows) {
        walk(std::true_type());
        rest = attn_pair_sum(rest);
        __syncthreads();
        if (WN > 1) {                                    // the waves' shares of the tile
            attn_lds_f32 *share = (attn_lds_f32 *)((attn_lds *)lds + 4 * KT * tile::kRow);
            share[wn * 32 + (lane & 31)] = rest;
            __syncthreads();
            rest = 0;
#pragma unroll
            for (int x = 0; x < WN; ++x) rest += share[x * 32 + (lane & 31)];
        }
        delta += rest;
        rest = 0;
    }
    walk(std::false_type());
    // For dkv_kernel, and what short rows go through their steps twice for.  The weights of a row that is whole here sum to 1, so what its ds
    // miss to sum to 0 is the error of a D made of an O that was rounded to 16 bits.
    rest = sizeof(T) == 2 && item.whole ? attn_pair_sum(rest) : 0.f;
    if (WN == 1 && me.valid && lane < 32 && item.c0 == item.chunk0) {
        f.delta[me.head * a.m + me.row] = delta + rest;
        if (POS && f.log_sum) f.log_sum[me.head * a.m + me.row] = log_sum;
    }
    float odd = 0;
#pragma unroll
    for (int x = 0; x < tile::kBlocks; ++x)
#pragma unroll
        for (int k = 0; k < 16; ++k) odd += acc[x][k] * 0.f;
    uint64_t again = __builtin_amdgcn_ballot_w64(me.valid && !(odd == 0.f));

    if (POS && hist) {
        __syncthreads();                                 // all waves are done with K
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            const int b = attn_far_place(a, side == 1);
            if (f.exact) {
                hist[(b * 64 + lane) * 2] += far_x[side];
                hist[(b * 64 + lane) * 2 + 1] += far_p[side];
            } else hist[b * 64 + lane] += far_x[side];
        }
        __syncthreads();
        const attn_lds_f32 *all = bias.table + (((places << bias.shift) + 3) & ~3);
        attn_lds_f32 *s_delta = (attn_lds_f32 *)(attn_lds *)lds;     // over K: [waves][32], each row's D
        // rows are a wave's own, or (WN) shared by all waves
        if (f.exact && lane < 32 && (WN == 1 || wave == 0)) {
            float d = 0;
            for (int w = wave; w < (WN == 1 ? wave + 1 : WN); ++w)
                for (int b = 0; b < places; ++b) d += all[w * hist_size + (b * 64 + lane) * 2] + all[w * hist_size + (b * 64 + 32 + lane) * 2];
            s_delta[wave * 32 + lane] = d;
        }
        __syncthreads();
        if (f.exact) {                                   // a row whose D is not a number adds nothing to the buckets that it has no weight in
            bool odd = false;
            for (int x = lane; x < (WN == 1 ? 32 * WM : 32); x += 64) odd = odd || !(s_delta[x] * 0.f == 0.f);
            if (__builtin_amdgcn_ballot_w64(odd) != 0) { // the whole workgroup
                const float d = s_delta[(WN == 1 ? wave : 0) * 32 + (lane & 31)];
                for (int b = 0; b < places; ++b) {
                    attn_lds_f32 *x = hist + (b * 64 + lane) * 2;
                    if (x[1] != 0) x[0] -= d * x[1];
                    x[1] = 0;
                }
                __syncthreads();
                if (tid < 32 * WM) s_delta[tid] = 0;
                __syncthreads();
            }
        }
        float *out = f.part_table + item.part * a.H * a.buckets;
        auto term = [&](int w, int b) {
            const attn_lds_f32 *x = all + w * hist_size + (b * 64 + lane) * (f.exact ? 2 : 1);
            return f.exact ? x[0] - s_delta[(WN == 1 ? w : 0) * 32 + (lane & 31)] * x[1] : x[0];
        };
        for (int b = wave; b < places; b += WM * WN) {
            float sum = 0;
            if (f.mode == kHeadsOfRows) {
                for (int w = 0; w < WM; ++w) {
                    const int y = group / a.Hk * WM + w;
                    sum = attn_wave_sum(term(w, b));
                    if (lane == 0 && y < a.G) out[(group % a.Hk * a.G + y) * a.buckets + attn_bucket_of(a, b)] = sum;
                }
                continue;
            }
            for (int w = 0; w < WM * WN; ++w) sum += term(w, b);
            if (f.mode == kHeadsTogether) {
                const int y = group / a.Hk * 32 + lane;
                sum = attn_pair_sum(sum);
                if (lane < 32 && y < a.G) out[(group % a.Hk * a.G + y) * a.buckets + attn_bucket_of(a, b)] = sum;
            } else {
                sum = attn_wave_sum(sum);
                if (lane == 0) out[(group % a.Hk * a.G + group / a.Hk) * a.buckets + attn_bucket_of(a, b)] = sum;
            }
        }
        __syncthreads();
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
        attn_lds_f32 *sums = (attn_lds_f32 *)(attn_lds *)lds, *bad = sums + WN * 32 * DT;
#pragma unroll
        for (int x = 0; x < tile::kBlocks; ++x)
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const int g = (8 * x + 2 * b + (lane >> 5)) ^ (lane & 7);
                *(attn_lds_f32x4 *)(sums + (wn * 32 + (lane & 31)) * DT + 4 * g) = (attn_f32x4){acc[x][4 * b], acc[x][4 * b + 1], acc[x][4 * b + 2], acc[x][4 * b + 3]};
            }
        if (lane < 32) {
            bad[wn * 32 + lane] = (again | again >> 32) >> lane & 1 ? 1.f : 0.f;
            bad[(WN + wn) * 32 + lane] = rest;
        }
        __syncthreads();
        constexpr int LANES = NT / 32, EACH = DT / LANES;
        const int mine = tid / LANES, part = tid % LANES;
        float any = 0, more = 0;
#pragma unroll
        for (int x = 0; x < WN; ++x) { any += bad[x * 32 + mine]; more += bad[(WN + x) * 32 + mine]; }
        const float delta2 = __shfl(delta, mine, 64), log_sum2 = POS ? __shfl(log_sum, mine, 64) : 0.f;
        const int64_t row2 = ((int64_t)__shfl((int)(me.row >> 32), mine, 64) << 32) | (uint32_t)__shfl((int)me.row, mine, 64);
        const int head2 = __shfl(me.head, mine, 64), r2 = __shfl(r, mine, 64);
        const bool valid2 = __shfl((int)me.valid, mine, 64) != 0;
        const int64_t place2 = (item.part * a.H + head2) * p.br + r2;
        if (valid2 && part == 0 && item.c0 == item.chunk0) {
            f.delta[head2 * a.m + row2] = delta2 + more;
            if (POS && f.log_sum) f.log_sum[head2 * a.m + row2] = log_sum2;
        }
        if (valid2 && any == 0) {
#pragma unroll
            for (int k = 0; k < EACH; k += 4) {
                const int d = part * EACH + k;
                attn_f32x4 v = (attn_f32x4)(0.f);
#pragma unroll
                for (int x = 0; x < WN; ++x) v += *(attn_lds_f32x4 *)(sums + (x * 32 + mine) * DT + 4 * ((d >> 2) ^ (mine & 7)));
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
                       __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(delta), x)), __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(log_sum), x)),
                       one);
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

// Does a workgroup of dkv_kernel take a compute unit's registers for itself?  Two sums and two operands of 128 numbers of 16 bits are 192
// registers; with the positions' work beside them the rest no longer fits half of the 512 (dK, dV of a band of 10763 tokens, 8 heads of
// 128, with bias: 262 us so, 86 alone), without it, it nearly does (8 sequences of about 860, 16 heads of 128: 446 us for the whole
// step, 476 alone).
constexpr bool attn_dkv_alone(int row_bytes, bool pos) { return row_bytes > (pos ? 128 : 256); }

// dK and dV: blocks of keys (lanes) over the queries that attend to them, head by head of the keys' group.  Q and dO come through
// LDS, K and V stay in registers; the scores are those of the forward kernel with the roles exchanged, so weights and ds are again
// operands as they lie.  WM waves take 32 keys each.  The sequences above: 66 us, 435 TFLOP/s for four products; the matrix cores work 19 % of
// the cycles, the vector units 32 %: two workgroups a compute unit, and a third round of them that is a third full.
template <typename T, int DT, int WM, int KW, bool POS>
__global__ __launch_bounds__(64 * WM, attn_dkv_alone(DT * (int)sizeof(T), POS) ? 1 : 2) void dkv_kernel(grad_args f)
{
    typedef attn_tile<T, DT> tile;
    typedef typename tile::frag frag;
    constexpr int NT = 64 * WM, KT = KW, TILES = KW / 32, SUB = kAttnChunk / KT;
    static_assert(KT <= kAttnChunk, "steps within a chunk");
    extern __shared__ __align__(1024) char lds[];
    // behind Q and dO, two places of everything: lse and D, with POS positions and attn_log_sum of a step's queries, the bias of a head
    attn_lds_f32 *s_lse = (attn_lds_f32 *)((attn_lds *)lds + 4 * KT * tile::kRow), *s_delta = s_lse + 2 * KT;
    attn_lds_i32 *s_qpos = (attn_lds_i32 *)(s_delta + 2 * KT);
    attn_lds_f32 *s_log = (attn_lds_f32 *)(s_qpos + 2 * KT);
    const attn_args &a = f.a;
    const attn_plan_view &p = f.p;                       // of the transposed pattern: rows are keys
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t item_no = blockIdx.x / a.Hk;
    const int kv = blockIdx.x % a.Hk;
    const attn_item item(p, item_no);
    const int r = 32 * wave + (lane & 31);
    const bool valid = r < item.rows;
    const int64_t key = item.row0 + (valid ? r : item.rows - 1);
    const bool busy = __builtin_amdgcn_ballot_w64(valid) != 0, some = valid && item.c1 > item.c0;
    const float cc = POS ? kLog2e : fabsf(a.c);
    frag kx[tile::kSteps], vx[tile::kSteps];
    tile::load_lane((const T *)a.K + key * a.ldk + kv * a.hdk, a.D, f.vec, some, POS ? 1.f : a.c, kx, lane);
    tile::load_lane((const T *)a.V + key * a.ldv + kv * a.hdv, a.D, f.vec, some, 1.f, vx, lane);
    int kp = 0, k_lo = 0, k_hi = 0;
    attn_bias bias = {};
    if (POS) {
        if (a.kpos) { kp = a.kpos[key]; k_lo = attn_wave_min(kp); k_hi = attn_wave_max(kp); }
        if (a.buckets) {
            // a slot for even heads and one for odd ones: the head at hand and the next
            bias = attn_make_bias<T>(a, (attn_lds *)(s_log + 2 * KT), 1, [&](int s) {
                const int x = (s ^ kv * a.G) & 1;
                return x < a.G ? kv * a.G + x : -1;
            });
        }
    }
    attn_f32x16 dk[tile::kBlocks], dv[tile::kBlocks];
#pragma unroll
    for (int x = 0; x < tile::kBlocks; ++x) dk[x] = dv[x] = (attn_f32x16)(0.f);

    const int64_t per_head = (int64_t)(item.c1 - item.c0) * SUB, steps = per_head * a.G;
    attn_ring<T, DT, NT, KT, POS, true> ring;
    ring.lds = (attn_lds *)lds;
    ring.ldx = a.ldq; ring.ldy = f.g.lddo;
    ring.cols = item.cols; ring.x0 = (int64_t)(item.c0 - item.chunk0) * kAttnChunk; ring.step = KT; ring.tid = tid;
    ring.pos = a.qpos; ring.sign = POS ? -a.causal : 0; ring.limit = k_lo;
    ring.D = a.D; ring.vec = f.vec;
    if (a.D != DT || ring.sign) ring.zero();
    if (POS && a.causal && WM > 1) {
        if (lane == 0) s_qpos[wave] = k_lo;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WM; ++w) ring.limit = s_qpos[w] < ring.limit ? s_qpos[w] : ring.limit;
    }
    if (POS || a.D != DT) __syncthreads();
    float lse_next = 0, delta_next = 0, log_next = 0;
    uint64_t word = 0, word_next = 0;
    int state = 0, state_next = 0;
    // a step: the head and the step among the head's
    struct place { int h; int64_t at; };
    auto after = [&](place x) { return ++x.at == per_head ? place{x.h + 1, 0} : x; };
    auto fetch = [&](place x) {
        if (busy) {
            const int chunk = item.c0 + (int)(x.at / SUB);
            state_next = item.state(p, chunk, r);
            word_next = item.word(p, chunk, r);
        }
        if (tid < KT) {
            lse_next = f.g.lse[x.h * a.m + ring.one];
            delta_next = f.delta[x.h * a.m + ring.one];
            if (POS && f.log_sum) log_next = f.log_sum[x.h * a.m + ring.one];
        }
    };
    auto rows = [&](int64_t s, place x) { ring.rows(s, (const T *)a.Q + x.h * a.hdq, (const T *)f.g.dO + x.h * f.g.hddo); };
    place now = {kv * a.G, 0}, soon = after(now), ahead = after(soon);
    if (ring.kAhead == 3) ahead = after(ahead);          // the step whose columns are asked for
    if (steps > 0) {
        place x[3] = {now, soon, after(soon)};
        ring.begin(steps, [&](int64_t s) { return x[s].at; });
        fetch(now);
        rows(0, now);
    }
    for (int64_t step = 0; step < steps; ++step) {
        ring.arrive();
        const int here = (int)(step & 1) * KT;
        if (tid < KT) {
            s_lse[here + tid] = lse_next == -INFINITY ? INFINITY : POS ? lse_next : lse_next * kLog2e;     // no weight left
            s_delta[here + tid] = delta_next;
            if (POS) { s_qpos[here + tid] = ring.kp_one; s_log[here + tid] = log_next; }
        }
        if (POS && a.buckets && now.at == 0) {           // the slot of the head before the last is free
            bias.slot = now.h & 1;
            if (a.G > 2)
                for (int b = tid; b < attn_places(a); b += NT) bias.table[2 * b + bias.slot] = (float)((const T *)a.table)[(int64_t)attn_bucket_of(a, b) * a.ldt + now.h];
        }
        __syncthreads();
        word = word_next; state = state_next;
        const attn_lds *sQ = ring.x_of(step), *sO = ring.y_of(step);
        if (step + 1 < steps) {
            ring.advance();
            if (step + ring.kAhead < steps) ring.columns(ahead.at);
            fetch(soon);
            rows(step + 1, soon);
        }
        const int col0 = (int)(now.at % SUB) * KT;
        now = soon; soon = after(soon); ahead = after(ahead);
        if (!busy) continue;
        state = __builtin_amdgcn_readfirstlane(state);
        if (state == 0) continue;
        word >>= col0;
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            attn_near near = {false, false, false, 0};
            if (POS) {
                const int qp = s_qpos[here + 32 * t + (lane & 31)];
                near = attn_look(a, attn_distance(k_lo, qp), attn_distance(k_hi, qp));
                if (near.nothing) continue;
            }
            attn_f32x16 s = tile::scores(sQ, 32 * t, kx, a.D, lane);
            attn_f32x16 dp = tile::scores(sO, 32 * t, vx, a.D, lane);
            const uint32_t bits = (valid ? (uint32_t)(word >> (32 * t)) : 0u) >> (4 * (lane >> 5));
            uint32_t there = bits;
            if (POS) {
                if (near.ask) {
#pragma unroll
                    for (int x = 0; x < 16; ++x)
                        there &= ~((uint32_t)(kp > s_qpos[here + 32 * t + 8 * (x >> 2) + 4 * (lane >> 5) + (x & 3)]) << (8 * (x >> 2) + (x & 3)));
                }
                if (!a.buckets || near.far) {
                    const float all_of = a.buckets ? bias.at(near.place) : 0.f;
#pragma unroll
                    for (int x = 0; x < 16; ++x) s[x] = __builtin_fmaf(s[x], a.scale, all_of);
                } else {
                    attn_add_bias(bias, s, a.scale, [&](int) { return kp; }, [&](int x) { return s_qpos[here + 32 * t + 8 * (x >> 2) + 4 * (lane >> 5) + (x & 3)]; });
                }
            }
            if (POS && attn_any_lowest(s)) {             // a score of minus infinity has weight 0, whatever dP is
#pragma unroll
                for (int x = 0; x < 16; ++x) there &= ~((uint32_t)(s[x] == -INFINITY) << (8 * (x >> 2) + (x & 3)));
            }
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const int q0 = here + 32 * t + 8 * b + 4 * (lane >> 5);
                const attn_f32x4 lse = *(const attn_lds_f32x4 *)(s_lse + q0), delta = *(const attn_lds_f32x4 *)(s_delta + q0);
                const attn_f32x4 log_sum = POS ? *(const attn_lds_f32x4 *)(s_log + q0) : (attn_f32x4)(0.f);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const int x = 4 * b + c;
                    s[x] = __builtin_amdgcn_exp2f(POS ? __builtin_fmaf(s[x] - lse[c], cc, -log_sum[c]) : __builtin_fmaf(s[x], cc, -lse[c]));
                    dp[x] = s[x] * (dp[x] - delta[c]);
                }
            }
            if (POS || state != 2) {                     // a lane of no key keeps its own nonsense to itself
#pragma unroll
                for (int x = 0; x < 16; ++x) {
                    s[x] = attn_where(there, 8 * (x >> 2) + (x & 3), s[x]);
                    dp[x] = attn_where(there, 8 * (x >> 2) + (x & 3), dp[x]);
                }
            }
            tile::add_rows(dv, sO, 32 * t, s, a.D, lane);
            tile::add_rows(dk, sQ, 32 * t, dp, a.D, lane);
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
            attn_row_dkv<T>(a, p, item.block, rr, item.c0, item.c1, j, g, lane, (const T *)f.g.dO, f.g.lddo, f.g.hddo, f.g.lse, f.delta, POS ? f.log_sum : nullptr, k1, v1);
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
// The grid: blocks that were cut, rows of a block, heads.
template <typename T, int LP, int PER>
__global__ __launch_bounds__(kThreads) void join_kernel(grad_args f, int64_t cut, int heads)
{
    const attn_plan_view &p = f.p;
    const int lane = threadIdx.x & 63, D = f.a.D;
    const int64_t x = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
    if (x >= cut * p.br * heads) return;
    const int h = (int)(x % heads), r = (int)(x / heads % p.br);
    const int64_t b = p.cut_block[x / heads / p.br], i = attn_first_row(p.row0, b, p.br, p.m) + r;
    if (i >= attn_first_row(p.row0, b + 1, p.br, p.m)) return;
    const int first = p.item0[b], parts = p.item0[b + 1] - first;
#pragma unroll
    for (int v = 0; v < PER; ++v) {
        T *out = PER == 1 ? (T *)f.g.dQ + i * f.g.lddq + h * f.g.hddq
                          : v == 0 ? (T *)f.g.dK + i * f.g.lddk + h * f.g.hddk : (T *)f.g.dV + i * f.g.lddv + h * f.g.hddv;
        const attn_f32x4 sum = attn_add_parts<LP>(parts, f.pd, lane, [&](int k) {
            return f.part + ((((int64_t)(first + k) * heads + h) * p.br + r) * PER + v) * f.pd;
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
    const bool none = a.bidirectional && b == a.side;    // no distance is in that bucket, and nothing was written for it
    if (threadIdx.x == 0) ((T *)f.g.dTable)[(int64_t)b * f.g.lddt + h] = (T)(none ? 0.f : s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3]);
}

template <typename K>
sp_status launch(K kernel, const grad_args &f, int64_t groups, int threads, size_t lds, hipStream_t st)
{
    if (!attn_launches(groups, threads)) return SP_ERR_TOO_LARGE;
    if (lds > (size_t)kAttnLds) return SP_ERR_UNSUPPORTED;
    if (lds > 65536) SP_HIP(hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
    hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(threads), lds, st, f);
    SP_HIP(hipGetLastError());
    return SP_OK;
}

template <typename T, int DT, int WM, int WN, int KW, bool POS>
sp_status launch_dq(const grad_args &f, const attn_mapping &c, int64_t items, hipStream_t st)
{
    const size_t lds = attn_dq_lds(f.a, c, DT * (int)sizeof(T), POS, POS && f.part_table, f.exact);
    const size_t join = WN > 1 ? (size_t)WN * 32 * (DT + 2) * 4 : 0;
    return launch(dq_kernel<T, DT, WM, WN, KW, POS>, f, items * c.groups, 64 * WM * WN, lds > join ? lds : join, st);
}
template <typename T, int DT, bool POS>
sp_status launch_dq_mode(const grad_args &f, const attn_mapping &c, int64_t items, hipStream_t st)
{
    constexpr int kRow = DT * (int)sizeof(T);
    if (c.wn > 1) return launch_dq<T, DT, 1, attn_dq_waves(kRow, POS), 32, POS>(f, c, items, st);
    return launch_dq<T, DT, 4, 1, attn_dq_columns(kRow, POS), POS>(f, c, items, st);
}
template <typename T, int DT, bool POS>
sp_status launch_dkv_mode(const grad_args &f, int br, int64_t items, hipStream_t st)
{
    constexpr int KW = sizeof(T) == 2 && (DT <= 64 || (DT == 128 && POS)) ? 64 : 32;
    const size_t lds = 4 * (size_t)KW * DT * sizeof(T) + KW * (POS ? 32 : 16) + (POS ? attn_bias_bytes(f.a, 2) : 0);
    if (br == 128) return launch(dkv_kernel<T, DT, 4, KW, POS>, f, items * f.a.Hk, 256, lds, st);
    return launch(dkv_kernel<T, DT, 1, KW, POS>, f, items * f.a.Hk, 64, lds, st);
}

template <typename T, int DT>
sp_status grad_d(const sp_tensor *S, grad_args &f, const grad_choice &c, hipStream_t st)
{
    attn_args &a = f.a;
    const sp_attn_plan *rows = S->attention[0], *keys = S->attention[1];
    const bool pos = (S->nvalues > 0 && (a.buckets || a.causal)) || a.scale == 0;
    const int row_threads = c.rows.wn > 1 ? 64 * attn_dq_waves(DT * (int)sizeof(T), pos) : 256;
    if (!attn_launches(rows->items[c.rows.level] * c.rows.groups, row_threads) || !attn_launches(keys->items[c.keys_level] * a.Hk, keys->br == 128 ? 256 : 64))
        return SP_ERR_TOO_LARGE;                         // before anything is written
    if (S->nvalues == 0) {                               // no pairs: zeros, and nothing of the problem is read
        // (by dTable: without rows the workspace has no bytes, and its parts no addresses)
        if (a.buckets && f.g.dTable) hipLaunchKernelGGL(table_kernel<T>, dim3((unsigned)(a.buckets * a.H)), dim3(kThreads), 0, st, f, (int64_t)0);
        SP_HIP(hipGetLastError());
        f.part_table = nullptr;
        a.buckets = a.causal = 0;
    }
    if (!a.buckets && !a.causal) a.qpos = a.kpos = nullptr;
    if (a.m > 0) {
        f.p = attn_view(rows, c.rows.level);
        f.groups = c.rows.groups; f.mode = c.rows.mode;
        const int64_t items = rows->items[c.rows.level];
        if (pos) SP_TRY((launch_dq_mode<T, DT, true>(f, c.rows, items, st)));
        else SP_TRY((launch_dq_mode<T, DT, false>(f, c.rows, items, st)));
        if (c.rows.cut) hipLaunchKernelGGL((join_kernel<T, DT / 4, 1>), dim3((unsigned)ceil_div(rows->cut[c.rows.level] * rows->br * a.H, 4)), dim3(kThreads), 0, st, f,
                                           rows->cut[c.rows.level], a.H);
        if (f.part_table) hipLaunchKernelGGL(table_kernel<T>, dim3((unsigned)(a.buckets * a.H)), dim3(kThreads), 0, st, f, items);
        SP_HIP(hipGetLastError());
    }
    if (a.n > 0) {
        f.p = attn_view(keys, c.keys_level);
        const int64_t items = keys->items[c.keys_level];
        if (pos) SP_TRY((launch_dkv_mode<T, DT, true>(f, keys->br, items, st)));
        else SP_TRY((launch_dkv_mode<T, DT, false>(f, keys->br, items, st)));
        if (c.keys_cut) hipLaunchKernelGGL((join_kernel<T, DT / 4, 2>), dim3((unsigned)ceil_div(keys->cut[c.keys_level] * keys->br * a.Hk, 4)), dim3(kThreads), 0, st, f,
                                       keys->cut[c.keys_level], a.Hk);
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
    // f32 ends at 128: a row and its sums of 256 numbers of 32 bits do not fit a lane's registers (0.6 to 2 KB of scratch a lane), nor, with a
    // bias, a step of K and V and the sums by bucket the LDS
    if constexpr (sizeof(T) == 2) return grad_d<T, 256>(S, f, c, st);
    return SP_ERR_SHAPE;
}
