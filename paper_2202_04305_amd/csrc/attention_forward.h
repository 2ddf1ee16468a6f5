// Attention over a stored pattern, forward: the kernel that makes O and lse, the join of rows that were cut.  Compiled once for each
// type (attention_forward_*.hip).
#pragma once
#include "attention_tiles.h"

namespace {

// A workgroup takes an item (a block of rows and a stretch of the columns that they store) and one head or a few that share K and V.
// Per step KT columns' rows of K and V come into LDS, gathered by the plan's list, while the step before is computed; every wave makes the 32 x KW scores of its tile, masks them with the plan's bits, keeps each row's running maximum and sum
// (f32), and adds the weighted rows of V to its 32 x D sums, which stay in registers.  Weights are rounded to the operands' type
// for that product (half a step of 16-bit types, as every operand of the matrix cores is); the sum that divides takes them unrounded.
//
// 16 sequences of 512 to 1024 queries over 2048 to 4096 keys, 16 heads of 128 over 4, bf16: 419 us, 763 TFLOP/s.  Of the cycles the matrix
// cores work 31 % and the vector units 47 %: an exponential takes four vector cycles, 32 of them a lane and step, beside 32 products,
// and two waves a SIMD (256 registers each) overlap them only in part.  Single tokens are bound by the rows of K and V: 64 of them over
// 800 to 1500 columns, 16 heads of 64, f16: 70 us, 4.1 TB/s.
//
// WM waves take different tiles over the same columns; WN waves share the columns of one tile and are joined through LDS at the end.
// POS: with positions (bias, causal); scores are held in units of e then, so that a bias of the type's lowest value stays a number,
// and as plain products of q and k otherwise.
template <typename T, int DT, int WM, int WN, int KW, bool POS>
__global__ __launch_bounds__(64 * WM * WN, DT * (int)sizeof(T) <= 128 ? 3 : DT <= 128 ? 2 : 1) void forward_kernel(forward_args f)
{
    typedef attn_tile<T, DT> tile;
    typedef typename tile::frag frag;
    constexpr int NT = 64 * WM * WN, KT = KW * WN, TILES = KW / 32;
    constexpr int STEP = KT > kAttnChunk ? KT / kAttnChunk : 1;         // chunks of a step (or one chunk in 64 / KT steps)
    constexpr int SUB = KT < kAttnChunk ? kAttnChunk / KT : 1;
    extern __shared__ __align__(1024) char lds[];
    // WM waves fetch a step together and meet at barriers; WN waves fetch a share of it each, into a place of their own, and do not meet
    constexpr int FT = WN > 1 ? 64 : NT, FC = WN > 1 ? KW : KT;
    const attn_args &a = f.a;
    const attn_plan_view &p = f.p;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wn = WN > 1 ? wave : 0;
    const int ftid = WN > 1 ? lane : tid;
    attn_lds_i32 *s_kpos = (attn_lds_i32 *)((attn_lds *)lds + 4 * KT * tile::kRow) + wn * 2 * FC;    // POS: two places of [FC]
    const int64_t item_no = blockIdx.x / f.groups;
    const int group = blockIdx.x % f.groups;
    const attn_item item(p, item_no);

    const attn_lane me(a, item, f.mode, group, lane, wave, WM);
    const int64_t row = me.row;
    const int head = me.head, kv = me.kv, r = me.r;
    const bool valid = me.valid;
    const bool busy = __builtin_amdgcn_ballot_w64(valid) != 0;
    const float cc = POS ? kLog2e : fabsf(a.c);

    frag q[tile::kSteps];
    tile::load_lane((const T *)a.Q + row * a.ldq + head * a.hdq, a.D, f.vec, valid && item.c1 > item.c0, POS ? 1.f : a.c, q, lane);
    int qp = 0, q_lo = 0, q_hi = 0;
    attn_bias bias = {};
    if (POS) {
        if (a.qpos) { qp = a.qpos[row]; q_lo = attn_wave_min(qp); q_hi = attn_wave_max(qp); }
        if (a.buckets) bias = attn_lane_bias<T>(a, (attn_lds *)lds + 4 * KT * tile::kRow + 2 * KT * 4, f.mode, group, lane, wave, WM);
    }

    attn_f32x16 acc[tile::kBlocks];
#pragma unroll
    for (int x = 0; x < tile::kBlocks; ++x) acc[x] = (attn_f32x16)(0.f);
    float top = -INFINITY, total = 0;

    const int64_t steps = (int64_t)(item.c1 - item.c0 + STEP - 1) / STEP * SUB;
    attn_ring<T, DT, FT, FC, POS> ring;
    ring.lds = (attn_lds *)lds + wn * 4 * FC * tile::kRow;
    ring.ldx = a.ldk; ring.ldy = a.ldv;
    ring.cols = item.cols; ring.x0 = (int64_t)(item.c0 - item.chunk0) * kAttnChunk + wn * FC; ring.step = KT; ring.tid = ftid;
    ring.pos = a.kpos; ring.sign = POS ? a.causal : 0; ring.limit = q_hi;
    ring.D = a.D; ring.vec = f.vec;
    const T *Kh = (const T *)a.K + (int64_t)kv * a.hdk, *Vh = (const T *)a.V + (int64_t)kv * a.hdv;
    if (a.D != DT || ring.sign) ring.zero();
    if (POS && a.causal && WM > 1) {                     // the last position that any row of the block attends to
        if (lane == 0) s_kpos[wave] = q_hi;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WM; ++w) ring.limit = s_kpos[w] > ring.limit ? s_kpos[w] : ring.limit;
    }
    if (POS || a.D != DT) __syncthreads();               // the bias's tables, the zeros
    // this wave's share of a step: columns col0 .. col0 + KW of the step's chunks
    auto my_chunk = [&](int64_t step, int &col0) {
        col0 = (int)(step % SUB) * KT + wn * KW;
        const int chunk = item.c0 + (int)(step / SUB) * STEP + col0 / kAttnChunk;
        return busy && chunk < item.c1 ? chunk : -1;
    };
    // its pairs are asked for before the rows of the same step: a wait for them leaves those on their way
    uint64_t word = 0, word_next = 0;
    int state = 0, state_next = 0;
    auto fetch_pairs = [&](int64_t step) {
        int col0;
        const int chunk = my_chunk(step, col0);
        state_next = 0;
        if (chunk >= 0) { state_next = item.state(p, chunk, r); word_next = item.word(p, chunk, r); }
    };
    if (steps > 0) {
        ring.begin(steps, [](int64_t s) { return s; });
        fetch_pairs(0);
        ring.rows(0, Kh, Vh);
    }
    for (int64_t step = 0; step < steps; ++step) {
        ring.arrive();
        if (POS && ftid < FC) s_kpos[(step & 1) * FC + ftid] = ring.kp_one;
        if (WN == 1) __syncthreads();                    // the step's rows are there, the step before has been computed
        else {                                           // a wave's own rows; LDS is in order for a wave
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
        const bool all = state == 2;

        attn_f32x16 s[TILES];
        float up = top;
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            const attn_lds_i32 *kp = s_kpos + (step & 1) * FC + 32 * t;
            attn_near near = {false, false, false, 0};
            if (POS) {
                const int col = kp[lane & 31];
                near = attn_look(a, attn_distance(col, q_hi), attn_distance(col, q_lo));
                if (near.nothing) {
                    s[t] = (attn_f32x16)(-INFINITY);
                    continue;
                }
            }
            s[t] = tile::scores(sK, 32 * t, q, a.D, lane);
            if (POS) {
                if (a.buckets && !near.far) {
                    attn_add_bias(bias, s[t], a.scale, [&](int x) { return kp[8 * (x >> 2) + 4 * (lane >> 5) + (x & 3)]; }, [&](int) { return qp; });
                } else {
                    const float all_of = a.buckets ? bias.at(near.place) : 0.f;
#pragma unroll
                    for (int x = 0; x < 16; ++x) s[t][x] = __builtin_fmaf(s[t][x], a.scale, all_of);
                }
                if (near.ask) {
#pragma unroll
                    for (int x = 0; x < 16; ++x) s[t][x] = kp[8 * (x >> 2) + 4 * (lane >> 5) + (x & 3)] > qp ? -INFINITY : s[t][x];
                }
            }
            if (!all) {
                const uint32_t bits = (uint32_t)(word >> (32 * t)) >> (4 * (lane >> 5));
#pragma unroll
                for (int x = 0; x < 16; ++x) s[t][x] = bits >> (8 * (x >> 2) + (x & 3)) & 1 ? s[t][x] : -INFINITY;
            }
#pragma unroll
            for (int x = 0; x < 16; ++x) up = fmaxf(up, s[t][x]);
        }
        up = attn_pair_max(up);
        const float base = up == -INFINITY ? 0.f : up;
        if (__builtin_amdgcn_ballot_w64(up != top) != 0) {
            const float old = __builtin_amdgcn_exp2f((top - base) * cc);
            total *= old;
#pragma unroll
            for (int x = 0; x < tile::kBlocks; ++x) acc[x] *= old;
            top = up;
        }
        const float off = -base * cc;
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
#pragma unroll
            for (int x = 0; x < 16; ++x) {
                s[t][x] = __builtin_amdgcn_exp2f(POS ? (s[t][x] - base) * cc : __builtin_fmaf(s[t][x], cc, off));
                total += s[t][x];
            }
            tile::add_rows(acc, sV, 32 * t, s[t], a.D, lane);
        }
    }
    total = attn_pair_sum(total);
    // a row whose sums are not all finite is made again by itself: see attn_row_forward
    float odd = total * 0.f;
#pragma unroll
    for (int x = 0; x < tile::kBlocks; ++x)
#pragma unroll
        for (int k = 0; k < 16; ++k) odd += acc[x][k] * 0.f;
    uint64_t again = __builtin_amdgcn_ballot_w64(valid && !(odd == 0.f));
    if (!POS && top != -INFINITY) top *= fabsf(a.scale);                  // from here on in units of e

    const int64_t place = ((item.part * a.H + head) * p.br + r);          // of a part
    float *stat = f.part_stat + 2 * place;
    T *out = (T *)f.O + row * f.ldo + head * f.hdo;
    if (WN == 1) {
        again |= again >> 32;
        if (valid && !(again >> (lane & 31) & 1)) {
            const float inv = total == 0 ? 0.f : 1.f / total;
            if (lane < 32) {
                if (!item.whole) { stat[0] = top; stat[1] = total; }
                else if (f.lse) f.lse[head * a.m + row] = total == 0 ? -INFINITY : top + __builtin_amdgcn_logf(total) * kLn2;
            }
#pragma unroll
            for (int x = 0; x < tile::kBlocks; ++x)
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const int d = 32 * x + 8 * b + 4 * (lane >> 5);
                    const attn_f32x4 v = {acc[x][4 * b], acc[x][4 * b + 1], acc[x][4 * b + 2], acc[x][4 * b + 3]};
                    if (item.whole) attn_store4(out, d, a.D, f.vec, v * inv);
                    else if (total != 0) attn_store4(f.part + place * f.pd, d, f.pd, true, v);
                }
        }
    } else {
        // the waves' shares of the tile meet in LDS, over K and V
        __syncthreads();
        attn_lds_f32 *sums = (attn_lds_f32 *)(attn_lds *)lds, *stats = sums + WN * 32 * DT;        // [WN][32][DT], numbers exchanged by row; [WN][32][3]
#pragma unroll
        for (int x = 0; x < tile::kBlocks; ++x)
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const int g = (8 * x + 2 * b + (lane >> 5)) ^ (lane & 7);
                *(attn_lds_f32x4 *)(sums + (wn * 32 + (lane & 31)) * DT + 4 * g) = (attn_f32x4){acc[x][4 * b], acc[x][4 * b + 1], acc[x][4 * b + 2], acc[x][4 * b + 3]};
            }
        if (lane < 32) {
            attn_lds_f32 *st = stats + (wn * 32 + lane) * 3;
            st[0] = top; st[1] = total;
            st[2] = (again | again >> 32) >> lane & 1 ? 1.f : 0.f;
        }
        __syncthreads();
        // a row at a time for NT / 32 threads
        constexpr int LANES = NT / 32, EACH = DT / LANES;
        const int mine = tid / LANES, part = tid % LANES;
        float high = -INFINITY, sum = 0, w[WN], bad = 0;
#pragma unroll
        for (int x = 0; x < WN; ++x) { high = fmaxf(high, stats[(x * 32 + mine) * 3]); bad += stats[(x * 32 + mine) * 3 + 2]; }
#pragma unroll
        for (int x = 0; x < WN; ++x) {
            w[x] = attn_weight(stats[(x * 32 + mine) * 3], high == -INFINITY ? 0.f : high);
            sum += stats[(x * 32 + mine) * 3 + 1] * w[x];
        }
        // the row's query and head are those of lane `mine` of any wave
        const int64_t row2 = ((int64_t)__shfl((int)(row >> 32), mine, 64) << 32) | (uint32_t)__shfl((int)row, mine, 64);
        const int head2 = __shfl(head, mine, 64), r2 = __shfl(r, mine, 64);
        const bool valid2 = __shfl((int)valid, mine, 64) != 0;
        const int64_t place2 = (item.part * a.H + head2) * p.br + r2;
        T *out2 = (T *)f.O + row2 * f.ldo + head2 * f.hdo;
        if (valid2 && bad == 0) {
            const float inv = sum == 0 ? 0.f : 1.f / sum;
            if (part == 0) {
                if (!item.whole) { f.part_stat[2 * place2] = high; f.part_stat[2 * place2 + 1] = sum; }
                else if (f.lse) f.lse[head2 * a.m + row2] = sum == 0 ? -INFINITY : high + __builtin_amdgcn_logf(sum) * kLn2;
            }
#pragma unroll
            for (int k = 0; k < EACH; k += 4) {
                const int d = part * EACH + k;
                attn_f32x4 v = (attn_f32x4)(0.f);
#pragma unroll
                for (int x = 0; x < WN; ++x) v += *(attn_lds_f32x4 *)(sums + (x * 32 + mine) * DT + 4 * ((d >> 2) ^ (mine & 7))) * w[x];
                if (item.whole) attn_store4(out2, d, a.D, f.vec, v * inv);
                else if (sum != 0) attn_store4(f.part + place2 * f.pd, d, f.pd, true, v);
            }
        }
        again = 0;
        for (int x = 0; x < 32; ++x) {
            float any = 0;
            for (int y = 0; y < WN; ++y) any += stats[(y * 32 + x) * 3 + 2];
            if (any != 0 && x % WN == wn) again |= (uint64_t)1 << x;
        }
    }
    for (again &= 0xffffffffu; again; again &= again - 1) {
        const int x = __builtin_ctzll(again);
        const int64_t i = ((int64_t)__builtin_amdgcn_readlane((int)(row >> 32), x) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)row, x);
        const int h = __builtin_amdgcn_readlane(head, x), rr = __builtin_amdgcn_readlane(r, x);
        float one[kAttnPer], hi, sum;
        attn_row_forward<T>(a, p, item.block, rr, item.c0, item.c1, i, h, lane, hi, sum, one);
        const int64_t at1 = (item.part * a.H + h) * p.br + rr;
        const float inv = sum == 0 ? 0.f : 1.f / sum;
        if (lane == 0) {
            if (!item.whole) { f.part_stat[2 * at1] = hi; f.part_stat[2 * at1 + 1] = sum; }
            else if (f.lse) f.lse[h * a.m + i] = sum == 0 ? -INFINITY : hi + __builtin_amdgcn_logf(sum) * kLn2;
        }
#pragma unroll
        for (int k = 0; k < kAttnPer; ++k) {
            const int d = lane + 64 * k;
            if (d >= a.D) continue;
            if (item.whole) ((T *)f.O)[i * f.ldo + h * f.hdo + d] = (T)(one[k] * inv);
            else f.part[at1 * f.pd + d] = one[k];
        }
    }
}

// Rows whose columns were cut into several items: a wave for a row and head.  Each part has its maximum and total; the parts' sums are
// weighted to the largest maximum and added in a fixed order.  Parts that have nothing of the row wrote no sums and are left out.
// The grid: blocks that were cut, rows of a block, heads.
template <typename T, int LP>
__global__ __launch_bounds__(256) void join_kernel(forward_args f, int64_t cut)
{
    __shared__ float s_weight[4][64];
    __shared__ int s_part[4][64];
    const attn_args &a = f.a;
    const attn_plan_view &p = f.p;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t x = (int64_t)blockIdx.x * 4 + wave;
    if (x >= cut * p.br * a.H) return;
    const int h = (int)(x % a.H), r = (int)(x / a.H % p.br);
    const int64_t b = p.cut_block[x / a.H / p.br], i = attn_first_row(p.row0, b, p.br, p.m) + r;
    if (i >= attn_first_row(p.row0, b + 1, p.br, p.m)) return;
    const int first = p.item0[b], parts = p.item0[b + 1] - first;
    auto place = [&](int k) { return ((int64_t)(first + k) * a.H + h) * p.br + r; };
    float top = -INFINITY;
    for (int k = lane; k < parts; k += 64) top = fmaxf(top, f.part_stat[2 * place(k)]);
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
    const float base = top == -INFINITY ? 0.f : top;
    float total = 0;
    attn_f32x4 acc = (attn_f32x4)(0.f);
    for (int k0 = 0; k0 < parts; k0 += 64) {
        const int k = k0 + lane;
        const float t = k < parts ? f.part_stat[2 * place(k) + 1] : 0.f;
        const float w = t == 0 ? 0.f : attn_weight(f.part_stat[2 * place(k)], base);
        total += t * w;
        const uint64_t some = __builtin_amdgcn_ballot_w64(t != 0);
        if (t != 0) {
            const int n = __builtin_popcountll(some & (((uint64_t)1 << lane) - 1));
            s_weight[wave][n] = w;
            s_part[wave][n] = k;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");       // the list is this wave's own
        __builtin_amdgcn_wave_barrier();
        acc += attn_add_parts<LP>(__builtin_popcountll(some), f.pd, lane, [&](int n) { return f.part + place(s_part[wave][n]) * f.pd; },
                                  [&](int n) { return s_weight[wave][n]; });
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    total = attn_wave_sum(total);
    const float inv = total == 0 ? 0.f : 1.f / total;
    if (lane < LP) attn_store4((T *)f.O + i * f.ldo + h * f.hdo, 4 * lane, a.D, f.vec, acc * inv);
    if (f.lse && lane == 0) f.lse[h * a.m + i] = total == 0 ? -INFINITY : top + __builtin_amdgcn_logf(total) * kLn2;
}

template <typename T, int DT, int WM, int WN, int KW, bool POS>
sp_status launch(const forward_args &f, const forward_choice &c, int64_t items, hipStream_t st)
{
    constexpr int KT = KW * WN;
    size_t lds = 4 * (size_t)KT * DT * sizeof(T) + (POS ? 2 * KT * 4 + attn_bias_bytes(f.a, c.slots()) : 0);
    const size_t join = WN > 1 ? (size_t)WN * 32 * (DT + 3) * 4 : 0;
    if (join > lds) lds = join;
    auto kernel = forward_kernel<T, DT, WM, WN, KW, POS>;
    if (!attn_launches(items * c.groups, 64 * WM * WN)) return SP_ERR_TOO_LARGE;
    if (lds > 65536) SP_HIP(hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
    hipLaunchKernelGGL(kernel, dim3((unsigned)(items * c.groups)), dim3(64 * WM * WN), lds, st, f);
    SP_HIP(hipGetLastError());
    return SP_OK;
}

template <typename T, int DT, bool POS>
sp_status launch_mode(const forward_args &f, const forward_choice &c, int64_t items, hipStream_t st)
{
    // Waves that share a tile's columns have two places for their rows each.  Four of them, or two where four would not fit the LDS, or
    // where two let five workgroups onto a compute unit instead of two (64 rows of 800 to 1500 columns, 16 heads of 64: 73 -> 70 us; 4096
    // rows of 96 scattered ones: 94 -> 86; with positions to be looked at it is the other way round, 32 -> 49 for caches of 1024).
    constexpr int row = DT * (int)sizeof(T);
    if (c.wn > 1) return launch<T, DT, 1, (row == 512 || (row == 128 && !POS) ? 2 : 4), 32, POS>(f, c, items, st);
    return launch<T, DT, 4, 1, (DT * (int)sizeof(T) <= 256 ? 64 : 32), POS>(f, c, items, st);
}

}  // namespace

template <typename T>
sp_status attn_forward(const sp_attn_plan *plan, forward_args &f, const forward_choice &c, hipStream_t st)
{
    // scale 0 goes with the positions: products of q and k by themselves would be scaled by zero after the mask's infinities
    const bool pos = f.a.buckets || f.a.causal || f.a.scale == 0;
    const int64_t items = plan->items[c.level];
#define SPMI_FORWARD(DT)                                                                                                          \
    do {                                                                                                                          \
        if (pos) SP_TRY((launch_mode<T, DT, true>(f, c, items, st)));                                                             \
        else SP_TRY((launch_mode<T, DT, false>(f, c, items, st)));                                                                \
        if (c.cut) hipLaunchKernelGGL((join_kernel<T, DT / 4>), dim3((unsigned)ceil_div(plan->cut[c.level] * plan->br * f.a.H, 4)), dim3(256), 0, st, f, plan->cut[c.level]); \
    } while (0)
    if (f.a.D <= 32) SPMI_FORWARD(32);
    else if (f.a.D <= 64) SPMI_FORWARD(64);
    else if (f.a.D <= 128) SPMI_FORWARD(128);
    else if constexpr (sizeof(T) == 2) SPMI_FORWARD(256);
    else return SP_ERR_SHAPE;
#undef SPMI_FORWARD
    SP_HIP(hipGetLastError());
    return SP_OK;
}
