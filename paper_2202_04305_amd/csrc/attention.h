// Shared by the sources of attention over a stored pattern (attention_plan.hip, attention.hip, attention_forward_*.hip, attention_backward_*.hip).
#pragma once
#include "spmi_internal.h"

constexpr int kAttnChunk = 64;           // columns of a chunk: one 64-bit word of pairs for each row of a block
constexpr int kAttnLevels = 28;

// What sp_prepare_attention makes of a pattern (or of its transpose, where rows are keys and columns are queries).  Rows are
// taken in blocks of at most `br`, which end where neighbouring rows' columns lie apart (the sequences of a batch) if that takes hardly
// more chunks than blocks of `br` throughout; a block's distinct columns, ascending, are cut into chunks of 64.  br = 1: a block is a row and its
// columns are its stretch of crd, no bits are needed.
//
// A block of many rows reads a row of K and V once for all of them, and is worth it where neighbouring rows store mostly the same
// columns (bands, sequences, shared prefixes); a row by itself where they do not.
struct attn_stretch {                    // what a workgroup has to know of its item, in one load
    int32_t block, chunk0;               // the block and its first chunk
    int32_t c0, c1;                      // the item's chunks
    int32_t first, count;                // the block's columns: place of the first one in cols (br = 1: in crd), how many places
    int32_t row0;                        // the block's first row
    int32_t rows_whole;                  // 2 * its number of rows + 1 where it is the block's only item
};

struct sp_attn_plan {
    int br;
    int64_t m, n;                        // rows and columns as this plan sees them
    int64_t nblocks, nchunks, max_chunks;
    int32_t *rowptr;                     // DEVICE [m + 1]
    int32_t *row0;                       // DEVICE [nblocks + 1]: first row of every block; null: b * br
    const int32_t *crd;                  // DEVICE [entries], rows ascending, columns ascending within
    int32_t *crd_own;                    // the same where the plan had to make it
    int32_t *chunk0;                     // DEVICE [nblocks + 1]: first chunk of every block
    int32_t *cols;                       // DEVICE [nchunks * 64]; behind a block's last column: that column again, without pairs
    uint64_t *bits;                      // DEVICE [nchunks * br]: bit c of word r of a chunk: row r of the block stores column c
    uint8_t *state;                      // DEVICE [nchunks * br / 32]: of the 32 rows' pairs of a chunk 0 = none, 1 = some, 2 = all are stored
    // Work items: a block's chunks in stretches of at most attn_level_chunks(level) of them (a block without any is one item).
    // The last level's items are the blocks.
    int levels;
    int64_t items[kAttnLevels];
    int32_t *item0[kAttnLevels];         // DEVICE [nblocks + 1]: first item of every block
    attn_stretch *item[kAttnLevels];     // DEVICE [items]
    int64_t cut[kAttnLevels];            // blocks of several items,
    int32_t *cut_block[kAttnLevels];     // DEVICE [cut]: ascending
    size_t bytes;
};

static inline __host__ __device__ int attn_level_chunks(int level) { return 1 << level; }
// A launch has fewer than 2^32 threads along a direction.
static inline bool attn_launches(int64_t groups, int threads) { return groups < ((int64_t)1 << 31) && groups * threads < ((int64_t)1 << 32); }

// A plan at one level, as kernels take it.
struct attn_plan_view {
    const int32_t *rowptr, *crd, *chunk0, *cols, *item0, *row0;
    const attn_stretch *item;
    const int32_t *cut_block;
    const uint64_t *bits;
    const uint8_t *state;
    int64_t m, n;
    int br;
};
static inline attn_plan_view attn_view(const sp_attn_plan *p, int level)
{
    return {p->rowptr, p->crd, p->chunk0, p->cols, p->item0[level], p->row0, p->item[level], p->cut_block[level], p->bits, p->state, p->m, p->n, p->br};
}

// The problem as kernels take it.
struct attn_args {
    const void *Q, *K, *V;
    int64_t ldq, hdq, ldk, hdk, ldv, hdv, ldt;
    const int32_t *qpos, *kpos;
    const void *table;
    int64_t m, n;                        // queries, keys
    int D, H, Hk, G;                     // G = H / Hk
    float scale, c;                      // c = scale * log2(e)
    int buckets, side, exact, borders, last, bidirectional, causal;
    int16_t border[64];                  // far bucket k begins at distance border[k - 1]; distances from `last` on share a bucket
};

// How finely the blocks are cut.  With `groups` workgroups an item, `chunk_us` for a chunk of one, `item_us` to begin and end one (the
// loads that depend on each other before the first rows arrive) and `row_bytes` for a part of one row of one item (written and read
// again in f32), the level with the least of: what one of 512 places for a workgroup (two on each compute unit) gets of the work,
// plus the longest item, plus the parts' traffic and the launch that joins them.
static inline double attn_level_us(const sp_attn_plan *p, int level, int64_t groups, double chunk_us, double item_us, double row_bytes)
{
    const double longest = p->max_chunks < attn_level_chunks(level) ? (double)p->max_chunks : (double)attn_level_chunks(level);
    const double extra = p->cut[level] ? 5 + (double)(p->items[level] - p->nblocks + p->cut[level]) * row_bytes * p->br * 2 / 4e6 : 0;
    return (double)groups / 512 * (chunk_us * (double)p->nchunks + item_us * (double)p->items[level]) + chunk_us * longest + extra;
}
static inline int attn_pick_level(const sp_attn_plan *p, int64_t groups, double chunk_us, double item_us, double row_bytes)
{
    int best = p->levels - 1;
    for (int l = p->levels - 2; l >= 0; --l)
        if (attn_level_us(p, l, groups, chunk_us, item_us, row_bytes) < attn_level_us(p, best, groups, chunk_us, item_us, row_bytes)) best = l;
    return best;
}

// ---- device -----------------------------------------------------------------------------------------------------------------
typedef __bf16 attn_bf16;
typedef _Float16 attn_f16;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ int attn_distance(int kp, int qp) { return __builtin_elementwise_sub_sat(kp, qp); }

// The bucket of a distance r = key's position - query's, by the problem's borders.
__device__ __forceinline__ int attn_bucket(const attn_args &a, int r)
{
    int base = 0, d;
    if (a.bidirectional) {
        base = r > 0 ? a.side : 0;
        d = r < 0 ? (r == INT32_MIN ? INT32_MAX : -r) : r;
    } else d = r < 0 ? (r == INT32_MIN ? INT32_MAX : -r) : 0;
    if (d < a.exact) return base + d;
    int b = a.exact;
    for (int k = 0; k < a.borders; ++k) b += d >= a.border[k] ? 1 : 0;
    return base + b;
}

// Kernels number the buckets without the one that no distance has: of two directions, distance 0 on the upper half.  (That leaves two
// workgroups on a compute unit for the gradient of 32 buckets, head size 64.)
__host__ __device__ __forceinline__ int attn_places(const attn_args &a) { return a.buckets - a.bidirectional; }
__device__ __forceinline__ int attn_place_of(const attn_args &a, int bucket) { return bucket - (a.bidirectional && bucket > a.side ? 1 : 0); }
__device__ __forceinline__ int attn_bucket_of(const attn_args &a, int place) { return place + (a.bidirectional && place >= a.side ? 1 : 0); }
// The place of all distances from the last border on, ahead of the query or behind it.
__device__ __forceinline__ int attn_far_place(const attn_args &a, bool ahead)
{
    return ahead ? (a.bidirectional ? 2 * a.side - 2 : 0) : a.side - 1;
}

// Block b's first row and the one behind its last.
__host__ __device__ __forceinline__ int64_t attn_first_row(const int32_t *row0, int64_t b, int br, int64_t m)
{
    const int64_t x = row0 ? (int64_t)row0[b] : b * br;
    return x < m ? x : m;
}

// Calls f(column) for every column that row r of block b stores in the block's chunks [c0, c1), until it returns false; for a whole
// wave, f's argument and answer uniform.
template <typename F>
__device__ __forceinline__ void attn_for_columns(const attn_plan_view &p, int64_t b, int r, int c0, int c1, F f)
{
    if (p.br == 1) {
        const int64_t s = p.rowptr[b], e = p.rowptr[b + 1], first = p.chunk0[b];
        const int64_t lo = s + (c0 - first) * kAttnChunk, hi = s + (c1 - first) * kAttnChunk;
        for (int64_t x = lo; x < (hi < e ? hi : e); ++x) if (!f(p.crd[x])) return;
        return;
    }
    for (int c = c0; c < c1; ++c) {
        const uint64_t w = p.bits[(int64_t)c * p.br + r];
        uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)w), hi = __builtin_amdgcn_readfirstlane((uint32_t)(w >> 32));
        for (uint64_t left = ((uint64_t)hi << 32) | lo; left; left &= left - 1)
            if (!f(p.cols[(int64_t)c * kAttnChunk + __builtin_ctzll(left)])) return;
    }
}

__device__ __forceinline__ float attn_wave_sum(float v)
{
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d, 64);
    return v;
}

// One row by itself, a wave per row and head, lanes across the head's numbers (d = lane, lane + 64, ...): every pair is looked at
// alone, so nothing that a row does not attend to can reach it.  The kernels that take 32 rows at a time fall back on these where a
// result is not finite: there a number that other rows attend to is multiplied with zero, which infinities and NaN survive.
constexpr int kAttnPer = 4;              // numbers of a lane: head sizes up to 256

template <typename T>
__device__ __forceinline__ void attn_load_row(const T *row, int D, int lane, float (&x)[kAttnPer])
{
#pragma unroll
    for (int k = 0; k < kAttnPer; ++k) x[k] = lane + 64 * k < D ? (float)row[lane + 64 * k] : 0.f;
}
__device__ __forceinline__ float attn_dot(const float (&x)[kAttnPer], const float (&y)[kAttnPer])
{
    float s = 0;
#pragma unroll
    for (int k = 0; k < kAttnPer; ++k) s += x[k] * y[k];
    return attn_wave_sum(s);
}
// The score.  (In units of e, not of 2: a bias of the type's lowest value must stay a number, so that a row of nothing else is one.)
template <typename T>
__device__ __forceinline__ float attn_score(const attn_args &a, float dot, int64_t i, int64_t j, int h)
{
    float s = dot * a.scale;
    if (a.buckets) s += (float)((const T *)a.table)[(int64_t)attn_bucket(a, attn_distance(a.kpos[j], a.qpos[i])) * a.ldt + h];
    return s;
}
__device__ __forceinline__ float attn_weight(float s, float top) { return __builtin_amdgcn_exp2f((s - top) * kLog2e); }
// The same in the gradients, where log_sum is log2 of what the row's weights e^(s - lse) sum to (see attn_log_sum).  That is of the tiles' scores;
// one that is made pair by pair may round to another step, and its weight stays at 1 then.
__device__ __forceinline__ float attn_weight(float s, float lse, float log_sum)
{
    const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s - lse, kLog2e, -log_sum));
    return log_sum != 0 && w > 1.f ? 1.f : w;
}
__device__ __forceinline__ bool attn_left_out(const attn_args &a, int64_t i, int64_t j) { return a.causal && a.kpos[j] > a.qpos[i]; }

// Is any of a row's D sums still a number?  (What is not a number stays so, and a row of nothing else is done.)
__device__ __forceinline__ bool attn_any_number(const float (&x)[kAttnPer], int D, int lane)
{
    bool any = false;
#pragma unroll
    for (int k = 0; k < kAttnPer; ++k) any = any || (lane + 64 * k < D && x[k] == x[k]);
    return __builtin_amdgcn_ballot_w64(any) != 0;
}

// top (running maximum), total and acc = sum of e^(s - top) V over a stretch of a row's columns.  Values that are not numbers spoil acc
// alone: top and total (lse) go on to the row's end, as the gradients of the row's other keys are weighted by them.
template <typename T>
__device__ __forceinline__ void attn_row_forward(const attn_args &a, const attn_plan_view &p, int64_t b, int r, int c0, int c1, int64_t i, int h,
                                                 int lane, float &top, float &total, float (&acc)[kAttnPer])
{
    const int g = h / a.G;
    float q[kAttnPer];
    attn_load_row((const T *)a.Q + i * a.ldq + h * a.hdq, a.D, lane, q);
    top = -INFINITY; total = 0;
    bool sums = true;                                    // is any of acc still a number?
#pragma unroll
    for (int k = 0; k < kAttnPer; ++k) acc[k] = 0;
    attn_for_columns(p, b, r, c0, c1, [&](int64_t j) {
        if (attn_left_out(a, i, j)) return true;
        float x[kAttnPer];
        attn_load_row((const T *)a.K + j * a.ldk + g * a.hdk, a.D, lane, x);
        const float s = attn_score<T>(a, attn_dot(q, x), i, j, h);
        if (s == -INFINITY) return true;                 // weight 0
        if (sums) attn_load_row((const T *)a.V + j * a.ldv + g * a.hdv, a.D, lane, x);
        const float up = s > top ? s : top;              // not a number: stays with the old maximum, the weight carries it
        const float old = top == -INFINITY ? 0.f : attn_weight(top, up), w = attn_weight(s, up == -INFINITY ? 0.f : up);
        top = up;
        total = total * old + w;
        if (sums) {
#pragma unroll
            for (int k = 0; k < kAttnPer; ++k) acc[k] = acc[k] * old + w * x[k];
            sums = attn_any_number(acc, a.D, lane);
        }
        return sums || total == total;
    });
}

// sum over the stretch of ds K (not yet scaled)
template <typename T>
__device__ __forceinline__ void attn_row_dq(const attn_args &a, const attn_plan_view &p, int64_t b, int r, int c0, int c1, int64_t i, int h, int lane,
                                            const T *dO, float lse, float delta, float log_sum, float (&acc)[kAttnPer])
{
    const int g = h / a.G;
    float q[kAttnPer], go[kAttnPer];
    attn_load_row((const T *)a.Q + i * a.ldq + h * a.hdq, a.D, lane, q);
    attn_load_row(dO, a.D, lane, go);
#pragma unroll
    for (int k = 0; k < kAttnPer; ++k) acc[k] = 0;
    if (lse == -INFINITY) lse = INFINITY;                // no weight left
    attn_for_columns(p, b, r, c0, c1, [&](int64_t j) {
        if (attn_left_out(a, i, j)) return true;
        float x[kAttnPer], y[kAttnPer];
        attn_load_row((const T *)a.K + j * a.ldk + g * a.hdk, a.D, lane, x);
        attn_load_row((const T *)a.V + j * a.ldv + g * a.hdv, a.D, lane, y);
        const float s = attn_score<T>(a, attn_dot(q, x), i, j, h);
        if (s == -INFINITY) return true;
        const float ds = attn_weight(s, lse, log_sum) * (attn_dot(go, y) - delta);
#pragma unroll
        for (int k = 0; k < kAttnPer; ++k) acc[k] += ds * x[k];
        return attn_any_number(acc, a.D, lane);
    });
}

// sums over a stretch of a key's queries, for one head h of the key's group: dk += ds Q (not yet scaled), dv += p dO.
// p: the plan of the transposed pattern
template <typename T>
__device__ __forceinline__ void attn_row_dkv(const attn_args &a, const attn_plan_view &p, int64_t b, int r, int c0, int c1, int64_t j, int h, int lane,
                                             const T *dO, int64_t lddo, int64_t hddo, const float *lse, const float *delta, const float *log_sum,
                                             float (&dk)[kAttnPer], float (&dv)[kAttnPer])
{
    const int g = h / a.G;
    float kx[kAttnPer], vx[kAttnPer];
    attn_load_row((const T *)a.K + j * a.ldk + g * a.hdk, a.D, lane, kx);
    attn_load_row((const T *)a.V + j * a.ldv + g * a.hdv, a.D, lane, vx);
    attn_for_columns(p, b, r, c0, c1, [&](int64_t i) {
        if (attn_left_out(a, i, j)) return true;
        float x[kAttnPer], y[kAttnPer];
        attn_load_row((const T *)a.Q + i * a.ldq + h * a.hdq, a.D, lane, x);
        attn_load_row(dO + i * lddo + h * hddo, a.D, lane, y);
        const float s = attn_score<T>(a, attn_dot(kx, x), i, j, h);
        if (s == -INFINITY) return true;
        const float L = lse[h * a.m + i];
        const float w = attn_weight(s, L == -INFINITY ? INFINITY : L, log_sum ? log_sum[h * a.m + i] : 0.f);
        const float ds = w * (attn_dot(vx, y) - delta[h * a.m + i]);
#pragma unroll
        for (int k = 0; k < kAttnPer; ++k) { dk[k] += ds * x[k]; dv[k] += w * y[k]; }
        return attn_any_number(dk, a.D, lane) || attn_any_number(dv, a.D, lane);
    });
}
