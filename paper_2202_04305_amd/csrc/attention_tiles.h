// Tiles of 32 x 32 scores on the matrix cores, for attention_forward.h and attention_backward.h.
//
// Every product is laid out so that the 32 rows that a wave works for (queries; keys in the gradients of K and V) are the lanes:
// the transposed scores S^T = K Q^T come out with row lane % 32 of the wave in each lane, and 16 of the 32 columns in its registers
// (column 8 b + 4 (lane / 32) + c in register 4 b + c).  Maxima, sums, masks and scale factors of a row are then private to a lane
// and its partner 32 lanes on, and the weights are, register by register, what the next product O^T = V^T P^T takes as its second
// operand: a matrix instruction sums over 8 numbers of each half wave, in any order that both operands agree on, so registers 0-7
// are the operand of the first 16 columns and 8-15 of the last 16.  V^T needs the columns' numbers transposed, which the LDS does
// on reading (ds_read_b64_tr_b16; plain 4-byte reads for f32).
//
// A tile of dense rows lies in LDS in granules of 16 bytes, granule g of row r at place g ^ attn_swizzle(r).  The exchange keeps
// both readers off each other's banks: 16 consecutive rows at one granule (first operand), and 4 consecutive rows at 4 granules
// (transposed).
#pragma once
#include "attention.h"

typedef float attn_f32x16 __attribute__((ext_vector_type(16)));
typedef float attn_f32x4 __attribute__((ext_vector_type(4)));
typedef short attn_s16x4 __attribute__((ext_vector_type(4)));
// Pointers into LDS say so: through a generic pointer every access would be a flat one, which waits for memory too.
typedef __attribute__((address_space(3))) char attn_lds;
typedef __attribute__((address_space(3))) float attn_lds_f32;
typedef __attribute__((address_space(3))) attn_f32x4 attn_lds_f32x4;
typedef __attribute__((address_space(3))) int attn_lds_i32;
typedef __attribute__((address_space(3))) uint8_t attn_lds_u8;

template <typename T> struct attn_mma;
template <> struct attn_mma<attn_bf16> {
    typedef attn_bf16 frag __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ attn_f32x16 mul(frag a, frag b, attn_f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <> struct attn_mma<attn_f16> {
    typedef attn_f16 frag __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ attn_f32x16 mul(frag a, frag b, attn_f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};
template <> struct attn_mma<float> {
    typedef attn_f32x4 frag;
    static __device__ __forceinline__ attn_f32x16 mul(frag a, frag b, attn_f32x16 c)
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[k], b[k], c, 0, 0, 0);
        return c;
    }
};

// What a tile of rows of DT numbers (the head size rounded up) looks like in LDS.
template <typename T, int DT>
struct attn_tile {
    typedef typename attn_mma<T>::frag frag;
    static constexpr int kRow = DT * (int)sizeof(T);     // bytes of a row
    static constexpr int kGranules = kRow / 16;
    static constexpr int kPer = 16 / (int)sizeof(T);     // numbers of a granule
    static constexpr int kSteps = kGranules / 2;         // products a score is summed up in: 2 granules each, one for each half wave
    static constexpr int kBlocks = DT / 32;              // blocks of 32 numbers of a transposed product

    static __device__ __forceinline__ int swizzle(int r)
    {
        if (sizeof(T) == 4) return kGranules >= 16 ? (r & 3) | ((r >> 2) & 1) << 3 | ((r >> 3) & 1) << 2 : (r >> 1) & 7;
        return kGranules >= 16 ? (r & 3) << 2 | ((r >> 2) & 3) : kGranules == 8 ? ((r >> 1) & 1) << 2 | ((r >> 2) & 3) : (r >> 2) & 3;
    }
    static __device__ __forceinline__ int place(int r, int g) { return r * kRow + ((g ^ swizzle(r)) << 4); }

    // Addresses are one number of a lane, exchanged by a constant for every read (a step, a block of numbers), plus a constant: the
    // exchange only touches bits within a row, and tiles begin at multiples of a row.
    template <typename V>
    static __device__ __forceinline__ V read(unsigned at) { return *(const __attribute__((address_space(3))) V *)(uintptr_t)at; }

    // f32, whose products are slow, does without those of a row's last quarter where the head ends before it.
    static constexpr int kQuarter = sizeof(T) == 4 ? DT / 4 * 3 : 0;

    // acc (32 rows x 32 lanes) = the tile's rows row0 ... (a multiple of 32) times the lanes' rows `b`
    static __device__ __forceinline__ attn_f32x16 scores(const attn_lds *t, int row0, const frag (&b)[kSteps], int D, int lane)
    {
        const unsigned base = (unsigned)(uintptr_t)t + (unsigned)place(lane & 31, lane >> 5);
        attn_f32x16 acc = (attn_f32x16)(0.f);
#pragma unroll
        for (int s = 0; s < kSteps - kSteps / 4; ++s) acc = attn_mma<T>::mul(read<frag>((base ^ (unsigned)(s << 5)) + row0 * kRow), b[s], acc);
        if (sizeof(T) == 2 || D > kQuarter) {
#pragma unroll
            for (int s = kSteps - kSteps / 4; s < kSteps; ++s) acc = attn_mma<T>::mul(read<frag>((base ^ (unsigned)(s << 5)) + row0 * kRow), b[s], acc);
        }
        return acc;
    }
    // acc[x] (numbers 32 x ... of a head, 32 lanes) += sum over the tile's 32 rows from row0 on of row[number] * w[row of the lane]
    static __device__ __forceinline__ void add_rows(attn_f32x16 (&acc)[kBlocks], const attn_lds *t, int row0, const attn_f32x16 &w, int D, int lane)
    {
        const int half = lane >> 5;
        if constexpr (sizeof(T) == 4) {
            const unsigned base = (unsigned)(uintptr_t)t + (unsigned)(place(4 * half, (lane & 31) >> 2) + (lane & 3) * 4);
            constexpr int kFirst = kBlocks - kBlocks / 4;        // blocks that are not of the last quarter
            auto block = [&](int x) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int row = 8 * (r >> 2) + (r & 3);      // and 4 for the upper half
                    acc[x] = __builtin_amdgcn_mfma_f32_32x32x2f32(read<float>((base ^ (unsigned)((x * 8 ^ swizzle(row)) << 4)) + (row0 + row) * kRow), w[r], acc[x], 0, 0, 0);
                }
            };
#pragma unroll
            for (int x = 0; x < kFirst; ++x) block(x);
            if (kFirst < kBlocks && D > kQuarter) {
#pragma unroll
                for (int x = kFirst; x < kBlocks; ++x) block(x);
            }
        } else {
            const unsigned base = (unsigned)(uintptr_t)t + (unsigned)(place(4 * half + ((lane & 15) >> 2), 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) + (lane & 1) * 8);
            frag p[2];
#pragma unroll
            for (int k = 0; k < 16; ++k) p[k >> 3][k & 7] = (T)w[k];
            auto block = [&](int x, int u) {
                union { attn_s16x4 q[2]; frag f; } v;
#pragma unroll
                for (int k = 0; k < 2; ++k)              // rows 16 u + 8 k on, whose swizzle is that of the first ones exchanged by 2 k
                    v.q[k] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) attn_s16x4 *)(uintptr_t)(
                        (base ^ (unsigned)((4 * x ^ 2 * k) << 4)) + (row0 + 16 * u + 8 * k) * kRow));
                acc[x] = attn_mma<T>::mul(v.f, p[u], acc[x]);
            };
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int x = 0; x < kBlocks; ++x) block(x, u);
        }
    }
    // one lane's row as the second operand: numbers past D are zero
    static __device__ __forceinline__ void load_lane(const T *row, int D, bool vec, bool valid, float sign, frag (&b)[kSteps], int lane)
    {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            b[s] = granule(row, (2 * s + (lane >> 5)) * kPer, D, vec, valid);
            if (sign < 0) b[s] = -b[s];
        }
    }
    // numbers d .. d + kPer - 1 of a row.  vec: rows are 16-byte aligned and D is a multiple of kPer
    static __device__ __forceinline__ frag granule(const T *row, int d, int D, bool vec, bool valid)
    {
        frag f;
        if (vec) {
            if (valid && d < D) f = *(const frag *)(row + d);
            else f = (frag)((T)0.f);
        } else {
#pragma unroll
            for (int k = 0; k < kPer; ++k) f[k] = valid && d + k < D ? row[d + k] : (T)0.f;
        }
        return f;
    }
};

// The larger of a lane's value and its partner's 32 lanes on; their sum.
__device__ __forceinline__ float attn_pair_max(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    const unsigned lo = r[0], hi = r[1];
    return fmaxf(__uint_as_float(lo), __uint_as_float(hi));
}
__device__ __forceinline__ float attn_pair_sum(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    const unsigned lo = r[0], hi = r[1];
    return __uint_as_float(lo) + __uint_as_float(hi);
}

// Where a work item's columns come from: a plan's list of a block, or a row's stretch of crd.
struct attn_columns {
    const int32_t *at;
    int64_t last;                        // the last one's place; behind it: that one again
    __device__ __forceinline__ int32_t get(int64_t x) const { return at[x < last ? x : last]; }
};

struct attn_item {
    int64_t block;
    int chunk0, c0, c1;                  // the block's first chunk, the item's chunks
    int64_t part;                        // number among all items
    bool whole;                          // the block's only item
    int64_t row0;                        // the block's first row
    int rows;                            // and how many it has
    attn_columns cols;
    int64_t count;                       // places of the block's columns; br = 1: columns of the row

    __device__ __forceinline__ attn_item(const attn_plan_view &p, int64_t item)
    {
        const attn_stretch x = p.item[item];
        part = item;
        block = x.block; chunk0 = x.chunk0; c0 = x.c0; c1 = x.c1;
        whole = x.rows_whole & 1;
        row0 = x.row0; rows = x.rows_whole >> 1;
        count = x.count;
        cols = {(p.br == 1 ? p.crd : p.cols) + x.first, count - 1};
    }
    // the pairs of chunk c and row r of the block, and whether the 32 rows around r have none (0), some (1) or all (2) of them
    __device__ __forceinline__ uint64_t word(const attn_plan_view &p, int c, int r) const
    {
        if (p.br != 1) return p.bits[(int64_t)c * p.br + r];
        const int64_t left = count - (int64_t)(c - chunk0) * kAttnChunk;
        return left >= kAttnChunk ? ~(uint64_t)0 : ((uint64_t)1 << left) - 1;
    }
    __device__ __forceinline__ int state(const attn_plan_view &p, int c, int r) const
    {
        if (p.br != 1) return p.state[(int64_t)c * (p.br >> 5) + (r >> 5)];
        return count - (int64_t)(c - chunk0) * kAttnChunk >= kAttnChunk ? 2 : 1;
    }
};

// The rows of two operands (K and V; Q and dO) on their way from memory into LDS (global_load_lds): no registers hold them, and a step's
// rows arrive while the step before is computed from the other of two places.  (Through registers, 16 sequences of up to 1024 queries over
// 4096 keys, 16 heads of 128: 600 us instead of 419.)  A wave's instruction fills 64 consecutive granules of LDS, so the granules' exchange
// (attn_tile::place) is made by which granule of memory each lane asks for.  Rows that nobody attends to and numbers past D are
// left out; the place was zeroed once.  Inline assembly, because for the compiler's own form of this load every later read of LDS waits
// for it; it has no destination register, and arrive() waits for it before anybody reads.  The place in LDS is an operand in m0, which the
// compiler so knows the contents of (a write to m0 that the assembly only lists as clobbered need not be preserved); the load may
// follow a write to m0 after one cycle at the earliest.
__device__ __forceinline__ void attn_to_lds(const void *from, unsigned to)
{
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "{m0}"(to), "v"(from) : "memory");
}
// CAUSAL rows that nobody attends to are not read either, so that what lies in a cache's free places does not matter.  ONE: keep each
// step's columns, one a thread (for positions, and what else belongs to a column).
template <typename T, int DT, int NT, int KT, bool POS, bool ONE = POS>
struct attn_ring {
    typedef attn_tile<T, DT> tile;
    typedef typename tile::frag frag;
    static constexpr int kPieces = KT * tile::kGranules / NT, kRowStep = NT / tile::kGranules, kBytes = KT * tile::kRow;
    static_assert(KT * tile::kGranules % NT == 0 && NT % tile::kGranules == 0 && KT <= NT, "every thread fetches the same number of granules");
    attn_lds *lds;                       // two places of X and Y each
    int64_t ldx, ldy;                    // numbers from row to row
    attn_columns cols;
    int64_t x0;                          // the item's first column among its block's
    const int32_t *pos;                  // positions of the columns, or null
    int limit, sign;                     // causal: rows are needed where sign * pos <= sign * limit; sign 0: everywhere
    int D, step, tid;                    // step: columns from one step to the next; tid: among the NT threads that fetch together
    bool vec;
    int32_t next[kPieces], one_next;     // columns on their way
    int32_t soon[kPieces], one_soon;     // POS: columns that are there, whose positions are on their way
    int32_t at[kPieces], one;            // columns of the rows to be fetched next
    int32_t kp_soon[kPieces], kp_one_soon, kp[kPieces], kp_one;

    __device__ __forceinline__ attn_lds *x_of(int64_t s) const { return lds + (s & 1) * (2 * kBytes); }
    __device__ __forceinline__ attn_lds *y_of(int64_t s) const { return x_of(s) + kBytes; }
    __device__ __forceinline__ int row(int k) const { return tid / tile::kGranules + k * kRowStep; }
    __device__ __forceinline__ void zero()
    {
        for (int x = tid; x < 4 * kBytes / 16; x += NT) *(__attribute__((address_space(3))) attn_f32x4 *)(lds + x * 16) = (attn_f32x4)(0.f);
    }
    __device__ __forceinline__ void columns(int64_t s)
    {
#pragma unroll
        for (int k = 0; k < kPieces; ++k) next[k] = cols.get(x0 + s * step + row(k));
        if (ONE) one_next = cols.get(x0 + s * step + (tid < KT ? tid : 0));
    }
    // moves the columns up a place: next -> soon (POS: their positions are asked for) -> at
    __device__ __forceinline__ void advance()
    {
        if constexpr (POS) {
#pragma unroll
            for (int k = 0; k < kPieces; ++k) { at[k] = soon[k]; kp[k] = kp_soon[k]; soon[k] = next[k]; }
            one = one_soon; kp_one = kp_one_soon; one_soon = one_next;
            if (pos) {
                kp_one_soon = pos[one_soon];
                if (sign != 0) {
#pragma unroll
                    for (int k = 0; k < kPieces; ++k) kp_soon[k] = pos[soon[k]];
                }
            }
        } else {
#pragma unroll
            for (int k = 0; k < kPieces; ++k) at[k] = next[k];
            if (ONE) one = one_next;
        }
    }
    // step_at(s): the place of step s among the columns' steps
    template <typename F>
    __device__ __forceinline__ void begin(int64_t steps, F step_at)
    {
#pragma unroll
        for (int k = 0; k < kPieces; ++k) soon[k] = kp_soon[k] = 0;
        one_soon = kp_one_soon = 0;
        columns(step_at(0));
        advance();
        if (POS) {
            if (steps > 1) columns(step_at(1));
            advance();
            if (steps > 2) columns(step_at(2));
        } else if (steps > 1) columns(step_at(1));
    }
    static constexpr int kAhead = POS ? 3 : 2;           // columns(s + kAhead) is asked for when the rows of s + 1 are
    __device__ __forceinline__ void rows(int64_t s, const T *X, const T *Y)
    {
        const unsigned to = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)x_of(s) + (unsigned)tid / 64 * 1024);
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {
            const int g = (tid % tile::kGranules) ^ tile::swizzle(row(k));
            const bool need = !POS || sign == 0 || (sign > 0 ? kp[k] <= limit : kp[k] >= limit);
            const T *x = X + ((int64_t)at[k] * ldx + g * tile::kPer), *y = Y + ((int64_t)at[k] * ldy + g * tile::kPer);
            if (vec) {
                if (need && g * tile::kPer < D) {
                    attn_to_lds(x, to + k * (NT * 16));
                    attn_to_lds(y, to + k * (NT * 16) + kBytes);
                }
            } else if (need) {
                attn_lds *place = x_of(s) + (k * NT + tid) * 16;
                *(__attribute__((address_space(3))) frag *)place = tile::granule(x - g * tile::kPer, g * tile::kPer, D, false, true);
                *(__attribute__((address_space(3))) frag *)(place + kBytes) = tile::granule(y - g * tile::kPer, g * tile::kPer, D, false, true);
            }
        }
    }
    // this thread's rows have arrived (the others': after a barrier)
    static __device__ __forceinline__ void arrive() { asm volatile("s_waitcnt vmcnt(0)" : : : "memory"); }
};

// Positions of a tile's 32 columns against those of the wave's rows.  A tile that lies wholly past the last border on one side has one
// bias for each head.
struct attn_near {
    bool nothing, ask, far;              // causal leaves nothing / something out; all distances share a bucket
    int place;                           // its place
};
// col: this lane's column's position (lane % 32).  lo, hi: the least and largest distance that the wave's rows give it; a: borders
__device__ __forceinline__ attn_near attn_look(const attn_args &a, int lo, int hi)
{
    attn_near n = {false, false, false, 0};
    if (a.causal) {
        n.ask = __builtin_amdgcn_ballot_w64(hi > 0) != 0;
        n.nothing = n.ask && __builtin_amdgcn_ballot_w64(lo <= 0) == 0;
    }
    if (a.buckets) {
        const bool ahead = __builtin_amdgcn_ballot_w64(lo < a.last) == 0, behind = __builtin_amdgcn_ballot_w64(hi > -a.last) == 0;
        n.far = ahead || behind;
        n.place = attn_far_place(a, ahead);
    }
    return n;
}
__device__ __forceinline__ int attn_wave_min(int v)
{
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) { const int o = __shfl_xor(v, d, 64); v = o < v ? o : v; }
    return v;
}
__device__ __forceinline__ int attn_wave_max(int v)
{
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) { const int o = __shfl_xor(v, d, 64); v = o > v ? o : v; }
    return v;
}

// The position bias in LDS: the place of every distance's bucket up to the last border, and the table's columns of the heads at hand (a
// slot each, 1 << shift of them).  (The bias of every distance instead, one read less, made no difference.)
struct attn_bias {
    const attn_lds_u8 *lut;              // [2 last + 1]
    attn_lds_f32 *table;                 // [places][slots]
    int last, shift, slot;
    __device__ __forceinline__ int index(int kp, int qp) const
    {
        const int r = attn_distance(kp, qp);
        return __builtin_elementwise_max(__builtin_elementwise_min(r, last), -last) + last;
    }
    __device__ __forceinline__ float at(int place) const { return table[(place << shift) + slot]; }
};
static inline size_t attn_bias_bytes(const attn_args &a, int slots)
{
    return a.buckets ? (size_t)((2 * a.last + 1 + 15) & ~15) + (size_t)((attn_places(a) * slots * 4 + 15) & ~15) : 0;
}
// by the whole workgroup; the caller synchronises.  head(slot): the head of a slot, or -1
template <typename T, typename HEAD>
__device__ __forceinline__ attn_bias attn_make_bias(const attn_args &a, attn_lds *lds, int shift, HEAD head)
{
    const int slots = 1 << shift, distances = 2 * a.last + 1;
    attn_lds_u8 *lut = (attn_lds_u8 *)lds;
    attn_lds_f32 *table = (attn_lds_f32 *)(lds + ((distances + 15) & ~15));
    for (int x = threadIdx.x; x < distances; x += blockDim.x) lut[x] = (uint8_t)attn_place_of(a, attn_bucket(a, x - a.last));
    for (int x = threadIdx.x; x < attn_places(a) * slots; x += blockDim.x) {
        const int h = head(x & (slots - 1));
        table[x] = h < 0 ? 0.f : (float)((const T *)a.table)[(int64_t)attn_bucket_of(a, x >> shift) * a.ldt + h];
    }
    return {lut, table, a.last, shift, 0};
}
// scores of a tile: s * scale + bias, of the distances k(x) - q(x) of its 16 pairs
template <typename K, typename Q>
__device__ __forceinline__ void attn_add_bias(const attn_bias &bias, attn_f32x16 &s, float scale, K k, Q q)
{
    int i[16];
#pragma unroll
    for (int x = 0; x < 16; ++x) i[x] = bias.index(k(x), q(x));
#pragma unroll
    for (int x = 0; x < 16; ++x) i[x] = bias.lut[i[x]];
#pragma unroll
    for (int x = 0; x < 16; ++x) s[x] = __builtin_fmaf(s[x], scale, bias.at(i[x]));
}
// Is any of a wave's scores minus infinity?
__device__ __forceinline__ bool attn_any_lowest(const attn_f32x16 &s)
{
    float low = s[0];
#pragma unroll
    for (int x = 1; x < 16; ++x) low = fminf(low, s[x]);
    return __builtin_amdgcn_ballot_w64(low == -INFINITY) != 0;
}

// How the 32 rows of a wave's tile are made of queries and heads.
enum { kRowsOfHead,                      // br = 128: the workgroup's waves take 32 rows each, of one head
       kHeadsOfRows,                     // br = 32: the workgroup's waves take a head each, of the same 32 rows
       kRowsTogether,                    // br = 32: one tile, 32 rows of one head; the waves share its columns out
       kHeadsTogether };                 // br = 1: one tile, up to 32 heads of one row; the waves share its columns out

// A lane's query and head.  group: which of an item's workgroups this is.  The heads of one key head are Hk workgroups apart, so that with 8 key
// heads or 4 they run on one compute die or two, whose L2 they share K and V in.
struct attn_lane {
    int head, kv, r;                     // r: the row's place in its block
    int64_t row;
    bool valid;                          // a pair of a row and a head that exists (clamped to one that does)
    __device__ __forceinline__ attn_lane(const attn_args &a, const attn_item &item, int mode, int group, int lane, int wave, int waves)
    {
        r = lane & 31;
        valid = true;
        if (mode == kRowsOfHead || mode == kRowsTogether) {
            kv = group % a.Hk;
            head = kv * a.G + group / a.Hk;
            if (mode == kRowsOfHead) r += 32 * wave;
        } else {
            const int per = mode == kHeadsOfRows ? waves : 32;
            kv = group % a.Hk;
            int x = group / a.Hk * per + (mode == kHeadsOfRows ? wave : lane & 31);
            valid = x < a.G;
            if (!valid) x = a.G - 1;
            head = kv * a.G + x;
            if (mode == kHeadsTogether) r = 0;
        }
        valid = valid && r < item.rows;
        row = item.row0 + (r < item.rows ? r : item.rows - 1);
    }
};
// the bias for the workgroup's heads, its slot for this lane
template <typename T>
__device__ __forceinline__ attn_bias attn_lane_bias(const attn_args &a, attn_lds *lds, int mode, int group, int lane, int wave, int waves)
{
    const int shift = mode == kHeadsTogether ? 5 : mode == kHeadsOfRows ? 2 : 0;         // of four waves
    attn_bias b = attn_make_bias<T>(a, lds, shift, [&](int s) {
        const int x = shift == 0 ? group / a.Hk : (group / a.Hk << shift) + s;
        return x < a.G ? group % a.Hk * a.G + x : -1;
    });
    b.slot = mode == kHeadsTogether ? lane & 31 : mode == kHeadsOfRows ? wave : 0;
    return b;
}

// The mapping for a plan and a problem, and how the plan is cut.
// A block of 32 rows: with three heads or more to a key, the waves take the heads and K and V are fetched once for them; with
// fewer, they share the columns out.
struct attn_mapping {
    int mode, wm, wn, groups, level;
    double us, whole_us;                 // modelled time of the level, and with whole blocks
    bool cut;                            // some rows have several items
    int slots() const { return mode == kHeadsTogether ? 32 : mode == kHeadsOfRows ? wm : 1; }
};
// About what a chunk of 64 columns takes a workgroup of four tiles that has a compute unit to itself, in microseconds, for a number of
// products (forward 2: 2.0 for 128 numbers of 16 bits; f32 15).
static inline double attn_chunk_us(int D, int size, int products)
{
    const double numbers = D <= 32 ? 32 : D <= 64 ? 64 : D <= 128 ? 128 : 256;
    return (size == 4 ? 0.06 : 0.008) * numbers * products;
}
static inline attn_mapping attn_map(const sp_attn_plan *plan, const attn_args &a, int size, int products)
{
    attn_mapping c;
    if (plan->br == 128) { c.mode = kRowsOfHead; c.groups = a.H; }
    else if (plan->br == 32 && a.G >= 3) { c.mode = kHeadsOfRows; c.groups = a.Hk * (int)ceil_div(a.G, 4); }
    else if (plan->br == 32) { c.mode = kRowsTogether; c.groups = a.H; }
    else { c.mode = kHeadsTogether; c.groups = a.Hk * (int)ceil_div(a.G, 32); }
    const bool share = c.mode == kRowsTogether || c.mode == kHeadsTogether;
    c.wm = share ? 1 : 4;
    c.wn = share ? 4 : 1;
    const double chunk_us = attn_chunk_us(a.D, size, products) / (share ? 2 : 1), item_us = share ? 6 : 3, row_bytes = 4.0 * a.D * a.H;
    c.level = attn_pick_level(plan, c.groups, chunk_us, item_us, row_bytes);
    c.us = attn_level_us(plan, c.level, c.groups, chunk_us, item_us, row_bytes);
    c.whole_us = attn_level_us(plan, plan->levels - 1, c.groups, chunk_us, item_us, row_bytes);
    c.cut = plan->cut[c.level] > 0;
    return c;
}

// Rows of all tensors made of whole 16-byte granules?
struct attn_alignment {
    bool vec;
    attn_alignment(int D, int size) : vec(D * size % 16 == 0), size_(size) {}
    void with(const void *x, int64_t ld, int64_t hd) { vec = vec && (uintptr_t)x % 16 == 0 && ld * size_ % 16 == 0 && hd * size_ % 16 == 0; }
private:
    int size_;
};

// Numbers of 4 columns of a row: whole, or cut at D.
template <typename T>
__device__ __forceinline__ void attn_store4(T *row, int d, int D, bool vec, attn_f32x4 v)
{
    if (vec) {
        typedef T out4 __attribute__((ext_vector_type(4)));
        if (d < D) *(out4 *)(row + d) = __builtin_convertvector(v, out4);
    } else {
#pragma unroll
        for (int c = 0; c < 4; ++c) if (d + c < D) row[d + c] = (T)v[c];
    }
}

// dq_kernel: how many waves share a tile's columns, and the LDS it takes.  K and V of a step and the bias's sums have to fit together.
constexpr int kAttnLds = 160 * 1024;
static constexpr int attn_dq_waves(int row_bytes, bool pos) { return row_bytes == 512 ? (pos ? 1 : 2) : row_bytes == 256 && pos ? 2 : 4; }
// Columns of a step for four tiles.  64 take long enough to compute for the next ones to arrive; with the bias's sums in LDS, 32 leave
// room for a second workgroup.
static constexpr int attn_dq_columns(int row_bytes, bool pos) { return row_bytes <= (pos ? 64 : 256) ? 64 : 32; }
// 16-bit rows of up to this many pairs, on average over a block of up to this many chunks, go through dq_kernel twice: the first time for what
// their D misses, which is made of an O that was rounded to 16 bits.  (A pattern of such rows is not cut finer.)  Beside dQ that error is
// the larger the fewer pairs there are: in units of one rounding of dQ, rows of 20 to 30 have an error of 1.5 to 1.63 with it and of 1.42
// (ds' rounding and dQ's) without; rows of 128 of 1.46 at most.  The second pass takes a tenth of such a step (64 sequences of 64 to 128: 52.4
// and 58.1 us; 16384 rows of a band of 65: 224 and 260); 16 sequences of 200 to 512 would take 195.4 us instead of 191 with it up to 256.
constexpr int kAttnTwiceLevel = 3, kAttnTwice = 1 << kAttnTwiceLevel, kAttnTwicePairs = 128;
static inline size_t attn_dq_lds(const attn_args &a, const attn_mapping &c, int row_bytes, bool pos, bool table, bool exact)
{
    const bool share = c.wn > 1;
    const int waves = share ? attn_dq_waves(row_bytes, pos) : 4, KT = share ? 32 * waves : attn_dq_columns(row_bytes, pos);
    const size_t lds = 4 * (size_t)KT * row_bytes + (share ? waves * 128 : 0) + (pos ? 2 * KT * 4 + attn_bias_bytes(a, c.slots()) : 0) +
                       (table ? (size_t)waves * attn_places(a) * (exact ? 512 : 256) : 0);
    return lds;
}

// ---- what attention.hip hands to the sources of one type ---------------------------------------------------------------------
struct forward_args {
    attn_args a;
    attn_plan_view p;
    void *O;
    int64_t ldo, hdo;
    float *lse;
    float *part, *part_stat;             // of rows that are cut: [item][head][row of the block][pd] and [..][2] (maximum, total)
    int groups, mode, vec;               // workgroups of an item; mapping; whether rows are made of whole aligned granules
    int pd;                              // numbers of a row of a part: D rounded up to a multiple of 4
};

struct forward_choice : attn_mapping {
    size_t part, part_stat;              // bytes
};
template <typename T>
sp_status attn_forward(const sp_attn_plan *plan, forward_args &f, const forward_choice &c, hipStream_t st);

struct grad_args {
    attn_args a;
    attn_plan_view p;
    sp_attention_grads g;
    float *delta;                        // [heads][m]: D of every row, made by dq_kernel
    float *log_sum;                      // with a bias, [heads][m]: attn_log_sum of every row, made by dq_kernel
    float *part;                         // of rows (keys) that are cut: dq [item][head][row of the block][pd]; dkv [item][kv head][key][2][pd]
    float *part_table;                   // [item][head][buckets]
    int groups, mode, vec, pd;
    int exact;                           // how the bias's gradient is summed: see dq_kernel
};

struct grad_choice {
    attn_mapping rows;
    bool exact;
    int keys_level;
    bool keys_cut;
    size_t delta, log_sum, part, table;  // bytes; the parts of dQ and of dK, dV use the same place one after the other
    size_t bytes() const { return delta + log_sum + part + table; }
};
template <typename T>
sp_status attn_backward(const sp_tensor *S, grad_args &f, const grad_choice &c, hipStream_t st);

// ---- parts of rows that were cut ----------------------------------------------------------------------------------------------
// Sums of f32 rows of pd numbers (a multiple of 4, at most 256), by a wave: LP lanes take a row, 4 numbers each, and 64 / LP rows are
// taken at a time; `count` rows in all, row k at at(k) with weight weight(k).  The result is in every group of LP lanes.
template <int LP, typename AT, typename WEIGHT>
__device__ __forceinline__ attn_f32x4 attn_add_parts(int count, int pd, int lane, AT at, WEIGHT weight)
{
    constexpr int S = 64 / LP;
    const int l = lane % LP, s = lane / LP;
    attn_f32x4 sum = (attn_f32x4)(0.f);
    for (int k0 = 0; k0 < count; k0 += 4 * S) {
        attn_f32x4 v[4];
        float w[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int k = k0 + u * S + s;
            const bool there = k < count && 4 * l < pd;
            w[u] = k < count ? weight(k) : 0.f;
            v[u] = there ? *(const attn_f32x4 *)(at(k) + 4 * l) : (attn_f32x4)(0.f);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) sum += v[u] * w[u];
    }
#pragma unroll
    for (int d = LP; d < 64; d <<= 1)
#pragma unroll
        for (int c = 0; c < 4; ++c) sum[c] += __shfl_xor(sum[c], d, 64);
    return sum;
}
