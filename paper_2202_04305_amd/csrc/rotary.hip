// Rotary positions.  The bytes of Q and K in and out bound it: a workgroup takes one token (or a few short ones), makes the cosines and sines of
// its pairs once, in LDS, and turns all heads of Q and K by them.  16384 bf16 tokens of 40 heads of 128 take 60 us, 5.5 TB/s (a thread for each pair that makes
// its own cosine: 190); 4099 f32 tokens of 24 heads of 80, 20 numbers of which turn, 13.6 us, 4.6 TB/s.
#include "spmi_internal.h"
#include <math.h>

namespace {

struct rotary_side { const void *in; void *out; int64_t ld, hd, ldo, hdo; int heads; };
struct rotary_args {
    rotary_side side[2];
    const int32_t *position;
    const double *frequency;
    int64_t tokens;
    int D, half, interleaved;
    float scale, sign;
    int per_head, items;                 // items of a head and of a token's heads
    spmi_divisor32 by_head, by_heads, by_half;
    int group;                           // tokens of a workgroup
};

// (cos, sin) of position * f.  The angle in quarter turns, in 64 bits, leaves a rest of at most an eighth of a turn, which 32 bits hold to
// 2^-24 of itself however far the position.
__device__ __forceinline__ float2 rotary_turn(int position, double f)
{
    const double turns = (double)position * (f * 0.15915494309189535);
    const double quarter = rint(turns * 4);
    const float rest = (float)(2 * (turns - quarter * 0.25));
    float s, c;
    sincospif(rest, &s, &c);
    const int q = (int)(quarter - 4 * floor(quarter * 0.25));
    const float x = q & 1 ? s : c, y = q & 1 ? c : s;
    return {q == 1 || q == 2 ? -x : x, q >= 2 ? -y : y};
}

constexpr int kRotaryPairs = 1024;       // pairs of a workgroup's tokens that the LDS has room for

// V pairs at a time and W of the numbers that stay (16 bytes of them where everything is aligned to that, single ones otherwise).  An item of a
// head is V pairs, of numbers that lie half apart or side by side, or W numbers that stay.  Where the pairs do not fit the LDS (heads beyond 2 kRotaryPairs numbers) every
// item makes its own.
template <typename T, int V, int W, bool INTERLEAVED>
__global__ __launch_bounds__(256) void rotary_kernel(rotary_args a)
{
    typedef T row __attribute__((ext_vector_type(V)));
    typedef T row2 __attribute__((ext_vector_type(2 * V), aligned(V == 1 ? sizeof(T) : 2 * V * sizeof(T))));
    static_assert(V > 1 || alignof(row2) == alignof(T), "V = 1 takes strides and addresses of any number of elements");
    typedef T rest __attribute__((ext_vector_type(W)));
    __shared__ float2 turn[kRotaryPairs];
    const int turning = a.half / V;
    const bool kept = a.half <= kRotaryPairs;
    for (int64_t i0 = (int64_t)blockIdx.x * a.group; i0 < a.tokens; i0 += (int64_t)gridDim.x * a.group) {
    const int group = (int)(a.tokens - i0 < a.group ? a.tokens - i0 : a.group);
    if (kept) {
        __syncthreads();
        for (int x = threadIdx.x; x < group * a.half; x += 256) {
            const int i = (int)spmi_div_by32(x, a.by_half);
            const float2 t = rotary_turn(a.position[i0 + i], a.frequency[x - i * a.half]);
            turn[x] = {t.x * a.scale, t.y * a.scale * a.sign};
        }
        __syncthreads();
    }
    for (uint32_t x = threadIdx.x + 256 * blockIdx.y; x < (uint32_t)group * (uint32_t)a.items; x += 256 * gridDim.y) {
        const int all = (int)spmi_div_by32(x, a.by_head), k = (int)x - all * a.per_head;       // the head of all tokens' heads; the item in its head
        const int heads = a.side[0].heads + a.side[1].heads, i = (int)spmi_div_by32(all, a.by_heads);
        int h = all - i * heads;
        const bool second = h >= a.side[0].heads;
        if (second) h -= a.side[0].heads;
        const rotary_side &s = a.side[second];
        const T *in = (const T *)s.in + (i0 + i) * s.ld + h * s.hd;
        T *out = (T *)s.out + (i0 + i) * s.ldo + h * s.hdo;
        if (k >= turning) {                              // behind the turning numbers
            const int d = 2 * a.half + (k - turning) * W;
            *(rest *)(out + d) = *(const rest *)(in + d);
            continue;
        }
        float u[V], v[V];
        if (INTERLEAVED) {
            const row2 both = *(const row2 *)(in + 2 * V * k);
#pragma unroll
            for (int j = 0; j < V; ++j) { u[j] = (float)both[2 * j]; v[j] = (float)both[2 * j + 1]; }
        } else {
            const row first = *(const row *)(in + V * k), last = *(const row *)(in + a.half + V * k);
#pragma unroll
            for (int j = 0; j < V; ++j) { u[j] = (float)first[j]; v[j] = (float)last[j]; }
        }
#pragma unroll
        for (int j = 0; j < V; ++j) {
            float2 t;
            if (kept) t = turn[i * a.half + V * k + j];
            else {
                t = rotary_turn(a.position[i0 + i], a.frequency[V * k + j]);
                t.x *= a.scale; t.y *= a.scale * a.sign;
            }
            const float x0 = u[j] * t.x - v[j] * t.y;
            v[j] = u[j] * t.y + v[j] * t.x;
            u[j] = x0;
        }
        if (INTERLEAVED) {
            row2 both;
#pragma unroll
            for (int j = 0; j < V; ++j) { both[2 * j] = (T)u[j]; both[2 * j + 1] = (T)v[j]; }
            *(row2 *)(out + 2 * V * k) = both;
        } else {
            row first, last;
#pragma unroll
            for (int j = 0; j < V; ++j) { first[j] = (T)u[j]; last[j] = (T)v[j]; }
            *(row *)(out + V * k) = first;
            *(row *)(out + a.half + V * k) = last;
        }
    }
    }
}

template <typename T, int V, int W>
void launch(rotary_args a, hipStream_t st)
{
    a.per_head = a.half / V + (a.D - 2 * a.half) / W;
    const int heads = a.side[0].heads + a.side[1].heads;
    a.items = heads * a.per_head;
    a.by_head = spmi_make_divisor32(a.per_head);
    a.by_heads = spmi_make_divisor32(heads);
    a.by_half = spmi_make_divisor32(a.half ? a.half : 1);
    // about 1024 items a workgroup, four for each thread, but a workgroup for each of up to 1024 tokens; of one with many items several share the token
    int64_t group = 1024 / a.items, most = ceil_div(a.tokens, 1024);
    if (a.half && group > kRotaryPairs / a.half) group = kRotaryPairs / a.half;
    a.group = (int)(group > most ? most : group < 1 ? 1 : group);
    const int64_t blocks = ceil_div(a.tokens, a.group), each = ceil_div((int64_t)a.group * a.items, 256), more = ceil_div(512, blocks);
    const dim3 grid((unsigned)(blocks < 1 << 20 ? blocks : 1 << 20), (unsigned)(each < more ? each : more < 1 ? 1 : more));
    if (a.interleaved) rotary_kernel<T, V, W, true><<<grid, 256, 0, st>>>(a);
    else rotary_kernel<T, V, W, false><<<grid, 256, 0, st>>>(a);
}

// Are addresses and strides of all tensors multiples of so many numbers?
bool aligned(const rotary_args &a, int64_t numbers, int64_t size)
{
    for (const rotary_side &s : a.side)
        if (s.heads && ((((uintptr_t)s.in | (uintptr_t)s.out) % (numbers * size)) || s.ld % numbers || s.hd % numbers || s.ldo % numbers || s.hdo % numbers)) return false;
    return true;
}

// The most numbers at a time that sizes, strides and addresses allow: 16 bytes, or half of that, or a quarter, ...; of those that stay 16 bytes or
// as many as of the pairs.
template <typename T, int V>
void launch_widest(const rotary_args &a, hipStream_t st)
{
    constexpr int most = 16 / sizeof(T);
    const int64_t run = a.interleaved ? 2 * V : V, rest = a.D - 2 * a.half;
    if constexpr (V > 1) {
        if (a.half % V || run > most || rest % V || !aligned(a, run, sizeof(T))) return launch_widest<T, V / 2>(a, st);
    }
    if (V < most && rest && rest % most == 0 && 2 * a.half % most == 0 && aligned(a, most, sizeof(T))) launch<T, V, most>(a, st);
    else launch<T, V, V>(a, st);
}

sp_status rotary(const sp_rotary_problem *p, float sign, void *stream)
{
    if (!p) return SP_ERR_NULL;
    if (p->dtype != (int)SP_F32 && p->dtype != (int)SP_F16 && p->dtype != (int)SP_BF16) return SP_ERR_DTYPE;
    if (p->headDim < 1 || p->rotDim < 0 || p->rotDim % 2 || p->rotDim > p->headDim || p->tokens < 0 || p->heads < 0 || p->kvHeads < 0) return SP_ERR_SHAPE;
    const float scale = (float)p->scale;
    if (!(scale - scale == 0)) return SP_ERR_SHAPE;
    for (int64_t s : {p->ldq, p->hdq, p->ldk, p->hdk}) if (s < 0) return SP_ERR_SHAPE;
    if ((p->tokens > 1 && p->heads > 0 && p->ldqo < p->headDim) || (p->heads > 1 && p->hdqo < p->headDim)) return SP_ERR_SHAPE;
    if ((p->tokens > 1 && p->kvHeads > 0 && p->ldko < p->headDim) || (p->kvHeads > 1 && p->hdko < p->headDim)) return SP_ERR_SHAPE;
    if (p->interleaved != 0 && p->interleaved != 1) return SP_ERR_UNSUPPORTED;
    if (((int64_t)p->heads + p->kvHeads) * p->headDim >= (int64_t)1 << 31) return SP_ERR_TOO_LARGE;
    if (p->tokens == 0 || p->heads + p->kvHeads == 0) return SP_OK;
    if ((p->rotDim && (!p->position || !p->frequency)) || (p->heads && (!p->Q || !p->Qout)) || (p->kvHeads && (!p->K || !p->Kout))) return SP_ERR_NULL;
    const rotary_args a = {{{p->Q, p->Qout, p->ldq, p->hdq, p->ldqo, p->hdqo, p->heads}, {p->K, p->Kout, p->ldk, p->hdk, p->ldko, p->hdko, p->kvHeads}},
                           p->position, p->frequency, p->tokens, p->headDim, p->rotDim / 2, p->interleaved, scale, sign, 0, 0, {}, {}, {}, 0};
    hipStream_t st = (hipStream_t)stream;
    if (p->dtype == SP_F32) launch_widest<float, 4>(a, st);
    else if (p->dtype == SP_F16) launch_widest<_Float16, 8>(a, st);
    else launch_widest<__bf16, 8>(a, st);
    SP_HIP(hipGetLastError());
    return SP_OK;
}

}  // namespace

extern "C" sp_status sp_rotary(const sp_rotary_problem *p, void *stream) { return rotary(p, 1.f, stream); }
extern "C" sp_status sp_rotary_grad(const sp_rotary_problem *p, void *stream) { return rotary(p, -1.f, stream); }

extern "C" sp_status sp_rotary_frequencies(int rotDim, double base, double factor, int64_t trained, double low, double high, double *frequency)
{
    if (!frequency && rotDim != 0) return SP_ERR_NULL;
    if (rotDim < 0 || rotDim % 2 || trained < 0 || !(base > 0) || !(base - base == 0) || !(factor > 0) || !(factor - factor == 0)) return SP_ERR_SHAPE;
    if (trained > 0 && !(high > low)) return SP_ERR_SHAPE;
    for (int k = 0; k < rotDim / 2; ++k) {
        const double f = pow(base, -2.0 * k / rotDim);
        double keep = 0;
        if (trained > 0) {
            keep = ((double)trained * f / 6.283185307179586 - low) / (high - low);
            keep = keep < 0 ? 0 : keep > 1 ? 1 : keep;
        }
        frequency[k] = (1 - keep) * f / factor + keep * f;
        if (!(frequency[k] - frequency[k] == 0)) return SP_ERR_SHAPE;
    }
    return SP_OK;
}
