// Rotary positions: a thread for each pair of a token's head and for each number that stays.
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

template <typename T>
__global__ __launch_bounds__(256) void rotary_kernel(rotary_args a)
{
    const int per = a.D - a.half;                        // pairs, then the numbers that stay
    const int64_t row = (int64_t)(a.side[0].heads + a.side[1].heads) * per, n = a.tokens * row;
    for (int64_t x = blockIdx.x * (int64_t)256 + threadIdx.x; x < n; x += (int64_t)gridDim.x * 256) {
        const int64_t i = x / row;
        int h = (int)((x - i * row) / per);
        const int k = (int)((x - i * row) % per);
        const int which = h >= a.side[0].heads;
        if (which) h -= a.side[0].heads;
        const rotary_side &s = a.side[which];
        const T *in = (const T *)s.in + i * s.ld + h * s.hd;
        T *out = (T *)s.out + i * s.ldo + h * s.hdo;
        if (k >= a.half) { out[k + a.half] = in[k + a.half]; continue; }
        const int d0 = a.interleaved ? 2 * k : k, d1 = a.interleaved ? 2 * k + 1 : k + a.half;
        const float2 t = rotary_turn(a.position[i], a.frequency[k]);
        const float c = t.x * a.scale, z = t.y * a.scale * a.sign, u = (float)in[d0], v = (float)in[d1];
        out[d0] = (T)(u * c - v * z);
        out[d1] = (T)(u * z + v * c);
    }
}

template <typename T>
void launch(const rotary_args &a, hipStream_t st)
{
    const int64_t n = a.tokens * (a.side[0].heads + a.side[1].heads) * (a.D - a.half), blocks = ceil_div(n, 256);
    rotary_kernel<T><<<(int)(blocks < 65536 ? blocks : 65536), 256, 0, st>>>(a);
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
    if (p->tokens == 0 || p->heads + (int64_t)p->kvHeads == 0) return SP_OK;
    if ((p->rotDim && (!p->position || !p->frequency)) || (p->heads && (!p->Q || !p->Qout)) || (p->kvHeads && (!p->K || !p->Kout))) return SP_ERR_NULL;
    const rotary_args a = {{{p->Q, p->Qout, p->ldq, p->hdq, p->ldqo, p->hdqo, p->heads}, {p->K, p->Kout, p->ldk, p->hdk, p->ldko, p->hdko, p->kvHeads}},
                           p->position, p->frequency, p->tokens, p->headDim, p->rotDim / 2, p->interleaved, scale, sign};
    hipStream_t st = (hipStream_t)stream;
    if (p->dtype == SP_F32) launch<float>(a, st);
    else if (p->dtype == SP_F16) launch<_Float16>(a, st);
    else launch<__bf16>(a, st);
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
    }
    return SP_OK;
}
