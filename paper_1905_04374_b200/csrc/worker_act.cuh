// Activations and the 8-bit codes of checkpoints (gar_worker.h), shared by the kernels that compute the one and
// write the other.
#pragma once
#include "worker_common.cuh"

namespace gar {
namespace worker {

__device__ __forceinline__ float rcp(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// Off by 4e-7 of itself (both functions are approximate to 2^-22) and, for negative x, 1e-7 |x| (the rounded product in
// the exponent): less than what 16-bit results round off.
__device__ __forceinline__ float sigmoid(float x) { return rcp(1.f + ex2(-x * kLog2e)); }

// The normal distribution at two places: cdf = P(X < x) and the density's e^(-x^2 / 2).  The tail behind |x| is
//     e^(-x^2 / 2) t P(t),   t = 1 / (1 + 0.275 |x|)
// (the form of Abramowitz and Stegun 26.2.17), P of degree 8 fitted to e^(x^2 / 2) erfc(x / sqrt 2) / 2 t: 2.8e-7 of the
// tail at most, in fp32 1e-6 down to -4 and 2e-6 at -6, where the exponent's rounding shows.  (1 + erf(x / sqrt 2)) / 2
// cancels for negative x: 4 % off at -5, 0 from -5.5 on.  bf16 8192 x 8192, forward and backward: 76 and 60 us; with
// erff 105 and 95 us, with erfcf 143 and 131.
__device__ __forceinline__ void normal2(float x0, float x1, float (&cdf)[2], float (&e)[2]) {
    const float t0 = rcp(fmaf(fabsf(x0), 0.275f, 1.f)), t1 = rcp(fmaf(fabsf(x1), 0.275f, 1.f));
    const f32x2 t = pack2(t0, t1), x = pack2(x0, x1), c = pack2(-0.5f * kLog2e, -0.5f * kLog2e);
    unpack2(mul2(mul2(x, x), c), e[0], e[1]);
    e[0] = ex2(e[0]);
    e[1] = ex2(e[1]);
    f32x2 p = pack2(0.0237322034f, 0.0237322034f);
    constexpr float P[8] = {-0.0965348071f, 0.106157018f, -0.0134071806f, 0.0766527223f, 0.0823775453f, 0.101610145f, 0.10970306f, 0.109709157f};
#pragma unroll
    for (int i = 0; i < 8; ++i) p = fma2(p, t, pack2(P[i], P[i]));
    float tail0, tail1;
    unpack2(mul2(mul2(p, t), pack2(e[0], e[1])), tail0, tail1);
    cdf[0] = x0 < 0.f ? tail0 : 1.f - tail0;
    cdf[1] = x1 < 0.f ? tail1 : 1.f - tail1;
}

// act(x) of eight elements
template <int ACT>
__device__ __forceinline__ void act8(const float (&x)[8], float (&y)[8]) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        if constexpr (ACT == GAR_ACT_GELU) {
            float cdf[2], e[2];
            normal2(x[i], x[i + 1], cdf, e);
            y[i] = x[i] * cdf[0];
            y[i + 1] = x[i + 1] * cdf[1];
        } else {
#pragma unroll
            for (int k = i; k < i + 2; ++k) y[k] = ACT == GAR_ACT_RELU ? max_nan(x[k], 0.f) : ACT == GAR_ACT_SILU ? x[k] * sigmoid(x[k]) : x[k];
        }
    }
}

// ---- codes ----------------------------------------------------------------------------------------
constexpr float CK_TINY = 7.888609052210118e-31f;     // 2^-100
constexpr float CK_LARGEST = 2.6793884e+36f;           // the largest scale whose 127-fold is finite in fp32

// What a group whose largest magnitude is `top` is divided by.
struct Step {
    bool  sound, live;             // no NaN or infinity; not stored as zeros
    float inv;
    __device__ __forceinline__ explicit Step(float top) {
        sound = top <= 3.402823466e38f;
        live = sound && top >= CK_TINY;
        inv = live ? __fmul_rn(__frcp_rn(top), 127.f) : 0.f;
    }
    __device__ __forceinline__ float scale(float top) const {
        // top / 127, correctly rounded: Markstein's correction of the product with the rounded reciprocal
        const float y = 1.f / 127.f, q0 = __fmul_rn(top, y);
        const float s = fminf(__fmaf_rn(__fmaf_rn(-127.f, q0, top), y, q0), CK_LARGEST);
        return !sound ? CUDART_NAN_F : live ? s : 0.f;
    }
};
// The codes of eight columns, four to a word.
__device__ __forceinline__ void codes8(const float (&v)[8], const Step& step, unsigned& lo, unsigned& hi) {
    // |v inv| <= 127 (1 + 2^-22): the low byte of the sum with 1.5 * 2^23 is the nearest integer, ties to even
    // (the products one by one: as a pair, product and sum were contracted to one rounding)
    const f32x2 magic = pack2(12582912.f, 12582912.f);
    float r[8];
#pragma unroll
    for (int i = 0; i < 8; i += 2) unpack2(add2(pack2(__fmul_rn(v[i], step.inv), __fmul_rn(v[i + 1], step.inv)), magic), r[i], r[i + 1]);
    lo = __byte_perm(__byte_perm(__float_as_uint(r[0]), __float_as_uint(r[1]), 0x0040),
                              __byte_perm(__float_as_uint(r[2]), __float_as_uint(r[3]), 0x0040), 0x5410);
    hi = __byte_perm(__byte_perm(__float_as_uint(r[4]), __float_as_uint(r[5]), 0x0040),
                              __byte_perm(__float_as_uint(r[6]), __float_as_uint(r[7]), 0x0040), 0x5410);
    if (!step.sound) lo = hi = 0u;
}

}  // namespace worker
}  // namespace gar
