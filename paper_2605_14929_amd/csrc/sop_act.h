// Activations and their slopes in binary32, over all of its range: 0 none, 1 relu, 2 silu, 3 gelu, 4 gelu by tanh (SOP_ACT_*).
//
// exp(-a), a >= 0, is kept as its root g = exp(-a / 2): what is small because of it leaves binary32's normal numbers only in the last step, a second multiplication by g.
// What grows (z, the inner derivative) meets the first g before it meets anything else, so that nothing overflows beside a result that does not.
//   logistic(u)    w = 1 / (1 + exp(-|u|)); u >= 0: w, else w exp(-|u|)
//   silu           z logistic(z);             slope s + z s (1 - s)
//   gelu by tanh   z logistic(2 v), v = sqrt(2 / pi) (z + 0.044715 z^3): (1 + tanh v) / 2 = logistic(2 v)
//   gelu           z Phi(z), Phi the normal distribution.  Phi(-a) = phi(a) R(a), phi its density, R the Mills ratio, which is smooth: with t = 1 / (1 + 0.3 a),
//                  R = t P(t), P of degree 7 fitted here to R in 64 bits at 400 Chebyshev nodes of a in [0, 14.5] for the least relative error (1.7e-7).
//                  Slope Phi(z) + z phi(z): from -a, phi (R - a).
// FINE: with the exponent h = a log2 e in two parts, so that the error of g is that of the hardware's 2^t.  Otherwise, for bf16 numbers, without:
// 1.4 h 2^-24 of the value more.
// Far out the arguments are clamped where the function has long been 0 or z: infinities give the limits, NaN stays.
#ifndef SOP_ACT_H
#define SOP_ACT_H
#include <hip/hip_runtime.h>

namespace sopk {

#define SOPK_LOG2E 1.44269504f                                          // log2(e) = LOG2E + LOG2E_LO
#define SOPK_LOG2E_LO 1.9259630e-08f
// 2^-(h + r) for h / 2 and r / 2, r small
template <bool FINE> __device__ __forceinline__ float root_of(float h, float r)
{
    const float g = __builtin_amdgcn_exp2f(-h);
    return FINE ? __builtin_fmaf(g, r * -0.693147181f, g) : g;
}
// exp(-a / 2), a >= 0
template <bool FINE> __device__ __forceinline__ float root(float a)
{
    const float h = a * (0.5f * SOPK_LOG2E);
    return root_of<FINE>(h, FINE ? __builtin_fmaf(a, 0.5f * SOPK_LOG2E, -h) + a * (0.5f * SOPK_LOG2E_LO) : 0.0f);
}
__device__ __forceinline__ float within(float z, float far) { return z < -far ? -far : z > far ? far : z; }   // (NaN stays)
// logistic(u): w, and exp(-|u| / 2)
struct Logistic { float g, w; };
template <bool FINE> __device__ __forceinline__ Logistic logistic_of(float u)
{
    const float a = fabsf(u), g = root<FINE>(FINE && a > 1200.0f ? 1200.0f : a);   // (a difference of infinities would be no number; NaN stays)
    return Logistic{g, __builtin_amdgcn_rcpf(__builtin_fmaf(g, g, 1.0f))};
}
// the coefficients of P / sqrt(2 pi), t = 1 / (1 + 0.3 a)
#define SOPK_MILLS_0 0.119632013f
#define SOPK_MILLS_1 0.120712146f
#define SOPK_MILLS_2 0.100175917f
#define SOPK_MILLS_3 0.12769191f
#define SOPK_MILLS_4 -0.0520343035f
#define SOPK_MILLS_5 0.204557121f
#define SOPK_MILLS_6 -0.156158671f
#define SOPK_MILLS_7 0.0354238003f
// the root of phi(a) sqrt(2 pi), and R(a) / sqrt(2 pi), 0 <= a <= 40
struct Tail { float g, r; };
template <bool FINE> __device__ __forceinline__ Tail tail(float a)
{
    const float q = a * a, h = q * (0.25f * SOPK_LOG2E);
    const float g = root_of<FINE>(h, FINE ? __builtin_fmaf(q, 0.25f * SOPK_LOG2E, -h) + __builtin_fmaf(q, 0.25f * SOPK_LOG2E_LO, __builtin_fmaf(a, a, -q) * (0.25f * SOPK_LOG2E)) : 0.0f);
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(a, 0.3f, 1.0f));
    constexpr float c[8] = {SOPK_MILLS_0, SOPK_MILLS_1, SOPK_MILLS_2, SOPK_MILLS_3, SOPK_MILLS_4, SOPK_MILLS_5, SOPK_MILLS_6, SOPK_MILLS_7};
    float r = c[7];
#pragma unroll
    for (int i = 6; i >= 0; --i) r = __builtin_fmaf(r, t, c[i]);
    return Tail{g, r * t};
}
#define SOPK_PHI0 0.398942280f                                          // 1 / sqrt(2 pi)
#define SOPK_TANH_A 1.59576912f                                         // 2 sqrt(2 / pi)
#define SOPK_TANH_B 0.0713548163f                                       // ... times 0.044715

template <bool FINE> __device__ __forceinline__ float act_of(int act, float z)
{
    if (act == 1) return z < 0.0f ? 0.0f : z;
    if (act == 2 || act == 4) {
        const Logistic s = logistic_of<FINE>(act == 2 ? z : z * __builtin_fmaf(z * z, SOPK_TANH_B, SOPK_TANH_A));
        const float m = z >= 0.0f ? 1.0f : s.g;
        return __builtin_amdgcn_fmed3f(z, -1e30f, __builtin_inff()) * s.w * m * m;   // (w of NaN is NaN)
    }
    if (act == 3) {
        const float c = __builtin_amdgcn_fmed3f(z, -40.0f, 40.0f);      // (of NaN -40, and z - u is NaN)
        const Tail t = tail<FINE>(fabsf(c));
        const float u = c * (t.g * t.r) * t.g;                          // z Phi(-|z|)
        return z < 0.0f ? u : z - u;
    }
    return z;
}
// d times the slope at z
template <bool FINE> __device__ __forceinline__ float act_slope(int act, float z, float d)
{
    if (act == 1) return z <= 0.0f ? 0.0f : d;
    if (act == 2 || act == 4) {
        const float c = within(z, 1200.0f), q = c * c;
        const Logistic s = logistic_of<FINE>(act == 2 ? c : c * __builtin_fmaf(q, SOPK_TANH_B, SOPK_TANH_A));
        const float inner = act == 2 ? c : c * __builtin_fmaf(q, 3.0f * SOPK_TANH_B, SOPK_TANH_A);
        const bool up = z >= 0.0f;
        const float m = up ? 1.0f : s.g;
        return m * __builtin_fmaf(inner, up ? s.g * s.g * s.w : s.w, 1.0f) * (d * s.w) * m;   // (m (1 + inner w) is at most 1.3 whatever z is)
    }
    if (act == 3) {
        const float b = fabsf(z), a = b > 40.0f ? 40.0f : b;            // (NaN stays)
        const Tail t = tail<FINE>(a);
        const float u = d * (t.g * __builtin_fmaf(-a, SOPK_PHI0, t.r)) * t.g;   // d (Phi(-a) - a phi(a))
        return z < 0.0f ? u : d - u;
    }
    return d;
}

}  // namespace sopk
#endif
