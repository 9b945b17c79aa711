// Activations and their slopes in binary32, over all of its range: 0 none, 1 relu, 2 silu, 3 gelu, 4 gelu by tanh (SOP_ACT_*).
//
// exp(-a) for a >= 0 is kept as p 2^-i, i = rint(a log2 e) and p within [0.7, 1.42]: what is small because of it leaves binary32's normal numbers only in the
// last step, where 2^-i is put on.  With a log2 e in two parts the error of p is that of the hardware's 2^t.
//   logistic(u)    w = 1 / (1 + exp(-|u|)); u >= 0: w, else p w 2^-i
//   silu           z logistic(z);             slope s + z s (1 - s)
//   gelu by tanh   z logistic(2 v), v = sqrt(2 / pi) (z + 0.044715 z^3): (1 + tanh v) / 2 = logistic(2 v)
//   gelu           z Phi(z), Phi the normal distribution.  Phi(-a) = phi(a) R(a), phi its density, R the Mills ratio, which is smooth: with t = 1 / (1 + 0.3 a),
//                  R = t P(t), P of degree 7 fitted here to R in 64 bits at 400 Chebyshev nodes of a in [0, 14.5] for the least relative error (1.7e-7).
//                  Slope Phi(z) + z phi(z): from -a, phi (R - a).
// Far out the arguments are clamped where the function has long been 0 or z: infinities give the limits, NaN stays.
#ifndef SOP_ACT_H
#define SOP_ACT_H
#include <hip/hip_runtime.h>

namespace sopk {

#define SOPK_LOG2E 1.44269504f                                          // log2(e) = LOG2E + LOG2E_LO
#define SOPK_LOG2E_LO 1.9259630e-08f
struct Fall { float p; int i; };                                        // p 2^-i
// 2^-(h + r), r small
__device__ __forceinline__ Fall fall_of(float h, float r)
{
    const float i = rintf(h), p = __builtin_amdgcn_exp2f(i - h);
    return Fall{__builtin_fmaf(p, r * -0.693147181f, p), (int)i};
}
// exp(-a), 0 <= a <= 1200
__device__ __forceinline__ Fall fall(float a)
{
    const float h = a * SOPK_LOG2E;
    return fall_of(h, __builtin_fmaf(a, SOPK_LOG2E, -h) + a * SOPK_LOG2E_LO);
}
__device__ __forceinline__ float within(float z, float far) { return z < -far ? -far : z > far ? far : z; }   // (NaN stays)
// logistic(u) = m w 2^-k, 1 - logistic(u) = rest
struct Logistic { float m, w, rest; int k; };
__device__ __forceinline__ Logistic logistic_of(float u)
{
    const Fall f = fall(fminf(fabsf(u), 1200.0f));
    const float e = __builtin_amdgcn_ldexpf(f.p, -f.i), w = __builtin_amdgcn_rcpf(1.0f + e);
    const bool up = u >= 0.0f;
    return Logistic{up ? 1.0f : f.p, w, up ? e * w : w, up ? 0 : -f.i};
}
// the coefficients of P / sqrt(2 pi)
#define SOPK_MILLS_0 0.119632013f
#define SOPK_MILLS_1 0.120712146f
#define SOPK_MILLS_2 0.100175917f
#define SOPK_MILLS_3 0.12769191f
#define SOPK_MILLS_4 -0.0520343035f
#define SOPK_MILLS_5 0.204557121f
#define SOPK_MILLS_6 -0.156158671f
#define SOPK_MILLS_7 0.0354238003f
// phi(a) sqrt(2 pi) = p 2^-i and R(a) / sqrt(2 pi), 0 <= a <= 40
struct Tail { Fall f; float r; };
__device__ __forceinline__ Tail tail(float a)
{
    const float q = a * a, lo = __builtin_fmaf(a, a, -q), h = q * (0.5f * SOPK_LOG2E);
    const Fall f = fall_of(h, __builtin_fmaf(q, 0.5f * SOPK_LOG2E, -h) + __builtin_fmaf(q, 0.5f * SOPK_LOG2E_LO, lo * (0.5f * SOPK_LOG2E)));
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(a, 0.3f, 1.0f));
    float r = SOPK_MILLS_7;
    r = __builtin_fmaf(r, t, SOPK_MILLS_6);
    r = __builtin_fmaf(r, t, SOPK_MILLS_5);
    r = __builtin_fmaf(r, t, SOPK_MILLS_4);
    r = __builtin_fmaf(r, t, SOPK_MILLS_3);
    r = __builtin_fmaf(r, t, SOPK_MILLS_2);
    r = __builtin_fmaf(r, t, SOPK_MILLS_1);
    r = __builtin_fmaf(r, t, SOPK_MILLS_0);
    return Tail{f, r * t};
}
#define SOPK_PHI0 0.398942280f                                          // 1 / sqrt(2 pi)
#define SOPK_TANH_A 1.59576912f                                         // 2 sqrt(2 / pi)
#define SOPK_TANH_B 0.0713548163f                                       // ... times 0.044715

__device__ __forceinline__ float act_of(int act, float z)
{
    if (act == 1) return z < 0.0f ? 0.0f : z;
    if (act == 2 || act == 4) {
        const Logistic s = logistic_of(act == 2 ? z : z * __builtin_fmaf(z * z, SOPK_TANH_B, SOPK_TANH_A));
        return __builtin_amdgcn_ldexpf((z < -1200.0f ? -1200.0f : z) * s.w * s.m, s.k);
    }
    if (act == 3) {
        const Tail t = tail(fminf(fabsf(z), 40.0f));
        const float below = t.f.p * t.r;
        return z >= 0.0f ? z * (1.0f - __builtin_amdgcn_ldexpf(below, -t.f.i)) : __builtin_amdgcn_ldexpf((z < -40.0f ? -40.0f : z) * below, -t.f.i);
    }
    return z;
}
// d times the slope at z
__device__ __forceinline__ float act_slope(int act, float z, float d)
{
    if (act == 1) return z <= 0.0f ? 0.0f : d;
    if (act == 2 || act == 4) {
        const float c = within(z, 1200.0f), q = c * c;
        const Logistic s = logistic_of(act == 2 ? c : c * __builtin_fmaf(q, SOPK_TANH_B, SOPK_TANH_A));
        const float inner = act == 2 ? c : c * __builtin_fmaf(q, 3.0f * SOPK_TANH_B, SOPK_TANH_A);
        return __builtin_amdgcn_ldexpf(d * s.m * s.w * __builtin_fmaf(inner, s.rest, 1.0f), s.k);
    }
    if (act == 3) {
        const float a = fminf(fabsf(z), 40.0f);
        const Tail t = tail(a);
        const float down = t.f.p * __builtin_fmaf(-a, SOPK_PHI0, t.r);  // (Phi(-a) - a phi(a)) 2^i
        const float r = z >= 0.0f ? d * (1.0f - __builtin_amdgcn_ldexpf(down, -t.f.i)) : __builtin_amdgcn_ldexpf(d * down, -t.f.i);
        return z != z ? z : r;
    }
    return d;
}

}  // namespace sopk
#endif
