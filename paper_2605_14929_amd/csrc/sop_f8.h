// Eight elements a lane: loads, stores, and the rounding of a block of 128 of a row (sixteen lanes) into 8-bit floats under its scale.
#ifndef SOP_F8_H
#define SOP_F8_H
#include "sop_linear.h"

namespace sopk {

template <bool E5M2> __device__ __forceinline__ unsigned int scale_byte(unsigned int amax_bits)
{
    const int E = (int)(amax_bits >> 23) - 127, e = E - (E5M2 ? 15 : 8) + ((amax_bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return amax_bits == 0 ? 127u : (unsigned int)((e < -126 ? -126 : e) + 127);
}
__device__ __forceinline__ float inverse_scale(unsigned int b) { return __uint_as_float((254u - b) << 23); }   // b within 1 .. 247

template <bool E5M2> __device__ __forceinline__ uint2 codes8(const float (&v)[8], float inv)
{
    int lo = 0, hi = 0;
    if (E5M2) {
        lo = __builtin_amdgcn_cvt_pk_bf8_f32(v[0] * inv, v[1] * inv, lo, false);
        lo = __builtin_amdgcn_cvt_pk_bf8_f32(v[2] * inv, v[3] * inv, lo, true);
        hi = __builtin_amdgcn_cvt_pk_bf8_f32(v[4] * inv, v[5] * inv, hi, false);
        hi = __builtin_amdgcn_cvt_pk_bf8_f32(v[6] * inv, v[7] * inv, hi, true);
    } else {
        lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * inv, v[1] * inv, lo, false);
        lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[2] * inv, v[3] * inv, lo, true);
        hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[4] * inv, v[5] * inv, hi, false);
        hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[6] * inv, v[7] * inv, hi, true);
    }
    return make_uint2((unsigned int)lo, (unsigned int)hi);
}

// eight elements of a row from column k on; zero beyond K
template <bool BF16, bool VEC> __device__ __forceinline__ void load8(const void* x, long long at, int left, float (&v)[8])
{
    if (BF16) {
        const uint16_t* p = reinterpret_cast<const uint16_t*>(x) + at;
        if (VEC && left >= 8) {
            const uint4 t = *reinterpret_cast<const uint4*>(p);
            const unsigned int w[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i < left ? __uint_as_float((unsigned int)p[i] << 16) : 0.0f;
        }
    } else {
        const float* p = reinterpret_cast<const float*>(x) + at;
        if (VEC && left >= 8) {
            const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i < left ? p[i] : 0.0f;
        }
    }
}
template <bool BF16, bool VEC> __device__ __forceinline__ void store8(void* y, long long at, int left, const float (&v)[8])
{
    if (BF16) {
        uint16_t* p = reinterpret_cast<uint16_t*>(y) + at;
        if (VEC && left >= 8) {
            *reinterpret_cast<uint4*>(p) = make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7]));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) if (i < left) p[i] = (uint16_t)bf16_bits(v[i]);
        }
    } else {
        float* p = reinterpret_cast<float*>(y) + at;
        if (VEC && left >= 8) {
            *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) if (i < left) p[i] = v[i];
        }
    }
}
__device__ __forceinline__ void store_codes8(unsigned char* p, int left, uint2 q)   // p: 8-byte aligned
{
    if (left >= 8) { *reinterpret_cast<uint2*>(p) = q; return; }
#pragma unroll
    for (int i = 0; i < 8; ++i) if (i < left) p[i] = (unsigned char)((i < 4 ? q.x >> (8 * i) : q.y >> (8 * i - 32)) & 0xFFu);
}

// largest |x| of eight elements, as bits (they order as the numbers do); infinities and NaN leave no trace in `finite`
__device__ __forceinline__ unsigned int amax8(const float (&v)[8], bool finite_only)
{
    unsigned int a = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const unsigned int b = __float_as_uint(v[i]) & 0x7FFFFFFFu;
        a = max(a, finite_only && b >= 0x7F800000u ? 0u : b);
    }
    return a;
}
// maximum over the sixteen lanes of a row (every lane of the row receives it)
__device__ __forceinline__ unsigned int row_max(unsigned int a)
{
    a = max(a, (unsigned int)__builtin_amdgcn_update_dpp(0, (int)a, 0x128, 0xF, 0xF, false));   // row_ror:8
    a = max(a, (unsigned int)__builtin_amdgcn_update_dpp(0, (int)a, 0x124, 0xF, 0xF, false));
    a = max(a, (unsigned int)__builtin_amdgcn_update_dpp(0, (int)a, 0x122, 0xF, 0xF, false));
    a = max(a, (unsigned int)__builtin_amdgcn_update_dpp(0, (int)a, 0x121, 0xF, 0xF, false));
    return a;
}
// a block of one row, eight elements in each of sixteen lanes (all lanes of the wavefront take part)
template <bool E5M2> __device__ __forceinline__ void quantize_row_block(const float (&v)[8], const F8Out& o, long long m, long long k, int left)
{
    unsigned int a = row_max(amax8(v, false));
    if (a >= 0x7F800000u) a = row_max(amax8(v, true));                  // (the same for all lanes of a row; rows apart do not meet)
    const unsigned int b = scale_byte<E5M2>(a);
    if (left <= 0) return;
    store_codes8(o.codes + m * o.ldc + k, left, codes8<E5M2>(v, inverse_scale(b)));
    if ((threadIdx.x & 15) == 0) o.scales[m * o.lds + (k >> 7)] = (unsigned char)b;
}

}  // namespace sopk
#endif
