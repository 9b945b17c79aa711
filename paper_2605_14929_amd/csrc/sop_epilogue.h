// Epilogue of a product: z = v + bias (kept where wanted), y = residual + scale act(z), all in binary32, each of z and y rounded once.  Results come by four
// neighbouring columns of a row a lane; what an epilogue reads for the next four is on its way while these are finished.
#ifndef SOP_EPILOGUE_H
#define SOP_EPILOGUE_H
#include "sop_act.h"
#include "sop_linear.h"

namespace sopk {

struct EpilogueOperands { v4f bias; unsigned int r[4]; };               // residual as it lies in memory: two words of bf16, or four

template <bool BF16, typename P> __device__ __forceinline__ EpilogueOperands epilogue_operands(const P& p, int m, int n)
{
    EpilogueOperands o{v4f{0.0f, 0.0f, 0.0f, 0.0f}, {0, 0, 0, 0}};
    const Epilogue& e = p.e;
    if (m >= p.M || n >= p.N) return o;
    if (n + 3 < p.N) {
        if (e.bias) o.bias = reinterpret_cast<const FourWords*>(e.bias + n)->v;
        if (e.residual) {
            const long long at = (long long)m * e.ldr + n;
            if constexpr (BF16) {
                const FourHalves h = *reinterpret_cast<const FourHalves*>(reinterpret_cast<const uint16_t*>(e.residual) + at);
                o.r[0] = h.v[0]; o.r[1] = h.v[1];
            } else {
                const v4f h = reinterpret_cast<const FourWords*>(reinterpret_cast<const float*>(e.residual) + at)->v;
#pragma unroll
                for (int i = 0; i < 4; ++i) o.r[i] = __float_as_uint(h[i]);
            }
        }
        return o;
    }
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        if (n + i >= p.N) continue;
        if (e.bias) o.bias[i] = e.bias[n + i];
        if (e.residual) {
            const long long at = (long long)m * e.ldr + n + i;
            if constexpr (BF16) o.r[i >> 1] |= (unsigned int)reinterpret_cast<const uint16_t*>(e.residual)[at] << (16 * (i & 1));
            else o.r[i] = reinterpret_cast<const unsigned int*>(e.residual)[at];
        }
    }
    return o;
}
template <bool BF16> __device__ __forceinline__ void put_columns(void* y, long long at, int left, v4f v)
{
    if constexpr (BF16) {
        uint16_t* to = reinterpret_cast<uint16_t*>(y) + at;
        if (left >= 4) { put_four(to, v); return; }
#pragma unroll
        for (int i = 0; i < 3; ++i) if (i < left) to[i] = (uint16_t)bf16_bits(v[i]);
    } else {
        float* to = reinterpret_cast<float*>(y) + at;
        if (left >= 4) { put_four(to, v); return; }
#pragma unroll
        for (int i = 0; i < 3; ++i) if (i < left) to[i] = v[i];
    }
}
template <int ACT> __device__ __forceinline__ v4f act_four(v4f z)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) z[i] = act_of(ACT, z[i]);
    return z;
}
template <bool BF16, typename P> __device__ __forceinline__ void finish_four(const P& p, int m, int n, v4f v, const EpilogueOperands& o)
{
    if (m >= p.M || n >= p.N) return;
    const Epilogue& e = p.e;
    const int left = p.N - n;
    v = v + o.bias;
    if (e.z) put_columns<BF16>(e.z, (long long)m * e.ldz + n, left, v);
    switch (e.act) {
    case 1: v = act_four<1>(v); break;
    case 2: v = act_four<2>(v); break;
    case 3: v = act_four<3>(v); break;
    case 4: v = act_four<4>(v);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned int h = BF16 ? ((i & 1) ? o.r[i >> 1] & 0xFFFF0000u : o.r[i >> 1] << 16) : o.r[i];
        v[i] = e.residual ? __builtin_fmaf(v[i], e.scale, __uint_as_float(h)) : v[i] * e.scale;
    }
    put_columns<BF16>(p.y, (long long)m * p.ldy + n, left, v);
}
// `count` squares of 32 x 32 that a wavefront has put into LDS from `place` on, 4 KB each: the first is square `first` of the wavefront's, FN to a row of squares;
// the wavefront's rows begin at m0, its columns at n0.
template <bool BF16, int FN, typename P> __device__ __forceinline__ void finish_squares(const P& p, const v4f* place, int first, int count, int m0, int n0, int lane)
{
    auto row = [&](int q) { return m0 + (first + (q >> 2)) / FN * 32 + 8 * (q & 3) + (lane >> 3); };
    auto column = [&](int q) { return n0 + (first + (q >> 2)) % FN * 32 + 4 * (lane & 7); };
    EpilogueOperands here = epilogue_operands<BF16>(p, row(0), column(0));
#pragma unroll 1
    for (int q = 0; q < 4 * count; ++q) {
        const EpilogueOperands next = q + 1 < 4 * count ? epilogue_operands<BF16>(p, row(q + 1), column(q + 1)) : here;
        finish_four<BF16>(p, row(q), column(q), place[(q >> 2) * 256 + quarter_slot(q & 3, lane)], here);
        here = next;
    }
}

}  // namespace sopk
#endif
