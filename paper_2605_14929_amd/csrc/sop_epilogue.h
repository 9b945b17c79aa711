// Epilogue of a product: z = v + bias (kept where wanted), y = residual + scale act(z), all in binary32, each of z and y rounded once.  Results come by four
// neighbouring columns of a row a lane; what an epilogue reads is asked for ahead.
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
template <bool BF16, int ACT, int N> __device__ __forceinline__ void act_all(v4f (&z)[N])
{
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) z[j][i] = act_of<!BF16>(ACT, z[j][i]);
}
template <bool BF16, int N> __device__ __forceinline__ void act_by(int act, v4f (&z)[N])
{
    switch (act) {
    case 1: act_all<BF16, 1>(z); break;
    case 2: act_all<BF16, 2>(z); break;
    case 3: act_all<BF16, 3>(z); break;
    case 4: act_all<BF16, 4>(z);
    }
}
// the residual of column i of four
template <bool BF16> __device__ __forceinline__ float residual_of(const unsigned int* r, int i)
{
    return __uint_as_float(BF16 ? ((i & 1) ? r[i >> 1] & 0xFFFF0000u : r[i >> 1] << 16) : r[i]);
}
template <bool BF16, typename P> __device__ __forceinline__ void finish_four(const P& p, int m, int n, v4f v, const EpilogueOperands& o)
{
    if (m >= p.M || n >= p.N) return;
    const Epilogue& e = p.e;
    const int left = p.N - n;
    v = v + o.bias;
    if (e.z) put_columns<BF16>(e.z, (long long)m * e.ldz + n, left, v);
    v4f z[1] = {v};
    act_by<BF16>(e.act, z);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = e.residual ? __builtin_fmaf(z[0][i], e.scale, residual_of<BF16>(o.r, i)) : z[0][i] * e.scale;
    put_columns<BF16>(p.y, (long long)m * p.ldy + n, left, v);
}
// Four columns of a lane to or from a matrix in a window: offsets of the lane and of the wavefront, in bytes.
template <bool BF16> __device__ __forceinline__ void ask_four(unsigned int (&r)[4], const Window& w, unsigned int at, unsigned int uni)
{
    if constexpr (BF16) {
        const auto v = __builtin_amdgcn_raw_buffer_load_b64(resource(w), (int)at, (int)uni, 0);
        r[0] = (unsigned int)v[0]; r[1] = (unsigned int)v[1];
    } else {
        const auto v = __builtin_amdgcn_raw_buffer_load_b128(resource(w), (int)at, (int)uni, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = (unsigned int)v[i];
    }
}
// (A store of 16 bytes takes its data registers a moment after it has been issued.  Without a scalar offset the compiler keeps the next instruction from writing them that
// soon; with one it does not, and the first of the four arrived as what came after it.  So the sum of both offsets is the lane's.)
typedef unsigned int v2u __attribute__((ext_vector_type(2)));
typedef unsigned int v4u __attribute__((ext_vector_type(4)));
template <bool BF16> __device__ __forceinline__ void give_four(const Window& w, unsigned int at, unsigned int uni, v4f v)
{
    if constexpr (BF16) __builtin_amdgcn_raw_buffer_store_b64(v2u{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])}, resource(w), (int)at, (int)uni, 0);
    else __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u, v), resource(w), (int)(at + uni), 0, 0);
}
// Whether the part of a matrix of `rows` x `columns` from (m0, n0) on can go by such windows: all of it there, fours on their own alignment, 32-bit offsets.
template <typename P> __device__ __forceinline__ bool by_windows(const P& p, int m0, int n0, int rows, int columns, unsigned int size)
{
    const Epilogue& e = p.e;
    const unsigned long long on = (reinterpret_cast<unsigned long long>(p.y) | (unsigned long long)p.ldy * size | (e.residual ? reinterpret_cast<unsigned long long>(e.residual) | (unsigned long long)e.ldr * size : 0) |
                                   (e.z ? reinterpret_cast<unsigned long long>(e.z) | (unsigned long long)e.ldz * size : 0)) & (4 * size - 1);
    const long long far = (long long)(1 << 30) / (rows * (int)size);
    return on == 0 && m0 + rows <= p.M && n0 + columns <= p.N && p.ldy < far && (!e.residual || e.ldr < far) && (!e.z || e.ldz < far);
}
// The bias of a wavefront's 32 FN columns, in a place of its own in LDS: zeros where there is none
template <int FN, typename P> __device__ __forceinline__ void put_bias(const P& p, float* to, int n0, int lane)
{
#pragma unroll
    for (int c = 0; c < 32 * FN; c += 64) {
        const int n = n0 + c + lane;
        if (32 * FN - c >= 64 || lane < 32) to[c + lane] = p.e.bias && n < p.N ? p.e.bias[n] : 0.0f;
    }
}
// `count` squares of 32 x 32 that a wavefront has put into LDS from `place` on, 4 KB each, all of them inside y: the first is square `first` of the wavefront's, FN to a row
// of squares; its ROWS rows begin at m0, its columns at n0.  RES, Z: there is a residual, z is kept.  No branch stands between loads and stores, so that a square's residual, asked
// for two squares ahead, is waited for without the stores in between.
template <bool BF16, int FN, int ROWS, bool RES, bool Z, typename P> __device__ __forceinline__ void finish_whole(const P& p, const v4f* place, const float* bias, int first, int count, int m0, int n0, int lane)
{
    constexpr unsigned int SIZE = BF16 ? 2 : 4;
    const Epilogue& e = p.e;
    auto over = [&](const void* x, long long ld) { return window(reinterpret_cast<const char*>(x) + ((long long)m0 * ld + n0) * SIZE, (unsigned int)((ROWS - 1) * ld + 32 * FN) * SIZE); };
    const Window wy = over(p.y, p.ldy), wz = Z ? over(e.z, e.ldz) : wy, wr = RES ? over(e.residual, e.ldr) : wy;
    const unsigned int r8 = (unsigned int)(lane >> 3), c4 = 4 * (unsigned int)(lane & 7);
    const unsigned int aty = (r8 * (unsigned int)p.ldy + c4) * SIZE, atz = (r8 * (unsigned int)e.ldz + c4) * SIZE, atr = (r8 * (unsigned int)e.ldr + c4) * SIZE;
    struct Residual { unsigned int r[RES ? 4 : 1][4]; };
    auto ask = [&](Residual& o, int s) {
        if constexpr (RES) {
            const unsigned int q = (unsigned int)(first + (s < count ? s : count - 1)), row = q / FN * 32, column = q % FN * 32;
#pragma unroll
            for (int i = 0; i < 4; ++i) ask_four<BF16>(o.r[i], wr, atr, ((row + 8 * i) * (unsigned int)e.ldr + column) * SIZE);
        }
    };
    Residual next, after;
    ask(next, 0);
    ask(after, 1);
#pragma unroll 1
    for (int s = 0; s < count; ++s) {
        const Residual o = next;
        next = after;
        ask(after, s + 2);
        const unsigned int row = (unsigned int)((first + s) / FN) * 32, column = (unsigned int)((first + s) % FN) * 32;
        const v4f b = *reinterpret_cast<const v4f*>(bias + column + c4);
        v4f v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] = place[s * 256 + quarter_slot(i, lane)] + b;
            if constexpr (Z) give_four<BF16>(wz, atz, ((row + 8 * i) * (unsigned int)e.ldz + column) * SIZE, v[i]);
        }
        act_by<BF16>(e.act, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (RES) v[i][j] = __builtin_fmaf(v[i][j], e.scale, residual_of<BF16>(o.r[i], j));
                else v[i][j] *= e.scale;
            }
            give_four<BF16>(wy, aty, ((row + 8 * i) * (unsigned int)p.ldy + column) * SIZE, v[i]);
        }
    }
}
// ... or some of them outside y, or on odd addresses: four by four, each with its checks.  (From an odd address, every wait being for all stores before it, 4096 x 11008 x 4096 with
// gelu and z takes 253 us.  By windows 213, and with a residual 245; without an epilogue 182, with a bias 182, and a residual 205 (its 90 MB come in bursts, when all tiles end), with
// silu 197, with gelu 207: the vector ALUs, which are busy for 64 k of the 77 k cycles that gelu and z add.)
template <bool BF16, int FN, int ROWS, typename P> __device__ __forceinline__ void finish_squares(const P& p, const v4f* place, const float* bias, int first, int count, int m0, int n0, int lane)
{
    if (by_windows(p, m0, n0, ROWS, 32 * FN, BF16 ? 2 : 4)) {
        if (p.e.residual && p.e.z) finish_whole<BF16, FN, ROWS, true, true>(p, place, bias, first, count, m0, n0, lane);
        else if (p.e.residual) finish_whole<BF16, FN, ROWS, true, false>(p, place, bias, first, count, m0, n0, lane);
        else if (p.e.z) finish_whole<BF16, FN, ROWS, false, true>(p, place, bias, first, count, m0, n0, lane);
        else finish_whole<BF16, FN, ROWS, false, false>(p, place, bias, first, count, m0, n0, lane);
        return;
    }
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
