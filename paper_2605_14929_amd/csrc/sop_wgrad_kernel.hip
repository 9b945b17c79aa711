// Weight gradient from an 8-bit activation checkpoint: dw[n, k] = sum_m dy[m, n] x[m, k], x = code * 2^e with a scale for every block
// of 128 along k.
//
// The sum runs over the rows, and along them the scale changes at every step, so the 8-bit matrix instruction (one scale a row of its
// operand and 32 elements of the sum) cannot take it.  An 8-bit number times a power of two is a bf16 number, though: the
// checkpoint becomes bf16 exactly on its way into LDS, and the bf16 matrix instruction adds nothing but binary32 sums.
//
// Both operands arrive with the summed index outermost, the matrix instruction wants it innermost: a thread loads eight rows of two
// (dy) or four (x) columns, turns them in registers by byte permutations, and writes eight sums' worth of a column as one chunk.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "sop_linear.h"

namespace sopk {

// two neighbouring bf16 of a row, aligned or not
struct __attribute__((packed)) Pair { unsigned int v; };

template <int BN, int BK, int WR, int WC, bool X5>
__global__ __launch_bounds__(WR * WC * 64) void wgrad_kernel(const WgradParams p, int tiles_n, int tiles_k, int group)
{
    constexpr int NT = WR * WC * 64, FA = BN / WR / 16, FB = BK / WC / 16, ID = BN * 4 / NT, IX = BK * 2 / NT, STAGE = (BN + BK) * 128;
    static_assert(ID * NT == BN * 4 && IX * NT == BK * 2, "whole items");
    extern __shared__ __align__(16) unsigned char lds[];
    int tn, tk;
    tile_of(blockIdx.x, tiles_n * tiles_k, tiles_n, tiles_k, group, tn, tk);
    const int n0 = tn * BN, k0 = tk * BK, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r16 = lane & 15, q = lane >> 4;
    const int wn = wave / WC * (BN / WR), wk = wave % WC * (BK / WC);

    // columns of this thread's items.  A pair that reaches beyond the last column is read one column earlier and shifted; columns
    // beyond the matrix hold something, and their sums go nowhere.
    long long od[ID], ox[IX];
    int shift[ID];
    long long os[IX];
#pragma unroll
    for (int i = 0; i < ID; ++i) {
        const int c = n0 + 2 * ((i * NT + tid) % (BN / 2)), at = p.N < 2 ? 0 : min(c, p.N - 2);
        shift[i] = c > at ? 16 : 0;
        od[i] = at;
    }
#pragma unroll
    for (int i = 0; i < IX; ++i) {
        const int c = min(k0 + 4 * ((i * NT + tid) % (BK / 4)), (p.K - 1) & ~3);
        ox[i] = c;
        os[i] = c >> 7;
    }
    unsigned int d[ID][8], e[IX][8], s[IX][8];
    auto load = [&](int step) {
        const int base = step * 64;
        const bool whole = base + 64 <= p.M;
#pragma unroll
        for (int i = 0; i < ID; ++i) {
            const int m = base + (i * NT + tid) / (BN / 2) * 8;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const long long at = (long long)min(m + j, p.M - 1) * p.lddy + od[i];
                unsigned int v;
                if (p.N < 2) v = p.dy[at]; else v = reinterpret_cast<const Pair*>(p.dy + at)->v;
                d[i][j] = whole || m + j < p.M ? v >> shift[i] : 0u;
            }
        }
#pragma unroll
        for (int i = 0; i < IX; ++i) {
            const int m = base + (i * NT + tid) / (BK / 4) * 8;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const long long r = min(m + j, p.M - 1);
                const unsigned int v = *reinterpret_cast<const unsigned int*>(p.x + r * p.ldx + ox[i]);
                const unsigned int b = p.xs[r * p.ldxs + os[i]];
                e[i][j] = whole || m + j < p.M ? v : 0u;
                s[i][j] = whole || m + j < p.M ? b : 127u;
            }
        }
    };
    auto store = [&](unsigned char* to) {
#pragma unroll
        for (int i = 0; i < ID; ++i) {
            const int c = 2 * ((i * NT + tid) % (BN / 2)), g = (i * NT + tid) / (BN / 2);
            v4i lo, hi;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                lo[j] = (int)__builtin_amdgcn_perm(d[i][2 * j + 1], d[i][2 * j], 0x05040100u);
                hi[j] = (int)__builtin_amdgcn_perm(d[i][2 * j + 1], d[i][2 * j], 0x07060302u);
            }
            *reinterpret_cast<v4i*>(to + c * 128 + ((g ^ swz(c)) << 4)) = lo;
            *reinterpret_cast<v4i*>(to + (c + 1) * 128 + ((g ^ swz(c + 1)) << 4)) = hi;
        }
        to += BN * 128;
#pragma unroll
        for (int i = 0; i < IX; ++i) {
            const int c = 4 * ((i * NT + tid) % (BK / 4)), g = (i * NT + tid) / (BK / 4);
            unsigned int v[8][2];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float f = e8m0_value(s[i][j]);
                const v2bf a = X5 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(e[i][j], f, false) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(e[i][j], f, false);
                const v2bf b = X5 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(e[i][j], f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(e[i][j], f, true);
                v[j][0] = __builtin_bit_cast(unsigned int, a);
                v[j][1] = __builtin_bit_cast(unsigned int, b);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                v4i lo, hi;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    lo[j] = (int)__builtin_amdgcn_perm(v[2 * j + 1][h], v[2 * j][h], 0x05040100u);
                    hi[j] = (int)__builtin_amdgcn_perm(v[2 * j + 1][h], v[2 * j][h], 0x07060302u);
                }
                const int r = c + 2 * h;
                *reinterpret_cast<v4i*>(to + r * 128 + ((g ^ swz(r)) << 4)) = lo;
                *reinterpret_cast<v4i*>(to + (r + 1) * 128 + ((g ^ swz(r + 1)) << 4)) = hi;
            }
        }
    };

    v4f acc[FA][FB];
#pragma unroll
    for (int a = 0; a < FA; ++a)
#pragma unroll
        for (int b = 0; b < FB; ++b) acc[a][b] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    const int steps = (p.M + 63) >> 6;
    if (steps) load(0);
    for (int t = 0; t < steps; ++t) {
        unsigned char* half = lds + (t & 1) * STAGE;
        store(half);
        __syncthreads();
        if (t + 1 < steps) load(t + 1);
        bf16_step<FA, FB>(half, half + BN * 128, wn + r16, wk + r16, q, acc);
    }
#pragma unroll
    for (int a = 0; a < FA; ++a) {
        const int n = n0 + wn + a * 16 + r16;
        if (n >= p.N) continue;
#pragma unroll
        for (int b = 0; b < FB; ++b) {
            const int k = k0 + wk + b * 16 + 4 * q;
            if (k >= p.K) continue;
            const long long at = (long long)n * p.lddw + k;
            const bool four = k + 3 < p.K;
            if (p.out_bf16) {
                uint16_t* w = reinterpret_cast<uint16_t*>(p.dw) + at;
                v4f v = acc[a][b];
                if (p.accumulate) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) if (k + i < p.K) v[i] += __uint_as_float((unsigned int)w[i] << 16);
                }
                if (four && (reinterpret_cast<uintptr_t>(w) & 7) == 0) *reinterpret_cast<uint2*>(w) = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
                else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) if (k + i < p.K) w[i] = (uint16_t)bf16_bits(v[i]);
                }
            } else {
                float* w = reinterpret_cast<float*>(p.dw) + at;
                v4f v = acc[a][b];
                if (four && (reinterpret_cast<uintptr_t>(w) & 15) == 0) {
                    if (p.accumulate) v += *reinterpret_cast<const v4f*>(w);
                    *reinterpret_cast<v4f*>(w) = v;
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) if (k + i < p.K) w[i] = p.accumulate ? v[i] + w[i] : v[i];
                }
            }
        }
    }
}

template <int BN, int BK, int WR, int WC, bool X5> static hipError_t wgrad_go(const WgradParams& p, hipStream_t st)
{
    const int tn = (p.N + BN - 1) / BN, tk = (p.K + BK - 1) / BK, bytes = 2 * (BN + BK) * 128;
    if (bytes > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&wgrad_kernel<BN, BK, WR, WC, X5>), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((wgrad_kernel<BN, BK, WR, WC, X5>), dim3((unsigned)(tn * tk)), dim3(WR * WC * 64), bytes, st, p, tn, tk, 8);
    return hipGetLastError();
}
template <bool X5> static hipError_t wgrad_pick(const WgradParams& p, int n_cu, hipStream_t st)
{
    auto tiles = [&](int a, int b) { return (long long)((p.N + a - 1) / a) * ((p.K + b - 1) / b); };
    if (tiles(256, 256) >= n_cu) return wgrad_go<256, 256, 2, 4, X5>(p, st);
    if (tiles(128, 128) >= n_cu) return wgrad_go<128, 128, 2, 2, X5>(p, st);
    return wgrad_go<64, 128, 2, 2, X5>(p, st);
}

}  // namespace sopk

extern "C" hipError_t sopk_wgrad_launch(const WgradParams* p, int x_e5m2, int n_cu, void* stream)
{
    return x_e5m2 ? sopk::wgrad_pick<true>(*p, n_cu, (hipStream_t)stream) : sopk::wgrad_pick<false>(*p, n_cu, (hipStream_t)stream);
}
