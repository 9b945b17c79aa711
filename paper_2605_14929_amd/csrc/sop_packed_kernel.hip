// Product with packed codebook weights: y[m, n] = sum_k x[m, k] w[n, k], w = s L_sel[code], with the scale words (sign, magnitude,
// selector) and n-bit code payloads that the packing writes.
//
// A weight is formed in binary32 from its scale and its codebook entry and rounded once, to bf16, for the bf16 matrix instruction (the
// activations are bf16 too, and the weight's own quantisation error is some hundred times larger than that rounding); sums are binary32.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "sop_linear.h"

namespace sopk {

struct __attribute__((packed)) U16 { uint16_t v; };
struct __attribute__((packed)) U32 { uint32_t v; };

// eight codes of NB bits: NB bytes at any address, no byte more
template <int NB> __device__ __forceinline__ unsigned long long eight_codes(const unsigned char* p)
{
    if (NB == 1) return p[0];
    if (NB == 2) return reinterpret_cast<const U16*>(p)->v;
    if (NB == 3) return (unsigned int)reinterpret_cast<const U16*>(p)->v | (unsigned int)p[2] << 16;
    if (NB == 4) return reinterpret_cast<const U32*>(p)->v;
    if (NB == 5) return reinterpret_cast<const U32*>(p)->v | (unsigned long long)p[4] << 32;
    return reinterpret_cast<const U32*>(p)->v | (unsigned long long)reinterpret_cast<const U16*>(p + 4)->v << 32;
}

// scale word -> the scale with its sign; which codebook
__device__ __forceinline__ float word_scale(const PackedMmParams& p, unsigned int w)
{
    const unsigned int mag = (w >> p.mag_shift) & (unsigned int)p.mag_mask, e = mag >> p.man_bits, f = mag & (unsigned int)p.man_mask;
    float s = __builtin_amdgcn_ldexpf((float)(e ? f + (unsigned int)p.man_mask + 1u : f), (int)(e ? e : 1u) + p.exp_off);
    if (p.sign_pos >= 0 && (w >> p.sign_pos & 1u)) s = -s;
    return s;
}
__device__ __forceinline__ int word_table(const PackedMmParams& p, unsigned int w)
{
    return p.sel_pos >= 0 ? (int)(w >> p.sel_pos & 1u) * SOP_K_PACKED_TAB : 0;
}

// eight weights as bf16
template <int NB> __device__ __forceinline__ v4i eight_weights(unsigned long long codes, const float* tab, float s)
{
    v4i r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int a = (int)(codes >> (2 * i * NB)) & ((1 << NB) - 1), b = (int)(codes >> ((2 * i + 1) * NB)) & ((1 << NB) - 1);
        r[i] = (int)bf16_pair(s * tab[a], s * tab[b]);
    }
    return r;
}

__device__ __forceinline__ void store_y(const PackedMmParams& p, int m, int n, v4f v)
{
    if (m >= p.M || n >= p.N) return;
    uint16_t* y = p.y + (long long)m * p.ldy + n;
    if (n + 3 < p.N && (reinterpret_cast<uintptr_t>(y) & 7) == 0) {
        *reinterpret_cast<uint2*>(y) = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) if (n + i < p.N) y[i] = (uint16_t)bf16_bits(v[i]);
    }
}

// ---- few rows of x: FM x 16 of them by 16 columns a workgroup, K dealt out to its eight wavefronts, 128 elements a step: a lane takes
// 32 neighbouring codes of its row, eight for each of four matrix instructions, and the same elements of x.
template <int NB, int FM>
__global__ __launch_bounds__(512) void packed_rows_kernel(const PackedMmParams p)
{
    constexpr int W = 8;
    __shared__ float tab[2 * SOP_K_PACKED_TAB];
    __shared__ v4f part[W][FM][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r16 = lane & 15, q = lane >> 4;
    if (tid < 2 * SOP_K_PACKED_TAB) tab[tid] = p.tab[tid / SOP_K_PACKED_TAB][tid % SOP_K_PACKED_TAB];
    __syncthreads();
    const int n0 = blockIdx.x * 16, n = min(n0 + r16, p.N - 1), lg = 31 - __builtin_clz(p.g);
    const uint16_t* words = p.words + (long long)n * (p.K >> lg);
    const unsigned char* pay = p.payload + (long long)n * (p.K / 8) * NB;
    const uint16_t* xr[FM];
#pragma unroll
    for (int a = 0; a < FM; ++a) xr[a] = p.x + (long long)min(a * 16 + r16, p.M - 1) * p.ldx;
    v4f acc[FM];
#pragma unroll
    for (int a = 0; a < FM; ++a) acc[a] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    const int steps = (p.K + 127) >> 7;
    for (int t = wave; t < steps; t += W) {
        const int k = t * 128 + q * 32;
        unsigned long long c[4];
        unsigned int w[4];
        v8bf x[FM][4];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int ks = k + 8 * s;
            const bool in = ks < p.K;
            c[s] = in ? eight_codes<NB>(pay + (ks >> 3) * NB) : 0;
            w[s] = in ? words[ks >> lg] : 0;
#pragma unroll
            for (int a = 0; a < FM; ++a) {
                v4i z = {0, 0, 0, 0};
                if (in) z = *reinterpret_cast<const v4i*>(xr[a] + ks);
                x[a][s] = __builtin_bit_cast(v8bf, z);
            }
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const bool in = k + 8 * s < p.K;
            v4i u = eight_weights<NB>(c[s], tab + word_table(p, w[s]), word_scale(p, w[s]));
            if (!in) u = v4i{0, 0, 0, 0};
#pragma unroll
            for (int a = 0; a < FM; ++a) acc[a] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, u), x[a][s], acc[a], 0, 0, 0);
        }
    }
#pragma unroll
    for (int a = 0; a < FM; ++a) part[wave][a][lane] = acc[a];
    __syncthreads();
    for (int a = wave; a < FM; a += W) {
        v4f s = part[0][a][lane];
#pragma unroll
        for (int i = 1; i < W; ++i) s += part[i][a][lane];
        store_y(p, a * 16 + r16, n0 + 4 * q, s);
    }
}

// ---- tiles: BM x BN of y, 64 elements along K a step, two steps in LDS.  The weights are formed once a tile, on their way into LDS.
template <int NB, int BM, int BN, int WR, int WC>
__global__ __launch_bounds__(WR * WC * 64) void packed_tile_kernel(const PackedMmParams p, int tiles_m, int tiles_n, int group)
{
    constexpr int NT = WR * WC * 64, FM = BM / WR / 16, FN = BN / WC / 16, CX = BM * 8 / NT, IW = BN * 4 / NT, STAGE = (BM + BN) * 128;
    static_assert(IW * NT == BN * 4, "whole items");
    extern __shared__ __align__(16) unsigned char lds[];
    __shared__ float tab[2 * SOP_K_PACKED_TAB];
    int tm, tn;
    tile_of(blockIdx.x, tiles_m * tiles_n, tiles_m, tiles_n, group, tm, tn);
    const int m0 = tm * BM, n0 = tn * BN, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r16 = lane & 15, q = lane >> 4;
    const int wm = wave / WC * (BM / WR), wn = wave % WC * (BN / WC), lg = 31 - __builtin_clz(p.g);
    if (tid < 2 * SOP_K_PACKED_TAB) tab[tid] = p.tab[tid / SOP_K_PACKED_TAB][tid % SOP_K_PACKED_TAB];
    const unsigned char* xb = reinterpret_cast<const unsigned char*>(p.x + (long long)m0 * p.ldx);
    unsigned int ox[CX];                                                // (a row of x has at most 2^22 elements: the entry point's check)
#pragma unroll
    for (int i = 0; i < CX; ++i) {
        const int c = i * NT + tid, r = c >> 3;
        ox[i] = (unsigned int)min(r, p.M - 1 - m0) * (unsigned int)(p.ldx * 2) + (((c & 7) ^ swz(r)) << 4);
    }
    const Window xw = window(xb, (unsigned int)(min(BM, p.M - m0) - 1) * (unsigned int)(p.ldx * 2) + (unsigned int)p.K * 2);
    auto load_x = [&](int t) {
        unsigned char* to = lds + (t & 1) * STAGE;
        const unsigned char* xk = xb + (long long)t * 128;
        if (t * 64 + 64 <= p.K) {
#pragma unroll
            for (int i = 0; i < CX; ++i) load_to_lds(xw, ox[i], t * 128, to + (i * NT + (wave << 6)) * 16);
        } else {
            const int left = (p.K - t * 64) * 2;
#pragma unroll
            for (int i = 0; i < CX; ++i) {
                const int c = i * NT + tid;
                v4i v = {0, 0, 0, 0};
                if ((((c & 7) ^ swz(c >> 3)) << 4) < left) v = *reinterpret_cast<const v4i*>(xk + ox[i]);   // (K is a multiple of eight: whole chunks)
                *reinterpret_cast<v4i*>(to + c * 16) = v;
            }
        }
    };
    // an item: sixteen codes of a row, four items a row and step
    const long long per_row = p.K >> lg;
    unsigned long long c[IW][2];
    unsigned int w[IW][2];
    auto load_w = [&](int t) {
#pragma unroll
        for (int i = 0; i < IW; ++i) {
            const int id = i * NT + tid, k = t * 64 + (id & 3) * 16;
            const long long n = min(n0 + (id >> 2), p.N - 1);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const bool in = k + 8 * h < p.K;
                c[i][h] = in ? eight_codes<NB>(p.payload + (n * (p.K >> 3) + ((k >> 3) + h)) * NB) : 0;
                w[i][h] = in ? p.words[n * per_row + ((k + 8 * h) >> lg)] : 0;
            }
        }
    };
    auto store_w = [&](int t) {
        unsigned char* to = lds + (t & 1) * STAGE + BM * 128;
#pragma unroll
        for (int i = 0; i < IW; ++i) {
            const int id = i * NT + tid, r = id >> 2, k = t * 64 + (id & 3) * 16;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                v4i u = eight_weights<NB>(c[i][h], tab + word_table(p, w[i][h]), word_scale(p, w[i][h]));
                if (k + 8 * h >= p.K) u = v4i{0, 0, 0, 0};
                *reinterpret_cast<v4i*>(to + r * 128 + ((((id & 3) * 2 + h) ^ swz(r)) << 4)) = u;
            }
        }
    };
    v4f acc[FM][FN];
#pragma unroll
    for (int a = 0; a < FM; ++a)
#pragma unroll
        for (int b = 0; b < FN; ++b) acc[a][b] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    const int steps = (p.K + 63) >> 6;
    load_x(0);
    load_w(0);
    __syncthreads();                                                    // the codebooks are there
    store_w(0);
    for (int t = 0; t < steps; ++t) {
        wait_loads();
        __syncthreads();
        const bool more = t + 1 < steps;
        if (more) { load_x(t + 1); load_w(t + 1); }
        const unsigned char* half = lds + (t & 1) * STAGE;
        bf16_step<FM, FN>(half, half + BM * 128, wm + r16, wn + r16, q, acc);
        if (more) store_w(t + 1);
    }
#pragma unroll
    for (int a = 0; a < FM; ++a)
#pragma unroll
        for (int b = 0; b < FN; ++b) store_y(p, m0 + wm + a * 16 + r16, n0 + wn + b * 16 + 4 * q, acc[a][b]);
}

template <int NB, int FM> static hipError_t rows_go(const PackedMmParams& p, hipStream_t st)
{
    hipLaunchKernelGGL((packed_rows_kernel<NB, FM>), dim3((unsigned)((p.N + 15) / 16)), dim3(512), 0, st, p);
    return hipGetLastError();
}
template <int NB, int BM, int BN, int WR, int WC> static hipError_t tile_go(const PackedMmParams& p, hipStream_t st)
{
    const int tm = (p.M + BM - 1) / BM, tn = (p.N + BN - 1) / BN, bytes = 2 * (BM + BN) * 128;
    if (bytes > 64 * 1024 - 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&packed_tile_kernel<NB, BM, BN, WR, WC>), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((packed_tile_kernel<NB, BM, BN, WR, WC>), dim3((unsigned)(tm * tn)), dim3(WR * WC * 64), bytes, st, p, tm, tn, 8);
    return hipGetLastError();
}
template <int NB> static hipError_t packed_pick(const PackedMmParams& p, int n_cu, hipStream_t st)
{
    auto tiles = [&](int bm, int bn) { return (long long)((p.M + bm - 1) / bm) * ((p.N + bn - 1) / bn); };
    if (p.M <= 16) return rows_go<NB, 1>(p, st);
    if (p.M <= 32) return rows_go<NB, 2>(p, st);
    if (tiles(256, 256) >= n_cu) return tile_go<NB, 256, 256, 2, 4>(p, st);
    if (tiles(128, 128) >= n_cu) return tile_go<NB, 128, 128, 2, 2>(p, st);
    return tile_go<NB, 64, 64, 2, 2>(p, st);
}

}  // namespace sopk

extern "C" hipError_t sopk_packed_launch(const PackedMmParams* p, int n_cu, void* stream)
{
    hipStream_t st = (hipStream_t)stream;
    switch (p->n_bits) {
    case 1: return sopk::packed_pick<1>(*p, n_cu, st);
    case 2: return sopk::packed_pick<2>(*p, n_cu, st);
    case 3: return sopk::packed_pick<3>(*p, n_cu, st);
    case 4: return sopk::packed_pick<4>(*p, n_cu, st);
    case 5: return sopk::packed_pick<5>(*p, n_cu, st);
    case 6: return sopk::packed_pick<6>(*p, n_cu, st);
    default: return hipErrorInvalidValue;
    }
}
