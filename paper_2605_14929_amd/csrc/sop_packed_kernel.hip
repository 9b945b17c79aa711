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
template <int N> struct __attribute__((packed)) Words { uint32_t v[N]; };
struct Codes { unsigned int lo, hi; };                                  // eight codes, the first in the lowest bits

// eight codes of NB bits: NB bytes at any address, no byte more
template <int NB> __device__ __forceinline__ Codes eight_codes(const unsigned char* p)
{
    if (NB == 1) return Codes{p[0], 0};
    if (NB == 2) return Codes{reinterpret_cast<const U16*>(p)->v, 0};
    if (NB == 3) return Codes{(unsigned int)reinterpret_cast<const U16*>(p)->v | (unsigned int)p[2] << 16, 0};
    if (NB == 4) return Codes{reinterpret_cast<const U32*>(p)->v, 0};
    if (NB == 5) return Codes{reinterpret_cast<const U32*>(p)->v, p[4]};
    return Codes{reinterpret_cast<const U32*>(p)->v, reinterpret_cast<const U16*>(p + 4)->v};
}
// the s-th eight of 32 codes that were read as NB words
template <int NB> __device__ __forceinline__ Codes eight_of(const unsigned int (&w)[NB], int s)
{
    const int bit = 8 * NB * s, at = bit >> 5, sh = bit & 31;
    Codes c;
    c.lo = sh == 0 ? w[at] : __builtin_amdgcn_alignbit(at + 1 < NB ? w[at + 1] : 0u, w[at], (unsigned int)sh);
    c.hi = NB <= 4 || at + 1 >= NB ? 0u : (sh == 0 ? w[at + 1] : __builtin_amdgcn_alignbit(at + 2 < NB ? w[at + 2] : 0u, w[at + 1], (unsigned int)sh));
    return c;
}

// scale word -> the scale with its sign; which codebook
__device__ __forceinline__ float word_scale(const PackedMmParams& p, unsigned int w)
{
    const unsigned int mag = (w >> p.mag_shift) & (unsigned int)p.mag_mask, e = mag >> p.man_bits, f = mag & (unsigned int)p.man_mask;
    const float s = __builtin_amdgcn_ldexpf((float)(e ? f + (unsigned int)p.man_mask + 1u : f), (int)(e ? e : 1u) + p.exp_off);
    return __uint_as_float(__float_as_uint(s) | (w << p.sign_up & 0x80000000u));
}
// Codebooks in LDS: the second behind the first at once, so that up to five bits a lane's look-up in either goes to a bank of its own entry.
template <int NB> __device__ __forceinline__ unsigned int word_table(const PackedMmParams& p, unsigned int w)   // in bytes
{
    return (w >> p.sel_pos & (unsigned int)p.sel_mask) << (NB + 2);
}
template <int NB> __device__ __forceinline__ void put_codebooks(const PackedMmParams& p, float* tab, int tid)
{
    if (tid < 2 << NB) tab[tid] = p.tab[tid >> NB][tid & ((1 << NB) - 1)];
}

// eight weights as bf16; `book` = the codebook's place in LDS, in bytes from tab (a multiple of its size)
template <int NB> __device__ __forceinline__ v4i eight_weights(Codes c, const float* tab, unsigned int book, float s)
{
    constexpr unsigned int MASK = ((1u << NB) - 1u) << 2;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {                                       // the code's entry, four bytes each: its bits moved to bit 2
        const int at = NB * i - 2;
        const unsigned int m = at < 0 ? c.lo << -at : at + NB + 2 <= 32 ? c.lo >> at : at >= 32 ? c.hi >> (at - 32) : __builtin_amdgcn_alignbit(c.hi, c.lo, (unsigned int)at);
        v[i] = *reinterpret_cast<const float*>(reinterpret_cast<const unsigned char*>(tab) + ((m & MASK) | book));
    }
    v4i r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = (int)bf16_pair(s * v[2 * i], s * v[2 * i + 1]);
    return r;
}
__device__ __forceinline__ v4i only_if(bool in, v4i v)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = in ? v[i] : 0;
    return v;
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

// ---- few rows of x: FM x 16 of them by 16 columns a workgroup, K dealt out to its W wavefronts, 128 elements a step, U steps of a
// wavefront in flight: a lane takes 32 neighbouring codes of its row, eight for each of four matrix instructions, and the same elements of x.
// WPL: scale words of 32 codes (4, 2 or 1 for g = 8, 16 and more).
template <int NB, int FM, int U, int W, int WPL>
__global__ __launch_bounds__(W * 64) void packed_rows_kernel(const PackedMmParams p)
{
    __shared__ __align__(16) float tab[2 << NB];
    __shared__ v4f part[W][FM][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r16 = lane & 15, q = lane >> 4;
    const int n0 = blockIdx.x * 16, n = min(n0 + r16, p.N - 1), lg = 31 - __builtin_clz(p.g);
    const uint16_t* words = p.words + (long long)n * (p.K >> lg);
    const unsigned char* pay = p.payload + (long long)n * (p.K / 8) * NB;
    const uint16_t* xr[FM];
#pragma unroll
    for (int a = 0; a < FM; ++a) xr[a] = p.x + (long long)min(a * 16 + r16, p.M - 1) * p.ldx;
    v4f acc[FM];
#pragma unroll
    for (int a = 0; a < FM; ++a) acc[a] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    const int whole = p.K >> 7, steps = (p.K + 127) >> 7;
    struct Step { unsigned int c[NB], w[WPL == 4 ? 2 : 1]; v4i x[FM][4]; };
    auto load = [&](int t, Step& z) {
        const int k = t * 128 + q * 32;
        const Words<NB> c = *reinterpret_cast<const Words<NB>*>(pay + (k >> 3) * NB);
#pragma unroll
        for (int i = 0; i < NB; ++i) z.c[i] = c.v[i];
        const uint16_t* w = words + (k >> lg);
        if (WPL == 1) z.w[0] = w[0];
        else {
            const Words<WPL == 4 ? 2 : 1> v = *reinterpret_cast<const Words<WPL == 4 ? 2 : 1>*>(w);
#pragma unroll
            for (int i = 0; i < (WPL == 4 ? 2 : 1); ++i) z.w[i] = v.v[i];
        }
#pragma unroll
        for (int a = 0; a < FM; ++a)
#pragma unroll
            for (int s = 0; s < 4; ++s) z.x[a][s] = *reinterpret_cast<const v4i*>(xr[a] + k + 8 * s);
    };
    auto add = [&](const Step& z) {
        float sc[WPL];
        unsigned int book[WPL];
#pragma unroll
        for (int i = 0; i < WPL; ++i) {
            const unsigned int w = z.w[i >> 1] >> (16 * (i & 1)) & 0xFFFFu;
            sc[i] = word_scale(p, w);
            book[i] = word_table<NB>(p, w);
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const v4i u = eight_weights<NB>(eight_of<NB>(z.c, s), tab, book[s * WPL / 4], sc[s * WPL / 4]);
#pragma unroll
            for (int a = 0; a < FM; ++a) acc[a] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, u), __builtin_bit_cast(v8bf, z.x[a][s]), acc[a], 0, 0, 0);
        }
    };
    put_codebooks<NB>(p, tab, tid);
    __syncthreads();
    int t = wave;
    for (; t + (U - 1) * W < whole; t += U * W) {
        Step z[U];
#pragma unroll
        for (int u = 0; u < U; ++u) load(t + u * W, z[u]);
        __builtin_amdgcn_sched_barrier(0);                              // (every load of the U steps is asked for before the first is used)
#pragma unroll
        for (int u = 0; u < U; ++u) add(z[u]);
    }
#pragma unroll 1
    for (; t < whole; t += W) {
        Step z;
        load(t, z);
        add(z);
    }
    if (t == whole && t < steps) {                                      // the last step of a K that is no multiple of 128: one wavefront's
        const int k = t * 128 + q * 32;
#pragma unroll 1
        for (int s = 0; s < 4; ++s) {
            const bool in = k + 8 * s < p.K;
            const int ks = in ? k + 8 * s : p.K - 8;
            const unsigned int w = words[ks >> lg];
            const v4i u = only_if(in, eight_weights<NB>(eight_codes<NB>(pay + (ks >> 3) * NB), tab, word_table<NB>(p, w), word_scale(p, w)));
#pragma unroll
            for (int a = 0; a < FM; ++a)
                acc[a] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, u), __builtin_bit_cast(v8bf, only_if(in, *reinterpret_cast<const v4i*>(xr[a] + ks))), acc[a], 0, 0, 0);
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
    constexpr int NT = WR * WC * 64, FM = BM / WR / 32, FN = BN / WC / 32, CX = BM * 8 / NT, IW = BN * 4 / NT, STAGE = (BM + BN) * 128;
    static_assert(IW * NT == BN * 4 && CX * NT == BM * 8 && FM * WR * 32 == BM && FN * WC * 32 == BN, "whole items and squares");
    extern __shared__ __align__(16) unsigned char lds[];
    __shared__ float tab[2 << NB];
    int tm, tn;
    tile_of(blockIdx.x, tiles_m * tiles_n, tiles_m, tiles_n, group, tm, tn);
    const int m0 = tm * BM, n0 = tn * BN, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WC * (BM / WR), wn = wave % WC * (BN / WC), lg = 31 - __builtin_clz(p.g);
    put_codebooks<NB>(p, tab, tid);
    const uint16_t* xb = p.x + (long long)m0 * p.ldx;
    unsigned int ox[CX];                                                // (a row of x has at most 2^22 elements: the entry point's check)
#pragma unroll
    for (int i = 0; i < CX; ++i) {
        const int c = i * NT + tid, r = c >> 3;
        ox[i] = (unsigned int)min(r, p.M - 1 - m0) * (unsigned int)(p.ldx * 2) + (((c ^ r >> 1) & 7) << 4);
    }
    const Window xw = window(xb, (unsigned int)(min(BM, p.M - m0) - 1) * (unsigned int)(p.ldx * 2) + (unsigned int)p.K * 2);
    auto load_x = [&](int t) {
        unsigned char* to = lds + (t & 1) * STAGE;
        if (t * 64 + 64 <= p.K) {
            const unsigned int at = lds_address(to) + (wave << 10);
#pragma unroll
            for (int i = 0; i < CX; ++i) load_to_lds(xw, ox[i], t * 128, at + i * NT * 16);
        } else {                                                        // (K is a multiple of eight: whole chunks)
            const int left = (p.K - t * 64) * 2;
#pragma unroll 1
            for (int c = tid; c < BM * 8; c += NT) {
                const int r = c >> 3, col = ((c ^ r >> 1) & 7) << 4;
                v4i v = {0, 0, 0, 0};
                if (col < left) v = *reinterpret_cast<const v4i*>(xb + (long long)min(r, p.M - 1 - m0) * p.ldx + t * 64 + (col >> 1));
                *reinterpret_cast<v4i*>(to + c * 16) = v;
            }
        }
    };
    // an item: sixteen codes of a row, four items a row and step
    const unsigned char* pay[IW];
    const uint16_t* words[IW];
    const int k16 = (tid & 3) * 16;
#pragma unroll
    for (int i = 0; i < IW; ++i) {
        const long long n = min(n0 + ((i * NT + tid) >> 2), p.N - 1);
        pay[i] = p.payload + n * (p.K >> 3) * NB;
        words[i] = p.words + n * (p.K >> lg);
    }
    struct Share { Codes c[IW][2]; unsigned int w[IW][2]; };            // what a thread forms weights of, a step
    auto load_w = [&](int t, Share& z) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k = min(t * 64 + k16 + 8 * h, p.K - 8);
#pragma unroll
            for (int i = 0; i < IW; ++i) {
                z.c[i][h] = eight_codes<NB>(pay[i] + (k >> 3) * NB);
                z.w[i][h] = words[i][k >> lg];
            }
        }
    };
    auto store_w = [&](int t, const Share& z, int i, int h) {           // eight weights: item i, half h
        const int r = (i * NT + tid) >> 2;
        const v4i u = eight_weights<NB>(z.c[i][h], tab, word_table<NB>(p, z.w[i][h]), word_scale(p, z.w[i][h]));
        *reinterpret_cast<v4i*>(lds + (t & 1) * STAGE + BM * 128 + r * 128 + ((((tid & 3) * 2 + h) ^ (r >> 1 & 7)) << 4)) = only_if(t * 64 + k16 + 8 * h < p.K, u);
    };
    v16f acc[FM][FN];
#pragma unroll
    for (int a = 0; a < FM; ++a)
#pragma unroll
        for (int b = 0; b < FN; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[a][b][i] = 0.0f;
    const int steps = (p.K + 63) >> 6;
    const unsigned int row_x = (unsigned int)(wm + (lane & 31)) * 128, row_w = (unsigned int)(wn + (lane & 31)) * 128;
    Share now, next;
    load_w(0, now);
    load_w(1, next);
    load_x(0);
    __syncthreads();                                                    // the codebooks are there
#pragma unroll
    for (int i = 0; i < 2 * IW; ++i) store_w(0, now, i >> 1, i & 1);
    for (int t = 0; t < steps; ++t) {
        wait_loads();
        __syncthreads();
        const bool more = t + 1 < steps;
        now = next;
        if (more) { load_w(t + 2, next); load_x(t + 1); }               // (codes are asked for two steps ahead, so that they are there when their turn comes)
        const unsigned char* half = lds + (t & 1) * STAGE;
        // sixteen elements of K are multiplied, then a part of the next step's weights is formed: of the two wavefronts on a SIMD one forms
        // weights while the other one's matrix instructions run
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            bf16_squares<FM, FN>(half, half + BM * 128, row_x, row_w, lane, s, acc);
            if (more)
#pragma unroll
                for (int i = s * IW / 2; i < (s + 1) * IW / 2; ++i) store_w(t + 1, now, i >> 1, i & 1);
        }
    }
#pragma unroll
    for (int a = 0; a < FM; ++a)
#pragma unroll
        for (int b = 0; b < FN; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                store_y(p, m0 + wm + a * 32 + (lane & 31), n0 + wn + b * 32 + 8 * i + 4 * (lane >> 5),
                        v4f{acc[a][b][4 * i], acc[a][b][4 * i + 1], acc[a][b][4 * i + 2], acc[a][b][4 * i + 3]});
}

template <int NB, int FM, int U, int W> static hipError_t rows_go(const PackedMmParams& p, hipStream_t st)
{
    auto fn = p.g == 8 ? &packed_rows_kernel<NB, FM, U, W, 4> : p.g == 16 ? &packed_rows_kernel<NB, FM, U, W, 2> : &packed_rows_kernel<NB, FM, U, W, 1>;
    hipLaunchKernelGGL(fn, dim3((unsigned)((p.N + 15) / 16)), dim3(W * 64), 0, st, p);
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
    if (p.M <= 16) return rows_go<NB, 1, 3, 16>(p, st);
    if (p.M <= 32) return rows_go<NB, 2, 2, 8>(p, st);
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
