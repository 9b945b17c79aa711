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

// ---- large products of 4-bit codes: 256 x 64 F of y (F = 4 or 3) by four wavefronts, one on a SIMD, each 128 x 32 F of it; 64 elements along
// K a step, two steps in LDS.  While sixteen elements are multiplied (4 F matrix instructions), the next sixteen's operands are read, and
// between two barriers (16 F matrix instructions) every thread forms 16 F weights of the step after the next, eight by eight: behind each matrix
// instruction stand a part of the look-ups and of the scale word of an eight, and a part of the products of the eight before.  A matrix
// instruction (32 cycles) hides seven others of its wavefront, so what a weight costs in instructions is what counts: two codes (a byte of
// the payload) are looked up at once, in a table of the 256 pairs of either codebook.  Halfway through a step comes its barrier: the
// next step is there, this one's place is free.
template <int F, bool G8>
__global__ __launch_bounds__(256) void packed_large_kernel(const PackedMmParams p, int tiles_m, int tiles_n, int group)
{
    constexpr int BM = 256, BN = 64 * F, SLOTS = 4 * F, STAGE = (BM + BN) * 128, TAB = 4096, WORDS = G8 ? 2 : 1;
    constexpr unsigned int NOWHERE = 0xE0000000u;                       // an offset beyond every window
    extern __shared__ __align__(4096) unsigned char lds[];
    int tm, tn;
    tile_of(blockIdx.x, tiles_m * tiles_n, tiles_m, tiles_n, group, tm, tn);
    const int m0 = tm * BM, n0 = tn * BN, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave >> 1 << 7, wn = (wave & 1) * (32 * F), lg = 31 - __builtin_clz(p.g), steps = (p.K + 63) >> 6;
    const unsigned int tab0 = lds_address(lds), lds0 = tab0 + TAB;
#pragma unroll
    for (int b = 0; b < 2; ++b) *reinterpret_cast<float2*>(lds + b * 2048 + tid * 8) = make_float2(p.tab[b][tid & 15], p.tab[b][tid >> 4]);

    // x: chunks of 16 bytes straight into LDS
    const unsigned int xcol = (unsigned int)((tid ^ tid >> 4) & 7) << 4;   // (rows 32 apart lie alike)
    unsigned int ox[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) ox[i] = (unsigned int)min(i * 32 + (tid >> 3), p.M - 1 - m0) * (unsigned int)(p.ldx * 2) + xcol;
    const Window xw = window(p.x + (long long)m0 * p.ldx, (unsigned int)(min(BM, p.M - m0) - 1) * (unsigned int)(p.ldx * 2) + (unsigned int)p.K * 2);
    auto load_x = [&](int t, int i) { load_to_lds(xw, ox[i], t * 128, lds0 + (t & 1) * STAGE + (wave << 10) + i * 4096); };
    // w: an item is sixteen codes of a row, four items a row and step, F of a thread
    const int rows = min(BN, p.N - n0), k16 = (tid & 3) * 16;
    const unsigned int prow = (unsigned int)(p.K >> 1), wrow = (unsigned int)(p.K >> lg) * 2u;
    const Window pw = window(p.payload + (long long)n0 * prow, (unsigned int)rows * prow), ww = window(p.words + (long long)n0 * (p.K >> lg), (unsigned int)rows * wrow);
    unsigned int op[F], ow[F][WORDS];
#pragma unroll
    for (int i = 0; i < F; ++i) {
        const unsigned int r = (unsigned int)min(i * 64 + (tid >> 2), rows - 1);
        op[i] = r * prow + (unsigned int)(k16 >> 1);
#pragma unroll
        for (int h = 0; h < WORDS; ++h) ow[i][h] = r * wrow + (unsigned int)((k16 >> lg) + h) * 2u;
    }
    // Elements of the last step beyond K: x is asked for nowhere, and zeros arrive; so are the scale words, whose scale is 0.
    const bool odd = (p.K & 63) != 0;
    auto end_x = [&](int t) {
        if (odd && t == steps - 1) {
#pragma unroll
            for (int i = 0; i < 8; ++i) ox[i] = t * 128 + (int)xcol < p.K * 2 ? ox[i] : NOWHERE;
        }
    };
    auto end_w = [&](int t) {
        if (odd && t == steps - 1) {
#pragma unroll
            for (int i = 0; i < F; ++i)
#pragma unroll
                for (int h = 0; h < WORDS; ++h) ow[i][h] = t * 64 + k16 + 8 * h < p.K ? ow[i][h] : NOWHERE;
        }
    };
    struct Item { unsigned int c[2], w[WORDS]; };
    auto load_w = [&](Item& z, int t, int i) {
        const auto c = __builtin_amdgcn_raw_buffer_load_b64(resource(pw), (int)op[i], t * 32, 0);
        z.c[0] = c[0]; z.c[1] = c[1];
#pragma unroll
        for (int h = 0; h < WORDS; ++h) z.w[h] = __builtin_amdgcn_raw_buffer_load_b16(resource(ww), (int)ow[i][h], t * (128 >> lg), 0);
    };

    v16f acc[4][F];
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int b = 0; b < F; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[a][b][i] = 0.0f;

    typedef __attribute__((address_space(3))) v4i* ldsi;
    typedef __attribute__((address_space(3))) v2f* ldsp;
    unsigned int put[2], putting[2] = {0, 0};                           // where this thread's weights go (rows 64 apart lie alike)
#pragma unroll
    for (int h = 0; h < 2; ++h) put[h] = lds0 + BM * 128 + (unsigned int)(tid >> 2) * 128 + (unsigned int)((((tid & 3) * 2 + h) ^ (tid >> 3 & 7)) << 4);
    v2f v[2][4];
    float scale[2];
    unsigned int book = 0, mag = 0, ex = 0, frac = 0;
    // eight weights (half h of item z; o = 0 or 1 in turn): the e-th of eight parts of the look-ups and the scale
    auto look_up = [&](const Item& z, int h, int o, int e) {
        const unsigned int w = z.w[h & (WORDS - 1)];
        if (e == 0) book = tab0 | (w >> p.sel_pos & (unsigned int)p.sel_mask) << 11;
        if (!(e & 1)) {
            const unsigned int m = e == 0 ? z.c[h] << 3 : z.c[h] >> (4 * e - 3);
            v[o][e >> 1] = *(ldsp)(uintptr_t)((m & 0x7F8u) | book);
        }
        if (e == 1) { mag = (w >> p.mag_shift) & (unsigned int)p.mag_mask; ex = mag >> p.man_bits; }
        if (e == 3) { frac = (mag & (unsigned int)p.man_mask) | min(ex, 1u) << p.man_bits; ex = max(ex, 1u); }
        if (e == 5) { scale[o] = __builtin_amdgcn_ldexpf((float)frac, (int)ex + p.exp_off); }
        if (e == 7) scale[o] = __uint_as_float(__float_as_uint(scale[o]) | (w << p.sign_up & 0x80000000u));
    };
    v4i u;
    // ... of their products, rounded and stored as item i
    auto form = [&](int i, int h, int o, int e) {
        if (e == 0) asm volatile("" : "+v"(v[o][0]), "+v"(v[o][1]), "+v"(v[o][2]), "+v"(v[o][3]));   // (one wait for all four)
        if (!(e & 1)) return;
        u[e >> 1] = (int)bf16_pair(scale[o] * v[o][e >> 1][0], scale[o] * v[o][e >> 1][1]);
        asm volatile("" : "+v"(u[e >> 1]));
        if (e == 7) *(ldsi)(uintptr_t)(putting[h] + i * 8192) = u;
    };

    const int r32 = lane & 31;
    unsigned int at[4];                                                 // the s-th sixteen elements of this lane's row, without the row
#pragma unroll
    for (int s = 0; s < 4; ++s) at[s] = lds0 + (unsigned int)r32 * 128 + ((unsigned int)(((lane >> 5) ^ (r32 >> 1 & 7)) << 4) ^ (unsigned int)(s << 5));
    v4i fx[2][4], fw[2][F];
    unsigned int rx = 0, rw = 0;
    auto from = [&](unsigned int stage, int s) { rx = at[s] + (stage + wm * 128); rw = at[s] + (stage + (BM + wn) * 128); };
    auto read = [&](int s, int i) {                                     // the i-th of F + 4 reads
        if (i < F) fw[s & 1][i] = *(ldsi)(uintptr_t)(rw + i * 4096);
        else if (i < F + 4) fx[s & 1][i - F] = *(ldsi)(uintptr_t)(rx + (i - F) * 4096);
    };
    auto multiply = [&](int s, int i) {
        const int a = i / F, b = i % F;
        acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, fw[s & 1][b]), __builtin_bit_cast(v8bf, fx[s & 1][a]), acc[a][b], 0, 0, 0);
    };

    Item now[F], next[F];
    auto settle = [&](Item (&z)[F]) {                                   // what has arrived is used as such (and not waited for again behind later loads)
#pragma unroll
        for (int i = 0; i < F; ++i) {
            asm volatile("" : "+v"(z[i].c[0]), "+v"(z[i].c[1]), "+v"(z[i].w[0]));
            if (G8) asm volatile("" : "+v"(z[i].w[WORDS - 1]));
        }
    };
    __syncthreads();                                                    // the codebooks are there
    // the first step whole; of the second, x and a quarter of the weights
    for (int t = 0; t < 2; ++t) {
        end_x(t);
#pragma unroll
        for (int i = 0; i < 8; ++i) load_x(t, i);
    }
    end_w(0);
#pragma unroll
    for (int i = 0; i < F; ++i) load_w(next[i], 0, i);
    end_w(1);
#pragma unroll
    for (int i = 0; i < F; ++i) load_w(now[i], 1, i);
    putting[0] = put[0]; putting[1] = put[1];
    // A quarter of a step's work is F / 2 eights; with F = 3 the second of them is looked up, and half formed.
    constexpr int PART = 4 * F;
#pragma unroll
    for (int g = 0; g < 2 * F; ++g) {
#pragma unroll
        for (int e = 0; e < 8; ++e) look_up(next[g >> 1], g & 1, g & 1, e);
#pragma unroll
        for (int e = 0; e < 8; ++e) form(g >> 1, g & 1, g & 1, e);
    }
    putting[0] += STAGE; putting[1] += STAGE;
#pragma unroll
    for (int e = 0; e < 8; ++e) look_up(now[0], 0, 0, e);
#pragma unroll
    for (int f = 0; f < PART; ++f) {
        const int g = f >> 3, e = f & 7;
        form(g >> 1, g & 1, g & 1, e);
        look_up(now[(g + 1) >> 1], (g + 1) & 1, (g + 1) & 1, e);
    }
    wait_loads();
    __syncthreads();
    settle(now);
    from(0, 0);
#pragma unroll
    for (int i = 0; i < F + 4; ++i) read(0, i);
    for (int t = 0; t < steps; ++t) {
        const unsigned int here = (t & 1) * STAGE, there = STAGE - here;
        // sixteen elements of K, and a quarter of the work between two barriers: behind a step's last sixteen elements the first quarter of the
        // step after the next, behind the next step's first three times sixteen the others
        auto part = [&](auto S) {
            constexpr int s = decltype(S)::value, Q = (s + 1) & 3;
            from(s == 3 ? there : here, (s + 1) & 3);
            if (s == 0) end_w(t + 2);
            if (s == 3) {
                end_x(t + 2);
                putting[0] = put[0] + here; putting[1] = put[1] + here;
            }
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) {
                multiply(s, i);
                if (F == 4 ? (i & 1) == 0 : i < F + 4) read((s + 1) & 3, F == 4 ? i >> 1 : i);
                const int f = Q * SLOTS + i, g = f >> 3, e = f & 7;     // the eight whose products are formed; the one after it is looked up
                form(g >> 1, g & 1, g & 1, e);
                if (f == 4 * SLOTS - 8) { wait_loads(); settle(next); }
                if (g < 2 * F - 1) look_up(now[(g + 1) >> 1], (g + 1) & 1, (g + 1) & 1, e);
                else look_up(next[0], 0, 0, e);
                if (s == 3 && i * 8 / SLOTS != (i + 1) * 8 / SLOTS) load_x(t + 2, i * 8 / SLOTS);
                if (s < 2 && i % 8 == 3) { if (s * (SLOTS / 8) + i / 8 < F) load_w(next[s * (SLOTS / 8) + i / 8], t + 2, s * (SLOTS / 8) + i / 8); }
                if constexpr (F == 3 && s == 1) if (i == 8) load_w(next[2], t + 2, 2);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        part(std::integral_constant<int, 0>{});
        part(std::integral_constant<int, 1>{});
        part(std::integral_constant<int, 2>{});
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");              // (the loads were waited for eight instructions ago)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int i = 0; i < F; ++i) now[i] = next[i];
        part(std::integral_constant<int, 3>{});
    }
    wait_loads();
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int b = 0; b < F; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                store_y(p, m0 + wm + a * 32 + r32, n0 + wn + b * 32 + 8 * i + 4 * (lane >> 5),
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
template <int F> static hipError_t large_go(const PackedMmParams& p, hipStream_t st)
{
    const int tm = (p.M + 255) / 256, tn = (p.N + 64 * F - 1) / (64 * F), bytes = 4096 + 2 * (256 + 64 * F) * 128;
    auto fn = p.g == 8 ? &packed_large_kernel<F, true> : &packed_large_kernel<F, false>;
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(fn), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(fn, dim3((unsigned)(tm * tn)), dim3(256), bytes, st, p, tm, tn, 8);
    return hipGetLastError();
}
// One workgroup a compute unit: the width whose last round is filled better.  A tile of 192 columns forms and reads more for a product: 2048 x
// 11008 x 4096 takes 242 us by it (464 tiles, two rounds) and 256 us by the wider (344 tiles, two rounds), 4096 x 4096 x 4096 208 us (352
// tiles, two rounds) and 145 us (256 tiles, one).
static hipError_t large_pick(const PackedMmParams& p, int n_cu, hipStream_t st)
{
    auto cost = [&](int f, int each) {
        const long long tiles = (long long)((p.M + 255) / 256) * ((p.N + 64 * f - 1) / (64 * f));
        return (tiles + n_cu - 1) / n_cu * f * each;
    };
    return cost(4, 20) <= cost(3, 25) ? large_go<4>(p, st) : large_go<3>(p, st);
}
template <int NB> static hipError_t packed_pick(const PackedMmParams& p, int n_cu, hipStream_t st)
{
    auto tiles = [&](int bm, int bn) { return (long long)((p.M + bm - 1) / bm) * ((p.N + bn - 1) / bn); };
    if (p.M <= 16) return rows_go<NB, 1, 3, 16>(p, st);
    if (p.M <= 32) return rows_go<NB, 2, 2, 8>(p, st);
    if (tiles(256, 256) >= n_cu) {
        if constexpr (NB == 4) return large_pick(p, n_cu, st);
        else return tile_go<NB, 256, 256, 2, 4>(p, st);
    }
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
