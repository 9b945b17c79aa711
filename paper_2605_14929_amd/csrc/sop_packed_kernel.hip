// Product with packed codebook weights: y[m, n] = sum_k x[m, k] w[n, k], w = s L_sel[code], with the scale words (sign, magnitude,
// selector) and n-bit code payloads that the packing writes.
//
// A weight is formed in binary32 from its scale and its codebook entry and rounded once, to bf16, for the bf16 matrix instruction (the
// activations are bf16 too, and the weight's own quantisation error is some hundred times larger than that rounding); sums are binary32.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "sop_linear.h"
#include "sop_linear_rules.h"

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
    if (n + 3 < p.N) put_four(y, v);
    else {
#pragma unroll
        for (int i = 0; i < 4; ++i) if (n + i < p.N) y[i] = (uint16_t)bf16_bits(v[i]);
    }
}

// ---- few rows of x: FM x 16 of them by 16 columns a workgroup, K dealt out to its W wavefronts, 128 elements a step, U steps of a
// wavefront in flight: a lane takes 32 neighbouring codes of its row, eight for each of four matrix instructions, and the same elements of x.
// One row through 4096 x 11008 (28 MB of codes and scale words) takes 10.6 us, 11.6 where they lie in HBM, through 28672 x 8192 (147 MB) 41 and 44; sixteen
// rows 17.4.  More steps in flight or more wavefronts take as long; nothing is busy most of the time (vector ALUs 31 % of the cycles, LDS 13 %), and what
// would shorten a wavefront's way from a code to its weight - codes looked up in pairs, as below - has not been built here.
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
    // U steps in flight all the time; what the last batch has beyond the wavefront's steps is asked for again and not added
    const int mine = wave < whole ? (whole - wave + W - 1) / W : 0, batches = (mine + U - 1) / U;
    if (mine) {
        Step z[U];
#pragma unroll
        for (int u = 0; u < U; ++u) load(wave + min(u, mine - 1) * W, z[u]);
#pragma unroll 1
        for (int b = 1; b < batches; ++b) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                add(z[u]);
                load(wave + min(b * U + u, mine - 1) * W, z[u]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) if ((batches - 1) * U + u < mine) add(z[u]);
    }
    if (whole < steps && wave == whole % W) {                                      // the last step of a K that is no multiple of 128: one wavefront's
        const int k = whole * 128 + q * 32;
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

// ---- narrow tiles, K dealt out: 32 FM x 32 FN of y a workgroup, its eight wavefronts taking steps of 64 S elements in turn.  A wavefront has its
// step of x in a place of its own in LDS (no barrier before the sums are joined), and forms the weights in the registers that the matrix
// instructions read: a lane takes 32 neighbouring codes of its row, eight for each of four instructions, and the same elements of x.  The next
// step is asked for when this one's operands have been read.  128 x 4096 x 4096 of 4-bit codes takes 11.7 us (wide tiles of 128 x 128: 60), 32 x 11008
// x 4096 16.1: forming the weights, code by code, once for 32 to 128 rows bounds it.
template <int NB, int FM, int FN, int S, int WPL>
__global__ __launch_bounds__(512) void packed_split_kernel(const PackedMmParams p, int tiles_m, int tiles_n, int group)
{
    constexpr int W = 8, OWN = (S > FN ? S : FN) * FM * 4096;
    extern __shared__ __align__(16) unsigned char lds[];
    __shared__ __align__(16) float tab[2 << NB];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r32 = lane & 31, h = lane >> 5, lg = 31 - __builtin_clz(p.g);
    int tm, tn;
    tile_of(blockIdx.x, tiles_m * tiles_n, tiles_m, tiles_n, group, tm, tn);
    const int m0 = tm * (32 * FM), n0 = tn * (32 * FN), whole = p.K / (64 * S);
    unsigned char* own = lds + wave * OWN;
    const unsigned int own0 = lds_address(own);
    const Window xw = window(p.x + (long long)m0 * p.ldx, ((unsigned int)(min(32 * FM, p.M - m0) - 1) * (unsigned int)p.ldx + (unsigned int)p.K) * 2);
    unsigned int off[4 * FM];                                           // rows beyond the matrix read its last
#pragma unroll
    for (int i = 0; i < 4 * FM; ++i) off[i] = (unsigned int)min(i * 8 + (lane >> 3), p.M - 1 - m0) * (unsigned int)p.ldx * 2 + (((lane ^ (i * 8 + (lane >> 3)) >> 1) & 7) << 4);
    const unsigned char* pay[FN];
    const uint16_t* words[FN];
#pragma unroll
    for (int b = 0; b < FN; ++b) {
        const long long n = min(n0 + b * 32 + r32, p.N - 1);
        pay[b] = p.payload + n * (p.K / 8) * NB;
        words[b] = p.words + n * (p.K >> lg);
    }
    struct Part { unsigned int c[NB], w[WPL == 4 ? 2 : 1]; };
    Part z[S][FN];
    auto load = [&](int t) {
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const int k = (t * S + s) * 64 + h * 32;
#pragma unroll
            for (int b = 0; b < FN; ++b) {
                const Words<NB> c = *reinterpret_cast<const Words<NB>*>(pay[b] + (k >> 3) * NB);
#pragma unroll
                for (int i = 0; i < NB; ++i) z[s][b].c[i] = c.v[i];
                const uint16_t* w = words[b] + (k >> lg);
                if (WPL == 1) z[s][b].w[0] = w[0];
                else {
                    const Words<WPL == 4 ? 2 : 1> v = *reinterpret_cast<const Words<WPL == 4 ? 2 : 1>*>(w);
#pragma unroll
                    for (int i = 0; i < (WPL == 4 ? 2 : 1); ++i) z[s][b].w[i] = v.v[i];
                }
            }
#pragma unroll
            for (int i = 0; i < 4 * FM; ++i) load_to_lds(xw, off[i], (t * S + s) * 128, own0 + (s * 4 * FM + i) * 1024);
        }
    };
    v16f acc[FM][FN];
#pragma unroll
    for (int a = 0; a < FM; ++a)
#pragma unroll
        for (int b = 0; b < FN; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[a][b][i] = 0.0f;
    put_codebooks<NB>(p, tab, tid);
    __syncthreads();
    if (wave < whole) load(wave);
    for (int t = wave; t < whole; t += W) {
        Part c[S][FN];
        v4i x[S][FM][4];
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int s = 0; s < S; ++s) {
#pragma unroll
            for (int b = 0; b < FN; ++b) {
                c[s][b] = z[s][b];
#pragma unroll
                for (int i = 0; i < NB; ++i) asm volatile("" : "+v"(c[s][b].c[i]));
#pragma unroll
                for (int i = 0; i < (WPL == 4 ? 2 : 1); ++i) asm volatile("" : "+v"(c[s][b].w[i]));
            }
#pragma unroll
            for (int a = 0; a < FM; ++a)
#pragma unroll
                for (int j = 0; j < 4; ++j) x[s][a][j] = *reinterpret_cast<const v4i*>(own + ((s * FM + a) * 32 + r32) * 128 + (((4 * h + j) ^ (r32 >> 1 & 7)) << 4));
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");              // (the reads have ended: the place is free)
        __builtin_amdgcn_sched_barrier(0);
        if (t + W < whole) load(t + W);
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int b = 0; b < FN; ++b) {
                float sc[WPL];
                unsigned int book[WPL];
#pragma unroll
                for (int i = 0; i < WPL; ++i) {
                    const unsigned int w = c[s][b].w[i >> 1] >> (16 * (i & 1)) & 0xFFFFu;
                    sc[i] = word_scale(p, w);
                    book[i] = word_table<NB>(p, w);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const v4i u = eight_weights<NB>(eight_of<NB>(c[s][b].c, j), tab, book[j * WPL / 4], sc[j * WPL / 4]);
#pragma unroll
                    for (int a = 0; a < FM; ++a) acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, u), __builtin_bit_cast(v8bf, x[s][a][j]), acc[a][b], 0, 0, 0);
                }
            }
    }
#pragma unroll 1
    for (int k0 = whole * 64 * S + wave * 16; k0 < p.K; k0 += W * 16) {  // what is left of K, sixteen elements a wavefront
        const int k = k0 + 8 * h;
        const bool in = k < p.K;
        const int ks = in ? k : p.K - 8;
        v4i u[FN];
#pragma unroll
        for (int b = 0; b < FN; ++b) {
            const unsigned int w = words[b][ks >> lg];
            u[b] = only_if(in, eight_weights<NB>(eight_codes<NB>(pay[b] + (ks >> 3) * NB), tab, word_table<NB>(p, w), word_scale(p, w)));
        }
#pragma unroll
        for (int a = 0; a < FM; ++a) {
            const v4i v = only_if(in, *reinterpret_cast<const v4i*>(p.x + (long long)min(m0 + a * 32 + r32, p.M - 1) * p.ldx + ks));
#pragma unroll
            for (int b = 0; b < FN; ++b) acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, u[b]), __builtin_bit_cast(v8bf, v), acc[a][b], 0, 0, 0);
        }
    }
    wait_loads();
    __syncthreads();
#pragma unroll
    for (int a = 0; a < FM; ++a)
#pragma unroll
        for (int b = 0; b < FN; ++b) put_square(reinterpret_cast<v4f*>(own) + (a * FN + b) * 256, lane, acc[a][b]);
    __syncthreads();
    for (int t = wave; t < FM * FN * 4; t += W) {                         // a quarter of a square
        const int a = (t >> 2) / FN, b = (t >> 2) % FN, i = t & 3, at = (t >> 2) * 256 + quarter_slot(i, lane);
        v4f s = reinterpret_cast<const v4f*>(lds)[at];
#pragma unroll
        for (int q = 1; q < W; ++q) s += reinterpret_cast<const v4f*>(lds + q * OWN)[at];
        store_y(p, m0 + a * 32 + 8 * i + (lane >> 3), n0 + b * 32 + 4 * (lane & 7), s);
    }
}

// ---- wide tiles: 64 E x 64 F of y (4 x 4, 4 x 3, 2 x 2) by four wavefronts, each 32 E x 32 F of it; 64 elements along K a step,
// two steps in LDS.  While sixteen elements are multiplied (E F matrix instructions), the next sixteen's operands are read, and between
// two barriers (4 E F matrix instructions) every thread forms 16 F weights of the step after the next, eight by eight: behind each matrix
// instruction stand a part of the look-ups and of the scale word of an eight, and a part of the products of the eight before.  A matrix
// instruction (32 cycles) hides seven others of its wavefront, so what a weight costs in instructions is what counts: two codes
// are looked up at once, in a table of the 4^NB pairs of either codebook.  Before a step's last sixteen elements comes its barrier: the
// next step is there, this one's place is free.  2048 x 11008 x 4096 of 4-bit codes takes 194 us, 950 TFLOP/s: matrix instructions are busy 41 % of the
// cycles; the others go to the look-ups and products of the weights, formed anew by every row of tiles, and 44 % of the cycles in which LDS is at work to
// bank conflicts of the pairs' look-ups.
template <int NB, int E, int F, bool G8>
__global__ __launch_bounds__(256, E == 2 ? 2 : 1) void packed_wide_kernel(const PackedMmParams p, int tiles_m, int tiles_n, int group)
{
    constexpr int BM = 64 * E, BN = 64 * F, SLOTS = E * F, EACH = 4 / E, XL = 2 * E, STAGE = (BM + BN) * 128, BOOK = 8 << 2 * NB, TAB = 2 * BOOK, CW = (NB + 1) / 2, WORDS = G8 ? 2 : 1;
    constexpr unsigned int NOWHERE = 0xE0000000u;                       // an offset beyond every window
    extern __shared__ __align__(TAB) unsigned char lds[];
    int tm, tn;
    tile_of(blockIdx.x, tiles_m * tiles_n, tiles_m, tiles_n, group, tm, tn);
    const int m0 = tm * BM, n0 = tn * BN, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = (wave >> 1) * (32 * E), wn = (wave & 1) * (32 * F), lg = 31 - __builtin_clz(p.g), steps = (p.K + 63) >> 6;
    const unsigned int tab0 = lds_address(lds), lds0 = tab0 + TAB;
    for (int i = tid; i < 2 << 2 * NB; i += 256) {
        const float* book = p.tab[i >> 2 * NB];
        *reinterpret_cast<float2*>(lds + i * 8) = make_float2(book[i & ((1 << NB) - 1)], book[i >> NB & ((1 << NB) - 1)]);
    }

    // x: chunks of 16 bytes straight into LDS
    const unsigned int xcol = (unsigned int)((tid ^ tid >> 4) & 7) << 4;   // (rows 32 apart lie alike)
    unsigned int ox[XL];
#pragma unroll
    for (int i = 0; i < XL; ++i) ox[i] = (unsigned int)min(i * 32 + (tid >> 3), p.M - 1 - m0) * (unsigned int)(p.ldx * 2) + xcol;
    const Window xw = window(p.x + (long long)m0 * p.ldx, (unsigned int)(min(BM, p.M - m0) - 1) * (unsigned int)(p.ldx * 2) + (unsigned int)p.K * 2);
    auto load_x = [&](int t, int i) { load_to_lds(xw, ox[i], packed_step_at(t, steps, NB, lg, false).x, lds0 + (t & 1) * STAGE + (wave << 10) + i * 4096); };
    // w: an item is sixteen codes of a row, four items a row and step, F of a thread
    const int rows = min(BN, p.N - n0), k16 = (tid & 3) * 16;
    const unsigned int prow = (unsigned int)(p.K >> 3) * NB, wrow = (unsigned int)(p.K >> lg) * 2u;
    const Window pw = window(p.payload + (long long)n0 * prow, (unsigned int)rows * prow), ww = window(p.words + (long long)n0 * (p.K >> lg), (unsigned int)rows * wrow);
    unsigned int op[F], ow[F][WORDS];
#pragma unroll
    for (int i = 0; i < F; ++i) {
        const unsigned int r = (unsigned int)min(i * 64 + (tid >> 2), rows - 1);
        op[i] = r * prow + (unsigned int)(k16 >> 3) * NB;
#pragma unroll
        for (int h = 0; h < WORDS; ++h) ow[i][h] = r * wrow + (unsigned int)((k16 >> lg) + h) * 2u;
    }
    unsigned int put[2], putting[2] = {0, 0};                           // where this thread's weights go (rows 64 apart lie alike)
#pragma unroll
    for (int h = 0; h < 2; ++h) put[h] = lds0 + BM * 128 + (unsigned int)(tid >> 2) * 128 + (unsigned int)((((tid & 3) * 2 + h) ^ (tid >> 3 & 7)) << 4);
    // Elements of the last step beyond K: x is asked for nowhere, and zeros arrive; so are the scale words, whose scale is 0.
    // Where K ends in the middle of an item (g = 8 alone), no byte beyond its codes is read: the last step's items are asked for one eight earlier,
    // this one's too, which has its eight in its second half then; the others' places are moved back by as much.
    const bool odd = (p.K & 63) != 0, half = G8 && (p.K & 15) != 0;
    auto end_x = [&](int t) {
        if (odd && t == steps - 1) {
#pragma unroll
            for (int i = 0; i < XL; ++i) ox[i] = t * 128 + (int)xcol < p.K * 2 ? ox[i] : NOWHERE;
        }
    };
    auto end_w = [&](int t) {
        if (odd && t == steps - 1) {
#pragma unroll
            for (int i = 0; i < F; ++i)
#pragma unroll
                for (int h = 0; h < WORDS; ++h) ow[i][h] = t * 64 + k16 + 8 * h < p.K ? ow[i][h] : NOWHERE;
            if (half) {
                const bool mine = t * 64 + k16 + 8 == p.K;
#pragma unroll
                for (int i = 0; i < F; ++i) {
                    op[i] += mine ? 0u : (unsigned int)NB;
                    ow[i][WORDS - 1] = mine ? ow[i][0] : ow[i][WORDS - 1];
                    ow[i][0] = mine ? NOWHERE : ow[i][0];
                }
                const unsigned int first = put[0];
                put[0] = mine ? put[1] : first;
                put[1] = mine ? first : put[1];
            }
        }
    };
    struct Item { unsigned int c[CW], w[WORDS]; };
    auto load_w = [&](Item& z, int t, int i) {
        const PackedStepAt step = packed_step_at(t, steps, NB, lg, half);
        const int at = step.codes;
        if constexpr (NB / 2 == 1) z.c[0] = (unsigned int)__builtin_amdgcn_raw_buffer_load_b32(resource(pw), (int)op[i], at, 0);
        if constexpr (NB / 2 == 2) {
            const auto c = __builtin_amdgcn_raw_buffer_load_b64(resource(pw), (int)op[i], at, 0);
            z.c[0] = c[0]; z.c[1] = c[1];
        }
        if constexpr (NB / 2 == 3) {
            const auto c = __builtin_amdgcn_raw_buffer_load_b96(resource(pw), (int)op[i], at, 0);
            z.c[0] = c[0]; z.c[1] = c[1]; z.c[2] = c[2];
        }
        if constexpr (NB % 2 == 1) z.c[CW - 1] = __builtin_amdgcn_raw_buffer_load_b16(resource(pw), (int)op[i], at + NB / 2 * 4, 0);
#pragma unroll
        for (int h = 0; h < WORDS; ++h) z.w[h] = __builtin_amdgcn_raw_buffer_load_b16(resource(ww), (int)ow[i][h], step.words, 0);
    };

    v16f acc[E][F];
#pragma unroll
    for (int a = 0; a < E; ++a)
#pragma unroll
        for (int b = 0; b < F; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[a][b][i] = 0.0f;

    typedef __attribute__((address_space(3))) v4i* ldsi;
    typedef __attribute__((address_space(3))) v2f* ldsp;
    v2f v[2][4];
    float scale[2];
    unsigned int book = 0, mag = 0, ex = 0, frac = 0;
    // eight weights (half h of item z; o = 0 or 1 in turn): the e-th of eight parts of the look-ups and the scale
    auto look_up = [&](const Item& z, int h, int o, int e) {
        const unsigned int w = z.w[h & (WORDS - 1)];
        if (e == 0) book = tab0 | (w >> p.sel_pos & (unsigned int)p.sel_mask) << (2 * NB + 3);
        if (!(e & 1)) {
            const int at = NB * (8 * h + e) - 3, i = at < 0 ? 0 : at >> 5, sh = at & 31;    // the pair's bits, moved to bit 3
            const unsigned int m = at < 0 ? z.c[0] << -at : sh + 2 * NB + 3 <= 32 || i + 1 >= CW ? z.c[i] >> sh : __builtin_amdgcn_alignbit(z.c[i + 1 < CW ? i + 1 : 0], z.c[i], (unsigned int)sh);
            v[o][e >> 1] = *(ldsp)(uintptr_t)((m & (unsigned int)(BOOK - 8)) | book);
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
    v4i fx[2][E], fw[2][F];
    unsigned int rx = 0, rw = 0;
    auto from = [&](unsigned int stage, int s) { rx = at[s] + (stage + wm * 128); rw = at[s] + (stage + (BM + wn) * 128); };
    auto read = [&](int s, int i) {                                     // the i-th of F + E reads
        if (i < F) fw[s & 1][i] = *(ldsi)(uintptr_t)(rw + i * 4096);
        else if (i < F + E) fx[s & 1][i - F] = *(ldsi)(uintptr_t)(rx + (i - F) * 4096);
    };
    auto multiply = [&](int s, int i) {
        const int a = i / F, b = i % F;
        acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, fw[s & 1][b]), __builtin_bit_cast(v8bf, fx[s & 1][a]), acc[a][b], 0, 0, 0);
    };

    Item now[F], next[F];
    auto settle = [&](Item (&z)[F]) {                                   // what has arrived is used as such (and not waited for again behind later loads)
#pragma unroll
        for (int i = 0; i < F; ++i) {
#pragma unroll
            for (int k = 0; k < CW; ++k) asm volatile("" : "+v"(z[i].c[k]));
#pragma unroll
            for (int h = 0; h < WORDS; ++h) asm volatile("" : "+v"(z[i].w[h]));
        }
    };
    __syncthreads();                                                    // the codebooks are there
    // the first step whole; of the second, x and a quarter of the weights
    for (int t = 0; t < 2; ++t) {
        end_x(t);
#pragma unroll
        for (int i = 0; i < XL; ++i) load_x(t, i);
    }
    end_w(0);
#pragma unroll
    for (int i = 0; i < F; ++i) load_w(next[i], 0, i);
    putting[0] = put[0]; putting[1] = put[1];
    end_w(1);
#pragma unroll
    for (int i = 0; i < F; ++i) load_w(now[i], 1, i);
    // A quarter of a step's work is F / 2 eights; with F = 3 the second of them is looked up, and half formed.
    constexpr int PART = 4 * F;                                         // parts of eights in a quarter
#pragma unroll
    for (int g = 0; g < 2 * F; ++g) {
#pragma unroll
        for (int e = 0; e < 8; ++e) look_up(next[g >> 1], g & 1, g & 1, e);
#pragma unroll
        for (int e = 0; e < 8; ++e) form(g >> 1, g & 1, g & 1, e);
    }
    putting[0] = put[0] + STAGE; putting[1] = put[1] + STAGE;
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
    for (int i = 0; i < F + E; ++i) read(0, i);
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
                // the reads, dealt out over the instructions
#pragma unroll
                for (int k = i * (F + E) / SLOTS; k < (i + 1) * (F + E) / SLOTS; ++k) read((s + 1) & 3, k);
#pragma unroll
                for (int k = 0; k < EACH; ++k) {
                    const int f = (Q * SLOTS + i) * EACH + k, g = f >> 3, e = f & 7;    // the eight whose products are formed; the one after it is looked up
                    form(g >> 1, g & 1, g & 1, e);
                    if (f == 16 * F - 8) { wait_loads(); settle(next); }
                    if (g < 2 * F - 1) look_up(now[(g + 1) >> 1], (g + 1) & 1, (g + 1) & 1, e);
                    else look_up(next[0], 0, 0, e);
                }
                if (s == 3 && i * XL / SLOTS != (i + 1) * XL / SLOTS) load_x(t + 2, i * XL / SLOTS);
                if (s < 2) {                                            // (the first two quarters ask for the next codes)
#pragma unroll
                    for (int k = 0; k < F; ++k) if (s * SLOTS + i == (2 * k + 1) * SLOTS / F) load_w(next[k], t + 2, k);
                }
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
    __syncthreads();                                                    // (LDS is free for the results)
    v4f* place = reinterpret_cast<v4f*>(lds + wave * 4096);
#pragma unroll
    for (int a = 0; a < E; ++a)
#pragma unroll
        for (int b = 0; b < F; ++b) {
            put_square(place, lane, acc[a][b]);
#pragma unroll
            for (int i = 0; i < 4; ++i) store_y(p, m0 + wm + a * 32 + 8 * i + (lane >> 3), n0 + wn + b * 32 + 4 * (lane & 7), place[quarter_slot(i, lane)]);
        }
}

template <int NB, int FM, int U, int W> static hipError_t rows_go(const PackedMmParams& p, hipStream_t st)
{
    auto fn = p.g == 8 ? &packed_rows_kernel<NB, FM, U, W, 4> : p.g == 16 ? &packed_rows_kernel<NB, FM, U, W, 2> : &packed_rows_kernel<NB, FM, U, W, 1>;
    hipLaunchKernelGGL(fn, dim3((unsigned)((p.N + 15) / 16)), dim3(W * 64), 0, st, p);
    return hipGetLastError();
}
template <int NB, int FM, int FN, int S> static hipError_t split_go(const PackedMmParams& p, hipStream_t st)
{
    const int tm = (p.M + 32 * FM - 1) / (32 * FM), tn = (p.N + 32 * FN - 1) / (32 * FN), bytes = 8 * (S > FN ? S : FN) * FM * 4096;
    auto fn = p.g == 8 ? &packed_split_kernel<NB, FM, FN, S, 4> : p.g == 16 ? &packed_split_kernel<NB, FM, FN, S, 2> : &packed_split_kernel<NB, FM, FN, S, 1>;
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(fn), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(fn, dim3((unsigned)(tm * tn)), dim3(512), bytes, st, p, tm, tn, 8);
    return hipGetLastError();
}
template <int NB, int E, int F> static hipError_t wide_go(const PackedMmParams& p, hipStream_t st)
{
    const int tm = (p.M + 64 * E - 1) / (64 * E), tn = (p.N + 64 * F - 1) / (64 * F), bytes = (16 << 2 * NB) + 2 * (64 * E + 64 * F) * 128;
    static_assert((16 << 2 * NB) + 2 * (64 * E + 64 * F) * 128 <= 160 * 1024, "the tables and two steps fit into LDS");
    auto fn = p.g == 8 ? &packed_wide_kernel<NB, E, F, true> : &packed_wide_kernel<NB, E, F, false>;
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(fn), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(fn, dim3((unsigned)(tm * tn)), dim3(256), bytes, st, p, tm, tn, 8);
    return hipGetLastError();
}
template <int NB> static hipError_t go(const PackedMmParams& p, int choice, hipStream_t st)
{
    switch (choice) {
    case sopr::PACKED_ROWS: return rows_go<NB, 1, 2, 8>(p, st);
    case sopr::PACKED_32x32: return split_go<NB, 1, 1, 1>(p, st);
    case sopr::PACKED_64x32: return split_go<NB, 2, 1, 1>(p, st);
    case sopr::PACKED_64x64: return split_go<NB, 2, 2, 1>(p, st);
    case sopr::PACKED_128x32: return split_go<NB, 4, 1, 1>(p, st);
    case sopr::PACKED_128x128: return wide_go<NB, 2, 2>(p, st);
    case sopr::PACKED_256x192:
        if constexpr (NB <= 5) return wide_go<NB, 4, 3>(p, st);
        break;
    case sopr::PACKED_256x256:
        if constexpr (NB <= 5) return wide_go<NB, 4, 4>(p, st);
    }
    return hipErrorInvalidValue;
}

}  // namespace sopk

extern "C" hipError_t sopk_packed_launch(const PackedMmParams* p, int choice, void* stream)
{
    hipStream_t st = (hipStream_t)stream;
    switch (p->n_bits) {
    case 1: return sopk::go<1>(*p, choice, st);
    case 2: return sopk::go<2>(*p, choice, st);
    case 3: return sopk::go<3>(*p, choice, st);
    case 4: return sopk::go<4>(*p, choice, st);
    case 5: return sopk::go<5>(*p, choice, st);
    case 6: return sopk::go<6>(*p, choice, st);
    }
    return hipErrorInvalidValue;
}
