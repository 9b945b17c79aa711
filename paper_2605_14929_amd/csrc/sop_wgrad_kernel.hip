// Weight gradient from an 8-bit activation checkpoint: dw[n, k] = sum_m dy[m, n] x[m, k], x = code * 2^e with a scale for every block
// of 128 along k.
//
// The sum runs over the rows, and along them the scale changes at every step, so the 8-bit matrix instruction (one scale a row of its
// operand and 32 elements of the sum) cannot take it.  An 8-bit number times a power of two is a bf16 number, though: the
// checkpoint becomes bf16 exactly on its way into LDS, and the bf16 matrix instruction adds nothing but binary32 sums.
//
// Both operands arrive with the summed index outermost, the matrix instruction wants it innermost.  Where dy's rows lie on 16 bytes,
// both go to LDS as they are, straight from memory, and are turned by LDS's transposing reads (a sixteen-lane group reads four rows of
// sixteen 16-bit, or eight rows of sixteen 8-bit elements and receives the columns); the checkpoint stays in 8 bits until then.
// Otherwise a thread loads eight rows of two (dy) or four (x) columns, turns them in registers, and writes columns (8192 x 11007 x 4096 takes 1339 us
// so, 8192 x 11008 x 4096 by the transposing reads 611).
#include <hip/hip_runtime.h>

#include <type_traits>

#include "sop_linear.h"
#include "sop_linear_rules.h"

namespace sopk {

// two neighbouring bf16 of a row, aligned or not
struct __attribute__((packed)) Pair { unsigned int v; };

// four neighbouring columns of a row of dw
__device__ __forceinline__ void store_dw(const WgradParams& p, int n, int k, v4f v)
{
    if (n >= p.N || k >= p.K) return;
    const long long at = (long long)n * p.lddw + k;
    const bool four = k + 3 < p.K;
    if (p.out_bf16) {
        uint16_t* w = reinterpret_cast<uint16_t*>(p.dw) + at;
        if (p.accumulate) {
#pragma unroll
            for (int i = 0; i < 4; ++i) if (k + i < p.K) v[i] += __uint_as_float((unsigned int)w[i] << 16);
        }
        if (four) put_four(w, v);
        else {
#pragma unroll
            for (int i = 0; i < 4; ++i) if (k + i < p.K) w[i] = (uint16_t)bf16_bits(v[i]);
        }
    } else {
        float* w = reinterpret_cast<float*>(p.dw) + at;
        // Whole lines are written past the caches.  Two results in turn: 64 x 11008 x 4096 takes 36.6 us so and 39.5 otherwise, with an update that reads
        // them 114 and 125; 777 x 1531 x 5024 21.3 and 23.1, 36 and 36; but 2048 x 4096 x 4096 67 and 64, 98 and 93, and 64 x 4096 x 4096 17.0 and
        // 16.4, 47 and 45.  (Lines in parts, 26 x 1920 x 4793: 26 and 14.)
        const bool lines = ((reinterpret_cast<uintptr_t>(p.dw) | (unsigned long long)p.lddw * 4) & 127) == 0;
        if (four) {
            if (p.accumulate) v += reinterpret_cast<const FourWords*>(w)->v;
            if (lines) __builtin_nontemporal_store(v, reinterpret_cast<v4f*>(w));
            else put_four(w, v);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) if (k + i < p.K) w[i] = p.accumulate ? v[i] + w[i] : v[i];
        }
    }
}

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
    for (int a = 0; a < FA; ++a)
#pragma unroll
        for (int b = 0; b < FB; ++b) store_dw(p, n0 + wn + a * 16 + r16, k0 + wk + b * 16 + 4 * q, acc[a][b]);
}

// two codes of a column (the low or the high half of a word) under the scales of their rows, as bf16
template <bool E5M2, bool HIGH> __device__ __forceinline__ int two_rows(int c, float s0, float s1)
{
    const v2bf a = E5M2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(c, s0, HIGH) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, s0, HIGH);
    const v2bf b = E5M2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(c, s1, HIGH) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, s1, HIGH);
    return (int)__builtin_amdgcn_perm(__builtin_bit_cast(unsigned int, b), __builtin_bit_cast(unsigned int, a), 0x07060100u);
}

// ---- rows of dy on 16 bytes.  64 rows a step, three steps in LDS: one being multiplied, one on its way or there, one being asked for.
// In LDS a row is chunks of 16 bytes; chunk c of row m stands at position c ^ 4 (m & 3) (dy, rows of 256 bytes) or c ^ 2 (m / 2 & 3) (x, rows of
// 128), so that the rows that 32 lanes read together fall on different banks.  777 x 1531 x 5024 takes 19.7 us: thirteen
// steps of two workgroups a compute unit (12 us), 31 MB of results (6 us), and the first loads.
template <int BN, int BK, int WR, int WC, bool X5>
__global__ __launch_bounds__(WR * WC * 64) void wgrad_turn_kernel(const WgradParams p, int tiles_n, int tiles_k, int group)
{
    constexpr int NT = WR * WC * 64, FA = BN / WR / 32, FB = BK / WC / 32;
    constexpr int CD = BN / 8, CX = BK / 16, LD = 64 * CD / NT, LX = 64 * CX / NT, XAT = 64 * BN * 2, SAT = XAT + 64 * BK, STAGE = SAT + 256;
    static_assert(LD * NT == 64 * CD && LX * NT == 64 * CX && LD == 4 && LX == 2 && NT / CD % 4 == 0 && NT / CX % 8 == 0 && BK == 128, "shares of a step, one scale a row");
    extern __shared__ __align__(16) unsigned char lds[];
    int tn, tk;
    tile_of(blockIdx.x, tiles_n * tiles_k, tiles_n, tiles_k, group, tn, tk);
    const int n0 = tn * BN, k0 = tk * BK, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wn = wave / WC * (BN / WR), wk = wave % WC * (BK / WC), i16 = lane & 15, g16 = lane >> 4 & 1, h = lane >> 5;
    const int steps = (p.M + 63) >> 6;

    auto turn_x = [](int m) { return (m >> 1 & 3) << 1; };
    // where this thread's chunks come from, within 64 rows; chunks beyond the last column read the last one, and their sums go nowhere.
    // (An aligned chunk with one element inside the matrix lies on its page.)
    unsigned int od[LD], ox[LX];
    {
        const int m = tid / CD, n = min(n0 + ((tid % CD) ^ ((m & 3) << 2)) * 8, (p.N - 1) & ~7);
#pragma unroll
        for (int i = 0; i < LD; ++i) od[i] = ((unsigned int)(m + i * (NT / CD)) * (unsigned int)p.lddy + (unsigned int)n) * 2u;
    }
    {
        const int m = tid / CX, k = min(k0 + ((tid % CX) ^ turn_x(m)) * 16, (p.K - 1) & ~15);
#pragma unroll
        for (int i = 0; i < LX; ++i) ox[i] = (unsigned int)(m + i * (NT / CX)) * (unsigned int)p.ldx + (unsigned int)k;
    }
    const unsigned int wide_n = (unsigned int)((p.N + 7) & ~7) * 2u, wide_k = (unsigned int)((p.K + 15) & ~15);
    auto load = [&](int t, unsigned char* to) {                         // rows beyond the last arrive as zeros
        const long long m0 = (long long)t * 64;
        const unsigned int last = (unsigned int)min(64, p.M - (int)m0) - 1;
        const Window d = window(p.dy + m0 * p.lddy, last * (unsigned int)p.lddy * 2u + wide_n);
        const Window x = window(p.x + m0 * p.ldx, last * (unsigned int)p.ldx + wide_k);
#pragma unroll
        for (int i = 0; i < LD; ++i) load_to_lds(d, od[i], 0, lds_address(to) + (i * NT + wave * 64) * 16);
#pragma unroll
        for (int i = 0; i < LX; ++i) load_to_lds(x, ox[i], 0, lds_address(to) + XAT + (i * NT + wave * 64) * 16);
    };
    // Scales: the words that hold this tile's bytes come into LDS a step ahead of the step's operands (the first wavefront asks for
    // them), and become numbers there while the step before is multiplied.
    unsigned char* const words = lds + 3 * STAGE;
    auto load_scales = [&](int t) {
        const long long m0 = (long long)t * 64;
        const unsigned int last = (unsigned int)min(64, p.M - (int)m0) - 1;
        load_word_to_lds(window(p.xs + m0 * p.ldxs, last * (unsigned int)p.ldxs + (unsigned int)p.ldxs), min((unsigned int)lane, last) * (unsigned int)p.ldxs + (unsigned int)(k0 >> 7 & ~3), 0,
                         lds_address(words) + t % 3 * 256);
    };
    auto put_scales = [&](int t, unsigned char* to) {
        if (tid < 64) {
            const unsigned int w = *reinterpret_cast<const unsigned int*>(words + t % 3 * 256 + tid * 4);
            *reinterpret_cast<float*>(to + SAT + tid * 4) = e8m0_value(w >> (8 * ((k0 >> 7) & 3)) & 255u);
        }
    };

    // what this lane reads of each square of 32 columns, relative to a step's place
    unsigned int ad[FA], ax[FB];
#pragma unroll
    for (int a = 0; a < FA; ++a) {
        const int c = (wn >> 3) + 4 * a + 2 * g16 + (i16 >> 1 & 1), m = 8 * h + (i16 >> 2);
        ad[a] = (unsigned int)(m * (BN * 2) + ((c ^ ((m & 3) << 2)) << 4) + (i16 & 1) * 8);
    }
#pragma unroll
    for (int b = 0; b < FB; ++b) {
        const int c = (wk >> 4) + 2 * b + g16, m = 8 * h + (i16 >> 1);
        ax[b] = (unsigned int)(XAT + m * BK + ((c ^ turn_x(m)) << 4) + (i16 & 1) * 8);
    }
    const unsigned int as = (unsigned int)(SAT + h * 32);

    v16f acc[FA][FB];
#pragma unroll
    for (int a = 0; a < FA; ++a)
#pragma unroll
        for (int b = 0; b < FB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[a][b][i] = 0.0f;
    typedef __attribute__((address_space(3))) v4s* lds16;
    typedef __attribute__((address_space(3))) v2i* lds8;

    auto compute = [&](const unsigned char* at) {
#pragma unroll
        for (int s = 0; s < 4; ++s) {                                   // sixteen rows
            const v4f s0 = *reinterpret_cast<const v4f*>(at + as + s * 64), s1 = *reinterpret_cast<const v4f*>(at + as + s * 64 + 16);
            const float sc[8] = {s0[0], s0[1], s0[2], s0[3], s1[0], s1[1], s1[2], s1[3]};
            v8bf x[FB];
#pragma unroll
            for (int b = 0; b < FB; ++b) {
                const v2i c = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds8)(at + ax[b] + s * (16 * BK)));
                v4i r;
#pragma unroll
                for (int i = 0; i < 2; ++i) {                           // rows 4i .. 4i + 3
                    r[2 * i] = two_rows<X5, false>(c[i], sc[4 * i], sc[4 * i + 1]);
                    r[2 * i + 1] = two_rows<X5, true>(c[i], sc[4 * i + 2], sc[4 * i + 3]);
                }
                x[b] = __builtin_bit_cast(v8bf, r);
            }
#pragma unroll
            for (int a = 0; a < FA; ++a) {
                const v4s d0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds16)(at + ad[a] + s * (32 * BN)));
                const v4s d1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds16)(at + ad[a] + s * (32 * BN) + 8 * BN));
                const v8bf d = __builtin_bit_cast(v8bf, __builtin_shufflevector(d0, d1, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                for (int b = 0; b < FB; ++b) acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[b], d, acc[a][b], 0, 0, 0);
            }
        }
    };

    unsigned char *now = lds, *next = lds + STAGE, *after = lds + 2 * STAGE;
    load(0, now);
    if (wave == 0) { load_scales(0); if (steps > 1) load_scales(1); }
    wait_loads();
    if (steps > 1) load(1, next);
    if (wave == 0 && steps > 2) load_scales(2);
    __syncthreads();
    put_scales(0, now);
    for (int t = 0; t < steps; ++t) {
        // what was asked for a step ago, and nothing older, may still be on its way: LD + LX loads, the first wavefront's scales
        if (t + 2 < steps && wave == 0) wait_loads<LD + LX + 1>(); else if (t + 1 < steps) wait_loads<LD + LX>(); else wait_loads();
        __syncthreads();
        if (t + 1 < steps) put_scales(t + 1, next);
        if (t + 2 < steps) load(t + 2, after);
        if (t + 3 < steps && wave == 0) load_scales(t + 3);
        compute(now);
        unsigned char* u = now;
        now = next; next = after; after = u;
    }
    __syncthreads();                                                    // (LDS is free for the results)
    v4f* place = reinterpret_cast<v4f*>(lds + wave * 4096);
#pragma unroll
    for (int a = 0; a < FA; ++a)
#pragma unroll
        for (int b = 0; b < FB; ++b) {
            put_square(place, lane, acc[a][b]);
#pragma unroll
            for (int i = 0; i < 4; ++i) store_dw(p, n0 + wn + a * 32 + 8 * i + (lane >> 3), k0 + wk + b * 32 + 4 * (lane & 7), place[quarter_slot(i, lane)]);
        }
}

// ---- small gradients, the rows dealt out: 32 FN x 64 of dw a workgroup, its eight wavefronts taking 64 rows in turn, each in a place of its own
// in LDS (no barrier before the sums are joined, in the order of the wavefronts).  The next rows are asked for when these have been read.
// Chunk c of row m stands at position c ^ 4 (m / 2 & 1) (dy, rows of 128 bytes; of 64: c), c ^ 2 (m / 4 & 1) (x, rows of 64).
template <int FN, bool X5>
__global__ __launch_bounds__(512) void wgrad_split_kernel(const WgradParams p, int tiles_n, int tiles_k, int group)
{
    constexpr int W = 8, FK = 2, BN = 32 * FN, BK = 64, CD = 4 * FN, LD = 4 * FN, LX = 4, XAT = 128 * BN, SAT = XAT + 64 * BK, SUMS = FN * FK * 4096, OWN = SAT + 256 > SUMS ? SAT + 256 : SUMS;
    extern __shared__ __align__(16) unsigned char lds[];
    int tn, tk;
    tile_of(blockIdx.x, tiles_n * tiles_k, tiles_n, tiles_k, group, tn, tk);
    const int n0 = tn * BN, k0 = tk * BK, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i16 = lane & 15, g16 = lane >> 4 & 1, h = lane >> 5;
    const int steps = (p.M + 63) >> 6;
    unsigned char* own = lds + wave * OWN;
    const unsigned int own0 = lds_address(own);
    auto turn_d = [](int m) { return FN == 2 ? (m >> 1 & 1) << 2 : 0; };
    auto turn_x = [](int m) { return (m >> 2 & 1) << 1; };
    unsigned int od[LD], ox[LX];                                        // (as above)
#pragma unroll
    for (int i = 0; i < LD; ++i) {
        const int m = lane / CD + i * (64 / CD), n = min(n0 + ((lane % CD) ^ turn_d(m)) * 8, (p.N - 1) & ~7);
        od[i] = ((unsigned int)m * (unsigned int)p.lddy + (unsigned int)n) * 2u;
    }
#pragma unroll
    for (int i = 0; i < LX; ++i) {
        const int m = (lane >> 2) + i * 16, k = min(k0 + ((lane & 3) ^ turn_x(m)) * 16, (p.K - 1) & ~15);
        ox[i] = (unsigned int)m * (unsigned int)p.ldx + (unsigned int)k;
    }
    const unsigned int wide_n = (unsigned int)((p.N + 7) & ~7) * 2u, wide_k = (unsigned int)((p.K + 15) & ~15);
    auto load = [&](int t) {                                            // rows beyond the last arrive as zeros
        const long long m0 = (long long)t * 64;
        const unsigned int last = (unsigned int)min(64, p.M - (int)m0) - 1;
        const Window d = window(p.dy + m0 * p.lddy, last * (unsigned int)p.lddy * 2u + wide_n);
        const Window x = window(p.x + m0 * p.ldx, last * (unsigned int)p.ldx + wide_k);
        load_word_to_lds(window(p.xs + m0 * p.ldxs, last * (unsigned int)p.ldxs + (unsigned int)p.ldxs), min((unsigned int)lane, last) * (unsigned int)p.ldxs + (unsigned int)(k0 >> 7 & ~3), 0, own0 + SAT);
#pragma unroll
        for (int i = 0; i < LD; ++i) load_to_lds(d, od[i], 0, own0 + i * 1024);
#pragma unroll
        for (int i = 0; i < LX; ++i) load_to_lds(x, ox[i], 0, own0 + XAT + i * 1024);
    };
    unsigned int ad[FN], ax[FK];
#pragma unroll
    for (int a = 0; a < FN; ++a) {
        const int c = 4 * a + 2 * g16 + (i16 >> 1 & 1), m = 8 * h + (i16 >> 2);     // (m + 4 stands alike)
        ad[a] = own0 + (unsigned int)(m * (BN * 2) + ((c ^ turn_d(m)) << 4) + (i16 & 1) * 8);
    }
#pragma unroll
    for (int b = 0; b < FK; ++b) {
        const int c = 2 * b + g16, m = 8 * h + (i16 >> 1);
        ax[b] = own0 + (unsigned int)(XAT + m * BK + ((c ^ turn_x(m)) << 4) + (i16 & 1) * 8);
    }
    typedef __attribute__((address_space(3))) v4s* lds16;
    typedef __attribute__((address_space(3))) v2i* lds8;
    v16f acc[FN][FK];
#pragma unroll
    for (int a = 0; a < FN; ++a)
#pragma unroll
        for (int b = 0; b < FK; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[a][b][i] = 0.0f;
    if (wave < steps) load(wave);
    for (int t = wave; t < steps; t += W) {
        v4s d[4][FN][2];
        v2i c[4][FK];
        v4f sc[4][2];
        wait_loads();
        {                                                               // the scale word of this lane's row becomes its number
            const unsigned int w = *reinterpret_cast<const unsigned int*>(own + SAT + lane * 4);
            *reinterpret_cast<float*>(own + SAT + lane * 4) = e8m0_value(w >> (8 * ((k0 >> 7) & 3)) & 255u);
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
#pragma unroll
            for (int a = 0; a < FN; ++a)
#pragma unroll
                for (int i = 0; i < 2; ++i) d[s][a][i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds16)(uintptr_t)(ad[a] + s * (32 * BN) + i * (8 * BN)));
#pragma unroll
            for (int b = 0; b < FK; ++b) c[s][b] = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds8)(uintptr_t)(ax[b] + s * (16 * BK)));
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");              // (the numbers are written)
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int i = 0; i < 2; ++i) sc[s][i] = *reinterpret_cast<const v4f*>(own + SAT + s * 64 + h * 32 + i * 16);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");              // (the reads have ended: the place is free)
        __builtin_amdgcn_sched_barrier(0);
        if (t + W < steps) load(t + W);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            v8bf x[FK];
#pragma unroll
            for (int b = 0; b < FK; ++b) {
                v4i r;
#pragma unroll
                for (int i = 0; i < 2; ++i) {                           // rows 4i .. 4i + 3
                    r[2 * i] = two_rows<X5, false>(c[s][b][i], sc[s][i][0], sc[s][i][1]);
                    r[2 * i + 1] = two_rows<X5, true>(c[s][b][i], sc[s][i][2], sc[s][i][3]);
                }
                x[b] = __builtin_bit_cast(v8bf, r);
            }
#pragma unroll
            for (int a = 0; a < FN; ++a) {
                const v8bf y = __builtin_bit_cast(v8bf, __builtin_shufflevector(d[s][a][0], d[s][a][1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                for (int b = 0; b < FK; ++b) acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[b], y, acc[a][b], 0, 0, 0);
            }
        }
    }
#pragma unroll
    for (int a = 0; a < FN; ++a)
#pragma unroll
        for (int b = 0; b < FK; ++b) put_square(reinterpret_cast<v4f*>(own) + (a * FK + b) * 256, lane, acc[a][b]);
    __syncthreads();
    for (int t = wave; t < FN * FK * 4; t += W) {                         // a quarter of a square
        const int a = (t >> 2) / FK, b = (t >> 2) % FK, i = t & 3, at = (t >> 2) * 256 + quarter_slot(i, lane);
        v4f s = reinterpret_cast<const v4f*>(lds)[at];
#pragma unroll
        for (int q = 1; q < W; ++q) s += reinterpret_cast<const v4f*>(lds + q * OWN)[at];
        store_dw(p, n0 + a * 32 + 8 * i + (lane >> 3), k0 + b * 32 + 4 * (lane & 7), s);
    }
}

// ---- large gradients: 256 x 256 of dw by four wavefronts, one on a SIMD, each 128 x 128 of it.  As above, but a wavefront overlaps its own
// work.  While sixteen rows are multiplied (sixteen matrix instructions), behind each of them stands a sixteenth of: the reads of the next
// sixteen rows of dy, the reads of the codes after the next, the conversion of the next codes, the loads of the step after the next.  A
// wavefront issues an instruction in four cycles, so a matrix instruction (32 cycles) hides seven others: they are dealt out evenly.
// Halfway through a step comes its barrier: the next step has arrived, the place of the step before is free.  8192 x 11008 x 4096 takes 611 us,
// 1210 TFLOP/s (a large library product in bf16 1619); the matrix instructions are busy 57 % of the cycles at a clock that they lower.
template <bool X5>
__global__ __launch_bounds__(256) void wgrad_large_kernel(const WgradParams p, int tiles_n, int tiles_k, int group)
{
    constexpr int BN = 256, BK = 256, XAT = 64 * BN * 2, SAT = XAT + 64 * BK, STAGE = SAT + 512, LD = 8, LX = 4;
    extern __shared__ __align__(16) unsigned char lds[];
    int tn, tk;
    tile_of(blockIdx.x, tiles_n * tiles_k, tiles_n, tiles_k, group, tn, tk);
    const int n0 = tn * BN, k0 = tk * BK, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wn = wave >> 1 << 7, wk = (wave & 1) << 7, i16 = lane & 15, g16 = lane >> 4 & 1, h = lane >> 5;
    const int steps = (p.M + 63) >> 6;
    const unsigned int lds0 = lds_address(lds);
    unsigned int od[LD], ox[LX];
    {
        const int m = tid >> 5, n = min(n0 + ((tid & 31) ^ ((m & 3) << 2)) * 8, (p.N - 1) & ~7);
#pragma unroll
        for (int i = 0; i < LD; ++i) od[i] = ((unsigned int)(m + i * 8) * (unsigned int)p.lddy + (unsigned int)n) * 2u;
    }
    {
        const int m = tid >> 4, k = min(k0 + ((tid & 15) ^ ((m & 7) << 1)) * 16, (p.K - 1) & ~15);
#pragma unroll
        for (int i = 0; i < LX; ++i) ox[i] = (unsigned int)(m + i * 16) * (unsigned int)p.ldx + (unsigned int)k;
    }
    const unsigned int wide_n = (unsigned int)((p.N + 7) & ~7) * 2u, wide_k = (unsigned int)((p.K + 15) & ~15);
    // the rows of step t; behind the last step nothing (zeros arrive, in a place that nobody reads)
    auto rows_of = [&](const void* base, long long ld, unsigned int wide, int t) {
        const int left = p.M - t * 64;
        return window(reinterpret_cast<const unsigned char*>(base) + (long long)min(t, steps - 1) * 64 * ld, left > 0 ? (unsigned int)(min(64, left) - 1) * (unsigned int)ld + wide : 0u);
    };
    auto load_d = [&](const Window& w, int i, unsigned int to) { load_to_lds(w, od[i], 0, to + i * 4096 + (wave << 10)); };
    auto load_x = [&](const Window& w, int i, unsigned int to) { load_to_lds(w, ox[i], 0, to + XAT + i * 4096 + (wave << 10)); };
    // the words that hold this tile's scale bytes: a place for every wavefront and three steps
    const unsigned int so = (unsigned int)lane * (unsigned int)p.ldxs + (unsigned int)(k0 >> 7 & ~3);
    auto load_scales = [&](int t, int place) { load_word_to_lds(rows_of(p.xs, p.ldxs, (unsigned int)p.ldxs, t), so, 0, lds0 + 3 * STAGE + (place * 4 + wave) * 256); };
    auto put_scales = [&](int place, unsigned char* to) {               // (rows beyond the last: byte 0, a finite scale of codes that are 0)
        if (tid < 128) {
            const unsigned int w = *reinterpret_cast<const unsigned int*>(lds + 3 * STAGE + (place * 4 + wave) * 256 + (tid & 63) * 4);
            *reinterpret_cast<float*>(to + SAT + tid * 4) = e8m0_value(w >> (8 * (((k0 >> 7) + (tid >> 6)) & 3)) & 255u);
        }
    };

    // where this lane reads: dy's squares, the codes' squares, the scales
    unsigned int ad[4], ax[4], as = lds0 + (unsigned int)(SAT + (wk >> 7) * 256 + h * 32);
#pragma unroll
    for (int a = 0; a < 4; ++a) {
        const int c = (wn >> 3) + 4 * a + 2 * g16 + (i16 >> 1 & 1), m = 8 * h + (i16 >> 2);
        ad[a] = lds0 + (unsigned int)(m * (BN * 2) + ((c ^ ((m & 3) << 2)) << 4) + (i16 & 1) * 8);
        const int cx = (wk >> 4) + 2 * a + g16, mx = 8 * h + (i16 >> 1);
        ax[a] = lds0 + (unsigned int)(XAT + mx * BK + ((cx ^ ((mx & 7) << 1)) << 4) + (i16 & 1) * 8);
    }
    typedef __attribute__((address_space(3))) v4s* lds16;
    typedef __attribute__((address_space(3))) v2i* lds8;
    typedef __attribute__((address_space(3))) v4f* ldsf;

    v16f acc[4][4];
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[a][b][i] = 0.0f;
    v4s d[2][4][2];
    v2i c[2][4];
    v4f sc[2][2];
    v4i x[2][4];
    auto read_d = [&](int s, int i) { d[s & 1][i >> 1][i & 1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds16)(uintptr_t)(ad[i >> 1] + s * (32 * BN) + (i & 1) * (8 * BN))); };
    auto read_c = [&](int s, int i) {
        if (i < 2) sc[s & 1][i] = *(ldsf)(uintptr_t)(as + s * 64 + i * 16);
        else c[s & 1][i - 2] = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds8)(uintptr_t)(ax[i - 2] + s * (16 * BK)));
    };
    auto convert = [&](int s, int i) {                                  // a word: two of a column's eight codes
        const int b = i >> 2, k = i & 3;
        const v4f f = sc[s & 1][k >> 1];
        const int w = k & 1 ? two_rows<X5, true>(c[s & 1][b][k >> 1], f[2], f[3]) : two_rows<X5, false>(c[s & 1][b][k >> 1], f[0], f[1]);
        x[s & 1][b][k] = w;
        asm volatile("" : "+v"(x[s & 1][b][k]));                        // (here, and not where it is used)
    };
    auto multiply = [&](int s, int i) {
        const int a = i >> 2, b = i & 3;
        const v8bf y = __builtin_bit_cast(v8bf, __builtin_shufflevector(d[s & 1][a][0], d[s & 1][a][1], 0, 1, 2, 3, 4, 5, 6, 7));
        acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, x[s & 1][b]), y, acc[a][b], 0, 0, 0);
    };

#pragma unroll
    for (int t = 0; t < 2; ++t) {                                       // two steps' operands, three steps' scale words
        const Window wd = rows_of(p.dy, p.lddy * 2, wide_n, t), wx = rows_of(p.x, p.ldx, wide_k, t);
#pragma unroll
        for (int i = 0; i < LD; ++i) load_d(wd, i, lds0 + t * STAGE);
#pragma unroll
        for (int i = 0; i < LX; ++i) load_x(wx, i, lds0 + t * STAGE);
        load_scales(t, t);
    }
    load_scales(2, 2);
    wait_loads();
    __syncthreads();
    put_scales(0, lds);
    put_scales(1, lds + STAGE);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) read_d(0, i);
#pragma unroll
    for (int i = 0; i < 6; ++i) { read_c(0, i); read_c(1, i); }
#pragma unroll
    for (int i = 0; i < 16; ++i) convert(0, i);
    int r = 0;                                                          // t modulo 3: the place of step t
    for (int t = 0; t < steps; ++t) {
        const int r1 = r == 2 ? 0 : r + 1, r2 = r1 == 2 ? 0 : r1 + 1;   // ... of step t + 1, of step t + 2
        const unsigned int hop = (unsigned int)(r1 - r) * STAGE;
        auto part = [&](auto S) {                                       // sixteen rows
            constexpr int s = decltype(S)::value;
            if (s == 2) {                                               // from here on codes and scales are the next step's, a sixteen later dy
#pragma unroll
                for (int a = 0; a < 4; ++a) ax[a] += hop;
                as += hop;
            }
            if (s == 3) {
#pragma unroll
                for (int a = 0; a < 4; ++a) ad[a] += hop;
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                multiply(s, i);
                if (i & 1) read_d((s + 1) & 3, i >> 1);
                else if (i < 12) read_c((s + 2) & 3, i >> 1);
                convert(s + 1, i);
                if (s == 2 && (i & 1) == 0) load_d(rows_of(p.dy, p.lddy * 2, wide_n, t + 2), i >> 1, lds0 + r2 * STAGE);
                if (s == 3 && i < 8 && (i & 1) == 0) load_x(rows_of(p.x, p.ldx, wide_k, t + 2), i >> 1, lds0 + r2 * STAGE);
                if (s == 3 && i == 8) load_scales(t + 3, r);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        part(std::integral_constant<int, 0>{});
        part(std::integral_constant<int, 1>{});
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        put_scales(r2, lds + r2 * STAGE);
        part(std::integral_constant<int, 2>{});
        part(std::integral_constant<int, 3>{});
        r = r1;
    }
    wait_loads();
    __syncthreads();                                                    // (LDS is free for the results)
    v4f* place = reinterpret_cast<v4f*>(lds + wave * 4096);
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            put_square(place, lane, acc[a][b]);
#pragma unroll
            for (int i = 0; i < 4; ++i) store_dw(p, n0 + wn + a * 32 + 8 * i + (lane >> 3), k0 + wk + b * 32 + 4 * (lane & 7), place[quarter_slot(i, lane)]);
        }
}

template <bool X5> static hipError_t wgrad_large_go(const WgradParams& p, hipStream_t st)
{
    const int tn = (p.N + 255) / 256, tk = (p.K + 255) / 256, bytes = 3 * (64 * 512 + 64 * 256 + 512) + 3 * 4 * 256;
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&wgrad_large_kernel<X5>), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(wgrad_large_kernel<X5>, dim3((unsigned)(tn * tk)), dim3(256), bytes, st, p, tn, tk, 8);
    return hipGetLastError();
}

template <int FN, bool X5> static hipError_t wgrad_split_go(const WgradParams& p, hipStream_t st)
{
    const int tn = (p.N + 32 * FN - 1) / (32 * FN), tk = (p.K + 63) / 64, own = 4096 * FN + 4096 + 256, bytes = 8 * (own > FN * 8192 ? own : FN * 8192);
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&wgrad_split_kernel<FN, X5>), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((wgrad_split_kernel<FN, X5>), dim3((unsigned)(tn * tk)), dim3(512), bytes, st, p, tn, tk, 8);
    return hipGetLastError();
}
template <int BN, int BK, int WR, int WC, bool X5> static hipError_t wgrad_turn_go(const WgradParams& p, hipStream_t st)
{
    const int tn = (p.N + BN - 1) / BN, tk = (p.K + BK - 1) / BK, bytes = 3 * (64 * BN * 2 + 64 * BK + 256) + 3 * 256;
    if (bytes > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&wgrad_turn_kernel<BN, BK, WR, WC, X5>), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((wgrad_turn_kernel<BN, BK, WR, WC, X5>), dim3((unsigned)(tn * tk)), dim3(WR * WC * 64), bytes, st, p, tn, tk, 8);
    return hipGetLastError();
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
template <bool X5> static hipError_t go(const WgradParams& p, int choice, hipStream_t st)
{
    switch (choice) {
    case sopr::WGRAD_32x64: return wgrad_split_go<1, X5>(p, st);
    case sopr::WGRAD_64x64: return wgrad_split_go<2, X5>(p, st);
    case sopr::WGRAD_128x128: return wgrad_turn_go<128, 128, 2, 2, X5>(p, st);
    case sopr::WGRAD_256x256: return wgrad_large_go<X5>(p, st);
    case sopr::WGRAD_ANY_64x128: return wgrad_go<64, 128, 2, 2, X5>(p, st);
    case sopr::WGRAD_ANY_128x128: return wgrad_go<128, 128, 2, 2, X5>(p, st);
    case sopr::WGRAD_ANY_256x256: return wgrad_go<256, 256, 2, 4, X5>(p, st);
    }
    return hipErrorInvalidValue;
}

}  // namespace sopk

extern "C" hipError_t sopk_wgrad_launch(const WgradParams* p, int x_e5m2, int choice, void* stream)
{
    return x_e5m2 ? sopk::go<true>(*p, choice, (hipStream_t)stream) : sopk::go<false>(*p, choice, (hipStream_t)stream);
}
