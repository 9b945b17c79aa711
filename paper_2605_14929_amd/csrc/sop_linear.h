// What the products of a linear layer with narrow operands share between the host side (sop_linear_api.cpp) and the
// kernels: launch parameters, the rules that choose a variant, and small device helpers.
#ifndef SOP_LINEAR_H
#define SOP_LINEAR_H
#include <stdint.h>

/* Quantiser into 8-bit floats with one power-of-two scale for each block of 128 (rows x 128, rows = 1 or 128) */
struct F8QuantParams {
    const void* x; long long ldx;            // elements
    long long M, K;
    unsigned char* codes; long long ldc;     // bytes
    unsigned char* scales; long long lds;    // bytes; [M or ceil(M/128)][ceil(K/128)]
    unsigned char* codes_t; long long ldct;  // null: not written; [K][M]
};

/* Gated unit: h = silu(gate) * up, all three into 8 bits */
struct F8Out { unsigned char* codes; long long ldc; unsigned char* scales; long long lds; };
struct F8In { const unsigned char* codes; long long ldc; const unsigned char* scales; long long lds; };
struct F8GatedParams {
    const void* gate; long long ldg;         // elements
    const void* up; long long ldu;
    long long M, F;
    F8Out h, g8, u8;
};
/* ... and its gradient from the 8-bit checkpoints */
struct F8GatedGradParams {
    F8In g8, u8;
    const void* dh; long long lddh;          // elements
    long long M, F;
    void* dgate; long long lddg;             // of dh's type
    void* dup; long long lddu;
    F8Out dg8, du8;
};

/* y[m, n] = sum over blocks b of 2^(xs[m, b] + ws[n / 128, b] - 254) sum_{k in b} x[m, k] w[n, k] */
struct F8MmParams {
    const unsigned char* x; long long ldx; const unsigned char* xs; long long ldxs;
    const unsigned char* w; long long ldw; const unsigned char* ws; long long ws_n, ws_k;   // scale of block (n / 128, k / 128) at n * ws_n + k * ws_k
    int M, N, K;
    void* y; long long ldy; int out_bf16;
};

/* dw[n, k] = sum_m dy[m, n] x[m, k] 2^(xs[m, k / 128] - 127) (+ dw) */
struct WgradParams {
    const uint16_t* dy; long long lddy;      // bf16
    const unsigned char* x; long long ldx; const unsigned char* xs; long long ldxs;
    int M, N, K;
    void* dw; long long lddw; int out_bf16, accumulate;
};

/* y[m, n] = sum_k x[m, k] s[n, k / g] L_sel[code[n, k]] */
#define SOP_K_PACKED_TAB 64
struct PackedMmParams {
    const uint16_t* x; long long ldx;        // bf16
    const uint16_t* words; const unsigned char* payload;
    int M, N, K, g, n_bits;
    int mag_shift, mag_mask, man_bits, man_mask, exp_off;   // scale = (mantissa with its leading one) * 2^(max(e, 1) + exp_off)
    int sign_up, sel_pos, sel_mask;          // word << sign_up has the sign in bit 31 (0: none); selector = word >> sel_pos & sel_mask
    uint16_t* y; long long ldy;              // bf16
    float tab[2][SOP_K_PACKED_TAB];
};

#if defined(__HIPCC__)
#define SOP_HD __host__ __device__ inline
#else
#define SOP_HD inline
#endif
/* What the wide packed kernel adds, the same for all lanes, to its lanes' offsets into its three windows at step t (64 elements along K each).  It asks
 * for two steps more than there are.  A window's check compares a lane's offset with what the window has left beyond this sum, so the sum
 * never passes the window's end, which with one row left is the end of K: the steps behind the last one ask for the last one again. */
struct PackedStepAt { int x, codes, words; };                              // bytes
SOP_HD PackedStepAt packed_step_at(int t, int steps, int nb, int lg, bool half)
{
    const bool end = t >= steps - 1;                                       // half: K ends in the middle of sixteen codes, and the last step's begin eight earlier
    const int k = end ? steps - 1 : t;
    return PackedStepAt{k * 128, k * 8 * nb - (half && end ? nb : 0), k * (128 >> lg)};
}

#if defined(__HIPCC__)
namespace sopk {
typedef int v2i __attribute__((ext_vector_type(2)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));

// 2^(b - 127); 255 stands for NaN
__device__ __forceinline__ float e8m0_value(unsigned int b)
{
    const unsigned int bits = b == 0 ? 0x00400000u : (b == 255 ? 0x7FC00000u : b << 23);
    return __uint_as_float(bits);
}
// nearest bf16 (ties to even) of a number that is no NaN, or a NaN, in the low 16 bits
__device__ __forceinline__ unsigned int bf16_bits(float x)
{
    return (unsigned int)__builtin_bit_cast(unsigned short, (__bf16)x);
}
__device__ __forceinline__ unsigned int bf16_pair(float lo, float hi)
{
    v2bf v;
    v[0] = (__bf16)lo; v[1] = (__bf16)hi;
    return __builtin_bit_cast(unsigned int, v);
}
// eight 8-bit floats times a scale, as bf16: exact within its normal numbers
template <bool E5M2> __device__ __forceinline__ v4i eight_bf16(unsigned int lo, unsigned int hi, float s)
{
    v4i r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const unsigned int w = i ? hi : lo;
        const v2bf a = E5M2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, s, false) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, false);
        const v2bf b = E5M2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, s, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, true);
        r[2 * i] = __builtin_bit_cast(int, a);
        r[2 * i + 1] = __builtin_bit_cast(int, b);
    }
    return r;
}
// The tiles of an operand in LDS: rows of 128 bytes, eight chunks of 16.  Chunk c of row r stands at position c ^ swz(r), so that
// the 16 rows that one matrix instruction reads at the same c, and rows 2 or 4 apart that a transposing store writes, fall on
// different banks.
__device__ __forceinline__ int swz(int r) { return (r ^ (r >> 3)) & 7; }

// One step of 64 elements of a product of bf16 operands whose tiles stand in LDS as above: acc[a][b] holds rows 4q .. 4q + 3 of b's
// sixteen and column r16 of a's sixteen.
template <int FA, int FB>
__device__ __forceinline__ void bf16_step(const unsigned char* ta, const unsigned char* tb, int ra, int rb, int q, v4f (&acc)[FA][FB])
{
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        v8bf fb[FB];
#pragma unroll
        for (int b = 0; b < FB; ++b) { const int r = rb + b * 16; fb[b] = *reinterpret_cast<const v8bf*>(tb + r * 128 + (((4 * s + q) ^ swz(r)) << 4)); }
#pragma unroll
        for (int a = 0; a < FA; ++a) {
            const int r = ra + a * 16;
            const v8bf fa = *reinterpret_cast<const v8bf*>(ta + r * 128 + (((4 * s + q) ^ swz(r)) << 4));
#pragma unroll
            for (int b = 0; b < FB; ++b) acc[a][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[b], fa, acc[a][b], 0, 0, 0);
        }
    }
}
// Operands read 16 bytes a lane for 32 x 32 squares: chunk c of a 128-byte row r stands at position c ^ (r >> 1 & 7).  LDS serves such a read
// sixteen lanes at a time (0-3, 12-15, 20-23 and 24-27, then the others of the first 32, ...), whose rows so fall on different banks.
// Results.  acc[i] of a 32 x 32 square is row 8 (i / 4) + 4 (lane >> 5) + i % 4, column lane & 31, and the rows are what lies side by side in memory: to be
// written line by line, a square passes through 4 KB of LDS.  Four rows j of a column m stand at slot 32 j + (m ^ 2 j), so that both ways
// the lanes served together fall on different banks.  Of the four quarters (eight columns) that come out again, lane l has rows 4 (l & 7), column
// 8 quarter + (l >> 3).  A weight gradient of
// 64 x 4096 x 4096 takes 16.8 us by it, 18.4 straight from the registers; one of 26 x 1920 x 4793, in bf16, whose rows lie on odd addresses, 12.1 and 28.5.
__device__ __forceinline__ void put_square(v4f* place, int lane, const v16f& acc)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int j = 2 * i + (lane >> 5);
        place[32 * j + ((lane & 31) ^ 2 * j)] = v4f{acc[4 * i], acc[4 * i + 1], acc[4 * i + 2], acc[4 * i + 3]};
    }
}
__device__ __forceinline__ int quarter_slot(int quarter, int lane) { return 32 * (lane & 7) + ((8 * quarter + (lane >> 3)) ^ 2 * (lane & 7)); }
// four neighbours in memory, on any address of their type: as binary32, or rounded to bf16
struct __attribute__((packed, aligned(4))) FourWords { v4f v; };
struct __attribute__((packed, aligned(2))) FourHalves { unsigned int v[2]; };
__device__ __forceinline__ void put_four(float* y, v4f v) { reinterpret_cast<FourWords*>(y)->v = v; }
__device__ __forceinline__ void put_four(uint16_t* y, v4f v)
{
    FourHalves* to = reinterpret_cast<FourHalves*>(y);
    to->v[0] = bf16_pair(v[0], v[1]);
    to->v[1] = bf16_pair(v[2], v[3]);
}
// zeroes the bytes of a 16-byte chunk beyond the first `n`
__device__ __forceinline__ v4i keep_bytes(v4i v, int n)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int k = n - 4 * i;
        v[i] = k >= 4 ? v[i] : k <= 0 ? 0 : (int)((unsigned int)v[i] & ((1u << (8 * k)) - 1u));
    }
    return v;
}
// `bytes` bytes from p on, for loads at byte offsets at + uni (uni the same for all lanes); what lies beyond arrives as zeros.
struct Window { v4i r; };
__device__ __forceinline__ Window window(const void* p, unsigned int bytes)
{
    const unsigned long long a = reinterpret_cast<unsigned long long>(p);
    return Window{v4i{__builtin_amdgcn_readfirstlane((int)a), __builtin_amdgcn_readfirstlane((int)(a >> 32) & 0xFFFF), __builtin_amdgcn_readfirstlane((int)bytes), 0x00027000}};
}
__device__ __forceinline__ auto resource(const Window& w)
{
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>((unsigned long long)(unsigned int)w.r[0] | (unsigned long long)(unsigned int)w.r[1] << 32), 0, w.r[2], 0x00027000);
}
__device__ __forceinline__ unsigned int load_word(const Window& w, unsigned int at, unsigned int uni)
{
    return (unsigned int)__builtin_amdgcn_raw_buffer_load_b32(resource(w), (int)at, (int)uni, 0);
}
// ... 16 (or 4) bytes a lane straight into LDS, lane by lane from `to` on (the same for all lanes).  Written out so that the compiler does not
// wait for them by itself before other reads of LDS: whoever reads what they bring waits for its own wavefront's loads (wait_loads),
// then meets the others at a barrier.  (m0, which holds the place in LDS, is written right before each use by whoever uses it.)
__device__ __forceinline__ unsigned int lds_address(const unsigned char* p)
{
    return (unsigned int)__builtin_amdgcn_readfirstlane((int)(unsigned int)reinterpret_cast<uintptr_t>((const __attribute__((address_space(3))) unsigned char*)p));
}
__device__ __forceinline__ void load_to_lds(const Window& w, unsigned int at, unsigned int uni, unsigned int to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(to), "v"(at), "s"(w.r), "s"(uni) : "memory");
}
__device__ __forceinline__ void load_word_to_lds(const Window& w, unsigned int at, unsigned int uni, unsigned int to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds" ::"s"(to), "v"(at), "s"(w.r), "s"(uni) : "memory");
}
// all but the N loads asked for last have arrived (N = 0: all)
template <int N = 0> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

// Workgroups that follow each other go to the eight XCDs in turn, each with an L2 of its own: XCD i gets the i-th part of the tiles,
// and walks it in groups of `group` tile rows, so that the tiles in flight on it share their operands' panels.
__device__ __forceinline__ void tile_of(int id, int n_tiles, int rows, int cols, int group, int& r, int& c)
{
    const int per = n_tiles >> 3, rest = n_tiles & 7, xcd = id & 7, k = id >> 3;
    const int at = xcd * per + (xcd < rest ? xcd : rest) + k;
    const int in = group * cols, g0 = at / in * group, span = rows - g0 < group ? rows - g0 : group;
    const int off = at - g0 * cols;
    r = g0 + off % span;
    c = off / span;
}
}  // namespace sopk
#endif
#endif
