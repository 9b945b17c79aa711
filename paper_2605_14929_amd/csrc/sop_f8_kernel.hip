// 8-bit floats (E4M3, E5M2) with one power-of-two scale for each block of 128: the quantiser, and the gated unit of an MLP whose
// forward pass writes 8-bit checkpoints and whose backward pass reads them.
//
// Block rule: a = largest finite |x| of the block, e = the smallest integer with a <= T * 2^e, T the format's largest number (448 or
// 57344, both 1.75 times a power of two), at least -126, and 0 where a = 0; scale byte e + 127 (E8M0), code = x * 2^-e rounded to
// nearest, ties to even.  With a = m * 2^E, 1 <= m < 2, that is e = E - 8 (E - 15) plus one where m > 1.75: integer work on the
// bits.  The multiplication by 2^-e is exact, so an element is rounded once, and nothing saturates.
//
// All passes read their inputs once and write their outputs once and are bound by HBM.  A lane takes eight neighbouring elements
// (one 16-byte load of bf16, one 8-byte store of codes), sixteen lanes a block of 128, which find its maximum by rotations inside
// a row of the wavefront: no LDS.  Measured, kernel times (a large copy moves 5.14 TB/s here): rows of 4096 x 11008 bf16, 26 us, 5.2 TB/s; squares of
// 28672 x 8192 bf16 with their transposed copy, 192 us, 4.9 TB/s; the gated unit of 8192 x 11008 bf16, 135 us, 4.7 TB/s; its gradient at 1531 x 5024,
// 17.5 us, 4.4 TB/s.
#include <hip/hip_runtime.h>

#include "sop_f8.h"
#include "sop_linear.h"

namespace sopk {

// One wavefront takes four blocks of a row; `units` = such quarters of rows, `per_row` of them a row.
template <bool BF16, bool E5M2, bool VEC>
__global__ __launch_bounds__(256) void f8_rows_kernel(const F8QuantParams p, long long units, int per_row)
{
    const int lane = threadIdx.x & 63;
    const F8Out o{p.codes, p.ldc, p.scales, p.lds};
    for (long long u = (long long)blockIdx.x * 4 + (threadIdx.x >> 6); u < units; u += (long long)gridDim.x * 4) {
        const long long m = u / per_row, k = (u - m * per_row) * 512 + lane * 8;
        const long long rest = p.K - k;
        const int left = rest > 8 ? 8 : (int)rest;
        float v[8];
        load8<BF16, VEC>(p.x, m * p.ldx + k, left, v);
        quantize_row_block<E5M2>(v, o, m, k, left);
    }
}

// One workgroup takes a block of 128 x 128: a thread eight columns of eight neighbouring rows, which it keeps in registers between
// the maximum and the rounding.  The transposed copy leaves through LDS, so that its rows are written 128 bytes at a time too.
template <bool BF16, bool E5M2, bool VEC>
__global__ __launch_bounds__(256) void f8_square_kernel(const F8QuantParams p, int blocks_k)
{
    __shared__ unsigned int wave_max[2][4];
    __shared__ __align__(16) unsigned char turned[128][128 + 16];
    const int t = threadIdx.x, c = (t & 15) * 8, r = (t >> 4) * 8;
    const long long bm = blockIdx.x / blocks_k, bk = blockIdx.x - bm * blocks_k;
    const long long m0 = bm * 128 + r, k0 = bk * 128 + c;
    const long long rest = p.K - k0;
    const int left = rest > 8 ? 8 : (int)rest;
    float v[8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (m0 + i < p.M) load8<BF16, VEC>(p.x, (m0 + i) * p.ldx + k0, left, v[i]);
        else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = 0.0f;
        }
    }
    unsigned int a = 0, f = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) { a = max(a, amax8(v[i], false)); f = max(f, amax8(v[i], true)); }
    a = row_max(a); f = row_max(f);
#pragma unroll
    for (int d = 16; d < 64; d <<= 1) { a = max(a, (unsigned int)__shfl_xor((int)a, d)); f = max(f, (unsigned int)__shfl_xor((int)f, d)); }
    if ((t & 63) == 0) { wave_max[0][t >> 6] = a; wave_max[1][t >> 6] = f; }
    __syncthreads();
    f = max(max(wave_max[1][0], wave_max[1][1]), max(wave_max[1][2], wave_max[1][3]));
    const unsigned int b = scale_byte<E5M2>(f);
    const float inv = inverse_scale(b);
    if (t == 0) p.scales[bm * p.lds + bk] = (unsigned char)b;
    uint2 q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        q[i] = codes8<E5M2>(v[i], inv);
        if (m0 + i < p.M && left > 0) store_codes8(p.codes + (m0 + i) * p.ldc + k0, left, q[i]);
    }
    if (!p.codes_t) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) {                                       // column c + j: its eight rows, in order
        unsigned int w[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            unsigned int s[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] = ((j < 4 ? q[4 * h + i].x : q[4 * h + i].y) >> (8 * (j & 3))) & 0xFFu;
            w[h] = s[0] | s[1] << 8 | s[2] << 16 | s[3] << 24;
        }
        *reinterpret_cast<uint2*>(&turned[c + j][r]) = make_uint2(w[0], w[1]);
    }
    __syncthreads();
    const long long mleft = p.M - bm * 128, kleft = p.K - bk * 128;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int id = i * 256 + t, kk = id >> 3, mm = (id & 7) * 16;
        if (kk >= kleft || mm >= mleft) continue;
        unsigned char* d = p.codes_t + (bk * 128 + kk) * p.ldct + bm * 128 + mm;
        const uint4 w = *reinterpret_cast<const uint4*>(&turned[kk][mm]);
        const int n = mleft - mm > 16 ? 16 : (int)(mleft - mm);
        store_codes8(d, n, make_uint2(w.x, w.y));
        if (n > 8) store_codes8(d + 8, n - 8, make_uint2(w.z, w.w));
    }
}

// ---- gated unit: s = 1 / (1 + exp(-g)), h = g s u
// exp(-g) = 2^t (1 + r ln 2) with t the binary32 product of -g and log2(e), r what the product left: as exact as the hardware's 2^t.
// Where 2^t is 0 (g beyond about 87), s is 1 to 32 bits; g is not below FAR_BELOW here, so that 2^t is finite and s a normal number.
#define SOPK_L2E 1.44269504f                                            // log2(e) = L2E + L2E_LO
#define SOPK_L2E_LO 1.9259630e-08f
#define SOPK_FAR_BELOW (-64.0f)
__device__ __forceinline__ float logistic(float g)
{
    const float t = -g * SOPK_L2E, r = __builtin_fmaf(-g, SOPK_L2E, -t) - g * SOPK_L2E_LO;
    const float p = __builtin_amdgcn_exp2f(t);
    const float q = p > 0.0f ? __builtin_fmaf(p, r * 0.693147181f, p) : p;
    return __builtin_amdgcn_rcpf(1.0f + q);
}
// s for g below that, where it is exp(g) to 32 bits.  It leaves binary32's normal numbers at g = -87 and binary32 at -104, and a large factor
// brings the product back into both: it is formed in binary64, whose smallest number lies at g = -745.
__device__ __forceinline__ double logistic_far_below(float g)
{
    const float c = fmaxf(g, -1200.0f), t = c * SOPK_L2E, r = __builtin_fmaf(c, SOPK_L2E, -t) + c * SOPK_L2E_LO, i = rintf(t);
    const float p = __builtin_amdgcn_exp2f(t - i);
    return ldexp((double)__builtin_fmaf(p, r * 0.693147181f, p), (int)i);
}
__device__ __forceinline__ bool any_far_below(const float (&g)[8])
{
    float least = g[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) least = fminf(least, g[i]);             // (of NaN and a number, the number)
    return least < SOPK_FAR_BELOW;
}

template <bool BF16, bool E5M2, bool VEC>
__global__ __launch_bounds__(256) void f8_gated_kernel(const F8GatedParams p, long long units, int per_row)
{
    const int lane = threadIdx.x & 63;
    for (long long w = (long long)blockIdx.x * 4 + (threadIdx.x >> 6); w < units; w += (long long)gridDim.x * 4) {
        const long long m = w / per_row, k = (w - m * per_row) * 512 + lane * 8;
        const long long rest = p.F - k;
        const int left = rest > 8 ? 8 : (int)rest;
        float g[8], u[8], h[8];
        load8<BF16, VEC>(p.gate, m * p.ldg + k, left, g);
        load8<BF16, VEC>(p.up, m * p.ldu + k, left, u);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = g[i] * logistic(g[i]) * u[i];
        if (any_far_below(g)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) if (g[i] < SOPK_FAR_BELOW) h[i] = (float)((double)g[i] * logistic_far_below(g[i]) * (double)u[i]);
        }
        quantize_row_block<E5M2>(h, p.h, m, k, left);
        quantize_row_block<E5M2>(g, p.g8, m, k, left);
        quantize_row_block<E5M2>(u, p.u8, m, k, left);
    }
}

template <bool E5M2> __device__ __forceinline__ void values8(const F8In& x, long long m, long long k, int left, float (&v)[8])
{
    if (left <= 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.0f;
        return;
    }
    const uint2 q = *reinterpret_cast<const uint2*>(x.codes + m * x.ldc + k);   // (rows are readable up to a multiple of 16)
    const float s = e8m0_value(x.scales[m * x.lds + (k >> 7)]);
    const int w[2] = {(int)q.x, (int)q.y};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const auto a = E5M2 ? __builtin_amdgcn_cvt_pk_f32_bf8(w[h], false) : __builtin_amdgcn_cvt_pk_f32_fp8(w[h], false);
        const auto b = E5M2 ? __builtin_amdgcn_cvt_pk_f32_bf8(w[h], true) : __builtin_amdgcn_cvt_pk_f32_fp8(w[h], true);
        v[4 * h] = a[0] * s; v[4 * h + 1] = a[1] * s; v[4 * h + 2] = b[0] * s; v[4 * h + 3] = b[1] * s;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) if (i >= left) v[i] = 0.0f;
}

// dup = dh g s,  dgate = dh u s (1 + g (1 - s)), g and u the checkpoints' numbers
template <bool BF16, bool C5M2, bool E5M2, bool VEC>
__global__ __launch_bounds__(256) void f8_gated_grad_kernel(const F8GatedGradParams p, long long units, int per_row)
{
    const int lane = threadIdx.x & 63;
    for (long long w = (long long)blockIdx.x * 4 + (threadIdx.x >> 6); w < units; w += (long long)gridDim.x * 4) {
        const long long m = w / per_row, k = (w - m * per_row) * 512 + lane * 8;
        const long long rest = p.F - k;
        const int left = rest > 8 ? 8 : (int)rest;
        float g[8], u[8], d[8], dg[8], du[8];
        values8<C5M2>(p.g8, m, k, left, g);
        values8<C5M2>(p.u8, m, k, left, u);
        load8<BF16, VEC>(p.dh, m * p.lddh + k, left, d);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float s = logistic(g[i]), ds = d[i] * s;
            du[i] = ds * g[i];
            dg[i] = ds * u[i] * __builtin_fmaf(g[i], 1.0f - s, 1.0f);
        }
        if (any_far_below(g)) {                                         // (1 - s is 1)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (g[i] < SOPK_FAR_BELOW) {
                    const double ds = (double)d[i] * logistic_far_below(g[i]);
                    du[i] = (float)(ds * (double)g[i]);
                    dg[i] = (float)(ds * (double)u[i] * (1.0 + (double)g[i]));
                }
            }
        }
        if (left > 0) {
            store8<BF16, VEC>(p.dgate, m * p.lddg + k, left, dg);
            store8<BF16, VEC>(p.dup, m * p.lddu + k, left, du);
        }
        quantize_row_block<E5M2>(dg, p.dg8, m, k, left);
        quantize_row_block<E5M2>(du, p.du8, m, k, left);
    }
}

// Wavefronts take further units in turn once every compute unit has eight workgroups.
static int rows_grid(long long units) { const long long wg = (units + 3) / 4; return (int)(wg < 256 * 8 ? wg : 256 * 8); }

}  // namespace sopk

extern "C" hipError_t sopk_f8_quant_launch(const F8QuantParams* pp, int bf16, int e5m2, int vec, int square, void* stream)
{
    const F8QuantParams p = *pp;
    hipStream_t st = (hipStream_t)stream;
    auto go = [&](auto B, auto E, auto V) {
        constexpr bool b = decltype(B)::value, e = decltype(E)::value, v = decltype(V)::value;
        if (square) {
            const long long bm = (p.M + 127) / 128, bk = (p.K + 127) / 128;
            hipLaunchKernelGGL((sopk::f8_square_kernel<b, e, v>), dim3((unsigned)(bm * bk)), dim3(256), 0, st, p, (int)bk);
        } else {
            const int per_row = (int)((p.K + 511) / 512);
            const long long units = p.M * per_row;
            hipLaunchKernelGGL((sopk::f8_rows_kernel<b, e, v>), dim3(sopk::rows_grid(units)), dim3(256), 0, st, p, units, per_row);
        }
    };
    using T = std::true_type; using F = std::false_type;
    auto go2 = [&](auto B, auto E) { if (vec) go(B, E, T{}); else go(B, E, F{}); };
    auto go3 = [&](auto B) { if (e5m2) go2(B, T{}); else go2(B, F{}); };
    if (bf16) go3(T{}); else go3(F{});
    return hipGetLastError();
}

extern "C" hipError_t sopk_f8_gated_launch(const F8GatedParams* pp, int bf16, int e5m2, int vec, void* stream)
{
    const F8GatedParams p = *pp;
    const int per_row = (int)((p.F + 511) / 512);
    const long long units = p.M * per_row;
    using T = std::true_type; using F = std::false_type;
    auto go = [&](auto B, auto E, auto V) {
        hipLaunchKernelGGL((sopk::f8_gated_kernel<decltype(B)::value, decltype(E)::value, decltype(V)::value>), dim3(sopk::rows_grid(units)), dim3(256), 0,
                           (hipStream_t)stream, p, units, per_row);
    };
    auto go2 = [&](auto B, auto E) { if (vec) go(B, E, T{}); else go(B, E, F{}); };
    auto go3 = [&](auto B) { if (e5m2) go2(B, T{}); else go2(B, F{}); };
    if (bf16) go3(T{}); else go3(F{});
    return hipGetLastError();
}

extern "C" hipError_t sopk_f8_gated_grad_launch(const F8GatedGradParams* pp, int bf16, int ckpt_e5m2, int e5m2, int vec, void* stream)
{
    const F8GatedGradParams p = *pp;
    const int per_row = (int)((p.F + 511) / 512);
    const long long units = p.M * per_row;
    using T = std::true_type; using F = std::false_type;
    auto go = [&](auto B, auto C, auto E, auto V) {
        hipLaunchKernelGGL((sopk::f8_gated_grad_kernel<decltype(B)::value, decltype(C)::value, decltype(E)::value, decltype(V)::value>),
                           dim3(sopk::rows_grid(units)), dim3(256), 0, (hipStream_t)stream, p, units, per_row);
    };
    auto go2 = [&](auto B, auto C, auto E) { if (vec) go(B, C, E, T{}); else go(B, C, E, F{}); };
    auto go3 = [&](auto B, auto C) { if (e5m2) go2(B, C, T{}); else go2(B, C, F{}); };
    auto go4 = [&](auto B) { if (ckpt_e5m2) go3(B, T{}); else go3(B, F{}); };
    if (bf16) go4(T{}); else go4(F{});
    return hipGetLastError();
}
