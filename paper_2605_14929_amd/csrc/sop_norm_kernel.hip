// Norms before and after a block with its gate and residual scale, forward and backward.  With rows m and columns k:
//   x = y s1, s1 = 1 / sqrt(mean_k y^2 + eps)  (no norm after the block: x = y)      s = r + f x, f = scale gate after
//   h = s s2, s2 = 1 / sqrt(mean_k s^2 + eps)                                        n = before h, as numbers, in 8 bits, or both
// and backward, s being the stored sum, p = before dn:
//   dr = ds + s2 (p - h mean_k(p h))             dbefore = sum_m dn h
//   dy = s1 (q - x mean_k(q x)), q = f dr        t = sum_m dr x over the rows of a gate: dgate = scale after t, dafter = sum scale gate t
//   (no norm after the block: dy = q)
//
// Every pass is bound by HBM.  A row stays in the registers of the threads that share it (T threads, C times eight neighbouring elements each), so that it is
// read once; its sums go over a wavefront by rotations and over a workgroup through LDS.  Threads keep their columns from row to row, so weights, and the
// backward pass's sums over rows, stay with them: a workgroup leaves one row of partial sums, and a second kernel adds those up in a fixed order.
// Backward, rows of 8193 to 16384 elements are read twice over, y a third time: 4096 x 12288 fetches 1.3 times one read from beyond L2 in bf16, 1.9 times in fp32.  Longer ones are read four
// times by a pass over rows (2.3 times one read from beyond L2 at 4096 x 20000 bf16) and once more by a pass over columns, which has their sums.
//
// Measured, kernel times (a large copy moves 5.1 TB/s): forward 8192 x 8192, y bf16 and stream fp32, 145 us, 5.1 TB/s, one token of 4096 4.1 us; backward 8192 x 4096 bf16 with a
// gate of one row 95 us, 4.8 TB/s with the partial sums, and 6 us to add those up (512 rows of 4096, twice); 777 x 5024 fp32 with three gates 25 and 7; 4096 x 12288 bf16 209 us in all,
// fp32 338; 4096 x 20000 bf16 forward 189, backward 506; a gate row for each of y, 8192 x 4096 bf16 134, 32768 x 512 148 (a gate of one row: 48).
// Backward, the next row is asked for while one is worked on (8192 x 4096 102 us in all, without that some 20 more).
//
// Sums of squares are binary32; where one leaves its range (elements beyond 2^51 to 2^61, by how many there are) the row's are formed once more from elements 2^-96 as large: 2^20 of the
// largest, 2^128, then add up to 2^84, and the smallest sum that is formed again, 2^20 elements of 2^51, to 2^-69.
// The means of p h and q x are no larger than what they are means of: a thread's part of the sum is divided by D before the parts meet.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "sop_block.h"
#include "sop_block_rules.h"
#include "sop_rows.h"

namespace sopk {

// The sum over sixteen lanes of a wavefront that stand in a row, and over all of it; for all lanes
__device__ __forceinline__ float sixteen_sum(float x)
{
    x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x128, 0xF, 0xF, false));   // row_ror:8, 4, 2, 1
    x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x124, 0xF, 0xF, false));
    x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x122, 0xF, 0xF, false));
    x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x121, 0xF, 0xF, false));
    return x;
}
__device__ __forceinline__ float wave_sum(float x)
{
    const int b = __float_as_int(sixteen_sum(x));
    return (__int_as_float(__builtin_amdgcn_readlane(b, 0)) + __int_as_float(__builtin_amdgcn_readlane(b, 16))) +
           (__int_as_float(__builtin_amdgcn_readlane(b, 32)) + __int_as_float(__builtin_amdgcn_readlane(b, 48)));
}
// Up to four sums over a row's threads: a wavefront's own, or those of a workgroup of up to sixteen, which leave theirs in LDS, where a lane reads the one of its place
// in a row of sixteen (places without a wavefront hold zeros).  Two sets of places by turns: whoever writes one has passed the barrier behind the other's reads.
// However they are added, all lanes get the same bits.
template <bool ONE> struct RowSums {
    v4f (*slot)[16];                                                    // [2]
    int turn = 0;
    __device__ __forceinline__ explicit RowSums(v4f (*at)[16]) : slot(at)
    {
        if (!ONE && threadIdx.x < 32) slot[threadIdx.x >> 4][threadIdx.x & 15] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        if (!ONE) __syncthreads();
    }
    template <int N> __device__ __forceinline__ void operator()(float (&v)[N])
    {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = wave_sum(v[j]);
        if constexpr (!ONE) {
            if ((threadIdx.x & 63) == 0) {
                v4f mine = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int j = 0; j < N; ++j) mine[j] = v[j];
                slot[turn][threadIdx.x >> 6] = mine;
            }
            __syncthreads();
            const v4f its = slot[turn][threadIdx.x & 15];
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = sixteen_sum(its[j]);
            turn ^= 1;
        }
    }
};
// 1 / sqrt(mean + eps) of a row whose sum of squares is `sum`; where that is beyond SOPK_MUCH, that of elements times SOPK_FEWER instead, and eps times its square
#define SOPK_MUCH 1e37f
__device__ __forceinline__ bool too_much(float sum) { return !(sum <= SOPK_MUCH); }
__device__ __forceinline__ float unit_of(float sum, float inv_d, float eps) { return __builtin_amdgcn_rsqf(__builtin_fmaf(sum, inv_d, eps)); }
// (beyond an rms of 2^126 it is no normal number, and known to 2^-150)
__device__ __forceinline__ float unit_of_fewer(float sum, float inv_d, float eps_fewer) { return __builtin_amdgcn_rsqf(__builtin_fmaf(sum, inv_d, eps_fewer)) * SOPK_FEWER; }

// ---- forward, a row in registers
template <bool ONE, int C, int MOST, bool YB, bool RB>
__global__ __launch_bounds__(MOST) void norm_kernel(const NormParams p, long long each)
{
    constexpr int RW = ONE ? MOST / 64 : 1;                             // rows at a time
    __shared__ v4f slot[2][16];
    RowSums<ONE> sums(slot);
    const int T = ONE ? 64 : blockDim.x, t = ONE ? threadIdx.x & 63 : threadIdx.x, who = ONE ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
    const float inv_d = 1.0f / (float)p.D;
    int k[C], left[C];
    float f[C][8], b[C][8];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        k[c] = (c * T + t) * 8;
        left[c] = p.D - k[c];
        vector8(p.before, k[c], left[c], 0.0f, b[c]);
    }
    const long long m0 = ((long long)blockIdx.x * RW + who) * each, m1 = m0 + each < p.M ? m0 + each : p.M;
    if (m0 >= m1) return;                                               // (wavefronts of a row each meet nowhere; a workgroup of one row leaves together)
    long long g = m0 / p.per_group, turn = m0;
    for (long long m = m0; m < m1; ++m) {
        if (p.y && m == turn) {                                         // the rows of a gate's row begin here
            if (m != m0) ++g;
            turn = (g + 1) * p.per_group;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float after[8];
                gate8(p.gate, p.ldg, p.gate_bf16, g, k[c], left[c], f[c]);
                vector8(p.after, k[c], left[c], 1.0f, after);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[c][i] = p.scale * f[c][i] * after[i];
            }
        }
        const char* row = reinterpret_cast<const char*>(p.r) + m * p.ldr * (RB ? 2 : 4);
        const char* rowy = reinterpret_cast<const char*>(p.y) + m * p.ldy * (YB ? 2 : 4);
        Raw<RB> r[C];
        Raw<YB> y[C];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            r[c] = ask<RB>(row, k[c], left[c]);
            y[c] = p.y ? ask<YB>(rowy, k[c], left[c]) : nothing<YB>();
        }
        float s[C][8];
        if (p.y) {
            float s1 = 1.0f;
            if (p.after) {
                float sum[1] = {0.0f};
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum[0] = __builtin_fmaf(at(y[c], i), at(y[c], i), sum[0]);
                sums(sum);
                s1 = unit_of(sum[0], inv_d, p.eps);
                if (too_much(sum[0])) {
                    sum[0] = 0.0f;
#pragma unroll
                    for (int c = 0; c < C; ++c)
#pragma unroll
                        for (int i = 0; i < 8; ++i) { const float z = at(y[c], i) * SOPK_FEWER; sum[0] = __builtin_fmaf(z, z, sum[0]); }
                    sums(sum);
                    s1 = unit_of_fewer(sum[0], inv_d, p.eps_fewer);
                }
            }
            char* out = reinterpret_cast<char*>(p.out) + m * p.ldo * (RB ? 2 : 4);
#pragma unroll
            for (int c = 0; c < C; ++c) {
#pragma unroll
                for (int i = 0; i < 8; ++i) s[c][i] = __builtin_fmaf(at(y[c], i) * s1, f[c][i], at(r[c], i));
                put<RB>(out, k[c], left[c], s[c]);
            }
        } else {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) s[c][i] = at(r[c], i);
        }
        if (!p.before) continue;
        float sum[1] = {0.0f};
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[0] = __builtin_fmaf(s[c][i], s[c][i], sum[0]);   // (zero beyond the row's end)
        sums(sum);
        float s2 = unit_of(sum[0], inv_d, p.eps);
        if (too_much(sum[0])) {
            sum[0] = 0.0f;
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) { const float z = s[c][i] * SOPK_FEWER; sum[0] = __builtin_fmaf(z, z, sum[0]); }
            sums(sum);
            s2 = unit_of_fewer(sum[0], inv_d, p.eps_fewer);
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
#pragma unroll
            for (int i = 0; i < 8; ++i) s[c][i] = s[c][i] * s2 * b[c][i];
            if (p.n) put_numbers(p.n, m, p.ldn, p.n_bf16, k[c], left[c], s[c]);
            if (p.q.codes) put_codes(p.q, p.e5m2, s[c], m, k[c], left[c]);
        }
    }
}

// ---- forward, rows of any length: three walks over a row (the last writes, so the sum may go where r was)
template <bool YB, bool RB>
__global__ __launch_bounds__(1024) void norm_long_kernel(const NormParams p)
{
    __shared__ v4f slot[2][16];
    RowSums<false> sums(slot);
    const float inv_d = 1.0f / (float)p.D;
    const int whole = (p.D + 8191) / 8192 * 8192;                       // (all lanes of sixteen take part in a block's maximum)
    for (long long m = blockIdx.x; m < p.M; m += gridDim.x) {
        const long long g = m / p.per_group;
        const char* row = reinterpret_cast<const char*>(p.r) + m * p.ldr * (RB ? 2 : 4);
        const char* rowy = reinterpret_cast<const char*>(p.y) + m * p.ldy * (YB ? 2 : 4);
        float s1 = 1.0f, s2 = 0.0f;
        auto total = [&](int k, float (&s)[8]) {
            const int left = p.D - k;
            const Raw<RB> r = ask<RB>(row, k, left);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] = at(r, i);
            if (!p.y) return;
            const Raw<YB> y = ask<YB>(rowy, k, left);
            float f[8], after[8];
            gate8(p.gate, p.ldg, p.gate_bf16, g, k, left, f);
            vector8(p.after, k, left, 1.0f, after);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] = __builtin_fmaf(at(y, i) * s1, p.scale * f[i] * after[i], s[i]);
        };
        auto squares = [&](bool of_y, float by) {
            float sum[1] = {0.0f};
            for (int k = threadIdx.x * 8; k < p.D; k += 8192) {
                float v[8];
                if (of_y) {
                    const Raw<YB> y = ask<YB>(rowy, k, p.D - k);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = at(y, i);
                } else total(k, v);
#pragma unroll
                for (int i = 0; i < 8; ++i) { const float z = v[i] * by; sum[0] = __builtin_fmaf(z, z, sum[0]); }
            }
            sums(sum);
            return sum[0];
        };
        auto unit = [&](bool of_y) {
            const float sum = squares(of_y, 1.0f);
            return too_much(sum) ? unit_of_fewer(squares(of_y, SOPK_FEWER), inv_d, p.eps_fewer) : unit_of(sum, inv_d, p.eps);
        };
        if (p.y && p.after) s1 = unit(true);
        if (p.before) s2 = unit(false);
        for (int k = threadIdx.x * 8; k < whole; k += 8192) {
            const int left = p.D - k;
            float s[8], b[8];
            total(k, s);
            if (p.y) put<RB>(reinterpret_cast<char*>(p.out) + m * p.ldo * (RB ? 2 : 4), k, left, s);
            if (!p.before) continue;
            vector8(p.before, k, left, 0.0f, b);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] = s[i] * s2 * b[i];
            if (p.n) put_numbers(p.n, m, p.ldn, p.n_bf16, k, left, s);
            if (p.q.codes) put_codes(p.q, p.e5m2, s, m, k, left);
        }
    }
}

// ---- backward.  The kernels' arguments once more, where few rows want them: read there, so that they hold no registers while rows go by.
__device__ __forceinline__ const NormGradParams& seldom()
{
    unsigned long long at = (unsigned long long)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(at));
    return *(const NormGradParams*)(const __attribute__((address_space(4))) NormGradParams*)at;
}
// The groups and rows of a workgroup
struct Share { long long g0, g1; int part, parts; };
__device__ __forceinline__ Share share_of(const NormGradParams& p, long long w)
{
    if (p.parts > 1) return Share{w / p.parts, w / p.parts + 1, (int)(w % p.parts), p.parts};
    return Share{w * p.groups / p.words, (w + 1) * p.groups / p.words, 0, 1};
}
__device__ __forceinline__ long long begin_of(const NormGradParams& p, long long g, int part) { return g * p.per_group + part * p.per_group / p.parts; }

// What sums over rows a thread has when a group ends, t = sum of dr x: a part of it, from which dgate and dafter are joined; or, of a whole group, dgate, and what dafter gets of it
template <int C> __device__ __forceinline__ void end_group(long long w, long long g, const int (&k)[C], const int (&left)[C], const float (&t)[C][8], float (&da)[C][8])
{
    const NormGradParams& p = seldom();
#pragma unroll
    for (int c = 0; c < C; ++c) {
        if (p.parts > 1) {
            put<false>(p.part_t + w * p.D, k[c], left[c], t[c]);
            continue;
        }
        float gate[8];
        gate8(p.gate, p.ldg, p.gate_bf16, g, k[c], left[c], gate);
        if (p.dgate) {
            float after[8];
            vector8(p.after, k[c], left[c], 1.0f, after);
#pragma unroll
            for (int i = 0; i < 8; ++i) after[i] = p.scale * after[i] * t[c][i];
            put_numbers(p.dgate, g, p.lddg, p.gate_bf16, k[c], left[c], after);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) da[c][i] = p.scale * gate[i] * t[c][i];
    }
}

// ---- backward, a row in registers.  The next row is on its way while one is worked on.  What a thread keeps of its columns beside the sums of the rows (weights, and dafter's
// sums, which a group's end adds to) stands in LDS, in places of its own.
template <bool ONE, int C, int MOST, bool YB, bool RB>
__global__ __launch_bounds__(MOST) void norm_grad_kernel(const NormGradParams p)
{
    constexpr int RW = ONE ? MOST / 64 : 1;
    extern __shared__ __align__(16) unsigned char kept[];
    __shared__ v4f slot[2][16];
    RowSums<ONE> sums(slot);
    const int NT = blockDim.x, T = ONE ? 64 : NT, t = ONE ? threadIdx.x & 63 : threadIdx.x, who = ONE ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
    const float inv_d = 1.0f / (float)p.D;
    enum { FACTOR, BEFORE, AFTER, JOIN };
    auto place = [&](int what, int c, int half, int thread) -> v4f& { return reinterpret_cast<v4f*>(kept)[((what * C + c) * 2 + half) * NT + thread]; };
    auto keep = [&](int what, int c, const float (&v)[8]) {
        place(what, c, 0, threadIdx.x) = v4f{v[0], v[1], v[2], v[3]};
        place(what, c, 1, threadIdx.x) = v4f{v[4], v[5], v[6], v[7]};
    };
    auto have = [&](int what, int c, float (&v)[8]) {
        const v4f a = place(what, c, 0, threadIdx.x), b = place(what, c, 1, threadIdx.x);
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
    };
    int k[C], left[C];
    float st[C][8], sb[C][8];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        k[c] = (c * T + t) * 8;
        left[c] = p.D - k[c];
        float b[8], none[8];
        vector8(seldom().before, k[c], left[c], 0.0f, b);
        keep(BEFORE, c, b);
#pragma unroll
        for (int i = 0; i < 8; ++i) st[c][i] = sb[c][i] = none[i] = 0.0f;
        keep(AFTER, c, none);
        keep(FACTOR, c, none);
    }
    // the wavefronts of a workgroup that have a row each put their sums together: the first one has them all
    auto join = [&](float (&v)[C][8]) {
        if constexpr (ONE) {
            __syncthreads();
#pragma unroll
            for (int c = 0; c < C; ++c) keep(JOIN, c, v[c]);
            __syncthreads();
            if (who != 0) return;
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int w = 1; w < RW; ++w)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const v4f a = place(JOIN, c, half, w * 64 + t);
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[c][4 * half + i] += a[i];
                    }
        }
    };
    struct Row { Raw<RB> s[C], d[C]; Raw<YB> n[C], y[C]; };
    auto load = [&](Row& r, long long m) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            r.s[c] = p.before ? ask<RB>(reinterpret_cast<const char*>(p.s) + m * p.lds * (RB ? 2 : 4), k[c], left[c]) : nothing<RB>();
            r.n[c] = p.before ? ask<YB>(reinterpret_cast<const char*>(p.dn) + m * p.lddn * (YB ? 2 : 4), k[c], left[c]) : nothing<YB>();
            r.y[c] = p.y ? ask<YB>(reinterpret_cast<const char*>(p.y) + m * p.ldy * (YB ? 2 : 4), k[c], left[c]) : nothing<YB>();
            r.d[c] = p.ds ? ask<RB>(reinterpret_cast<const char*>(p.ds) + m * p.ldds * (RB ? 2 : 4), k[c], left[c]) : nothing<RB>();
        }
    };
    const Share z = share_of(seldom(), blockIdx.x);
    Row row;
    long long held = -1;                                                // the row that has been asked for
    for (long long g = z.g0; g < z.g1; ++g) {
        if (p.y) {
            const NormGradParams& p = seldom();
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float f[8], after[8];
                gate8(p.gate, p.ldg, p.gate_bf16, g, k[c], left[c], f);
                vector8(p.after, k[c], left[c], 1.0f, after);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = p.scale * f[i] * after[i];
                keep(FACTOR, c, f);
            }
        }
        const long long begin = begin_of(seldom(), g, z.part), end = begin_of(seldom(), g, z.part + 1);
        const long long after_end = g + 1 < z.g1 ? end + who : -1;      // (rows of a workgroup's groups follow each other)
        for (long long m = begin + who; m < end; m += RW) {
            if (held != m) load(row, m);
            const Row now = row;
            held = m + RW < end ? m + RW : after_end;
            if (held >= 0 && held < p.M) load(row, held);
            float sum[3] = {0.0f, 0.0f, 0.0f};                          // of s^2, p s and y^2
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float b[8];
                have(BEFORE, c, b);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float s = at(now.s[c], i), y = at(now.y[c], i);
                    sum[0] = __builtin_fmaf(s, s, sum[0]);
                    sum[1] = __builtin_fmaf(b[i] * at(now.n[c], i), s, sum[1]);
                    sum[2] = __builtin_fmaf(y, y, sum[2]);
                }
            }
            sum[1] *= inv_d;
            sums(sum);
            float s2 = unit_of(sum[0], inv_d, p.eps), s1 = p.after ? unit_of(sum[2], inv_d, p.eps) : 1.0f, mean = sum[1] * s2;
            if (too_much(sum[0]) || too_much(fabsf(sum[1])) || (p.after && too_much(sum[2]))) {
                float few[2] = {0.0f, 0.0f};
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float s = at(now.s[c], i) * SOPK_FEWER, y = at(now.y[c], i) * SOPK_FEWER;
                        few[0] = __builtin_fmaf(s, s, few[0]);
                        few[1] = __builtin_fmaf(y, y, few[1]);
                    }
                sums(few);
                if (too_much(sum[0])) s2 = unit_of_fewer(few[0], inv_d, p.eps_fewer);
                if (p.after && too_much(sum[2])) s1 = unit_of_fewer(few[1], inv_d, p.eps_fewer);
                float ph[1] = {0.0f};
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    float b[8];
                    have(BEFORE, c, b);
#pragma unroll
                    for (int i = 0; i < 8; ++i) ph[0] = __builtin_fmaf(b[i] * at(now.n[c], i), at(now.s[c], i) * s2, ph[0]);
                }
                ph[0] *= inv_d;
                sums(ph);
                mean = ph[0];
            }
            float dr[C][8], qx[1] = {0.0f};
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float b[8];
                have(BEFORE, c, b);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float h = at(now.s[c], i) * s2, x = at(now.y[c], i) * s1, dn = at(now.n[c], i);
                    dr[c][i] = __builtin_fmaf(s2, __builtin_fmaf(-h, mean, b[i] * dn), at(now.d[c], i));
                    sb[c][i] = __builtin_fmaf(dn, h, sb[c][i]);
                    st[c][i] = __builtin_fmaf(dr[c][i], x, st[c][i]);
                }
                put<RB>(reinterpret_cast<char*>(p.dr) + m * p.lddr * (RB ? 2 : 4), k[c], left[c], dr[c]);
            }
            if (!p.y) continue;
#pragma unroll
            for (int c = 0; c < C; ++c) {                               // dr becomes q
                float f[8];
                have(FACTOR, c, f);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    dr[c][i] *= f[i];
                    qx[0] = __builtin_fmaf(dr[c][i], at(now.y[c], i) * s1, qx[0]);
                }
            }
            if (p.after) {
                qx[0] *= inv_d;
                sums(qx);
                const float c1 = qx[0];
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int i = 0; i < 8; ++i) dr[c][i] = s1 * __builtin_fmaf(-at(now.y[c], i) * s1, c1, dr[c][i]);
            }
#pragma unroll
            for (int c = 0; c < C; ++c) {
                put<YB>(reinterpret_cast<char*>(p.dy) + m * p.lddy * (YB ? 2 : 4), k[c], left[c], dr[c]);
                if (p.q.codes) put_codes(p.q, p.e5m2, dr[c], m, k[c], left[c]);
            }
        }
        const NormGradParams& r = seldom();
        if (r.dafter || r.dgate) {
            join(st);
            if (who == 0) {
                float da[C][8], had[8];
                end_group<C>(blockIdx.x, g, k, left, st, da);
#pragma unroll
                for (int c = 0; c < C && r.parts == 1; ++c) {
                    have(AFTER, c, had);
#pragma unroll
                    for (int i = 0; i < 8; ++i) had[i] += da[c][i];
                    keep(AFTER, c, had);
                }
            }
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) st[c][i] = 0.0f;
        }
    }
    const NormGradParams& r = seldom();
    if (r.dbefore) join(sb);
    if (who != 0) return;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        float da[8];
        have(AFTER, c, da);
        if (r.dafter && r.parts == 1) put<false>(r.part_a + (long long)blockIdx.x * r.D, k[c], left[c], da);
        if (r.dbefore) put<false>(r.part_b + (long long)blockIdx.x * r.D, k[c], left[c], sb[c]);
    }
}

// Rows that no thread keeps: eight elements of their operands at a time.
template <bool YB, bool RB> struct LongRow {
    const NormGradParams& p;
    long long m, g;
    __device__ __forceinline__ const char* row(const void* x, long long ld, bool bf16) const { return reinterpret_cast<const char*>(x) + m * ld * (bf16 ? 2 : 4); }
    // s, p = before dn (or dn), y and f of eight columns; dr from them
    __device__ __forceinline__ void read(int k, float (&s)[8], float (&dn)[8], float (&y)[8], float (&b)[8]) const
    {
        const int left = p.D - k;
        const Raw<RB> rs = p.before ? ask<RB>(row(p.s, p.lds, RB), k, left) : nothing<RB>();
        const Raw<YB> rn = p.before ? ask<YB>(row(p.dn, p.lddn, YB), k, left) : nothing<YB>(), ry = p.y ? ask<YB>(row(p.y, p.ldy, YB), k, left) : nothing<YB>();
        vector8(p.before, k, left, 0.0f, b);
#pragma unroll
        for (int i = 0; i < 8; ++i) { s[i] = at(rs, i); dn[i] = at(rn, i); y[i] = at(ry, i); }
    }
    __device__ __forceinline__ void sum_grad(int k, const float (&s)[8], const float (&dn)[8], const float (&b)[8], float s2, float mean, float (&dr)[8]) const
    {
        const Raw<RB> rd = p.ds ? ask<RB>(row(p.ds, p.ldds, RB), k, p.D - k) : nothing<RB>();
#pragma unroll
        for (int i = 0; i < 8; ++i) dr[i] = __builtin_fmaf(s2, __builtin_fmaf(-(s[i] * s2), mean, b[i] * dn[i]), at(rd, i));
    }
    __device__ __forceinline__ void factors(int k, float (&f)[8]) const
    {
        float after[8];
        gate8(p.gate, p.ldg, p.gate_bf16, g, k, p.D - k, f);
        vector8(p.after, k, p.D - k, 1.0f, after);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = p.scale * f[i] * after[i];
    }
};

// ---- backward, rows of up to 16384 elements: 1024 threads with sixteen columns each.  Their sums over rows stay in registers and LDS, a row does not: it is read again, and, one
// workgroup a compute unit, mostly out of L2.  (Raw, a row of bf16 would take 32 of a thread's 128 registers, one of fp32 64; that has not been built.)  The compiler keeps some 40 registers
// of a thread in scratch memory: 31 of the 309 MB written at 4096 x 12288 bf16.
template <bool YB, bool RB>
__global__ __launch_bounds__(1024) void norm_grad_wide_kernel(const NormGradParams p)
{
    constexpr int C = 2;
    extern __shared__ __align__(16) unsigned char kept[];               // dafter's sums, and t
    __shared__ v4f slot[2][16];
    RowSums<false> sums(slot);
    const float inv_d = 1.0f / (float)p.D;
    auto after_sum = [&](int c, int half) -> v4f& { return reinterpret_cast<v4f*>(kept)[(c * 2 + half) * 1024 + threadIdx.x]; };
    auto t_sum = [&](int c, int half) -> v4f& { return reinterpret_cast<v4f*>(kept)[(4 + c * 2 + half) * 1024 + threadIdx.x]; };
    int k[C], left[C];
    float sb[C][8];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        k[c] = (c * 1024 + (int)threadIdx.x) * 8;
        left[c] = p.D - k[c];
        after_sum(c, 0) = after_sum(c, 1) = t_sum(c, 0) = t_sum(c, 1) = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < 8; ++i) sb[c][i] = 0.0f;
    }
    const Share z = share_of(seldom(), blockIdx.x);
    for (long long g = z.g0; g < z.g1; ++g) {
        const long long begin = begin_of(seldom(), g, z.part), end = begin_of(seldom(), g, z.part + 1);
        for (long long m = begin; m < end; ++m) {
            const LongRow<YB, RB> w{p, m, g};
            auto squares = [&](float by, float (&sum)[3]) {             // of s and y, and p s
                sum[0] = sum[1] = sum[2] = 0.0f;
#pragma unroll 1
                for (int c = 0; c < C; ++c) {
                    float s[8], dn[8], y[8], b[8];
                    w.read((c * 1024 + (int)threadIdx.x) * 8, s, dn, y, b);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float u = s[i] * by, v = y[i] * by;
                        sum[0] = __builtin_fmaf(u, u, sum[0]);
                        sum[1] = __builtin_fmaf(b[i] * dn[i], s[i], sum[1]);
                        sum[2] = __builtin_fmaf(v, v, sum[2]);
                    }
                }
                sum[1] *= inv_d;
                sums(sum);
            };
            float sum[3];
            squares(1.0f, sum);
            float s2 = unit_of(sum[0], inv_d, p.eps), s1 = p.after ? unit_of(sum[2], inv_d, p.eps) : 1.0f, mean = sum[1] * s2;
            if (too_much(sum[0]) || too_much(fabsf(sum[1])) || (p.after && too_much(sum[2]))) {
                float few[3], ph[1] = {0.0f};
                squares(SOPK_FEWER, few);
                if (too_much(sum[0])) s2 = unit_of_fewer(few[0], inv_d, p.eps_fewer);
                if (p.after && too_much(sum[2])) s1 = unit_of_fewer(few[2], inv_d, p.eps_fewer);
#pragma unroll 1
                for (int c = 0; c < C; ++c) {
                    float s[8], dn[8], y[8], b[8];
                    w.read((c * 1024 + (int)threadIdx.x) * 8, s, dn, y, b);
#pragma unroll
                    for (int i = 0; i < 8; ++i) ph[0] = __builtin_fmaf(b[i] * dn[i], s[i] * s2, ph[0]);
                }
                ph[0] *= inv_d;
                sums(ph);
                mean = ph[0];
            }
            float q[C][8], qx[1] = {0.0f};
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float s[8], dn[8], y[8], b[8], f[8];
                w.read(k[c], s, dn, y, b);
                w.sum_grad(k[c], s, dn, b, s2, mean, q[c]);
                put<RB>(reinterpret_cast<char*>(p.dr) + m * p.lddr * (RB ? 2 : 4), k[c], left[c], q[c]);
#pragma unroll
                for (int i = 0; i < 8; ++i) sb[c][i] = __builtin_fmaf(dn[i], s[i] * s2, sb[c][i]);
                if (!p.y) continue;
                w.factors(k[c], f);
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    v4f t = t_sum(c, half);
#pragma unroll
                    for (int i = 0; i < 4; ++i) t[i] = __builtin_fmaf(q[c][4 * half + i], y[4 * half + i] * s1, t[i]);
                    t_sum(c, half) = t;
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    q[c][i] *= f[i];
                    qx[0] = __builtin_fmaf(q[c][i], y[i] * s1, qx[0]);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            if (!p.y) continue;
            qx[0] *= inv_d;
            if (p.after) sums(qx);
            const float c1 = qx[0];
#pragma unroll
            for (int c = 0; c < C; ++c) {
                if (p.after) {
                    const Raw<YB> y = ask<YB>(w.row(p.y, p.ldy, YB), k[c], left[c]);
#pragma unroll
                    for (int i = 0; i < 8; ++i) q[c][i] = s1 * __builtin_fmaf(-at(y, i) * s1, c1, q[c][i]);
                }
                put<YB>(reinterpret_cast<char*>(p.dy) + m * p.lddy * (YB ? 2 : 4), k[c], left[c], q[c]);
                if (p.q.codes) put_codes(p.q, p.e5m2, q[c], m, k[c], left[c]);
            }
        }
        const NormGradParams& r = seldom();
        if (r.dafter || r.dgate) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int kc[1] = {(c * 1024 + (int)threadIdx.x) * 8}, lc[1] = {r.D - kc[0]};
                const v4f lo = t_sum(c, 0), hi = t_sum(c, 1);
                const float tc[1][8] = {{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]}};
                float da[1][8];
                t_sum(c, 0) = t_sum(c, 1) = v4f{0.0f, 0.0f, 0.0f, 0.0f};
                end_group<1>(blockIdx.x, g, kc, lc, tc, da);
                if (r.parts > 1) continue;
                after_sum(c, 0) += v4f{da[0][0], da[0][1], da[0][2], da[0][3]};
                after_sum(c, 1) += v4f{da[0][4], da[0][5], da[0][6], da[0][7]};
            }
        }
    }
    const NormGradParams& r = seldom();
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const v4f a = after_sum(c, 0), b = after_sum(c, 1);
        const float da[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
        if (r.dafter && r.parts == 1) put<false>(r.part_a + (long long)blockIdx.x * r.D, k[c], left[c], da);
        if (r.dbefore) put<false>(r.part_b + (long long)blockIdx.x * r.D, k[c], left[c], sb[c]);
    }
}

// ---- backward, longer rows: first the rows (dr, dy, and what the sums need of a row), then strips of 512 columns
template <bool YB, bool RB>
__global__ __launch_bounds__(1024) void norm_grad_long_kernel(const NormGradParams p)
{
    __shared__ v4f slot[2][16];
    RowSums<false> sums(slot);
    const float inv_d = 1.0f / (float)p.D;
    const int whole = (p.D + 8191) / 8192 * 8192;
    for (long long m = blockIdx.x; m < p.M; m += gridDim.x) {
        const LongRow<YB, RB> w{p, m, m / p.per_group};
        float s[8], dn[8], y[8], b[8], dr[8], f[8];
        auto squares = [&](float by) {
            v2f r = {0.0f, 0.0f};
            float sum[2] = {0.0f, 0.0f};
            for (int k = threadIdx.x * 8; k < p.D; k += 8192) {
                w.read(k, s, dn, y, b);
#pragma unroll
                for (int i = 0; i < 8; ++i) { const float u = s[i] * by, v = y[i] * by; sum[0] = __builtin_fmaf(u, u, sum[0]); sum[1] = __builtin_fmaf(v, v, sum[1]); }
            }
            sums(sum);
            r[0] = sum[0]; r[1] = sum[1];
            return r;
        };
        const v2f sq = squares(1.0f);
        float s2 = unit_of(sq[0], inv_d, p.eps), s1 = p.after ? unit_of(sq[1], inv_d, p.eps) : 1.0f;
        if (too_much(sq[0]) || (p.after && too_much(sq[1]))) {
            const v2f few = squares(SOPK_FEWER);
            if (too_much(sq[0])) s2 = unit_of_fewer(few[0], inv_d, p.eps_fewer);
            if (p.after && too_much(sq[1])) s1 = unit_of_fewer(few[1], inv_d, p.eps_fewer);
        }
        float sum[1] = {0.0f};
        if (p.before) {
            for (int k = threadIdx.x * 8; k < p.D; k += 8192) {
                w.read(k, s, dn, y, b);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[0] = __builtin_fmaf(b[i] * dn[i], s[i] * s2, sum[0]);
            }
            sum[0] *= inv_d;
            sums(sum);
        }
        const float mean = sum[0];
        sum[0] = 0.0f;
        if (p.y && p.after) {
            for (int k = threadIdx.x * 8; k < p.D; k += 8192) {
                w.read(k, s, dn, y, b);
                w.sum_grad(k, s, dn, b, s2, mean, dr);
                w.factors(k, f);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[0] = __builtin_fmaf(f[i] * dr[i], y[i] * s1, sum[0]);
            }
            sum[0] *= inv_d;
            sums(sum);
        }
        const float c1 = sum[0];
        for (int k = threadIdx.x * 8; k < whole; k += 8192) {
            const int left = p.D - k;
            w.read(k, s, dn, y, b);
            w.sum_grad(k, s, dn, b, s2, mean, dr);
            put<RB>(reinterpret_cast<char*>(p.dr) + m * p.lddr * (RB ? 2 : 4), k, left, dr);
            if (!p.y) continue;
            w.factors(k, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float q = f[i] * dr[i];
                dr[i] = p.after ? s1 * __builtin_fmaf(-y[i] * s1, c1, q) : q;
            }
            put<YB>(reinterpret_cast<char*>(p.dy) + m * p.lddy * (YB ? 2 : 4), k, left, dr);
            if (p.q.codes) put_codes(p.q, p.e5m2, dr, m, k, left);
        }
        if (threadIdx.x == 0) { p.stats[3 * m] = s1; p.stats[3 * m + 1] = s2; p.stats[3 * m + 2] = mean; }
    }
}
template <bool YB, bool RB>
__global__ __launch_bounds__(256) void norm_grad_columns_kernel(const NormGradParams p)
{
    __shared__ float joined[4][8 * 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int k[1] = {((int)blockIdx.x * 64 + lane) * 8}, left[1] = {p.D - k[0]};
    float st[1][8] = {}, sa[1][8] = {}, sb[1][8] = {};
    auto join = [&](float (&v)[1][8]) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) joined[wave][i * 64 + lane] = v[0][i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) v[0][i] = (joined[0][i * 64 + lane] + joined[1][i * 64 + lane]) + (joined[2][i * 64 + lane] + joined[3][i * 64 + lane]);
    };
    const long long word = blockIdx.y;
    const Share z = share_of(p, word);
    for (long long g = z.g0; g < z.g1; ++g) {
        const long long end = begin_of(p, g, z.part + 1);
        for (long long m = begin_of(p, g, z.part) + wave; m < end; m += 4) {
            const LongRow<YB, RB> w{p, m, g};
            const float s1 = p.stats[3 * m], s2 = p.stats[3 * m + 1], mean = p.stats[3 * m + 2];
            float s[8], dn[8], y[8], b[8], dr[8];
            w.read(k[0], s, dn, y, b);
            w.sum_grad(k[0], s, dn, b, s2, mean, dr);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                sb[0][i] = __builtin_fmaf(dn[i], s[i] * s2, sb[0][i]);
                st[0][i] = __builtin_fmaf(dr[i], y[i] * s1, st[0][i]);
            }
        }
        if (p.dafter || p.dgate) {
            join(st);
            if (wave == 0) {
                float da[1][8];
                end_group<1>(word, g, k, left, st, da);
#pragma unroll
                for (int i = 0; i < 8 && p.parts == 1; ++i) sa[0][i] += da[0][i];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) st[0][i] = 0.0f;
        }
    }
    if (p.dbefore) join(sb);
    if (wave != 0) return;
    if (p.dafter && p.parts == 1) put<false>(p.part_a + word * p.D, k[0], left[0], sa[0]);
    if (p.dbefore) put<false>(p.part_b + word * p.D, k[0], left[0], sb[0]);
}

// ---- the rows of partial sums added up, in binary64, in a fixed order: 32 columns a workgroup, its 32 half-wavefronts share the rows.  Row i of the first set has the
// weight of its gate's row, i / share.  A gate of one row: its own set's sum, weighted, is the first set's too.
__global__ __launch_bounds__(1024) void join_kernel(const JoinParams p)
{
    __shared__ double part[32][33];
    const int col = threadIdx.x & 31, row = threadIdx.x >> 5, d = blockIdx.x * 32 + col;
    long long set = blockIdx.y;
    int j = 0;
    while (j < 2 && set >= p.sets[j]) { set -= p.sets[j]; ++j; }
    const int rows = (int)p.rows[j], at = d < p.D ? d : p.D - 1;
    const float* from = p.part[j] + set * rows * p.D + at;
    const bool weighted = j == 0 && p.gate;
    auto weight = [&](int i) {
        const long long k = (unsigned int)i / (unsigned int)p.share * p.ldg + at;
        return (double)(p.gate_bf16 ? __uint_as_float((unsigned int)reinterpret_cast<const uint16_t*>(p.gate)[k] << 16) : reinterpret_cast<const float*>(p.gate)[k]);
    };
    double s = 0.0;
    const long long step = 32ll * p.D;
    const float* q = from + (long long)row * p.D;
    int i = row;
    for (; i + 224 < rows; i += 256, q += 8 * step) {
        float v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = q[u * step];
        if (weighted) {
#pragma unroll
            for (int u = 0; u < 8; ++u) s = __builtin_fma((double)v[u], weight(i + 32 * u), s);
        } else {
            s += (((double)v[0] + (double)v[1]) + ((double)v[2] + (double)v[3])) + (((double)v[4] + (double)v[5]) + ((double)v[6] + (double)v[7]));
        }
    }
    if (i < rows) {                                                     // the last ones, asked for together too
        float v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = from[(long long)(i + 32 * u < rows ? i + 32 * u : rows - 1) * p.D];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const bool in = i + 32 * u < rows;
            if (weighted) s = in ? __builtin_fma((double)v[u], weight(in ? i + 32 * u : i), s) : s;
            else s += in ? (double)v[u] : 0.0;
        }
    }
    part[row][col] = s;
    __syncthreads();
    if (row != 0 || d >= p.D) return;
    s = 0.0;
#pragma unroll
    for (int u = 0; u < 32; ++u) s += part[u][col];
    if (j == 2 && p.also) reinterpret_cast<float*>(p.out[0])[d] = (float)(s * (double)p.factor * weight(0));
    if (rows > 0 && j != 1) s *= (double)p.factor;                      // (sums of no rows are zero, whatever the weights are)
    if (rows > 0 && j == 2 && p.after) s *= (double)p.after[d];
    if (p.out_bf16[j]) reinterpret_cast<uint16_t*>(p.out[j])[set * p.ldo[j] + d] = (uint16_t)bf16_bits((float)s);
    else reinterpret_cast<float*>(p.out[j])[set * p.ldo[j] + d] = (float)s;
}

// Workgroups take rows that follow each other, as many workgroups as there are threads for twice over (eight elements each), or once.  4096 x 5024 fp32 takes 57 us by twice as many,
// 60 by once; with sixteen elements 8192 x 4096 bf16 takes 45 and 42.
template <bool ONE, int C, int MOST, bool YB, bool RB> static hipError_t norm_go(const NormParams& p, int T, int n_cu, hipStream_t st)
{
    const int RW = ONE ? MOST / 64 : 1, NT = ONE ? MOST : T;
    const long long most = (long long)n_cu * ((C == 1 ? 4096 : 2048) / NT) * RW, each = (p.M + most - 1) / most, units = (p.M + each - 1) / each;
    hipLaunchKernelGGL((norm_kernel<ONE, C, MOST, YB, RB>), dim3((unsigned)((units + RW - 1) / RW)), dim3(NT), 0, st, p, each);
    return hipGetLastError();
}
template <bool ONE, int C, int MOST, bool YB, bool RB> static hipError_t norm_grad_go(const NormGradParams& p, int T, hipStream_t st)
{
    const int NT = ONE ? MOST : T, bytes = (ONE ? 4 : 3) * C * 32 * NT;
    auto fn = &norm_grad_kernel<ONE, C, MOST, YB, RB>;
    if (bytes > 64 * 1024 - 512) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(fn), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(fn, dim3((unsigned)p.words), dim3(NT), bytes, st, p);
    return hipGetLastError();
}
static long long grid_of(long long n, long long most) { return n < most ? n : most; }

template <bool YB, bool RB> static hipError_t norm_shape_go(const NormParams& p, int n_cu, hipStream_t st)
{
    const sopr::RowShape s = sopr::norm_shape(p.D);
    if (s.T == 64) return s.C == 1 ? norm_go<true, 1, 256, YB, RB>(p, s.T, n_cu, st) : norm_go<true, 2, 256, YB, RB>(p, s.T, n_cu, st);
    if (s.C == 1) return norm_go<false, 1, 1024, YB, RB>(p, s.T, n_cu, st);
    if (s.C == 2) return norm_go<false, 2, 1024, YB, RB>(p, s.T, n_cu, st);
    hipLaunchKernelGGL((norm_long_kernel<YB, RB>), dim3((unsigned)grid_of(p.M, 2 * n_cu)), dim3(1024), 0, st, p);
    return hipGetLastError();
}
template <bool YB, bool RB> static hipError_t norm_grad_shape_go(const NormGradParams& p, int n_cu, hipStream_t st)
{
    const sopr::RowShape s = sopr::norm_grad_shape(p.D);
    if (s.T == 64) return norm_grad_go<true, 1, 256, YB, RB>(p, s.T, st);
    if (s.C == 1) return norm_grad_go<false, 1, 1024, YB, RB>(p, s.T, st);
    if (s.T == 1024) {
        auto fn = &norm_grad_wide_kernel<YB, RB>;
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(fn), hipFuncAttributeMaxDynamicSharedMemorySize, 128 * 1024);
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(fn, dim3((unsigned)p.words), dim3(1024), 128 * 1024, st, p);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((norm_grad_long_kernel<YB, RB>), dim3((unsigned)grid_of(p.M, 2 * n_cu)), dim3(1024), 0, st, p);
    if (p.dafter || p.dbefore || p.dgate) hipLaunchKernelGGL((norm_grad_columns_kernel<YB, RB>), dim3((unsigned)((p.D + 511) / 512), (unsigned)p.words), dim3(256), 0, st, p);
    return hipGetLastError();
}

}  // namespace sopk

extern "C" hipError_t sopk_norm_launch(const NormParams* p, int y_bf16, int r_bf16, int n_cu, void* stream)
{
    hipStream_t st = (hipStream_t)stream;
    if (y_bf16) return r_bf16 ? sopk::norm_shape_go<true, true>(*p, n_cu, st) : sopk::norm_shape_go<true, false>(*p, n_cu, st);
    return r_bf16 ? sopk::norm_shape_go<false, true>(*p, n_cu, st) : sopk::norm_shape_go<false, false>(*p, n_cu, st);
}
extern "C" hipError_t sopk_norm_grad_launch(const NormGradParams* p, int y_bf16, int r_bf16, int n_cu, void* stream)
{
    hipStream_t st = (hipStream_t)stream;
    if (y_bf16) return r_bf16 ? sopk::norm_grad_shape_go<true, true>(*p, n_cu, st) : sopk::norm_grad_shape_go<true, false>(*p, n_cu, st);
    return r_bf16 ? sopk::norm_grad_shape_go<false, true>(*p, n_cu, st) : sopk::norm_grad_shape_go<false, false>(*p, n_cu, st);
}
extern "C" hipError_t sopk_join_launch(const JoinParams* p, void* stream)
{
    const long long sets = p->sets[0] + p->sets[1] + p->sets[2];
    hipLaunchKernelGGL(sopk::join_kernel, dim3((unsigned)((p->D + 31) / 32), (unsigned)sets), dim3(1024), 0, (hipStream_t)stream, *p);   // (D at most 2^23)
    return hipGetLastError();
}
