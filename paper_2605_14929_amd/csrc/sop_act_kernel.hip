// Gradient of an epilogue's activation, dz = scale dy act'(z), as numbers and in 8 bits, and of its bias, dbias = sum of dz over the rows.
//
// One pass, bound by HBM.  A wavefront takes a strip of 512 columns, eight a lane, and goes down its share of the rows, so that the sums of a column stay in
// registers; the four wavefronts of a workgroup take rows by turns and join their sums in LDS, and workgroups leave a row of partial sums each, which a
// second kernel adds up in a fixed order (none where one workgroup has all rows).
#include <hip/hip_runtime.h>

#include <type_traits>

#include "sop_act.h"
#include "sop_block.h"
#include "sop_rows.h"

namespace sopk {

template <bool BF16, bool E5M2, bool SUMS>
__global__ __launch_bounds__(256) void act_grad_kernel(const ActGradParams p)
{
    __shared__ float joined[SUMS ? 4 : 1][SUMS ? 512 : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int strip = (int)(blockIdx.x % (unsigned)p.strips), k = strip * 512 + lane * 8, left = p.N - k;
    const long long word = blockIdx.x / (unsigned)p.strips, m0 = word * p.M / p.words, m1 = (word + 1) * p.M / p.words;
    float sum[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    const F8Out q = p.q;
    for (long long m = m0 + wave; m < m1; m += 4) {
        const Raw<BF16> rd = ask<BF16>(reinterpret_cast<const char*>(p.dy) + m * p.lddy * (BF16 ? 2 : 4), k, left);
        const Raw<BF16> rz = p.z ? ask<BF16>(reinterpret_cast<const char*>(p.z) + m * p.ldz * (BF16 ? 2 : 4), k, left) : nothing<BF16>();
        float d[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] = p.scale * at(rd, i);
        switch (p.act) {
        case 1:
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] = act_slope(1, at(rz, i), d[i]);
            break;
        case 2:
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] = act_slope(2, at(rz, i), d[i]);
            break;
        case 3:
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] = act_slope(3, at(rz, i), d[i]);
            break;
        case 4:
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] = act_slope(4, at(rz, i), d[i]);
        }
        if (p.dz) put<BF16>(reinterpret_cast<char*>(p.dz) + m * p.lddz * (BF16 ? 2 : 4), k, left, d);
        quantize_row_block<E5M2>(d, q, m, k, left);
        if constexpr (SUMS) {
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += d[i];
        }
    }
    if constexpr (SUMS) {
#pragma unroll
        for (int i = 0; i < 8; ++i) joined[wave][i * 64 + lane] = sum[i];
        __syncthreads();
        if (wave != 0) return;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] = (joined[0][i * 64 + lane] + joined[1][i * 64 + lane]) + (joined[2][i * 64 + lane] + joined[3][i * 64 + lane]);
        put<false>(p.part ? p.part + word * p.N : p.dbias, k, left, sum);
    }
}

}  // namespace sopk

extern "C" hipError_t sopk_act_grad_launch(const ActGradParams* pp, int bf16, int e5m2, void* stream)
{
    const ActGradParams p = *pp;
    using T = std::true_type; using F = std::false_type;
    auto go = [&](auto B, auto E, auto S) {
        hipLaunchKernelGGL((sopk::act_grad_kernel<decltype(B)::value, decltype(E)::value, decltype(S)::value>), dim3((unsigned)(p.words * p.strips)), dim3(256), 0, (hipStream_t)stream, p);
    };
    auto go2 = [&](auto B, auto E) { if (p.dbias) go(B, E, T{}); else go(B, E, F{}); };
    auto go3 = [&](auto B) { if (e5m2) go2(B, T{}); else go2(B, F{}); };
    if (bf16) go3(T{}); else go3(F{});
    return hipGetLastError();
}
