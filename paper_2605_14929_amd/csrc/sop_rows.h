// Eight neighbouring elements of a row a lane, rows on any address of their type.
#ifndef SOP_ROWS_H
#define SOP_ROWS_H
#include "sop_f8.h"

namespace sopk {

// eight neighbours of a row on any address of their type, as they lie in memory
struct __attribute__((packed, aligned(4))) Row4 { v4i v; };
struct __attribute__((packed, aligned(2))) Row2 { v4i v; };
template <bool BF16> struct Raw { v4i v[BF16 ? 1 : 2]; };

template <bool BF16> __device__ __forceinline__ Raw<BF16> ask(const void* row, int k, int left)
{
    Raw<BF16> r;
    if (left >= 8) {
        if constexpr (BF16) r.v[0] = reinterpret_cast<const Row2*>(reinterpret_cast<const uint16_t*>(row) + k)->v;
        else {
            const Row4* p = reinterpret_cast<const Row4*>(reinterpret_cast<const float*>(row) + k);
            r.v[0] = p[0].v; r.v[1] = p[1].v;
        }
        return r;
    }
#pragma unroll
    for (int i = 0; i < (BF16 ? 1 : 2); ++i) r.v[i] = v4i{0, 0, 0, 0};
    if (left > 0) {
        asm volatile("" : "+v"(left));                                  // (the end's comparisons are made here, and not kept from row to row)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (BF16) r.v[0][i >> 1] |= i < left ? (int)reinterpret_cast<const uint16_t*>(row)[k + i] << (16 * (i & 1)) : 0;
            else if (i < left) r.v[i >> 2][i & 3] = reinterpret_cast<const int*>(row)[k + i];
        }
    }
    return r;
}
template <bool BF16> __device__ __forceinline__ Raw<BF16> nothing()
{
    Raw<BF16> r;
#pragma unroll
    for (int i = 0; i < (BF16 ? 1 : 2); ++i) r.v[i] = v4i{0, 0, 0, 0};
    return r;
}
template <bool BF16> __device__ __forceinline__ float at(const Raw<BF16>& r, int i)
{
    if constexpr (BF16) return __int_as_float((i & 1) ? r.v[0][i >> 1] & (int)0xFFFF0000 : r.v[0][i >> 1] << 16);
    else return __int_as_float(r.v[i >> 2][i & 3]);
}
template <bool BF16> __device__ __forceinline__ void put(void* row, int k, int left, const float (&v)[8])
{
    if (left >= 8) {
        if constexpr (BF16) {
            reinterpret_cast<Row2*>(reinterpret_cast<uint16_t*>(row) + k)->v =
                v4i{(int)bf16_pair(v[0], v[1]), (int)bf16_pair(v[2], v[3]), (int)bf16_pair(v[4], v[5]), (int)bf16_pair(v[6], v[7])};
        } else {
            Row4* p = reinterpret_cast<Row4*>(reinterpret_cast<float*>(row) + k);
            p[0].v = __builtin_bit_cast(v4i, v4f{v[0], v[1], v[2], v[3]});
            p[1].v = __builtin_bit_cast(v4i, v4f{v[4], v[5], v[6], v[7]});
        }
        return;
    }
    if (left <= 0) return;
    asm volatile("" : "+v"(left));
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (i >= left) continue;
        if constexpr (BF16) reinterpret_cast<uint16_t*>(row)[k + i] = (uint16_t)bf16_bits(v[i]);
        else reinterpret_cast<float*>(row)[k + i] = v[i];
    }
}
__device__ __forceinline__ void put_numbers(void* base, long long row, long long ld, int bf16, int k, int left, const float (&v)[8])
{
    if (bf16) put<true>(reinterpret_cast<uint16_t*>(base) + row * ld, k, left, v);
    else put<false>(reinterpret_cast<float*>(base) + row * ld, k, left, v);
}
__device__ __forceinline__ void put_codes(const F8Out& q, int e5m2, const float (&v)[8], long long m, int k, int left)
{
    asm volatile("" : "+v"(left));
    if (e5m2) quantize_row_block<true>(v, q, m, k, left);
    else quantize_row_block<false>(v, q, m, k, left);
}
// eight values of a vector of D, or of a gate's row; `none` where there is no vector
__device__ __forceinline__ void vector8(const float* p, int k, int left, float none, float (&v)[8])
{
    const Raw<false> r = p ? ask<false>(p, k, left) : nothing<false>();
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = p ? at(r, i) : none;
}
__device__ __forceinline__ void gate8(const void* gate, long long ldg, int bf16, long long g, int k, int left, float (&v)[8])
{
    if (!gate) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 1.0f;
    } else if (bf16) {
        const Raw<true> r = ask<true>(reinterpret_cast<const uint16_t*>(gate) + g * ldg, k, left);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = at(r, i);
    } else {
        const Raw<false> r = ask<false>(reinterpret_cast<const float*>(gate) + g * ldg, k, left);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = at(r, i);
    }
}

}  // namespace sopk
#endif
