// Which kernel takes a product of a linear layer with narrow operands: the one that is expected to take least, among those whose launch is
// possible.  Plain C++, so that the rules can be evaluated on a host.  The times beside the rules are those that the costs were taken from; they compare kernels
// of one run.
#ifndef SOP_LINEAR_RULES_H
#define SOP_LINEAR_RULES_H

namespace sopr {

inline long long tiles(long long rows, long long cols, int a, int b) { return ((rows + a - 1) / a) * ((cols + b - 1) / b); }
// how many workgroups a compute unit gets
inline float each(long long rows, long long cols, int a, int b, int n_cu) { return (float)((tiles(rows, cols, a, b) + n_cu - 1) / n_cu); }
// a launch has fewer than 2^32 threads along a dimension
inline bool can(long long workgroups, int threads) { return workgroups * threads < 1ll << 32; }
const float kNever = 3.4e38f;
inline int least(const float* cost, int n)
{
    int best = 0;
    for (int i = 1; i < n; ++i) best = cost[i] < cost[best] ? i : best;
    return cost[best] < kNever ? best : -1;
}

// ---- product of two 8-bit matrices.  The cost is counted from how many workgroups a compute unit gets.  Microseconds at K = 4096 on 256 compute units,
// bf16 results: by c workgroups each, the narrow tiles take 4 c + 2 (32 x 32), 6.5 c + 1.5 (32 x 64), 9.3 c + 1 (64 x 64); tiles of 64 x 128 23 for
// one and 13.5 c for more, of 128 x 128 29 for one and 38.5 for every two, of 256 x 256 60 c (bf16 results alone).  Where the choice falls wrong it costs
// little: measured, the best and the next at 300 x 4096 x 4096: 19.0 and 20.1 us; 1024 x 4096 x 4096: 27.9 (64 x 128) and 30.5 (128 x
// 128); 777 x 5000 x 3000: 31 (128 x 128) and 37; 1024 x 11008 x 4096: 60 (256 x 256) and 70 (64 x 128).  32-bit results go by the same costs, which
// were not measured for them, and K is not in them.  Up to four rows operands go straight to
// registers, two steps in flight: one row through 28672 x 8192 takes 41 us, 45 by 32 x 32 tiles, through 4096 x 11008 9.8 and 10.1; eight rows
// through 11008 x 4096 12.7 and 9.7.
enum F8mm { F8MM_32x32, F8MM_32x64, F8MM_64x64, F8MM_64x128, F8MM_128x128, F8MM_256x256, F8MM_ROWS };
inline int f8mm_choice(long long M, long long N, bool f32, int n_cu)
{
    if (M <= 4 && can(tiles(M, N, 16, 16), 512)) return F8MM_ROWS;
    auto c = [&](int a, int b) { return each(M, N, a, b, n_cu); };
    auto if_can = [&](int a, int b, int threads, float cost) { return can(tiles(M, N, a, b), threads) ? cost : kNever; };
    const float c24 = c(64, 128), c44 = c(128, 128);
    const float cost[6] = {if_can(32, 32, 512, 4.0f * c(32, 32) + 2.0f), if_can(32, 64, 512, 6.5f * c(32, 64) + 1.5f), if_can(64, 64, 512, 9.3f * c(64, 64) + 1.0f),
                           if_can(64, 128, 256, c24 <= 1.0f ? 23.0f : 13.5f * c24),
                           if_can(128, 128, 256, c44 <= 1.0f ? 29.0f : 19.25f * (c44 + (float)((long long)c44 & 1))), f32 ? kNever : if_can(256, 256, 512, 60.0f * c(256, 256))};
    return least(cost, 6);
}

// ---- weight gradient from an 8-bit checkpoint; on16: rows of dy lie on 16 bytes.  The cost is counted from how many workgroups c a compute unit gets and how
// many times 64 rows there are (t).
// Microseconds on 256 compute units, 32-bit results: the rows dealt out 1.4 + c (1.2 + 0.16 t) (32 x 64) and 1.2 + c (2.9 + 0.21 t) (64 x 64);
// 128 x 128 4.4 + 0.82 t for one and c (4 + 0.6 t) for more; 256 x 256 c (19 + 1.65 t).  Measured (rows x N x K), the best and the next:
// 8192 x 512 x 512 24 (32 x 64) and 33, by 128 x 128 107; 8192 x 1024 x 1024 32 (64 x 64) and 49; 777 x 1531 x 5024 23 (128 x 128) and 30;
// 2048 x 4096 x 4096 72 (256 x 256) and 92; 500 x 8192 x 4096 67 (256 x 256) and 71.
enum Wgrad { WGRAD_32x64, WGRAD_64x64, WGRAD_128x128, WGRAD_256x256, WGRAD_ANY_64x128, WGRAD_ANY_128x128, WGRAD_ANY_256x256 };
inline int wgrad_choice(long long M, long long N, long long K, bool on16, int n_cu)
{
    if (M == 0 || !on16)
        return tiles(N, K, 256, 256) >= n_cu ? WGRAD_ANY_256x256 : tiles(N, K, 128, 128) >= n_cu ? WGRAD_ANY_128x128 : WGRAD_ANY_64x128;
    auto c = [&](int a, int b) { return each(N, K, a, b, n_cu); };
    const float t = (float)((M + 63) / 64), c44 = c(128, 128);
    const float cost[4] = {1.4f + c(32, 64) * (1.2f + 0.16f * t), 1.2f + c(64, 64) * (2.9f + 0.21f * t), c44 <= 1.0f ? 4.4f + 0.82f * t : c44 * (4.0f + 0.6f * t),
                           c(256, 256) * (19.0f + 1.65f * t)};
    return least(cost, 4);
}

// ---- product with packed codes of n_bits.  The cost is counted from how many workgroups a compute unit gets.  Microseconds at K = 4096 on 256 compute
// units, 4-bit codes, by c workgroups each: the narrow tiles 8 c + 2 (32 x 32), 11 c + 2 (64 x 32), 20.5 c (64 x 64), 19.5 c (128 x 32); the wide ones 64 for one
// and 51 c for more (128 x 128), 110 c (256 x 192), 128 c (256 x 256; 146 when every unit has one).  Measured, the best and the next: 32 x 11008 x
// 4096 17.8 (32 x 32) and 19.6; 64 x 11008 x 4096 20.9 (64 x 64) and 23.0; 128 x 4096 x 4096 14.5 (64 x 32) and 18.7; 512 x 4096 x 4096 39 (128 x 32)
// and 42; 1024 x 4096 x 4096 71 (128 x 128) and 77; 2048 x 11008 x 4096 212 (256 x 192) and 244; 4096 x 4096 x 4096 146 (256 x 256) and 199.  Codes
// of 3 and 5 bits take up to a quarter more, in the same order.  Up to 16 rows a workgroup takes 16 columns and reads x
// itself: one row through 4096 x 11008 11.5 us, 20.9 by tiles of 32 x 32.  Tables of pairs of 6-bit codes fit beside 128 x 128 tiles only.
// The wide ones take K from 64 on; below it none can be launched from some 2^35 numbers of y on (-1).
enum Packed { PACKED_32x32, PACKED_64x32, PACKED_64x64, PACKED_128x32, PACKED_128x128, PACKED_256x192, PACKED_256x256, PACKED_ROWS };
inline int packed_choice(long long M, long long N, long long K, int n_bits, int n_cu)
{
    if (M <= 16 && can(tiles(1, N, 1, 16), 512)) return PACKED_ROWS;
    auto c = [&](int a, int b) { return each(M, N, a, b, n_cu); };
    auto if_can = [&](int a, int b, int threads, float cost) { return can(tiles(M, N, a, b), threads) ? cost : kNever; };
    auto wide = [&](int a, int b, float cost) { return K < 64 ? kNever : if_can(a, b, 256, cost); };
    const float c22 = c(128, 128);
    const float cost[7] = {if_can(32, 32, 512, 8.0f * c(32, 32) + 1.7f), if_can(64, 32, 512, 11.0f * c(64, 32) + 2.0f), if_can(64, 64, 512, 20.5f * c(64, 64)),
                           if_can(128, 32, 512, 19.5f * c(128, 32)), wide(128, 128, c22 <= 1.0f ? 64.0f : 51.0f * c22),
                           n_bits > 5 ? kNever : wide(256, 192, 110.0f * c(256, 192)), n_bits > 5 ? kNever : wide(256, 256, 128.0f * c(256, 256))};
    return least(cost, 7);
}

}  // namespace sopr
#endif
