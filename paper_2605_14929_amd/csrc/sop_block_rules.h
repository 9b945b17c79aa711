// How the norms with the residual stream and the gradients of an epilogue share their rows out.  Plain C++, so that the rules can be evaluated on a host.
#ifndef SOP_BLOCK_RULES_H
#define SOP_BLOCK_RULES_H

namespace sopr {

// A row of D elements by T threads, C times eight elements each, which keep it in registers (T = 64: a wavefront, four of them a workgroup); D beyond 16384 is
// read several times instead (T = 0).  Measured, by eight and by sixteen elements, 2^25 elements in bf16 (and in fp32): rows of 512 45 and 54 us (87 and 95), of 768 57 and 53 (90 and 93), of 1024
// 49 and 50 (84 and 87), of 1536 47 and 51 (93 and 92), of 2048 48 and 52 (83 and 86), of 2560 55 and 54 (90 and 95), of 3000 55 and 50 (94 and 95), of 4096 48 and 46 (86 and 87);
// 2^26 elements: of 4104 128 and 138 (180 and 200), of 5024 123 and 125 (186 and 211), of 6144 103 and 108 (177 and 180), of 8192 115 and 100 (175 and 173; y in bf16, stream in fp32 146 and 149).
// Beyond 512 and up to 4096 the two are within a tenth of each other; in bf16 alone, rows of 7168 to 8192 would gain by sixteen (132 and 100, 115 and 100), which has not been taken.
struct RowShape { int T, C; };
inline int threads_for(long long D, int C) { return (int)((D + 512 * C - 1) / (512 * C)) * 64; }
inline RowShape norm_shape(long long D)
{
    const int C = D <= 512 ? 1 : D <= 1024 ? 2 : D <= 2048 ? 1 : D <= 4096 ? 2 : D <= 8192 ? 1 : 2;
    return D > 16384 ? RowShape{0, 0} : RowShape{threads_for(D, C), C};
}
// Backward, where a thread holds four times as much: eight elements up to 8192 (8192 x 4096 bf16 105 us, sixteen 108; 777 x 5024 fp32 32 and 34; 8192 x 1024 fp32 49, sixteen a
// wavefront's thread 58), then
// sixteen of a row that it does not keep (4096 x 12288 bf16 209 us, by the way of still longer rows 330).
inline RowShape norm_grad_shape(long long D)
{
    return D <= 512 ? norm_shape(D) : D <= 8192 ? RowShape{threads_for(D, 1), 1} : D <= 16384 ? RowShape{1024, 2} : RowShape{0, 0};
}

// Rows in G groups of `each` (a group shares a row of the gate), to `words` workgroups: as many groups as there are workgroups and more are dealt out whole
// (parts = 1, workgroup i has groups i G / words ..), fewer are cut into `parts` each (workgroup i has part i % parts of group i / parts).
struct RowShare { long long words; int parts; };
inline RowShare norm_share(long long G, long long each, long long most)
{
    if (G >= most) return RowShare{most, 1};
    long long parts = most / G;
    parts = parts < each ? parts : each;
    return RowShare{G * parts, (int)parts};
}

// How many workgroups the backward pass has at most: about what the compute units hold at once (each leaves a row of partial sums).
inline long long norm_grad_most(long long D, int n_cu)
{
    const RowShape s = norm_grad_shape(D);
    if (s.T == 0) {                                                     // (strips of 512 columns are workgroups too)
        const long long words = 16ll * n_cu / ((D + 511) / 512);
        return words < 1 ? 1 : words;
    }
    return (s.T < 256 ? 4ll : 1024ll / s.T) * n_cu;                     // (sixteen wavefronts a compute unit, but four workgroups at most)
}

// Rows of an activation's gradient to workgroups: strips of 512 columns times `words` shares of the rows, four rows each at least.
inline long long act_grad_words(long long M, long long N, int n_cu)
{
    const long long strips = (N + 511) / 512, all = 8ll * n_cu, words = all / strips, rows = (M + 3) / 4;
    return words < 1 ? 1 : words < rows ? words : rows < 1 ? 1 : rows;
}
// ... with their sums: whether one workgroup takes all rows of 128 columns, without a second launch.  In a graph 128 x 11008 takes 7.8 us so; from there on it is bound by the
// vector ALUs of the few compute units at work (256 x 1531 14.9 us, by two launches 9).
inline bool act_grad_few(long long M) { return M <= 128; }

// Many tensors: launches of up to `list` of them, and the workgroups of each, which leave a partial sum each.
inline long long clip_launches(long long count, int list) { return (count + list - 1) / list; }
inline long long clip_words(long long chunks, long long launches, int n_cu)
{
    long long words = 8ll * n_cu / (launches < 1 ? 1 : launches);
    words = words < 64 ? 64 : words;
    return chunks < words ? chunks : words;
}

}  // namespace sopr
#endif
