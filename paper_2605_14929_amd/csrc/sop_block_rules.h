// How the norms with the residual stream and the gradients of an epilogue share their rows out.  Plain C++, so that the rules can be evaluated on a host.
#ifndef SOP_BLOCK_RULES_H
#define SOP_BLOCK_RULES_H

namespace sopr {

// A row of D elements by T threads, C times eight elements each, which keep it in registers; D beyond 16384 is read several times instead (T = 0).
struct RowShape { int T, C; };
inline RowShape norm_shape(long long D)
{
    return D <= 512 ? RowShape{64, 1} : D <= 1024 ? RowShape{64, 2} : D <= 2048 ? RowShape{256, 1} : D <= 4096 ? RowShape{256, 2} : D <= 8192 ? RowShape{512, 2}
         : D <= 12288 ? RowShape{512, 3} : D <= 16384 ? RowShape{512, 4} : RowShape{0, 0};
}
// Backward, where a thread holds four times as much, from 8192 on.
inline RowShape norm_grad_shape(long long D) { return D <= 8192 ? norm_shape(D) : RowShape{0, 0}; }

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

// How many workgroups the backward pass has at most: what the compute units hold at once (each leaves a row of partial sums).
inline long long norm_grad_most(long long D, int n_cu)
{
    const RowShape s = norm_grad_shape(D);
    return (long long)n_cu * (s.T == 512 ? 1 : s.T == 0 || s.C == 2 ? 2 : 4);
}

// Rows of an activation's gradient to workgroups: strips of 512 columns times `words` shares of the rows, four rows each at least.
inline long long act_grad_words(long long M, long long N, int n_cu)
{
    const long long strips = (N + 511) / 512, all = 8ll * n_cu, words = all / strips, rows = (M + 3) / 4;
    return words < 1 ? 1 : words < rows ? words : rows < 1 ? 1 : rows;
}

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
