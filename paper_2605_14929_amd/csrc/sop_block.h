// What stands around a linear layer in a block of a model: launch parameters shared by the host side (sop_block_api.cpp) and the kernels.
#ifndef SOP_BLOCK_H
#define SOP_BLOCK_H
#include "sop_linear.h"

#define SOPK_FEWER 1.262177448e-29f                                     // 2^-96: what elements are multiplied by whose squares' sum leaves binary32

/* s = r + scale gate after y / rms(y), n = before s / rms(s) */
struct NormParams {
    const void* y; long long ldy;            // null: s = r
    const void* r; long long ldr;
    const float* after; const float* before; // null: no such norm
    const void* gate; long long ldg; int gate_bf16; long long per_group;   // row m takes row m / per_group
    float scale, eps, eps_fewer;             // eps_fewer: eps SOPK_FEWER^2
    long long M; int D;
    void* out; long long ldo;                // of r's type, null: not written
    void* n; long long ldn; int n_bf16;
    F8Out q; int e5m2;                       // codes null: not written
};
/* its gradients: dr = ds + d(n) / d(s), dy, and the sums over rows that weights and gates get */
struct NormGradParams {
    const void* ds; long long ldds;          // null: zero
    const void* dn; long long lddn;          // before null: not looked at
    const void* s; long long lds;
    const void* y; long long ldy;            // null: no dy
    const float* after; const float* before;
    const void* gate; long long ldg; int gate_bf16; long long groups, per_group;
    float scale, eps, eps_fewer;             // eps_fewer: eps SOPK_FEWER^2
    long long M; int D;
    void* dr; long long lddr;
    void* dy; long long lddy;
    F8Out q; int e5m2;
    float* dafter; float* dbefore; void* dgate; long long lddg;   // null: not wanted
    float* part_a; float* part_b; float* part_t;                  // a row of D for each workgroup: dafter's (parts = 1) or t (parts > 1), dbefore's
    float* stats;                                                 // rows read several times: 1 / rms(y), 1 / rms(s) and mean(p h) of each
    long long words; int parts;
};
/* Rows of partial sums added up: out[j] of set s, column d = sum over `rows` rows i of part[j][s rows + i][d] (j = 0: times factor and gate[i / share][d], 2: times factor
 * and after[d]) */
struct JoinParams {
    const float* part[3]; void* out[3]; long long rows[3];
    long long sets[3]; long long ldo[3]; int out_bf16[3];
    const float* after; float factor;
    const void* gate; long long ldg; int gate_bf16, share;             // gate null: weights of 1
    int also;                                                     // out[0] comes of set 2, the only one, times factor and gate
    int D;
};

/* dz = scale dy act'(z) as numbers and in 8 bits, and its sums over the rows */
struct ActGradParams {
    const void* dy; long long lddy;
    const void* z; long long ldz;            // null: no activation
    long long M; int N;
    float scale; int act;
    void* dz; long long lddz;                // null: not written
    F8Out q;
    float* part; float* dbias;               // null: no sums; part null: a workgroup has all rows of its columns
    long long words; int strips;
};

/* Many tensors: their sum of squares, and their product with a factor */
#define SOP_K_CLIP_LIST 96
struct ClipEntry { const void* x; void* out; long long n; int end; int types; };   // end: chunks up to and with this tensor; types: 1 bf16, 2 out bf16
struct ClipParams {
    ClipEntry e[SOP_K_CLIP_LIST];
    int count, chunks;
    double* part; int first, parts;          // this launch's partial sums begin at first; there are `parts` in all
    float* norm; double most;
};
#define SOP_K_CLIP_CHUNK 8192
#endif
