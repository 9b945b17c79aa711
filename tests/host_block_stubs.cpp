// The entry points around a linear layer without a GPU: what the kernels would be launched with is written down and looked at here.
#include <cstdarg>
#include <cstdio>
#include <cstring>

#include "../paper_2605_14929_amd/csrc/sop_checks.h"
#include "../paper_2605_14929_amd/csrc/sop_block.h"

struct sop_ctx { int cu; char text[512]; };
static char record[1 << 20];
static size_t used;
static void note(const char* f, ...)
{
    va_list a;
    va_start(a, f);
    used += (size_t)std::vsnprintf(record + used, sizeof(record) - used, f, a);
    va_end(a);
}
namespace sopc {
sop_status fail(sop_ctx* c, sop_status s, const char* msg) { std::snprintf(c->text, sizeof(c->text), "%s", msg); return s; }
int device(const sop_ctx*) { return 0; }
int compute_units(const sop_ctx* c) { return c->cu; }
}  // namespace sopc
extern "C" {
hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
hipError_t hipSetDevice(int) { return hipSuccess; }
const char* hipGetErrorString(hipError_t) { return "error"; }
static sop_ctx the_ctx;
sop_ctx* stub_ctx(int cu) { the_ctx.cu = cu; return &the_ctx; }
const char* stub_error(void) { return the_ctx.text; }
const char* stub_record(void) { record[used] = 0; used = 0; return record; }
hipError_t sopk_f8_quant_launch(const F8QuantParams*, int, int, int, int, void*) { note("quant\n"); return hipSuccess; }
hipError_t sopk_f8_gated_launch(const F8GatedParams*, int, int, int, void*) { note("gated\n"); return hipSuccess; }
hipError_t sopk_f8_gated_grad_launch(const F8GatedGradParams*, int, int, int, int, void*) { note("gated_grad\n"); return hipSuccess; }
hipError_t sopk_wgrad_launch(const WgradParams*, int, int, void*) { note("wgrad\n"); return hipSuccess; }
hipError_t sopk_f8mm_launch(const F8MmParams* p, int, int, void*) { note("f8mm %d %d\n", p->M, p->N); return hipSuccess; }
hipError_t sopk_packed_launch(const PackedMmParams* p, int, void*) { note("packed %d %d\n", p->M, p->N); return hipSuccess; }
hipError_t sopk_f8mm_epilogue_launch(const F8MmParams* p, int, int, void*) { note("f8mm_epilogue %d %d %d %g\n", p->M, p->N, p->e.act, (double)p->e.scale); return hipSuccess; }
hipError_t sopk_packed_epilogue_launch(const PackedMmParams* p, int, void*)
{
    note("packed_epilogue %d %d %llu %llu %llu %llu\n", p->M, p->N, (unsigned long long)p->e.bias, (unsigned long long)p->e.residual, (unsigned long long)p->e.z, (unsigned long long)p->y);
    return hipSuccess;
}
hipError_t sopk_norm_launch(const NormParams* p, int y, int r, int, void*) { note("norm %lld %d %lld %d %d\n", p->M, p->D, p->per_group, y, r); return hipSuccess; }
hipError_t sopk_norm_grad_launch(const NormGradParams* p, int, int, int, void*)
{
    note("norm_grad %lld %d %lld %d %lld %lld %llu %llu %llu %llu\n", p->M, p->D, p->words, p->parts, p->groups, p->per_group,
         (unsigned long long)p->part_a, (unsigned long long)p->part_b, (unsigned long long)p->part_t, (unsigned long long)p->stats);
    return hipSuccess;
}
hipError_t sopk_join_launch(const JoinParams* p, void*)
{
    for (int j = 0; j < 3; ++j)
        if (p->sets[j]) note("join %d %lld %lld %llu %llu\n", j, p->sets[j], p->rows[j], (unsigned long long)p->part[j], (unsigned long long)p->out[j]);
    return hipSuccess;
}
hipError_t sopk_act_grad_launch(const ActGradParams* p, int, int, void*) { note("act_grad %lld %d %lld %d %llu\n", p->M, p->N, p->words, p->strips, (unsigned long long)p->part); return hipSuccess; }
static void clip(const char* what, const ClipParams* p, int words)
{
    note("%s %d %d %d %d %d\n", what, p->count, p->chunks, words, p->first, p->parts);
    for (int i = 0; i < p->count; ++i) note("entry %lld %d %d\n", p->e[i].n, p->e[i].end, p->e[i].types);
}
hipError_t sopk_square_sum_launch(const ClipParams* p, int words, void*) { clip("square_sum", p, words); return hipSuccess; }
hipError_t sopk_norm_of_parts_launch(const ClipParams* p, void*) { note("norm_of_parts %d\n", p->parts); return hipSuccess; }
hipError_t sopk_clip_launch(const ClipParams* p, int words, void*) { clip("clip", p, words); return hipSuccess; }
}
