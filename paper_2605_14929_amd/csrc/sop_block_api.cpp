// Entry points of what stands around a linear layer: the gradient of an epilogue, norms with the residual stream, gradients clipped together.
// Every argument is checked here, before a launch; the kernels' own bounds rest on what these checks let through.
#include <algorithm>
#include <cmath>
#include <cstdlib>
#include <cstring>

#include "sop_checks.h"
#include "sop_block.h"
#include "sop_block_rules.h"

extern "C" hipError_t sopk_norm_launch(const NormParams* p, int y_bf16, int r_bf16, int n_cu, void* stream);
extern "C" hipError_t sopk_norm_grad_launch(const NormGradParams* p, int y_bf16, int r_bf16, int n_cu, void* stream);
extern "C" hipError_t sopk_join_launch(const JoinParams* p, void* stream);
extern "C" hipError_t sopk_act_grad_launch(const ActGradParams* p, int bf16, int e5m2, void* stream);
extern "C" hipError_t sopk_square_sum_launch(const ClipParams* p, int words, void* stream);
extern "C" hipError_t sopk_norm_of_parts_launch(const ClipParams* p, void* stream);
extern "C" hipError_t sopk_clip_launch(const ClipParams* p, int words, void* stream);

namespace {

constexpr int64_t kMaxRow = (int64_t)1 << 20, kMaxTensor = (int64_t)1 << 36;

// Sums over rows: sets of a launch are numbered in its grid's second dimension, which ends at 65535
hipError_t join(JoinParams p, void* stream)
{
    const int64_t most = 32768;
    for (int j = 0; j < 3; ++j) {
        const int64_t size = p.out_bf16[j] ? 2 : 4;
        while (p.sets[j] > most) {
            JoinParams q;
            std::memset(&q, 0, sizeof(q));
            q.D = p.D; q.after = p.after; q.factor = p.factor; q.gate = p.gate; q.ldg = p.ldg; q.gate_bf16 = p.gate_bf16; q.share = p.share;
            q.part[j] = p.part[j]; q.out[j] = p.out[j]; q.rows[j] = p.rows[j]; q.sets[j] = most; q.ldo[j] = p.ldo[j]; q.out_bf16[j] = p.out_bf16[j];
            const hipError_t e = sopk_join_launch(&q, stream);
            if (e != hipSuccess) return e;
            if (p.part[j]) p.part[j] += most * p.rows[j] * p.D;
            p.out[j] = static_cast<char*>(p.out[j]) + most * p.ldo[j] * size;
            p.sets[j] -= most;
        }
    }
    return p.sets[0] + p.sets[1] + p.sets[2] > 0 ? sopk_join_launch(&p, stream) : hipSuccess;
}
void one_sum(JoinParams& p, int j, const float* part, int64_t rows, int64_t sets, void* out, int64_t ldo, bool bf16)
{
    p.part[j] = part; p.rows[j] = rows; p.sets[j] = sets; p.out[j] = out; p.ldo[j] = ldo; p.out_bf16[j] = bf16;
}

// the options of a norm: null if they are some
const char* norm_fault(const sop_residual_norm_opts* o, int64_t M, int64_t D)
{
    if (!o) return "the options are NULL";
    if (off(o->after, 4) || off(o->before, 4)) return "a norm's weight is not aligned to its elements";
    if (!(o->eps >= 5.421010862e-20f) || std::isinf(o->eps)) return "eps is at least 2^-64, and finite";
    if (o->gate) {
        if (!dtype_ok(o->gate_dtype)) return "the gate is fp32 or bf16";
        if (o->groups < 1 || M % o->groups) return "the rows of the gate divide the rows of y";
        if (const char* why = plain_fault(o->gate, D, o->ld_gate, size_of(o->gate_dtype))) return why;
    }
    return nullptr;
}

struct GradPlan { int64_t groups, each; sopr::RowShare share; size_t part_a, part_b, stats, bytes; };
GradPlan plan_of(int64_t M, int64_t D, int64_t groups, int n_cu)
{
    GradPlan g;
    g.groups = groups < 1 ? 1 : groups;
    g.each = M / g.groups;
    g.share = sopr::norm_share(g.groups, g.each < 1 ? 1 : g.each, sopr::norm_grad_most(D, n_cu));
    const size_t row = (size_t)g.share.words * (size_t)D * 4;
    g.part_a = 0;
    g.part_b = row;
    g.stats = 2 * row;
    g.bytes = g.stats + (sopr::norm_grad_shape(D).T == 0 ? (size_t)M * 12 : 0);
    return g;
}

}  // namespace

extern "C" sop_status sop_fp8_linear_grad_workspace(sop_ctx* c, int64_t M, int64_t N, size_t* bytes)
{
    if (!c) return SOP_EINVAL;
    if (!bytes) return bad(c, "sop_fp8_linear_grad_workspace", SOP_EINVAL, "bytes is NULL");
    if (!dims_ok(M, N, 1)) return bad(c, "sop_fp8_linear_grad_workspace", SOP_ESHAPE, kDims);
    *bytes = sopr::act_grad_few(M) ? 0 : (size_t)sopr::act_grad_words(M, N, sopc::compute_units(c)) * (size_t)N * 4;
    return SOP_OK;
}

extern "C" sop_status sop_fp8_linear_grad(sop_ctx* c, const void* dy, int64_t lddy, const void* z, int64_t ldz, sop_dtype dtype, int64_t M, int64_t N,
                                          sop_act act, float scale, void* dz, int64_t lddz, const sop_f8_matrix* dz8, float* dbias,
                                          void* workspace, size_t workspace_bytes, void* stream)
{
    const char* call = "sop_fp8_linear_grad";
    if (!c) return SOP_EINVAL;
    if (!dims_ok(M, N, 1)) return bad(c, call, SOP_ESHAPE, kDims);
    if (!dtype_ok(dtype)) return bad(c, call, SOP_EINVAL, "dy, z and dz are fp32 or bf16");
    if (act < SOP_ACT_NONE || act > SOP_ACT_GELU_TANH) return bad(c, call, SOP_EINVAL, "no known activation");
    if (off(dbias, 4)) return bad(c, call, SOP_EINVAL, "dbias is not aligned to its elements");
    const int64_t size = size_of(dtype);
    ActGradParams p;
    std::memset(&p, 0, sizeof(p));
    if (M > 0) {
        if (const char* why = plain_fault(dy, N, lddy, size)) return bad(c, call, SOP_EINVAL, why);
        if (act != SOP_ACT_NONE) if (const char* why = plain_fault(z, N, ldz, size)) return bad(c, call, SOP_EINVAL, why);
        if (dz) if (const char* why = plain_fault(dz, N, lddz, size)) return bad(c, call, SOP_EINVAL, why);
        if (dz && M > 1 && ((dz == dy && lddz != lddy) || (act != SOP_ACT_NONE && dz == z && lddz != ldz))) return bad(c, call, SOP_EINVAL, "a dz in dy's or z's place has its row stride");
        if (const char* why = f8_fault(dz8, N, blocks(N), 1)) return bad(c, call, SOP_EINVAL, why);
        p.q = out_of(dz8);
    }
    p.dy = dy; p.lddy = lddy; p.z = act == SOP_ACT_NONE ? nullptr : z; p.ldz = ldz; p.M = M; p.N = (int)N; p.scale = scale; p.act = (int)act;
    p.dz = dz; p.lddz = lddz; p.dbias = dbias;
    p.words = sopr::act_grad_words(M, N, sopc::compute_units(c));
    p.strips = (int)((N + 511) / 512);
    if (dbias && M > 0 && !sopr::act_grad_few(M)) {
        if (!workspace || off(workspace, 16) || workspace_bytes < (size_t)p.words * (size_t)N * 4) return bad(c, call, SOP_ENOMEM, "the workspace is NULL, not on 16 bytes, or too small");
        p.part = static_cast<float*>(workspace);
    }
    OnDevice on(sopc::device(c));
    if (on.err != hipSuccess) return launched(c, call, on.err);
    if (M > 0) {
        const hipError_t e = sopk_act_grad_launch(&p, dtype == SOP_BF16, dz8->format == SOP_E5M2, stream);
        if (e != hipSuccess || !p.part) return launched(c, call, e);
    }
    if (!dbias) return SOP_OK;
    JoinParams j;
    std::memset(&j, 0, sizeof(j));
    j.D = (int)N; j.factor = 1.0f;
    one_sum(j, 0, p.part, M > 0 ? p.words : 0, 1, dbias, 0, false);
    return launched(c, call, join(j, stream));
}

extern "C" sop_status sop_residual_norm(sop_ctx* c, const sop_residual_norm_opts* o, int64_t M, int64_t D, const void* y, int64_t ld_y, sop_dtype y_dtype,
                                        const void* r, int64_t ld_r, sop_dtype r_dtype, void* s, int64_t ld_s, void* n, int64_t ld_n, sop_dtype n_dtype,
                                        const sop_f8_matrix* n8, void* stream)
{
    const char* call = "sop_residual_norm";
    if (!c) return SOP_EINVAL;
    if (!dims_ok(M, 1, D) || D > kMaxRow) return bad(c, call, SOP_ESHAPE, "M within 0 .. 2^30, D within 1 .. 2^20");
    if (!dtype_ok(r_dtype) || (y && !dtype_ok(y_dtype)) || (n && !dtype_ok(n_dtype))) return bad(c, call, SOP_EINVAL, "r, y and n are fp32 or bf16");
    if (const char* why = norm_fault(o, M, D)) return bad(c, call, SOP_EINVAL, why);
    if (M == 0) return SOP_OK;                                          // (matrices without rows have no address)
    if ((n || n8) != (o->before != nullptr)) return bad(c, call, SOP_EINVAL, "n or n8 with `before`, neither without");
    if (!y && (s || o->after || o->gate)) return bad(c, call, SOP_EINVAL, "without y there is no sum, no `after` and no gate");
    if (!y && !o->before) return bad(c, call, SOP_EINVAL, "nothing to do: neither y nor `before`");
    if (const char* why = plain_fault(r, D, ld_r, size_of(r_dtype))) return bad(c, call, SOP_EINVAL, why);
    if (y) {
        if (const char* why = plain_fault(y, D, ld_y, size_of(y_dtype))) return bad(c, call, SOP_EINVAL, why);
        if (const char* why = plain_fault(s, D, ld_s, size_of(r_dtype))) return bad(c, call, SOP_EINVAL, why);
        if (s == r && ld_s != ld_r && M > 1) return bad(c, call, SOP_EINVAL, "a sum in r's place has its row stride");
        if (s == y) return bad(c, call, SOP_EINVAL, "the sum may take r's place, not y's");
    }
    if (n) {
        if (const char* why = plain_fault(n, D, ld_n, size_of(n_dtype))) return bad(c, call, SOP_EINVAL, why);
        if (n == r || n == y || n == s) return bad(c, call, SOP_EINVAL, "n has memory of its own");
    }
    if (n8) if (const char* why = f8_fault(n8, D, blocks(D), 1)) return bad(c, call, SOP_EINVAL, why);
    NormParams p;
    std::memset(&p, 0, sizeof(p));
    p.y = y; p.ldy = ld_y; p.r = r; p.ldr = ld_r; p.after = o->after; p.before = o->before;
    p.gate = o->gate; p.ldg = o->ld_gate; p.gate_bf16 = o->gate && o->gate_dtype == SOP_BF16; p.per_group = o->gate ? M / o->groups : M;
    p.scale = o->scale; p.eps = o->eps; p.eps_fewer = o->eps * SOPK_FEWER * SOPK_FEWER; p.M = M; p.D = (int)D;
    p.out = s; p.ldo = ld_s; p.n = n; p.ldn = ld_n; p.n_bf16 = n && n_dtype == SOP_BF16;
    if (n8) { p.q = out_of(n8); p.e5m2 = n8->format == SOP_E5M2; }
    OnDevice on(sopc::device(c));
    if (on.err != hipSuccess) return launched(c, call, on.err);
    return launched(c, call, sopk_norm_launch(&p, (y ? y_dtype : r_dtype) == SOP_BF16, r_dtype == SOP_BF16, sopc::compute_units(c), stream));
}

extern "C" sop_status sop_residual_norm_grad_workspace(sop_ctx* c, int64_t M, int64_t D, int64_t groups, size_t* bytes)
{
    const char* call = "sop_residual_norm_grad_workspace";
    if (!c) return SOP_EINVAL;
    if (!bytes) return bad(c, call, SOP_EINVAL, "bytes is NULL");
    if (!dims_ok(M, 1, D) || D > kMaxRow || groups < 0 || (groups > 0 && M % groups)) return bad(c, call, SOP_ESHAPE, "M within 0 .. 2^30, D within 1 .. 2^20, groups 0 or a divisor of M");
    *bytes = M > 0 ? plan_of(M, D, groups, sopc::compute_units(c)).bytes : 0;
    return SOP_OK;
}

extern "C" sop_status sop_residual_norm_grad(sop_ctx* c, const sop_residual_norm_opts* o, int64_t M, int64_t D, const sop_residual_norm_grads* t,
                                             void* workspace, size_t workspace_bytes, void* stream)
{
    const char* call = "sop_residual_norm_grad";
    if (!c) return SOP_EINVAL;
    if (!dims_ok(M, 1, D) || D > kMaxRow) return bad(c, call, SOP_ESHAPE, "M within 0 .. 2^30, D within 1 .. 2^20");
    if (!t) return bad(c, call, SOP_EINVAL, "the gradients are NULL");
    const bool has_y = t->y != nullptr || (M == 0 && o && (o->after || o->gate));
    if (!dtype_ok(t->r_dtype) || ((has_y || (o && o->before)) && !dtype_ok(t->y_dtype))) return bad(c, call, SOP_EINVAL, "matrices are fp32 or bf16");
    if (const char* why = norm_fault(o, M, D)) return bad(c, call, SOP_EINVAL, why);
    if (!has_y && (o->after || o->gate)) return bad(c, call, SOP_EINVAL, "without y there is no `after` and no gate");
    if ((t->dbefore && !o->before) || (t->dafter && !o->after) || (t->dgate && !o->gate)) return bad(c, call, SOP_EINVAL, "a gradient is asked for that there is nothing to have");
    if (off(t->dbefore, 4) || off(t->dafter, 4)) return bad(c, call, SOP_EINVAL, "dbefore or dafter is not aligned to its elements");
    if ((t->dbefore && t->dbefore == o->before) || (t->dafter && t->dafter == o->after) || (t->dgate && t->dgate == o->gate))   // (which other workgroups still read)
        return bad(c, call, SOP_EINVAL, "the gradients of weights and gate have memory of their own");
    const int64_t zr = size_of(t->r_dtype), zy = size_of(t->y_dtype);
    if (t->dgate) if (const char* why = plain_fault(t->dgate, D, t->ld_dgate, size_of(o->gate_dtype))) return bad(c, call, SOP_EINVAL, why);
    if (M > 0) {
        if (!t->ds && !o->before) return bad(c, call, SOP_EINVAL, "no gradient to go from: neither ds nor dn");
        if (t->ds) if (const char* why = plain_fault(t->ds, D, t->ld_ds, zr)) return bad(c, call, SOP_EINVAL, why);
        if (const char* why = plain_fault(t->dr, D, t->ld_dr, zr)) return bad(c, call, SOP_EINVAL, why);
        if (o->before) {
            if (const char* why = plain_fault(t->s, D, t->ld_s, zr)) return bad(c, call, SOP_EINVAL, why);
            if (const char* why = plain_fault(t->dn, D, t->ld_dn, zy)) return bad(c, call, SOP_EINVAL, why);
        }
        if (t->y) {
            if (const char* why = plain_fault(t->y, D, t->ld_y, zy)) return bad(c, call, SOP_EINVAL, why);
            if (const char* why = plain_fault(t->dy, D, t->ld_dy, zy)) return bad(c, call, SOP_EINVAL, why);
        }
        for (const void* in : {t->ds, t->dn, t->s, t->y})
            if (in && (in == t->dr || in == t->dy)) return bad(c, call, SOP_EINVAL, "dr and dy have memory of their own");
        if (t->dr == t->dy) return bad(c, call, SOP_EINVAL, "dr and dy have memory of their own");
        if (t->dy8) {
            if (!t->y) return bad(c, call, SOP_EINVAL, "without y there is no dy8");
            if (const char* why = f8_fault(t->dy8, D, blocks(D), 1)) return bad(c, call, SOP_EINVAL, why);
        }
    }
    const GradPlan g = plan_of(M, D, o->gate ? o->groups : 0, sopc::compute_units(c));
    if (M > 0 && (!workspace || off(workspace, 16) || workspace_bytes < g.bytes)) return bad(c, call, SOP_ENOMEM, "the workspace is NULL, not on 16 bytes, or too small");
    char* at = static_cast<char*>(workspace);
    NormGradParams p;
    std::memset(&p, 0, sizeof(p));
    OnDevice on(sopc::device(c));
    if (on.err != hipSuccess) return launched(c, call, on.err);
    if (M > 0) {
        p.ds = t->ds; p.ldds = t->ld_ds; p.dn = t->dn; p.lddn = t->ld_dn; p.s = t->s; p.lds = t->ld_s; p.y = t->y; p.ldy = t->ld_y;
        p.after = o->after; p.before = o->before; p.gate = o->gate; p.ldg = o->ld_gate; p.gate_bf16 = o->gate && o->gate_dtype == SOP_BF16;
        p.groups = g.groups; p.per_group = g.each; p.scale = o->scale; p.eps = o->eps; p.eps_fewer = o->eps * SOPK_FEWER * SOPK_FEWER; p.M = M; p.D = (int)D;
        p.dr = t->dr; p.lddr = t->ld_dr; p.dy = t->dy; p.lddy = t->ld_dy;
        if (t->dy8) { p.q = out_of(t->dy8); p.e5m2 = t->dy8->format == SOP_E5M2; }
        p.dafter = t->dafter; p.dbefore = t->dbefore; p.dgate = t->dgate; p.lddg = t->ld_dgate;
        p.part_a = reinterpret_cast<float*>(at + g.part_a); p.part_b = reinterpret_cast<float*>(at + g.part_b); p.part_t = p.part_a;
        p.stats = reinterpret_cast<float*>(at + g.stats);
        p.words = g.share.words; p.parts = g.share.parts;
        const hipError_t e = sopk_norm_grad_launch(&p, (t->y || o->before ? t->y_dtype : t->r_dtype) == SOP_BF16, t->r_dtype == SOP_BF16, sopc::compute_units(c), stream);
        if (e != hipSuccess) return launched(c, call, e);
    }
    JoinParams j;
    std::memset(&j, 0, sizeof(j));
    j.D = (int)D; j.after = o->after;
    const int64_t words = M > 0 ? g.share.words : 0;
    const bool shared = g.share.parts > 1;                              // (what the workgroups left is t: dafter = sum of scale gate t, dgate = scale after t)
    if (t->dafter) one_sum(j, 0, p.part_a, words, 1, t->dafter, 0, false);
    if (t->dbefore) one_sum(j, 1, p.part_b, words, 1, t->dbefore, 0, false);
    if (t->dgate && (M == 0 || shared)) one_sum(j, 2, p.part_t, M > 0 ? g.share.parts : 0, o->groups, t->dgate, t->ld_dgate, o->gate_dtype == SOP_BF16);
    if (shared && o->gate) { j.gate = o->gate; j.ldg = o->ld_gate; j.gate_bf16 = o->gate_dtype == SOP_BF16; j.share = g.share.parts; }
    if (shared && t->dafter && t->dgate && o->groups == 1) { j.sets[0] = 0; j.also = 1; }
    j.factor = shared ? o->scale : 1.0f;                                // (whole groups: workgroups have put scale and gate on their sums)
    return launched(c, call, join(j, stream));
}

namespace {

const char* tensors_fault(const sop_grad* t, int64_t count, bool outs)
{
    if (count < 0 || (count > 0 && !t)) return "the tensors are NULL";
    for (int64_t i = 0; i < count; ++i) {
        if (t[i].n < 0 || t[i].n > kMaxTensor) return "a tensor has 0 .. 2^36 elements";
        if (t[i].n == 0) continue;
        if (!dtype_ok(t[i].x_dtype)) return "tensors are fp32 or bf16";
        if (!t[i].x || off(t[i].x, (uintptr_t)size_of(t[i].x_dtype))) return "a tensor is NULL or not aligned to its elements";
        if (!outs) continue;
        if (!dtype_ok(t[i].out_dtype)) return "tensors are fp32 or bf16";
        if (!t[i].out || off(t[i].out, (uintptr_t)size_of(t[i].out_dtype))) return "a tensor is NULL or not aligned to its elements";
        if (t[i].out == t[i].x && t[i].out_dtype != t[i].x_dtype) return "a tensor in its own place keeps its type";
    }
    return nullptr;
}
// Whether what is written is written once, and read by nobody else: no out overlaps another, or a tensor that it is not the place of.
// (Two walks over the ranges in order of their beginnings; memory for them is all that can be missing: then it is not known, and -1.)
struct Range { uintptr_t from, to; int64_t of; bool written; };
int tensors_apart(const sop_grad* t, int64_t count)
{
    Range* r = static_cast<Range*>(std::malloc(sizeof(Range) * 2 * (size_t)(count > 0 ? count : 1)));
    if (!r) return -1;
    int64_t k = 0;
    for (int64_t i = 0; i < count; ++i) {
        if (t[i].n == 0) continue;
        const uintptr_t x = reinterpret_cast<uintptr_t>(t[i].x), o = reinterpret_cast<uintptr_t>(t[i].out);
        r[k++] = Range{o, o + (uintptr_t)(t[i].n * size_of(t[i].out_dtype)), i, true};
        if (t[i].x != t[i].out) r[k++] = Range{x, x + (uintptr_t)(t[i].n * size_of(t[i].x_dtype)), i, false};
    }
    std::sort(r, r + k, [](const Range& a, const Range& b) { return a.from < b.from; });
    uintptr_t read = 0, written = 0;                                    // where what was read, and what was written, ends so far
    int apart = 1;
    for (int64_t i = 0; i < k && apart; ++i) {
        apart = r[i].from >= written && (!r[i].written || r[i].from >= read);
        uintptr_t& end = r[i].written ? written : read;
        end = r[i].to > end ? r[i].to : end;
    }
    std::free(r);
    return apart;
}
size_t clip_bytes(int64_t count, int n_cu) { return (size_t)(8 * n_cu + 64 * sopr::clip_launches(count, SOP_K_CLIP_LIST)) * 8; }

// `pass` is called with each launch's tensors, one launch after the other
template <typename F> hipError_t each_list(const sop_grad* t, int64_t count, ClipParams& p, F pass)
{
    p.count = p.chunks = 0;
    auto go = [&]() {
        const hipError_t e = p.count ? pass() : hipSuccess;
        p.count = p.chunks = 0;
        return e;
    };
    for (int64_t i = 0; i < count; ++i) {
        if (t[i].n == 0) continue;
        const int64_t chunks = (t[i].n + SOP_K_CLIP_CHUNK - 1) / SOP_K_CLIP_CHUNK;
        if (p.count == SOP_K_CLIP_LIST) {                               // (a list of the largest tensors has 96 x 2^23 chunks)
            const hipError_t e = go();
            if (e != hipSuccess) return e;
        }
        p.chunks += (int)chunks;
        p.e[p.count++] = ClipEntry{t[i].x, t[i].out, t[i].n, p.chunks, (t[i].x_dtype == SOP_BF16 ? 1 : 0) | (t[i].out_dtype == SOP_BF16 ? 2 : 0)};
    }
    return go();
}

sop_status norm_and_clip(const char* call, sop_ctx* c, const sop_grad* t, int64_t count, bool clip, float most, float* norm, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!c) return SOP_EINVAL;
    if (const char* why = tensors_fault(t, count, clip)) return bad(c, call, SOP_EINVAL, why);
    if (!norm || off(norm, 4)) return bad(c, call, SOP_EINVAL, "norm is NULL or not on 4 bytes");
    if (clip && !(most >= 0.0f)) return bad(c, call, SOP_EINVAL, "the largest norm is a number of at least 0");
    if (clip) {
        const int apart = tensors_apart(t, count);
        if (apart < 0) return bad(c, call, SOP_ENOMEM, "no memory to compare the tensors' places");
        if (!apart) return bad(c, call, SOP_EINVAL, "an out overlaps another out, or a tensor that it does not take the place of");
    }
    const int n_cu = sopc::compute_units(c);
    if (!workspace || off(workspace, 8) || workspace_bytes < clip_bytes(count, n_cu)) return bad(c, call, SOP_ENOMEM, "the workspace is NULL, not on 8 bytes, or too small");
    ClipParams p;
    std::memset(&p, 0, sizeof(p));
    p.part = static_cast<double*>(workspace); p.norm = norm; p.most = (double)most;
    int64_t some = 0;
    for (int64_t i = 0; i < count; ++i) some += t[i].n > 0;
    const int64_t launches = sopr::clip_launches(some, SOP_K_CLIP_LIST);
    OnDevice on(sopc::device(c));
    if (on.err != hipSuccess) return launched(c, call, on.err);
    hipError_t e = each_list(t, count, p, [&]() {
        const int64_t words = sopr::clip_words(p.chunks, launches, n_cu);
        p.first = p.parts;
        p.parts += (int)words;
        return sopk_square_sum_launch(&p, (int)words, stream);
    });
    if (e != hipSuccess) return launched(c, call, e);
    if (!clip || launches == 0) return launched(c, call, sopk_norm_of_parts_launch(&p, stream));
    p.first = 0;
    e = each_list(t, count, p, [&]() {
        const hipError_t f = sopk_clip_launch(&p, (int)sopr::clip_words(p.chunks, 1, n_cu), stream);
        ++p.first;                                                      // (the first of them writes the norm)
        return f;
    });
    return launched(c, call, e);
}

}  // namespace

extern "C" sop_status sop_clip_grads_workspace(sop_ctx* c, int64_t count, size_t* bytes)
{
    if (!c) return SOP_EINVAL;
    if (!bytes || count < 0) return bad(c, "sop_clip_grads_workspace", SOP_EINVAL, "bytes is NULL, or count negative");
    *bytes = clip_bytes(count, sopc::compute_units(c));
    return SOP_OK;
}
extern "C" sop_status sop_grad_norm(sop_ctx* c, const sop_grad* tensors, int64_t count, float* norm, void* workspace, size_t workspace_bytes, void* stream)
{
    return norm_and_clip("sop_grad_norm", c, tensors, count, false, 0.0f, norm, workspace, workspace_bytes, stream);
}
extern "C" sop_status sop_clip_grads(sop_ctx* c, const sop_grad* tensors, int64_t count, float most, float* norm, void* workspace, size_t workspace_bytes, void* stream)
{
    return norm_and_clip("sop_clip_grads", c, tensors, count, true, most, norm, workspace, workspace_bytes, stream);
}
