// Entry points of the products of a linear layer with narrow operands: every argument is checked here, before a launch; the kernels'
// own bounds rest on what these checks let through.
#include <cstring>

#include "sop_checks.h"
#include "sop_linear_rules.h"

extern "C" hipError_t sopk_f8_quant_launch(const F8QuantParams* p, int bf16, int e5m2, int vec, int square, void* stream);
extern "C" hipError_t sopk_f8_gated_launch(const F8GatedParams* p, int bf16, int e5m2, int vec, void* stream);
extern "C" hipError_t sopk_f8_gated_grad_launch(const F8GatedGradParams* p, int bf16, int ckpt_e5m2, int e5m2, int vec, void* stream);
extern "C" hipError_t sopk_f8mm_launch(const F8MmParams* p, int x_e5m2, int choice, void* stream);
extern "C" hipError_t sopk_f8mm_epilogue_launch(const F8MmParams* p, int x_e5m2, int choice, void* stream);
extern "C" hipError_t sopk_wgrad_launch(const WgradParams* p, int x_e5m2, int choice, void* stream);
extern "C" hipError_t sopk_packed_launch(const PackedMmParams* p, int choice, void* stream);
extern "C" hipError_t sopk_packed_epilogue_launch(const PackedMmParams* p, int choice, void* stream);

namespace {

// One launch, or, where none can be large enough (fewer than 64 elements along K, and some 2^35 numbers of y), halves of its longer side
hipError_t packed_parts(const PackedMmParams& p, bool epilogue, int n_cu, void* stream)
{
    const int choice = sopr::packed_choice(p.M, p.N, p.K, p.n_bits, n_cu);
    if (choice >= 0) return epilogue ? sopk_packed_epilogue_launch(&p, choice, stream) : sopk_packed_launch(&p, choice, stream);
    PackedMmParams a = p, b = p;
    if (p.M >= p.N) {
        a.M = p.M / 2; b.M = p.M - a.M;
        b.x += a.M * p.ldx; b.y += a.M * p.ldy;
        if (p.e.residual) b.e.residual = static_cast<const uint16_t*>(p.e.residual) + a.M * p.e.ldr;
        if (p.e.z) b.e.z = static_cast<uint16_t*>(p.e.z) + a.M * p.e.ldz;
    } else {
        a.N = p.N / 2; b.N = p.N - a.N;
        b.words += (int64_t)a.N * (p.K / p.g); b.payload += (int64_t)a.N * (p.K / 8) * p.n_bits; b.y += a.N;
        if (p.e.bias) b.e.bias += a.N;
        if (p.e.residual) b.e.residual = static_cast<const uint16_t*>(p.e.residual) + a.N;
        if (p.e.z) b.e.z = static_cast<uint16_t*>(p.e.z) + a.N;
    }
    const hipError_t e = packed_parts(a, epilogue, n_cu, stream);
    return e != hipSuccess ? e : packed_parts(b, epilogue, n_cu, stream);
}

// an epilogue of [M, N] results of `size` bytes: null if it is one
const char* epilogue_fault(const sop_epilogue* e, int64_t N, int64_t size, const void* y, int64_t ldy)
{
    if (!e) return "the epilogue is NULL";
    if (e->act < SOP_ACT_NONE || e->act > SOP_ACT_GELU_TANH) return "no known activation";
    if (off(e->bias, 4)) return "the bias is not aligned to its elements";
    if (e->residual) {
        if (const char* why = plain_fault(e->residual, N, e->ldr, size)) return why;
        if (e->residual == y && e->ldr != ldy) return "a residual that is y has its row stride";
    }
    if (e->z) {
        if (const char* why = plain_fault(e->z, N, e->ldz, size)) return why;
        if (e->z == y || e->z == e->residual) return "z has memory of its own";
    }
    return nullptr;
}
Epilogue epilogue_of(const sop_epilogue* e) { return Epilogue{e->bias, e->residual, e->ldr, e->z, e->ldz, e->scale, (int)e->act}; }

}  // namespace

extern "C" sop_status sop_fp8_quantize(sop_ctx* c, const void* x, sop_dtype dtype, int64_t M, int64_t K, int64_t ldx, const sop_f8_matrix* q,
                                       uint8_t* codes_t, int64_t ld_codes_t, void* stream)
{
    const char* call = "sop_fp8_quantize";
    if (!c) return SOP_EINVAL;
    if (!dims_ok(M, 1, K)) return bad(c, call, SOP_ESHAPE, kDims);
    if (!dtype_ok(dtype)) return bad(c, call, SOP_EINVAL, "x is fp32 or bf16");
    if (!q) return bad(c, call, SOP_EINVAL, "an 8-bit matrix is NULL");
    const int rows = q->block_rows;
    if (rows != 1 && rows != 128) return bad(c, call, SOP_EINVAL, "blocks have 1 or 128 rows");
    if (M > 0) if (const char* why = plain_fault(x, K, ldx, size_of(dtype))) return bad(c, call, SOP_EINVAL, why);
    if (M > 0) if (const char* why = f8_fault(q, K, blocks(K), rows)) return bad(c, call, SOP_EINVAL, why);
    if (codes_t) {
        if (rows != 128) return bad(c, call, SOP_EINVAL, "a transposed copy is made of square blocks only: blocks of one row have no scales for it");
        if (off(codes_t, 16) || (ld_codes_t & 15) || ld_codes_t < M || ld_codes_t > kMaxStride) return bad(c, call, SOP_EINVAL, "codes_t is on 16 bytes, its row stride a multiple of 16, at least M and at most 2^23");
    }
    if (M == 0) return SOP_OK;
    F8QuantParams p;
    std::memset(&p, 0, sizeof(p));
    p.x = x; p.ldx = ldx; p.M = M; p.K = K;
    p.codes = q->codes; p.ldc = q->ld_codes; p.scales = q->scales; p.lds = q->ld_scales;
    p.codes_t = codes_t; p.ldct = ld_codes_t;
    if (rows == 128 && blocks(M) * blocks(K) > 0x7FFFFFFF) return bad(c, call, SOP_ESHAPE, "too many blocks");
    OnDevice on(sopc::device(c));
    if (on.err != hipSuccess) return launched(c, call, on.err);
    return launched(c, call, sopk_f8_quant_launch(&p, dtype == SOP_BF16, q->format == SOP_E5M2, rows16(x, ldx, size_of(dtype)), rows == 128, stream));
}

static sop_status fp8_product(const char* call, sop_ctx* c, const sop_f8_matrix* x, const sop_f8_matrix* w, int w_transposed, int64_t M, int64_t N, int64_t K,
                              const sop_epilogue* e, bool epilogue, void* y, sop_dtype dtype, int64_t ldy, void* stream)
{
    if (!c) return SOP_EINVAL;
    if (!dims_ok(M, N, K)) return bad(c, call, SOP_ESHAPE, kDims);
    if (!dtype_ok(dtype)) return bad(c, call, SOP_EINVAL, "y is fp32 or bf16");
    if (const char* why = f8_fault(w, K, blocks(w_transposed ? N : K), 128)) return bad(c, call, SOP_EINVAL, why);
    if (w->format != SOP_E4M3) return bad(c, call, SOP_EINVAL, "weights are E4M3");
    if (M == 0) return SOP_OK;
    if (const char* why = f8_fault(x, K, blocks(K), 1)) return bad(c, call, SOP_EINVAL, why);
    if (const char* why = plain_fault(y, N, ldy, size_of(dtype))) return bad(c, call, SOP_EINVAL, why);
    if (epilogue) if (const char* why = epilogue_fault(e, N, size_of(dtype), y, ldy)) return bad(c, call, SOP_EINVAL, why);
    F8MmParams p;
    std::memset(&p, 0, sizeof(p));
    p.x = x->codes; p.ldx = x->ld_codes; p.xs = x->scales; p.ldxs = x->ld_scales;
    p.w = w->codes; p.ldw = w->ld_codes; p.ws = w->scales;
    p.ws_n = w_transposed ? 1 : w->ld_scales; p.ws_k = w_transposed ? w->ld_scales : 1;
    p.M = (int)M; p.N = (int)N; p.K = (int)K;
    p.y = y; p.ldy = ldy; p.out_bf16 = dtype == SOP_BF16;
    if (epilogue) p.e = epilogue_of(e);
    const int choice = sopr::f8mm_choice(M, N, dtype == SOP_F32, sopc::compute_units(c));
    if (choice < 0) return bad(c, call, SOP_ESHAPE, "y is too large for a launch");
    OnDevice on(sopc::device(c));
    if (on.err != hipSuccess) return launched(c, call, on.err);
    return launched(c, call, epilogue ? sopk_f8mm_epilogue_launch(&p, x->format == SOP_E5M2, choice, stream) : sopk_f8mm_launch(&p, x->format == SOP_E5M2, choice, stream));
}

extern "C" sop_status sop_fp8_matmul(sop_ctx* c, const sop_f8_matrix* x, const sop_f8_matrix* w, int w_transposed, int64_t M, int64_t N, int64_t K,
                                     void* y, sop_dtype dtype, int64_t ldy, void* stream)
{
    return fp8_product("sop_fp8_matmul", c, x, w, w_transposed, M, N, K, nullptr, false, y, dtype, ldy, stream);
}

extern "C" sop_status sop_fp8_linear(sop_ctx* c, const sop_f8_matrix* x, const sop_f8_matrix* w, int w_transposed, int64_t M, int64_t N, int64_t K,
                                     const sop_epilogue* e, void* y, sop_dtype dtype, int64_t ldy, void* stream)
{
    return fp8_product("sop_fp8_linear", c, x, w, w_transposed, M, N, K, e, true, y, dtype, ldy, stream);
}

extern "C" sop_status sop_fp8_weight_grad(sop_ctx* c, const void* dy, int64_t lddy, const sop_f8_matrix* x, int64_t M, int64_t N, int64_t K,
                                          void* dw, sop_dtype dtype, int64_t lddw, int accumulate, void* stream)
{
    const char* call = "sop_fp8_weight_grad";
    if (!c) return SOP_EINVAL;
    if (!dims_ok(M, N, K)) return bad(c, call, SOP_ESHAPE, kDims);
    if (!dtype_ok(dtype)) return bad(c, call, SOP_EINVAL, "dw is fp32 or bf16");
    if (const char* why = plain_fault(dw, K, lddw, size_of(dtype))) return bad(c, call, SOP_EINVAL, why);
    if (M == 0 && accumulate) return SOP_OK;
    WgradParams p;
    std::memset(&p, 0, sizeof(p));
    if (M > 0) {
        if (const char* why = plain_fault(dy, N, lddy, 2)) return bad(c, call, SOP_EINVAL, why);
        if (const char* why = f8_fault(x, K, blocks(K), 1)) return bad(c, call, SOP_EINVAL, why);
        p.dy = static_cast<const uint16_t*>(dy); p.lddy = lddy;
        p.x = x->codes; p.ldx = x->ld_codes; p.xs = x->scales; p.ldxs = x->ld_scales;
    }
    p.M = (int)M; p.N = (int)N; p.K = (int)K;
    p.dw = dw; p.lddw = lddw; p.out_bf16 = dtype == SOP_BF16; p.accumulate = accumulate != 0;
    if (((N + 63) / 64) * ((K + 127) / 128) > 0x7FFFFFFF) return bad(c, call, SOP_ESHAPE, "dw is too large");
    const bool on16 = rows16(dy, lddy, 2) && lddy <= (int64_t)1 << 22;
    OnDevice on(sopc::device(c));
    if (on.err != hipSuccess) return launched(c, call, on.err);
    return launched(c, call, sopk_wgrad_launch(&p, M > 0 && x->format == SOP_E5M2, sopr::wgrad_choice(M, N, K, on16, sopc::compute_units(c)), stream));
}

extern "C" sop_status sop_fp8_gated(sop_ctx* c, const void* gate, int64_t ld_gate, const void* up, int64_t ld_up, sop_dtype dtype, int64_t M, int64_t F,
                                    const sop_f8_matrix* h, const sop_f8_matrix* gate8, const sop_f8_matrix* up8, void* stream)
{
    const char* call = "sop_fp8_gated";
    if (!c) return SOP_EINVAL;
    if (!dims_ok(M, 1, F)) return bad(c, call, SOP_ESHAPE, kDims);
    if (!dtype_ok(dtype)) return bad(c, call, SOP_EINVAL, "gate and up are fp32 or bf16");
    if (M == 0) return SOP_OK;
    if (const char* why = plain_fault(gate, F, ld_gate, size_of(dtype))) return bad(c, call, SOP_EINVAL, why);
    if (const char* why = plain_fault(up, F, ld_up, size_of(dtype))) return bad(c, call, SOP_EINVAL, why);
    for (const sop_f8_matrix* q : {h, gate8, up8}) if (const char* why = f8_fault(q, F, blocks(F), 1)) return bad(c, call, SOP_EINVAL, why);
    if (h->format != gate8->format || h->format != up8->format) return bad(c, call, SOP_EINVAL, "h, gate8 and up8 are of one format");
    F8GatedParams p;
    std::memset(&p, 0, sizeof(p));
    p.gate = gate; p.ldg = ld_gate; p.up = up; p.ldu = ld_up; p.M = M; p.F = F;
    p.h = out_of(h); p.g8 = out_of(gate8); p.u8 = out_of(up8);
    OnDevice on(sopc::device(c));
    if (on.err != hipSuccess) return launched(c, call, on.err);
    const int64_t z = size_of(dtype);
    return launched(c, call, sopk_f8_gated_launch(&p, dtype == SOP_BF16, h->format == SOP_E5M2, rows16(gate, ld_gate, z) && rows16(up, ld_up, z), stream));
}

extern "C" sop_status sop_fp8_gated_grad(sop_ctx* c, const sop_f8_matrix* gate8, const sop_f8_matrix* up8, const void* dh, int64_t ld_dh, sop_dtype dtype,
                                         int64_t M, int64_t F, void* dgate, int64_t ld_dgate, void* dup, int64_t ld_dup,
                                         const sop_f8_matrix* dgate8, const sop_f8_matrix* dup8, void* stream)
{
    const char* call = "sop_fp8_gated_grad";
    if (!c) return SOP_EINVAL;
    if (!dims_ok(M, 1, F)) return bad(c, call, SOP_ESHAPE, kDims);
    if (!dtype_ok(dtype)) return bad(c, call, SOP_EINVAL, "dh, dgate and dup are fp32 or bf16");
    if (M == 0) return SOP_OK;
    const int64_t z = size_of(dtype);
    if (const char* why = plain_fault(dh, F, ld_dh, z)) return bad(c, call, SOP_EINVAL, why);
    if (const char* why = plain_fault(dgate, F, ld_dgate, z)) return bad(c, call, SOP_EINVAL, why);
    if (const char* why = plain_fault(dup, F, ld_dup, z)) return bad(c, call, SOP_EINVAL, why);
    for (const sop_f8_matrix* q : {gate8, up8, dgate8, dup8}) if (const char* why = f8_fault(q, F, blocks(F), 1)) return bad(c, call, SOP_EINVAL, why);
    if (gate8->format != up8->format || dgate8->format != dup8->format) return bad(c, call, SOP_EINVAL, "gate8 and up8 are of one format, dgate8 and dup8 too");
    F8GatedGradParams p;
    std::memset(&p, 0, sizeof(p));
    p.g8 = in_of(gate8); p.u8 = in_of(up8); p.dh = dh; p.lddh = ld_dh; p.M = M; p.F = F;
    p.dgate = dgate; p.lddg = ld_dgate; p.dup = dup; p.lddu = ld_dup;
    p.dg8 = out_of(dgate8); p.du8 = out_of(dup8);
    OnDevice on(sopc::device(c));
    if (on.err != hipSuccess) return launched(c, call, on.err);
    const int vec = rows16(dh, ld_dh, z) && rows16(dgate, ld_dgate, z) && rows16(dup, ld_dup, z);
    return launched(c, call, sopk_f8_gated_grad_launch(&p, dtype == SOP_BF16, gate8->format == SOP_E5M2, dgate8->format == SOP_E5M2, vec, stream));
}

static sop_status packed_product(const char* call, sop_ctx* c, const void* x, int64_t ldx, const sop_packed_weights* w, int64_t M, const sop_epilogue* e, bool epilogue,
                                 void* y, int64_t ldy, void* stream)
{
    if (!c) return SOP_EINVAL;
    if (!w) return bad(c, call, SOP_EINVAL, "the weights are NULL");
    if (!dims_ok(M, w->N, w->K)) return bad(c, call, SOP_ESHAPE, kDims);
    const int g = w->g;
    if ((g != 8 && g != 16 && g != 32 && g != 64) || w->K % g) return bad(c, call, SOP_ESHAPE, "g is 8, 16, 32 or 64 and divides K");
    if (w->n_bits < 1 || w->n_bits > 6) return bad(c, call, SOP_EINVAL, "codes have 1 to 6 bits");
    if (!w->words_dev || !w->payload_dev || off(w->words_dev, 2) || off(w->payload_dev, 8)) return bad(c, call, SOP_EINVAL, "words and payload must not be NULL, words on 2 bytes, payload on 8");
    if (!w->table_a || w->entries_a < 1 || w->entries_a > SOP_MAX_ENTRIES) return bad(c, call, SOP_EATOM, "the first codebook has 1 to 64 entries");
    if ((w->table_b != nullptr) != (w->entries_b > 0) || w->entries_b < 0 || w->entries_b > SOP_MAX_ENTRIES) return bad(c, call, SOP_EATOM, "the second codebook has 1 to 64 entries, or is NULL with 0");
    const int sb = w->fmt.sign_bits, xb = w->fmt.exp_bits, yb = w->fmt.man_bits, b = w->fmt.container_bits, m = b - sb - xb - yb;
    if ((sb != 0 && sb != 1) || xb < 1 || yb < 0 || b < 1 || b > 16 || xb + yb > 15 || m < 0) return bad(c, call, SOP_EFMT, "not a SwExMy word in a container of at most 16 bits");
    if (w->table_b && m == 0) return bad(c, call, SOP_EFMT, "the scale format has no metabit for the selector");
    if (w->layer_shift_k < -64 || w->layer_shift_k > 64) return bad(c, call, SOP_EFMT, "layer shift outside [-64, 64]");
    const int bias = w->fmt.bias < 0 ? (1 << (xb - 1)) - 1 : w->fmt.bias;
    if (bias > 1 << 15) return bad(c, call, SOP_EFMT, "bias out of range");
    if (M == 0) return SOP_OK;
    if (const char* why = plain_fault(x, w->K, ldx, 2)) return bad(c, call, SOP_EINVAL, why);
    if (!rows16(x, ldx, 2)) return bad(c, call, SOP_EINVAL, "x is on 16 bytes, its row stride a multiple of 8 elements");
    if (w->K > kMaxStride / 2 || (ldx > kMaxStride / 2 && M > 1)) return bad(c, call, SOP_ESHAPE, "rows of x are at most 2^22 elements apart");
    if (const char* why = plain_fault(y, w->N, ldy, 2)) return bad(c, call, SOP_EINVAL, why);
    if (epilogue) if (const char* why = epilogue_fault(e, w->N, 2, y, ldy)) return bad(c, call, SOP_EINVAL, why);
    PackedMmParams p;
    std::memset(&p, 0, sizeof(p));
    p.x = static_cast<const uint16_t*>(x); p.ldx = M > 1 ? ldx : w->K; p.words = w->words_dev; p.payload = w->payload_dev;
    p.M = (int)M; p.N = (int)w->N; p.K = (int)w->K; p.g = g; p.n_bits = w->n_bits;
    p.mag_shift = sb ? m : (m > 0 ? m - 1 : 0);
    p.mag_mask = (1 << (xb + yb)) - 1; p.man_bits = yb; p.man_mask = (1 << yb) - 1;
    p.exp_off = -bias - yb - w->layer_shift_k;
    p.sign_up = sb ? 32 - b : 0;                                        // (16-bit words: bit 31 stays empty where there is no sign)
    p.sel_mask = w->table_b ? 1 : 0;
    p.sel_pos = !w->table_b ? 0 : (sb ? m - 1 : b - 1);
    p.y = static_cast<uint16_t*>(y); p.ldy = ldy;
    for (int i = 0; i < SOP_K_PACKED_TAB; ++i) {
        p.tab[0][i] = w->table_a[i < w->entries_a ? i : w->entries_a - 1];
        if (w->table_b) p.tab[1][i] = w->table_b[i < w->entries_b ? i : w->entries_b - 1];
    }
    if (epilogue) p.e = epilogue_of(e);
    OnDevice on(sopc::device(c));
    if (on.err != hipSuccess) return launched(c, call, on.err);
    return launched(c, call, packed_parts(p, epilogue, sopc::compute_units(c), stream));
}

extern "C" sop_status sop_packed_matmul(sop_ctx* c, const void* x, int64_t ldx, const sop_packed_weights* w, int64_t M, void* y, int64_t ldy, void* stream)
{
    return packed_product("sop_packed_matmul", c, x, ldx, w, M, nullptr, false, y, ldy, stream);
}

extern "C" sop_status sop_packed_linear(sop_ctx* c, const void* x, int64_t ldx, const sop_packed_weights* w, int64_t M, const sop_epilogue* e, void* y, int64_t ldy, void* stream)
{
    return packed_product("sop_packed_linear", c, x, ldx, w, M, e, true, y, ldy, stream);
}
