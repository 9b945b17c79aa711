// Checks of arguments that the entry points around a linear layer share: a kernel's own bounds rest on what these let through.
#ifndef SOP_CHECKS_H
#define SOP_CHECKS_H
#include "../../include/sop.h"

#include <hip/hip_runtime.h>

#include <cstdio>

#include "sop_ctx.h"
#include "sop_linear.h"

namespace {

constexpr int64_t kMaxDim = (int64_t)1 << 30, kMaxStride = (int64_t)1 << 23;

struct OnDevice {
    int prev = 0;
    bool switched = false;
    hipError_t err = hipSuccess;
    explicit OnDevice(int dev) { (void)hipGetDevice(&prev); if (prev != dev) { err = hipSetDevice(dev); switched = err == hipSuccess; } }
    ~OnDevice() { if (switched) (void)hipSetDevice(prev); }
};

inline bool off(const void* p, uintptr_t unit) { return (reinterpret_cast<uintptr_t>(p) & (unit - 1)) != 0; }
inline bool dtype_ok(sop_dtype d) { return d == SOP_F32 || d == SOP_BF16; }
inline int64_t size_of(sop_dtype d) { return d == SOP_F32 ? 4 : 2; }

// a matrix of numbers: null if it is one
inline const char* plain_fault(const void* p, int64_t cols, int64_t ld, int64_t size)
{
    if (!p) return "a matrix is NULL";
    if (off(p, (uintptr_t)size)) return "a matrix is not aligned to its elements";
    if (ld < cols) return "a row stride is smaller than the row";
    return nullptr;
}
// a matrix in 8 bits: null if it is one
inline const char* f8_fault(const sop_f8_matrix* q, int64_t cols, int64_t scale_cols, int block_rows)
{
    if (!q || !q->codes || !q->scales) return "an 8-bit matrix is NULL";
    if (q->format != SOP_E4M3 && q->format != SOP_E5M2) return "an 8-bit matrix is of no known format";
    if (q->block_rows != block_rows) return block_rows == 1 ? "activations and gradients have blocks of one row" : "weights have blocks of 128 rows";
    if (off(q->codes, 16) || (q->ld_codes & 15) || off(q->scales, 4) || (q->ld_scales & 3)) return "codes are on 16 bytes with a row stride of a multiple of 16, scales on 4 with one of 4";
    if (q->ld_codes < cols || q->ld_scales < scale_cols) return "a row stride is smaller than the row";
    if (q->ld_codes > kMaxStride || q->ld_scales > kMaxStride) return "a row stride is larger than 2^23";
    return nullptr;
}
inline sop_status bad(sop_ctx* c, const char* call, sop_status s, const char* why)
{
    char text[256];
    std::snprintf(text, sizeof(text), "%s: %s", call, why);
    return sopc::fail(c, s, text);
}
inline sop_status launched(sop_ctx* c, const char* call, hipError_t e)
{
    if (e == hipSuccess) return SOP_OK;
    char text[256];
    std::snprintf(text, sizeof(text), "%s: kernel launch: %s", call, hipGetErrorString(e));
    return sopc::fail(c, SOP_EHIP, text);
}
inline bool dims_ok(int64_t M, int64_t N, int64_t K) { return M >= 0 && N >= 1 && K >= 1 && M <= kMaxDim && N <= kMaxDim && K <= kMaxDim; }
const char* const kDims = "M >= 0 and N, K >= 1, at most 2^30 each";
inline int64_t blocks(int64_t n) { return (n + 127) / 128; }
inline F8Out out_of(const sop_f8_matrix* q) { return F8Out{q->codes, q->ld_codes, q->scales, q->ld_scales}; }
inline F8In in_of(const sop_f8_matrix* q) { return F8In{q->codes, q->ld_codes, q->scales, q->ld_scales}; }
inline bool rows16(const void* p, int64_t ld, int64_t size) { return !off(p, 16) && (ld * size) % 16 == 0; }

}  // namespace
#endif
