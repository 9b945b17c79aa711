// What translation units beside sop_api.cpp, which owns the structure, see of a context.
#ifndef SOP_CTX_H
#define SOP_CTX_H
#include "../../include/sop.h"

namespace sopc {
sop_status fail(sop_ctx* c, sop_status s, const char* msg);   // notes the text, returns s
int device(const sop_ctx* c);
int compute_units(const sop_ctx* c);
}  // namespace sopc
#endif
