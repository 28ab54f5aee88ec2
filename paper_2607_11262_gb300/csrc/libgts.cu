// The simulator's translation unit, with its error text made available to the library's other ones.
#include "gts.cu"

#include "internal.h"

namespace gts {
gts_status fail(gts_status s, const char *msg) { return ::fail(s, msg); }
gts_status cuda_fail(cudaError_t e, const char *what) { return ::cuda_fail(e, what); }
void clear_error() { ::clear_error(); }
}  // namespace gts
