// What libgts's translation units share: the calling thread's error text (gts_last_error).
#ifndef GTS_INTERNAL_H
#define GTS_INTERNAL_H

#include <cuda_runtime.h>

#include "gts_serving.h"

#define GTS_HIDDEN __attribute__((visibility("hidden")))

namespace gts {
GTS_HIDDEN gts_status fail(gts_status s, const char *msg);            // sets the text, returns s
GTS_HIDDEN gts_status cuda_fail(cudaError_t e, const char *what);     // GTS_ERR_CUDA with the runtime's words
GTS_HIDDEN void clear_error();
}  // namespace gts

#endif
