// What the operators of a language model (embed.cu, attention.cu, distill.cu) need of a context.
// The context itself is omni.cu's; these three calls are the whole seam.
#pragma once
#include "../../include/omni.h"

namespace omni {

struct ContextDevice {
    int sm_count;
    unsigned int *status;  // device word a kernel sets when a bounded wait runs out (OMNI_ERR_TIMEOUT)
};

// Binds the context to the current device on its first use; an omni_status.
int context_bind(omni_ctx *ctx, ContextDevice *out);
// Books one kernel launch: counts it, or records the cudaError_t it failed with; an omni_status.
int context_launched(omni_ctx *ctx, int cuda_error);
// Opts a kernel into `bytes` of dynamic shared memory, once per context (a context stays on one device).
int context_shared(omni_ctx *ctx, const void *kernel, int bytes);

}  // namespace omni
