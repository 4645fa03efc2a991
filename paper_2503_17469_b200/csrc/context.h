// What the operators of a language model (embed.cu, attention.cu, distill.cu) need of a context.
// The context itself is omni.cu's; these three calls are the whole seam.
#pragma once
#include <cuda_runtime.h>

#include "../../include/omni.h"

namespace omni {

struct ContextDevice {
    int sm_count;
    bool overlap;          // the context allows launches that begin while their predecessor ends (not OMNI_NO_BULK_COPY)
    unsigned int *status;  // device word a kernel sets when a bounded wait runs out (OMNI_ERR_TIMEOUT)
};

// Binds the context to the current device on its first use; an omni_status.
int context_bind(omni_ctx *ctx, ContextDevice *out);
// Books one kernel launch: counts it, or records the cudaError_t it failed with; an omni_status.
int context_launched(omni_ctx *ctx, int cuda_error);
// Launch configuration of a kernel that sets itself up while its predecessor, the call's own previous kernel, ends, and
// executes griddepcontrol.wait before it touches what that one wrote.
struct Dependent {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    Dependent(const ContextDevice &dev, dim3 grid, int threads, size_t smem, cudaStream_t stream)
    {
        cfg.gridDim = grid;
        cfg.blockDim = dim3(threads);
        cfg.dynamicSmemBytes = smem;
        cfg.stream = stream;
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = dev.overlap ? 1 : 0;
    }
};

// Opts a kernel into `bytes` of dynamic shared memory, once per context (a context stays on one device).
int context_shared(omni_ctx *ctx, const void *kernel, int bytes);

}  // namespace omni
