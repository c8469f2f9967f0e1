// The norm over many tensors, and the tensors scaled down to a bound on it: host interface.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

#include "product.h"

namespace redist {

struct ClipTensor {
    const void *data;
    void *out;
    int64_t elements;
    int32_t type;
};

// tensors is read during the call only.  partials: clip_partials(...) doubles.
int64_t clip_partials(const ClipTensor *tensors, int64_t count, int sms);
cudaError_t launch_clip(const ClipTensor *tensors, int64_t count, float max_norm, float eps, float *norm, double *partials, int sms,
                        const LaunchOptions &o, cudaStream_t stream);

}  // namespace redist
