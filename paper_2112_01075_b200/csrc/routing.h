// The router of a block of experts, and tokens moved to their experts' rows and back: host interface.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

#include "product.h"

namespace redist {

constexpr int kMostExperts = 1024, kMostChosen = 32;

struct Route {
    int64_t tokens;
    int32_t experts, chosen, type, normalize;
    const void *logits;
    int64_t ld;
    float *weights;                     // written by the forward pass, read by the backward pass
    int32_t *choice, *position, *offsets;
    // backward
    const float *dweights;
    void *dlogits;
    int64_t ld_dlogits;
};

int64_t route_scratch_bytes(int64_t tokens, int experts, int sms);
cudaError_t launch_route(const Route &r, void *scratch, int sms, const LaunchOptions &o, cudaStream_t stream);
cudaError_t launch_route_gradient(const Route &r, const LaunchOptions &o, cudaStream_t stream);

struct Move {
    int64_t tokens, rows, cols;
    int32_t type, chosen;
    void *token, *row, *drow;
    const void *residual;               // or null
    int64_t ld_token, ld_row, ld_drow, ld_residual;
    const int32_t *position;
    const float *weights;               // or null: all 1
    float *dweights;
};

cudaError_t launch_dispatch(const Move &m, const LaunchOptions &o, cudaStream_t stream);             // token -> row
cudaError_t launch_combine(const Move &m, const LaunchOptions &o, cudaStream_t stream);              // row -> token
cudaError_t launch_combine_gradient(const Move &m, const LaunchOptions &o, cudaStream_t stream);     // token, row -> drow, dweights

}  // namespace redist
