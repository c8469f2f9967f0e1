// Kernels that stream over matrices once: layer norm, and what has to be done to operands before a matrix product.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

#include "product.h"

namespace redist {

struct LayerNorm {
    int64_t rows, cols;
    int32_t type, weight_type;
    float eps;
    const void *x;
    int64_t ld_x;
    const void *gamma, *beta;           // of weight_type, or null
    float *mean, *rstd;                 // written by the forward pass, read by the backward pass
    void *y;
    int64_t ld_y;
    // backward
    const void *dy;
    int64_t ld_dy;
    void *dx;
    int64_t ld_dx;
    float *dgamma, *dbeta;              // either may be null
};

size_t layer_norm_backward_bytes(int64_t rows, int64_t cols, int type, int sms);
cudaError_t launch_layer_norm_forward(const LayerNorm &l, const LaunchOptions &o, cudaStream_t stream);
cudaError_t launch_layer_norm_backward(const LayerNorm &l, void *workspace, const LaunchOptions &o, cudaStream_t stream);

// dst (row-major, ld_dst a multiple of 8, 16-byte aligned) = src, or src times the activation's slope at z; 16-bit
// elements.  With `sums`, sums[c] = sum of column c of the unrounded product.  partials: column_partial_bytes.
struct Lay {
    int64_t rows, cols;
    int32_t type, activation;
    const void *src;
    int64_t ld_src;
    const void *z;                      // or null
    int64_t ld_z;
    void *dst;                          // or null: sums only
    int64_t ld_dst;
    float *sums;                        // or null
    float *partials;
};
size_t column_partial_bytes(int64_t rows, int64_t cols);
// Up to three of them in one launch (all of one type).
cudaError_t launch_lay(const Lay *l, int count, const LaunchOptions &o, cudaStream_t stream);

// The input of the orthogonalisation: |X|_F of every matrix, and X times a power of two that brings the norm to
// [2^13, 2^14), as f16 (hi) and, for 32-bit inputs, the rest times 2048 (lo).  scale[matrix] = 1 / (norm times that).
struct Scaled {
    int64_t rows, cols;
    int32_t batch, type;
    const void *x;
    int64_t ld_x, x_batch;
    void *hi, *lo;
    int64_t ld, plane;
    float *scale;
    double *partials;                   // batch * kNormParts
    double eps;
};
constexpr int kNormParts = 128;
cudaError_t launch_scaled(const Scaled &s, const LaunchOptions &o, cudaStream_t stream);

// The linear epilogue of product `p` on the sum of `splits` parts, parts[s][row][ld], added in this order.
cudaError_t launch_join(const Product &p, const float *parts, int64_t ld, int splits, const LaunchOptions &o, cudaStream_t stream);

}  // namespace redist
