// Matrix products grouped by expert: host interface.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

#include "product.h"

namespace redist {

// The rows of expert e are offsets[e] ... offsets[e + 1] - 1, known on the device only.
//
// ROWS: out[r] = act(b[r] a[e]^T + bias[e]) for the rows of each expert; a: a stack of `experts` operands of m rows, b: one
// operand of `rows` rows, sums of k.  SUMS: out[e] = (b's rows)^T (a's rows), sums over the rows of expert e; a and b: operands
// whose columns (the rows of the arrays, `rows` of them) are summed over, m and n features; out: a stack of n x m.
struct Grouped {
    int64_t rows, m, n, k;
    int32_t experts, type, sums;
    Operand a, b;
    const int32_t *offsets;
    void *out, *pre;                    // pre or null
    int64_t ld_out, out_batch, ld_pre;
    const void *bias;                   // or null
    int64_t bias_stride;
    int32_t bias_type, activation;
};

// Scratch of one launch: with `sums` a tensor map of both operands for every expert.
int64_t grouped_scratch_bytes(const Grouped &g);
cudaError_t launch_grouped(const Grouped &g, void *scratch, const LaunchOptions &o, cudaStream_t stream);

// ROWS for up to kFewRows rows, both operands contiguous along the sum, at any alignment (few.cu).
cudaError_t launch_few_grouped(const Grouped &g, const LaunchOptions &o, cudaStream_t stream);

// dz = dy times the activation's slope at z for the rows of the experts (dst or null: not kept), and the sums of an expert's
// rows (sums[e][col], or null), of the unrounded values in a fixed order.
struct ExpertSlope {
    int64_t rows, cols;
    int32_t experts, type, activation;
    const int32_t *offsets;
    const void *dy, *z;                 // z or null
    int64_t ld_dy, ld_z;
    void *dst;
    int64_t ld_dst;
    float *sums, *partials;             // partials: expert_partial_bytes
};
int64_t expert_partial_bytes(int64_t rows, int64_t cols, int experts);
cudaError_t launch_expert_slope(const ExpertSlope &s, const LaunchOptions &o, cudaStream_t stream);

// Thread blocks whose bounded wait ran out on the current device.  Synchronizes the device.
cudaError_t read_grouped_timeouts(unsigned int *out);

}  // namespace redist
