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

// The sums of the experts' rows whose parts launch_prepare has left (see ExpertSlope): a product computes them in passing where
// it has blocks enough (returns whether it did).
struct ExpertSums {
    int64_t rows, cols, per;
    int32_t experts;
    const int32_t *offsets;
    const float *partials;
    float *sums;                        // null: none
};

// With `sums` scratch are the tensor maps that launch_prepare has made.
cudaError_t launch_grouped(const Grouped &g, void *scratch, ExpertSums *columns, const LaunchOptions &o, cudaStream_t stream);
cudaError_t launch_expert_sums(const ExpertSums &s, const LaunchOptions &o, cudaStream_t stream);

// ROWS for up to kFewRows rows, both operands contiguous along the sum, at any alignment (few.cu).
cudaError_t launch_few_grouped(const Grouped &g, const LaunchOptions &o, cudaStream_t stream);

// What has to be done before the products, in one launch.
//
// dz = dy times the activation's slope at z for the rows of the experts (dst or null: not kept), and with `partials` the sums of
// the unrounded values over stretches of an expert's rows.
struct ExpertSlope {
    int64_t rows, cols;
    int32_t experts, activation;
    const int32_t *offsets;
    const void *dy, *z;                 // dy null: nothing of this; z or null
    int64_t ld_dy, ld_z;
    void *dst;
    int64_t ld_dst;
    float *partials;                    // expert_partial_bytes
};

// `count` matrices of `lines` lines laid out anew on 16-byte boundaries (dst null: none); with offsets only those of experts that
// have rows.
struct StackLay {
    const void *src;
    void *dst;
    int64_t count, lines, line, ld_src, plane_src, ld_dst, plane_dst;
    const int32_t *offsets;             // or null
    int64_t rows;                       // of all experts
    int32_t by_row;                     // set by launch_prepare
};

struct Prepare {
    int32_t type;
    ExpertSlope slope;
    StackLay lay[2];
    const Grouped *sums;                // the product of sums whose maps are made, or null
    void *maps;                         // grouped_maps_bytes
};
int64_t grouped_maps_bytes(int experts);
int64_t expert_partial_bytes(int64_t rows, int64_t cols, int experts);
int64_t slope_rows(int64_t rows, int64_t cols);         // of a part
cudaError_t launch_prepare(const Prepare &p, const LaunchOptions &o, cudaStream_t stream);

// Thread blocks whose bounded wait ran out on the current device.  Synchronizes the device.
cudaError_t read_grouped_timeouts(unsigned int *out);

}  // namespace redist
