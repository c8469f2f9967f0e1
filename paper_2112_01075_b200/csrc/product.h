// Matrix product with a fused epilogue on the tensor cores: host interface.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

namespace redist {

enum Type { T_BF16 = 0, T_F16 = 1, T_F32 = 2 };
enum Activation { ACT_NONE = 0, ACT_RELU = 1, ACT_GELU = 2, ACT_SILU = 3 };

constexpr int64_t type_bytes(int t) { return t == T_F32 ? 4 : 2; }

// One operand of the product, 16-bit elements.  Rows are the index that survives (m of A, n of B), columns the
// index that is summed over.  along_rows = 0: element (r, c) at r * ld + c; 1: at c * ld + r.  The base address,
// ld and batch_stride (elements) must put every line on a 16-byte boundary (the TMA's rule).
struct Operand {
    const void *data;
    int64_t ld, batch_stride;
    int along_rows;
};

// How an accumulator becomes an output.  LINEAR: z = acc + bias[n]; pre = z; out = act(z) + residual.
// SCALED: v = alpha * acc + beta * (hi + lo / 2048), alpha and beta multiplied by powers of a device scalar
// per matrix; out = v as f16 (with out_lo = the rest, times 2048) or as bf16.  PARTIAL (inside launch_product only): the
// 32-bit accumulators of each part of a split sum, out[part][row][ld_out].
enum EpilogueKind { EPI_LINEAR = 0, EPI_SCALED = 1, EPI_PARTIAL = 2 };

struct Epilogue {
    void *out;
    int64_t ld_out, out_batch;
    // LINEAR
    const void *bias;
    const void *residual;
    int64_t ld_residual;
    void *pre;
    int64_t ld_pre;
    int32_t bias_type, activation;
    // SCALED
    const void *hi, *lo;
    void *out_lo;
    int64_t ld_add, add_batch;      // of hi, lo and out_lo
    const float *scale;             // scale[matrix], or null
    float alpha, beta;
    int32_t alpha_power, beta_power;// how often scale[matrix] multiplies alpha / beta
    int32_t out_type;
    // SCALED, centred: t = mean_scale * the sum of diagonal_n f16 elements, diagonal_step apart from diagonal + i *
    // diagonal_batch on (a sample of the diagonal of matrix i); c = t (center_1 + t center_2) where t is at least 1/4, else 0.
    // on_diagonal * c is subtracted from the result's diagonal, to_beta * c (scaled as beta is) added to beta.  Null: neither.
    const void *diagonal;
    int64_t diagonal_step, diagonal_batch;
    int32_t diagonal_n;
    float mean_scale, center_1, center_2, on_diagonal, to_beta;
};

struct Product {
    int64_t m, n, k;
    int32_t batch;
    int32_t type;                   // of both operands: T_BF16 or T_F16
    int32_t symmetric;              // the result is symmetric (m == n): tiles above the diagonal are mirrored, not computed
    int32_t kind;                   // EpilogueKind
    Operand a, b;
    Epilogue e;
};

// What a launch takes from the tuning values.
struct LaunchOptions {
    int32_t pdl;
    uint32_t wait_polls;
    uint32_t test_extra_tx;
    int32_t test_shape, test_parts;     // test only: 1 + the Shape, and the parts of a sum, that every product takes; 0: chosen
};

// Whether an operand may be read as it lies (16-byte boundaries), or has to be laid out anew first.
bool operand_fits(const void *data, int64_t ld, int64_t batch_stride, int batch);

// The current device and its number of SMs (asked for once per device).
cudaError_t current_device(int *device, int *sms);

// Scratch that launch_product needs with the same options: the 32-bit parts of a sum that is split (only sizes are read).
int64_t product_scratch_bytes(const Product &p, const LaunchOptions &o);

// Asynchronous on `stream`; allocates nothing.
cudaError_t launch_product(const Product &p, void *scratch, const LaunchOptions &o, cudaStream_t stream);

// The linear epilogue on up to kFewRows rows, both operands contiguous along the sum, at any alignment; no scratch.
constexpr int kFewRows = 32;
cudaError_t launch_few_rows(const Product &p, const LaunchOptions &o, cudaStream_t stream);

// Thread blocks of the product kernels whose bounded wait ran out on the current device.  Synchronizes the device.
cudaError_t read_product_timeouts(unsigned int *out);

}  // namespace redist
