// Layer norm and the preparation of operands: kernels bound by the memory they stream over.
#include "rows.h"

#include <algorithm>

#include "activation.cuh"
#include "elements.cuh"

namespace redist {

namespace {

// ---- helpers -----------------------------------------------------------------------------------------

// VEC neighbours of a row as they lie in memory.
template <typename T, int VEC> struct Raw {
    uint4 u;
    __device__ __forceinline__ void load(const T *p) { u = __ldg(reinterpret_cast<const uint4 *>(p)); }
    __device__ __forceinline__ void clear() { u = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void get(float (&v)[VEC]) const
    {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(w[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 f = unpack2<T>(w[i]);
                v[2 * i] = f.x;
                v[2 * i + 1] = f.y;
            }
        }
    }
    static __device__ __forceinline__ void put(T *p, const float (&v)[VEC], int count)
    {
        if (count >= VEC) {
            uint4 u;
            if constexpr (sizeof(T) == 4)
                u = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
            else
                u = make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
            *reinterpret_cast<uint4 *>(p) = u;
        } else {
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (i < count) p[i] = from_float<T>(v[i]);
        }
    }
};
template <typename T> struct Raw<T, 1> {
    T u;
    __device__ __forceinline__ void load(const T *p) { u = __ldg(p); }
    __device__ __forceinline__ void clear() { u = from_float<T>(0.0f); }
    __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = to_float(u); }
    static __device__ __forceinline__ void put(T *p, const float (&v)[1], int) { *p = from_float<T>(v[0]); }
};

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}

// Sum over the W warps that share a row; every thread gets it.  W > 1: the whole block calls it, `slot` alternates.
template <int W> __device__ __forceinline__ float row_sum(float v, float *slot)
{
    v = warp_sum(v);
    if constexpr (W > 1) {
        if ((threadIdx.x & 31) == 0) slot[threadIdx.x >> 5] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int i = 0; i < W; ++i) v += slot[i];
    }
    return v;
}

// The same for two sums at once.
template <int W> __device__ __forceinline__ float2 row_sum2(float a, float b, float2 *slot)
{
    a = warp_sum(a);
    b = warp_sum(b);
    if constexpr (W > 1) {
        if ((threadIdx.x & 31) == 0) slot[threadIdx.x >> 5] = make_float2(a, b);
        __syncthreads();
        a = b = 0.0f;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            a += slot[i].x;
            b += slot[i].y;
        }
    }
    return make_float2(a, b);
}

// ---- layer norm, forward -------------------------------------------------------------------------------

constexpr int kNormWarps = 8;           // warps of a block whose rows belong to one warp each

// W warps hold a row in registers, NV pieces of VEC neighbours per lane.  Mean first, then the differences d from it,
// sum of d^2 and sum of d: the latter is what rounding left in the mean, and corrects both (var = mean d^2 - (mean d)^2),
// so a mean far larger than the spread costs no digits.
template <typename T, int VEC, int W, int NV>
__global__ void __launch_bounds__(W == 1 ? 32 * kNormWarps : 32 * W) redist_layer_norm_kernel(const LayerNorm l)
{
    constexpr int kRows = W == 1 ? kNormWarps : 1;
    __shared__ float slots[32];
    __shared__ float2 slots2[32];
    const int t = W == 1 ? threadIdx.x & 31 : threadIdx.x;
    const int group = W == 1 ? threadIdx.x >> 5 : 0;
    let_next_start();
    wait_for_previous();
    float gamma[NV][VEC], beta[NV][VEC];
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const int64_t c = int64_t(j * W * 32 + t) * VEC + i;
            gamma[j][i] = l.gamma && c < l.cols ? load_any(l.gamma, l.weight_type, c) : 1.0f;
            beta[j][i] = l.beta && c < l.cols ? load_any(l.beta, l.weight_type, c) : 0.0f;
        }
    const float over = 1.0f / float(l.cols);
    const int64_t step = int64_t(gridDim.x) * kRows;
    Raw<T, VEC> next[NV];
    auto fetch = [&](int64_t row) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int64_t c = int64_t(j * W * 32 + t) * VEC;
            if (row < l.rows && c < l.cols) next[j].load(static_cast<const T *>(l.x) + row * l.ld_x + c);
            else next[j].clear();
        }
    };
    int64_t row = int64_t(blockIdx.x) * kRows + group;
    fetch(row);
    for (; row < l.rows; row += step) {
        float v[NV][VEC];
#pragma unroll
        for (int j = 0; j < NV; ++j) next[j].get(v[j]);
        fetch(row + step);
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const int64_t c = int64_t(j * W * 32 + t) * VEC + i;
                if (c < l.cols) sum += v[j][i];
            }
        float mean = row_sum<W>(sum, slots) * over;
        float rest = 0.0f, square = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const int64_t c = int64_t(j * W * 32 + t) * VEC + i;
                v[j][i] -= mean;
                if (c < l.cols) {
                    rest += v[j][i];
                    square = fmaf(v[j][i], v[j][i], square);
                }
            }
        const float2 both = row_sum2<W>(rest, square, slots2);
        rest = both.x * over;
        mean += rest;
        float var = both.y * over - rest * rest;
        if (var < 0.0f) var = 0.0f;                     // by rounding alone; NaN stays
        const float rstd = 1.0f / sqrtf(var + l.eps);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int64_t c = int64_t(j * W * 32 + t) * VEC;
            if (c >= l.cols) continue;
            float y[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) y[i] = fmaf((v[j][i] - rest) * rstd, gamma[j][i], beta[j][i]);
            Raw<T, VEC>::put(static_cast<T *>(l.y) + row * l.ld_y + c, y, int(min(l.cols - c, int64_t(VEC))));
        }
        if (t == 0) {
            if (l.mean) l.mean[row] = mean;
            if (l.rstd) l.rstd[row] = rstd;
        }
    }
}

// Rows that do not fit into the registers of a block: three passes over a row, which its first pass left in L2.
template <typename T>
__global__ void __launch_bounds__(1024) redist_layer_norm_long_kernel(const LayerNorm l)
{
    __shared__ float slots[32];
    __shared__ float2 slots2[32];
    let_next_start();
    wait_for_previous();
    const float over = 1.0f / float(l.cols);
    for (int64_t row = blockIdx.x; row < l.rows; row += gridDim.x) {
        const T *x = static_cast<const T *>(l.x) + row * l.ld_x;
        T *y = static_cast<T *>(l.y) + row * l.ld_y;
        float sum = 0.0f, rest = 0.0f, square = 0.0f;
        for (int64_t c = threadIdx.x; c < l.cols; c += 1024) sum += to_float(x[c]);
        float mean = row_sum<32>(sum, slots) * over;
        for (int64_t c = threadIdx.x; c < l.cols; c += 1024) {
            const float d = to_float(x[c]) - mean;
            rest += d;
            square = fmaf(d, d, square);
        }
        const float2 both = row_sum2<32>(rest, square, slots2);
        rest = both.x * over;
        float var = both.y * over - rest * rest;
        if (var < 0.0f) var = 0.0f;                     // by rounding alone; NaN stays
        const float rstd = 1.0f / sqrtf(var + l.eps);
        for (int64_t c = threadIdx.x; c < l.cols; c += 1024) {
            const float g = l.gamma ? load_any(l.gamma, l.weight_type, c) : 1.0f;
            const float b = l.beta ? load_any(l.beta, l.weight_type, c) : 0.0f;
            y[c] = from_float<T>(fmaf((to_float(x[c]) - mean - rest) * rstd, g, b));
        }
        if (threadIdx.x == 0) {
            if (l.mean) l.mean[row] = mean + rest;
            if (l.rstd) l.rstd[row] = rstd;
        }
    }
}

// ---- layer norm, backward ------------------------------------------------------------------------------

// With c = dy gamma and xh = (x - mean) rstd: dx = rstd (c - mean(c) - xh mean(c xh)).  A block walks over its rows
// and keeps the column sums of dy xh and dy in registers; partials holds them per block, gamma's before beta's.
template <typename T, int VEC, int W, int NV>
__global__ void __launch_bounds__(W == 1 ? 32 * kNormWarps : 32 * W) redist_layer_norm_grad_kernel(const LayerNorm l, float *partials)
{
    constexpr int kRows = W == 1 ? kNormWarps : 1;
    __shared__ float slots[2][32];
    const int t = W == 1 ? threadIdx.x & 31 : threadIdx.x;
    const int group = W == 1 ? threadIdx.x >> 5 : 0;
    let_next_start();
    wait_for_previous();
    float gamma[NV][VEC], dgamma[NV][VEC], dbeta[NV][VEC];
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const int64_t c = int64_t(j * W * 32 + t) * VEC + i;
            gamma[j][i] = l.gamma && c < l.cols ? load_any(l.gamma, l.weight_type, c) : 1.0f;
            dgamma[j][i] = dbeta[j][i] = 0.0f;
        }
    const float over = 1.0f / float(l.cols);
    const int64_t step = int64_t(gridDim.x) * kRows;
    Raw<T, VEC> next_x[NV], next_dy[NV];
    auto fetch = [&](int64_t row) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int64_t c = int64_t(j * W * 32 + t) * VEC;
            if (row < l.rows && c < l.cols) {
                next_x[j].load(static_cast<const T *>(l.x) + row * l.ld_x + c);
                next_dy[j].load(static_cast<const T *>(l.dy) + row * l.ld_dy + c);
            } else {
                next_x[j].clear();
                next_dy[j].clear();
            }
        }
    };
    int64_t row = int64_t(blockIdx.x) * kRows + group;
    fetch(row);
    int turn = 0;
    for (; row < l.rows; row += step, turn ^= 1) {
        const float mean = l.mean[row], rstd = l.rstd[row];
        float xh[NV][VEC], c1[NV][VEC];
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            next_x[j].get(xh[j]);
            next_dy[j].get(c1[j]);
        }
        fetch(row + step);
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const int64_t c = int64_t(j * W * 32 + t) * VEC + i;
                const bool in = VEC == 1 || c < l.cols;     // VEC == 1: what lies outside was fetched as zero
                const float dy = in ? c1[j][i] : 0.0f;
                const float h = c < l.cols ? (xh[j][i] - mean) * rstd : 0.0f;
                dgamma[j][i] = fmaf(dy, h, dgamma[j][i]);
                dbeta[j][i] += dy;
                c1[j][i] = dy * gamma[j][i];
                xh[j][i] = h;
                s1 += c1[j][i];
                s2 = fmaf(c1[j][i], h, s2);
            }
        s1 = warp_sum(s1);
        s2 = warp_sum(s2);
        if constexpr (W > 1) {
            if ((threadIdx.x & 31) == 0) {
                slots[turn][2 * (threadIdx.x >> 5) % 32] = s1;
                slots[turn][(2 * (threadIdx.x >> 5) + 1) % 32] = s2;
            }
            __syncthreads();
            s1 = s2 = 0.0f;
#pragma unroll
            for (int i = 0; i < W; ++i) {
                s1 += slots[turn][2 * i];
                s2 += slots[turn][2 * i + 1];
            }
        }
        s1 *= over;
        s2 *= over;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int64_t c = int64_t(j * W * 32 + t) * VEC;
            if (c >= l.cols) continue;
            float d[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) d[i] = (c1[j][i] - s1 - xh[j][i] * s2) * rstd;
            Raw<T, VEC>::put(static_cast<T *>(l.dx) + row * l.ld_dx + c, d, int(min(l.cols - c, int64_t(VEC))));
        }
    }
    if (!partials) return;
    float *out = partials + int64_t(blockIdx.x) * 2 * l.cols;
    if constexpr (W == 1) {
        // the block's eight warps hold sums of the same columns
        __shared__ float all[kNormWarps][32 * VEC];
#pragma unroll
        for (int which = 0; which < 2; ++which)
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                __syncthreads();
#pragma unroll
                for (int i = 0; i < VEC; ++i) all[group][t * VEC + i] = which ? dbeta[j][i] : dgamma[j][i];
                __syncthreads();
                for (int q = threadIdx.x; q < 32 * VEC; q += 32 * kNormWarps) {
                    float s = 0.0f;
#pragma unroll
                    for (int w = 0; w < kNormWarps; ++w) s += all[w][q];
                    const int64_t c = int64_t(j) * 32 * VEC + q;
                    if (c < l.cols) out[which * l.cols + c] = s;
                }
            }
    } else {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const int64_t c = int64_t(j * W * 32 + t) * VEC + i;
                if (c < l.cols) {
                    out[c] = dgamma[j][i];
                    out[l.cols + c] = dbeta[j][i];
                }
            }
    }
}

// Long rows: dx alone, with a second pass over a row that the first left in L2 ...
template <typename T>
__global__ void __launch_bounds__(1024) redist_layer_norm_grad_long_kernel(const LayerNorm l)
{
    __shared__ float slots[2][32];
    let_next_start();
    wait_for_previous();
    const float over = 1.0f / float(l.cols);
    for (int64_t row = blockIdx.x; row < l.rows; row += gridDim.x) {
        const T *x = static_cast<const T *>(l.x) + row * l.ld_x, *dy = static_cast<const T *>(l.dy) + row * l.ld_dy;
        T *dx = static_cast<T *>(l.dx) + row * l.ld_dx;
        const float mean = l.mean[row], rstd = l.rstd[row];
        float s1 = 0.0f, s2 = 0.0f;
        for (int64_t c = threadIdx.x; c < l.cols; c += 1024) {
            const float g = to_float(dy[c]) * (l.gamma ? load_any(l.gamma, l.weight_type, c) : 1.0f);
            s1 += g;
            s2 = fmaf(g, (to_float(x[c]) - mean) * rstd, s2);
        }
        s1 = row_sum<32>(s1, slots[0]) * over;
        s2 = row_sum<32>(s2, slots[1]) * over;
        for (int64_t c = threadIdx.x; c < l.cols; c += 1024) {
            const float g = to_float(dy[c]) * (l.gamma ? load_any(l.gamma, l.weight_type, c) : 1.0f);
            dx[c] = from_float<T>((g - s1 - (to_float(x[c]) - mean) * rstd * s2) * rstd);
        }
        __syncthreads();
    }
}

// ... and the column sums on their own: a thread per column, a slice of the rows per block row.
template <typename T>
__global__ void __launch_bounds__(256) redist_layer_norm_columns_kernel(const LayerNorm l, float *partials)
{
    let_next_start();
    wait_for_previous();
    const int64_t c = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (c >= l.cols) return;
    const int64_t per = (l.rows + gridDim.y - 1) / gridDim.y, lo = per * blockIdx.y, hi = min(l.rows, lo + per);
    float g = 0.0f, b = 0.0f;
    for (int64_t row = lo; row < hi; ++row) {
        const float dy = to_float(static_cast<const T *>(l.dy)[row * l.ld_dy + c]);
        const float x = to_float(static_cast<const T *>(l.x)[row * l.ld_x + c]);
        g = fmaf(dy, (x - l.mean[row]) * l.rstd[row], g);
        b += dy;
    }
    float *out = partials + int64_t(blockIdx.y) * 2 * l.cols;
    out[c] = g;
    out[l.cols + c] = b;
}

// out[c] = sum over the parts of partials[part][c], in the same order every time.
__global__ void __launch_bounds__(256) redist_column_sum_kernel(const float *partials, int parts, int64_t stride, int64_t cols,
                                                               float *first, float *second)
{
    __shared__ float all[8][33];
    let_next_start();
    wait_for_previous();
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int64_t c = int64_t(blockIdx.x) * 32 + lane;
    const float *p = partials + (blockIdx.y ? cols : 0);
    float *out = blockIdx.y ? second : first;
    float s = 0.0f;
    if (out && c < cols)
        for (int q = w; q < parts; q += 8) s += p[q * stride + c];
    all[w][lane] = s;
    __syncthreads();
    if (w == 0 && out && c < cols) {
        s = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s += all[i][lane];
        out[c] = s;
    }
}

// ---- operands of a product -------------------------------------------------------------------------------

__device__ __forceinline__ float slope(float z, int act)
{
    if (act == ACT_RELU) return z > 0.0f ? 1.0f : 0.0f;
    if (act == ACT_GELU)
        return 0.5f * (1.0f + erff(z * 0.70710678118654752f)) + z * __expf(-0.5f * z * z) * 0.39894228040143268f;
    if (act == ACT_SILU) {
        const float s = 1.0f / (1.0f + __expf(-z));
        return s * (1.0f + z * (1.0f - s));
    }
    return 1.0f;
}

constexpr int kLayCols = 256;

// Rows of a block: 64, or more where the grid would grow beyond its limit.
int64_t lay_rows(int64_t rows) { return 64 * ((rows + 64 * 32768 - 1) / (64 * 32768)); }

template <typename T> __device__ __forceinline__ void split8(const uint4 &u, float (&v)[8])
{
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = unpack2<T>(w[i]);
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}

// A block takes rows_per_block rows by 256 columns, a warp every eighth row, a lane eight neighbours.
template <typename T>
__global__ void __launch_bounds__(256) redist_lay_kernel(const Lay l, int64_t rows_per_block)
{
    __shared__ float all[8][kLayCols];
    let_next_start();
    wait_for_previous();
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int64_t c = int64_t(blockIdx.x) * kLayCols + lane * 8;
    const int count = int(min(l.cols - c, int64_t(8)));
    float sums[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    const int64_t lo = int64_t(blockIdx.y) * rows_per_block, hi = min(l.rows, lo + rows_per_block);
    if (count > 0)
#pragma unroll 4
        for (int64_t row = lo + w; row < hi; row += 8) {
            uint4 u = load16_any(static_cast<const T *>(l.src) + row * l.ld_src + c, count * 2);
            if (l.z || l.sums) {
                float v[8];
                split8<T>(u, v);
                if (l.z) {
                    float z[8];
                    split8<T>(load16_any(static_cast<const T *>(l.z) + row * l.ld_z + c, count * 2), z);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] *= slope(z[i], l.activation);
                    u = make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) sums[i] += v[i];
            }
            if (l.dst) *reinterpret_cast<uint4 *>(static_cast<T *>(l.dst) + row * l.ld_dst + c) = u;
        }
    if (!l.sums) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) all[w][lane * 8 + i] = sums[i];
    __syncthreads();
    const int64_t cc = int64_t(blockIdx.x) * kLayCols + threadIdx.x;
    if (cc < l.cols) {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s += all[i][threadIdx.x];
        l.partials[int64_t(blockIdx.y) * l.cols + cc] = s;
    }
}

// ---- the input of the orthogonalisation --------------------------------------------------------------------

template <typename T> struct Eight {     // eight neighbours at any alignment; what is not wanted reads as zero
    static __device__ __forceinline__ void load(const T *p, int count, float (&v)[8])
    {
        if constexpr (sizeof(T) == 2) {
            split8<T>(load16_any(p, count * 2), v);
        } else {
            const uint4 a = load16_any(p, min(count, 4) * 4);
            uint4 b = make_uint4(0, 0, 0, 0);
            if (count > 4) b = load16_any(p + 4, (count - 4) * 4);
            const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < count ? v[i] : 0.0f;
    }
};

__device__ __forceinline__ double block_sum(double v, double *slots)
{
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) slots[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.0;
    for (int i = 0; i < int(blockDim.x) / 32; ++i) v += slots[i];
    return v;
}

// Squares are summed in 64 bits: their range (2^-298 to 2^256) does not fit into 32, and the kernel stays bound by memory.
template <typename T>
__global__ void __launch_bounds__(256) redist_norm_parts_kernel(const Scaled s)
{
    __shared__ double slots[8];
    let_next_start();
    wait_for_previous();
    const T *x = static_cast<const T *>(s.x) + int64_t(blockIdx.y) * s.x_batch;
    const int64_t per_row = (s.cols + 7) / 8, all = s.rows * per_row, step = int64_t(gridDim.x) * 256;
    double sum = 0.0;
    for (int64_t q = int64_t(blockIdx.x) * 256 + threadIdx.x; q < all; q += step) {
        const int64_t row = q / per_row, c = (q - row * per_row) * 8;
        float v[8];
        Eight<T>::load(x + row * s.ld_x + c, int(min(s.cols - c, int64_t(8))), v);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = fma(double(v[i]), double(v[i]), sum);
    }
    sum = block_sum(sum, slots);
    if (threadIdx.x == 0) s.partials[int64_t(blockIdx.y) * kNormParts + blockIdx.x] = sum;
}

template <typename T>
__global__ void __launch_bounds__(256) redist_scaled_kernel(const Scaled s, int parts)
{
    __shared__ double slots[8];
    let_next_start();
    wait_for_previous();
    const double norm = sqrt(block_sum(threadIdx.x < parts ? s.partials[int64_t(blockIdx.y) * kNormParts + threadIdx.x] : 0.0, slots)) + s.eps;
    int exponent = 0;
    const double fraction = frexp(norm, &exponent);                       // norm = fraction 2^exponent, fraction in [1/2, 1)
    const bool finite = norm - norm == 0.0;
    const float power = finite ? ldexpf(1.0f, 14 - exponent) : __int_as_float(0x7fffffff);
    if (blockIdx.x == 0 && threadIdx.x == 0) s.scale[blockIdx.y] = finite ? float(1.0 / ldexp(fraction, 14)) : 1.0f;
    const T *x = static_cast<const T *>(s.x) + int64_t(blockIdx.y) * s.x_batch;
    __half *hi = static_cast<__half *>(s.hi) + int64_t(blockIdx.y) * s.plane, *lo = s.lo ? static_cast<__half *>(s.lo) + int64_t(blockIdx.y) * s.plane : nullptr;
    const int64_t per_row = (s.cols + 7) / 8, all = s.rows * per_row, step = int64_t(gridDim.x) * 256;
    for (int64_t q = int64_t(blockIdx.x) * 256 + threadIdx.x; q < all; q += step) {
        const int64_t row = q / per_row, c = (q - row * per_row) * 8;
        float v[8], h[8];
        Eight<T>::load(x + row * s.ld_x + c, int(min(s.cols - c, int64_t(8))), v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= power;
        const uint4 u = make_uint4(pack2<__half>(v[0], v[1]), pack2<__half>(v[2], v[3]), pack2<__half>(v[4], v[5]), pack2<__half>(v[6], v[7]));
        *reinterpret_cast<uint4 *>(hi + row * s.ld + c) = u;
        if (lo) {
            split8<__half>(u, h);
#pragma unroll
            for (int i = 0; i < 8; ++i) h[i] = (v[i] - h[i]) * 2048.0f;
            *reinterpret_cast<uint4 *>(lo + row * s.ld + c) =
                make_uint4(pack2<__half>(h[0], h[1]), pack2<__half>(h[2], h[3]), pack2<__half>(h[4], h[5]), pack2<__half>(h[6], h[7]));
        }
    }
}

// ---- joining the parts of a split product --------------------------------------------------------------------

// A thread takes eight neighbours of a row.
template <typename T>
__global__ void __launch_bounds__(256) redist_join_kernel(const Epilogue e, const float *parts, int64_t ld, int splits, int64_t m, int64_t n)
{
    let_next_start();
    wait_for_previous();
    const int64_t per_row = ld / 8, q = int64_t(blockIdx.x) * 256 + threadIdx.x;
    const int64_t row = q / per_row, c = (q - row * per_row) * 8;
    if (row >= m || c >= n) return;
    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll 4
    for (int s = 0; s < splits; ++s) {
        const float4 *at = reinterpret_cast<const float4 *>(parts + (int64_t(s) * m + row) * ld + c);
        const float4 a = at[0], b = at[1];
        v[0] += a.x;
        v[1] += a.y;
        v[2] += a.z;
        v[3] += a.w;
        v[4] += b.x;
        v[5] += b.y;
        v[6] += b.z;
        v[7] += b.w;
    }
    const int count = int(min(n - c, int64_t(8)));
    auto put = [&](void *base, int64_t pitch) {
        T *to = static_cast<T *>(base) + row * pitch + c;
        if (count == 8 && (reinterpret_cast<uintptr_t>(to) & 15) == 0) {
            *reinterpret_cast<uint4 *>(to) = make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < count) to[i] = from_float<T>(v[i]);
        }
    };
    if (e.bias)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count) v[i] += load_any(e.bias, e.bias_type, c + i);
    if (e.pre) put(e.pre, e.ld_pre);
    activate8(v, e.activation);
    if (e.residual) {
        float w[8];
        split8<T>(load16_any(static_cast<const T *>(e.residual) + row * e.ld_residual + c, count * 2), w);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += w[i];
    }
    put(e.out, e.ld_out);
}

// ---- host ---------------------------------------------------------------------------------------------------

template <typename... P, typename... A>
cudaError_t launch(void (*kernel)(P...), dim3 grid, int block, const LaunchOptions &o, cudaStream_t stream, A... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(unsigned(block));
    cfg.stream = stream;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = o.pdl ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}

cudaError_t sm_count(int *sms)
{
    int device = 0;
    return current_device(&device, sms);
}

bool on_16(const void *p, int64_t ld, int64_t element) { return p == nullptr || (uintptr_t(p) % 16 == 0 && ld * element % 16 == 0); }

template <typename T, int VEC> cudaError_t forward_as(const LayerNorm &l, int sms, const LaunchOptions &o, cudaStream_t stream)
{
    const int64_t pieces = (l.cols + VEC - 1) / VEC;
    auto grid = [&](int rows_per_block, int blocks_per_sm) {
        return dim3(unsigned(std::min<int64_t>((l.rows + rows_per_block - 1) / rows_per_block, int64_t(sms) * blocks_per_sm)));
    };
    if (pieces <= 32) return launch(redist_layer_norm_kernel<T, VEC, 1, 1>, grid(kNormWarps, 8), 32 * kNormWarps, o, stream, l);
    if (pieces <= 64) return launch(redist_layer_norm_kernel<T, VEC, 1, 2>, grid(kNormWarps, 6), 32 * kNormWarps, o, stream, l);
    if (pieces <= 256) return launch(redist_layer_norm_kernel<T, VEC, 8, 1>, grid(1, 8), 256, o, stream, l);
    if (pieces <= 512) return launch(redist_layer_norm_kernel<T, VEC, 8, 2>, grid(1, 6), 256, o, stream, l);
    if (pieces <= 1024) return launch(redist_layer_norm_kernel<T, VEC, 16, 2>, grid(1, 3), 512, o, stream, l);
    if (pieces <= 2048) return launch(redist_layer_norm_kernel<T, VEC, 32, 2>, grid(1, 1), 1024, o, stream, l);
    return launch(redist_layer_norm_long_kernel<T>, grid(1, 2), 1024, o, stream, l);
}

// Parts of the column sums and, through `run`, the launches of the backward pass: one place that knows both.
constexpr int kGradPerSm = 2, kLongParts = 64;

template <typename T, int VEC>
cudaError_t backward_as(const LayerNorm &l, float *partials, int sms, const LaunchOptions &o, cudaStream_t stream)
{
    const int64_t pieces = (l.cols + VEC - 1) / VEC;
    auto grid = [&](int rows_per_block, int blocks_per_sm) {
        return int(std::min<int64_t>((l.rows + rows_per_block - 1) / rows_per_block, int64_t(sms) * blocks_per_sm));
    };
    int parts = 0;
    cudaError_t ce;
    if (pieces <= 32) ce = launch(redist_layer_norm_grad_kernel<T, VEC, 1, 1>, dim3(parts = grid(kNormWarps, 2)), 32 * kNormWarps, o, stream, l, partials);
    else if (pieces <= 64) ce = launch(redist_layer_norm_grad_kernel<T, VEC, 1, 2>, dim3(parts = grid(kNormWarps, 2)), 32 * kNormWarps, o, stream, l, partials);
    else if (pieces <= 256) ce = launch(redist_layer_norm_grad_kernel<T, VEC, 8, 1>, dim3(parts = grid(1, 2)), 256, o, stream, l, partials);
    else if (pieces <= 512) ce = launch(redist_layer_norm_grad_kernel<T, VEC, 8, 2>, dim3(parts = grid(1, 2)), 256, o, stream, l, partials);
    else if (pieces <= 1024) ce = launch(redist_layer_norm_grad_kernel<T, VEC, 16, 2>, dim3(parts = grid(1, 1)), 512, o, stream, l, partials);
    else {
        ce = launch(redist_layer_norm_grad_long_kernel<T>, dim3(grid(1, 2)), 1024, o, stream, l);
        if (ce != cudaSuccess || !partials) return ce;
        parts = int(std::min<int64_t>(l.rows, kLongParts));
        ce = launch(redist_layer_norm_columns_kernel<T>, dim3(unsigned((l.cols + 255) / 256), unsigned(parts)), 256, o, stream, l, partials);
    }
    if (ce != cudaSuccess || !partials) return ce;
    return launch(redist_column_sum_kernel, dim3(unsigned((l.cols + 31) / 32), 2), 256, o, stream, static_cast<const float *>(partials), parts,
                  int64_t(2) * l.cols, l.cols, l.dgamma, l.dbeta);
}

template <typename F> cudaError_t by_type(int type, F f)
{
    if (type == T_BF16) return f(__nv_bfloat16());
    if (type == T_F16) return f(__half());
    return f(float());
}

}  // namespace

size_t layer_norm_backward_bytes(int64_t rows, int64_t cols, int, int sms)
{
    const int64_t parts = std::min<int64_t>(rows, std::max(int64_t(sms) * kGradPerSm, int64_t(kLongParts)));
    return size_t(parts * 2 * cols * 4);
}

cudaError_t launch_layer_norm_forward(const LayerNorm &l, const LaunchOptions &o, cudaStream_t stream)
{
    int sms = 0;
    cudaError_t ce = sm_count(&sms);
    if (ce != cudaSuccess || l.rows == 0) return ce;
    return by_type(l.type, [&](auto t) {
        using T = decltype(t);
        constexpr int VEC = 16 / sizeof(T);
        if (on_16(l.x, l.ld_x, sizeof(T)) && on_16(l.y, l.ld_y, sizeof(T))) return forward_as<T, VEC>(l, sms, o, stream);
        return forward_as<T, 1>(l, sms, o, stream);
    });
}

cudaError_t launch_layer_norm_backward(const LayerNorm &l, void *workspace, const LaunchOptions &o, cudaStream_t stream)
{
    int sms = 0;
    cudaError_t ce = sm_count(&sms);
    if (ce != cudaSuccess) return ce;
    if (l.rows == 0) {
        if (l.dgamma) ce = cudaMemsetAsync(l.dgamma, 0, size_t(l.cols) * 4, stream);
        if (ce == cudaSuccess && l.dbeta) ce = cudaMemsetAsync(l.dbeta, 0, size_t(l.cols) * 4, stream);
        return ce;
    }
    float *partials = l.dgamma || l.dbeta ? static_cast<float *>(workspace) : nullptr;
    return by_type(l.type, [&](auto t) {
        using T = decltype(t);
        constexpr int VEC = 16 / sizeof(T);
        if (on_16(l.x, l.ld_x, sizeof(T)) && on_16(l.dy, l.ld_dy, sizeof(T)) && on_16(l.dx, l.ld_dx, sizeof(T)))
            return backward_as<T, VEC>(l, partials, sms, o, stream);
        return backward_as<T, 1>(l, partials, sms, o, stream);
    });
}

size_t column_partial_bytes(int64_t rows, int64_t cols)
{
    return rows > 0 ? size_t((rows + lay_rows(rows) - 1) / lay_rows(rows) * cols * 4) : 0;
}

cudaError_t launch_lay(const Lay &l, const LaunchOptions &o, cudaStream_t stream)
{
    if (l.rows == 0) return l.sums ? cudaMemsetAsync(l.sums, 0, size_t(l.cols) * 4, stream) : cudaSuccess;
    const int64_t per = lay_rows(l.rows), parts = (l.rows + per - 1) / per;
    const dim3 grid(unsigned((l.cols + kLayCols - 1) / kLayCols), unsigned(parts));
    cudaError_t ce = l.type == T_BF16 ? launch(redist_lay_kernel<__nv_bfloat16>, grid, 256, o, stream, l, per)
                                      : launch(redist_lay_kernel<__half>, grid, 256, o, stream, l, per);
    if (ce != cudaSuccess || !l.sums) return ce;
    return launch(redist_column_sum_kernel, dim3(unsigned((l.cols + 31) / 32), 1), 256, o, stream, static_cast<const float *>(l.partials),
                  int(parts), l.cols, l.cols, l.sums, static_cast<float *>(nullptr));
}

cudaError_t launch_join(const Product &p, const float *parts, int64_t ld, int splits, const LaunchOptions &o, cudaStream_t stream)
{
    const dim3 grid(unsigned((p.m * (ld / 8) + 255) / 256));
    return p.type == T_BF16 ? launch(redist_join_kernel<__nv_bfloat16>, grid, 256, o, stream, p.e, parts, ld, splits, p.m, p.n)
                            : launch(redist_join_kernel<__half>, grid, 256, o, stream, p.e, parts, ld, splits, p.m, p.n);
}

cudaError_t launch_scaled(const Scaled &s, const LaunchOptions &o, cudaStream_t stream)
{
    const int64_t pieces = s.rows * ((s.cols + 7) / 8);
    const int parts = int(std::min<int64_t>(kNormParts, (pieces + 1023) / 1024));
    const int blocks = int(std::min<int64_t>(1024, (pieces + 511) / 512));
    return by_type(s.type, [&](auto t) {
        using T = decltype(t);
        cudaError_t ce = launch(redist_norm_parts_kernel<T>, dim3(unsigned(parts), unsigned(s.batch)), 256, o, stream, s);
        if (ce != cudaSuccess) return ce;
        return launch(redist_scaled_kernel<T>, dim3(unsigned(blocks), unsigned(s.batch)), 256, o, stream, s, parts);
    });
}

}  // namespace redist
