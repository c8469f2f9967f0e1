// The norm over many tensors, and the tensors scaled down to a bound on it.
//
// Two passes over the data, the second only where it changes something or goes elsewhere.  The tensors' addresses travel as
// arguments of the launch (nothing is copied to the device, so a call can be captured), up to 1000 of them.  The tensors are cut
// into units of 32 KB; every block takes a stretch of units, adds their squares and leaves a partial sum in 64 bits; the
// blocks of the second pass all add all partial sums, in the same order, so that no block waits for another, and go through
// their stretch backwards: what the first pass read last is still in L2.
#include "clip.h"

#include <algorithm>
#include <cstring>

#include "elements.cuh"

namespace redist {

namespace {

constexpr int kThreads = 256, kPieces = 8, kUnit = kThreads * kPieces * 16, kBlocksPerSm = 3;

template <int MOST> struct ClipTable {
    const void *data[MOST];
    void *out[MOST];
    int64_t elements[MOST];
    int32_t begin[MOST + 1];            // its first unit
    uint8_t type[MOST];
    int32_t count;
    // the second pass
    int32_t partials;
    const double *sums;
    float *norm;
    float max_norm, eps;
};

template <typename T> __device__ __forceinline__ void values(const uint4 &u, float (&v)[16 / sizeof(T)])
{
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            v[i] = __uint_as_float(w[i]);
        } else {
            const float2 f = unpack2<T>(w[i]);
            v[2 * i] = f.x;
            v[2 * i + 1] = f.y;
        }
    }
}

// A unit's share of a thread: the 16-byte blocks number at, at + kThreads, ... of the tensor (counted from the block in
// which it begins), cleared where they reach beyond it.
template <typename T> struct Share {
    static constexpr int N = 16 / int(sizeof(T));
    const char *base;                   // the block in which the tensor begins
    int64_t head, end;                  // its first element and the one behind its last, counted from there
    int64_t at;
    __device__ __forceinline__ Share(const void *data, int64_t elements, int64_t unit)
    {
        const uintptr_t p = reinterpret_cast<uintptr_t>(data);
        base = reinterpret_cast<const char *>(p & ~uintptr_t(15));
        head = int64_t(p & 15) / int64_t(sizeof(T));
        end = head + elements;
        at = unit * (kUnit / 16) + threadIdx.x;
    }
    __device__ __forceinline__ int64_t block(int j) const { return at + j * kThreads; }
    __device__ __forceinline__ bool some(int j) const { return block(j) * N < end; }
    __device__ __forceinline__ bool whole(int j) const { return block(j) * N >= head && block(j) * N + N <= end; }
    __device__ __forceinline__ void load(uint4 (&u)[kPieces]) const
    {
#pragma unroll
        for (int j = 0; j < kPieces; ++j) u[j] = some(j) ? *(reinterpret_cast<const uint4 *>(base) + block(j)) : make_uint4(0, 0, 0, 0);
    }
};

// The sum of squares of a thread's share, in 32 bits where that loses nothing: neither an overflow nor squares that are
// flushed to zero next to a sum of their size.
template <typename T> __device__ __forceinline__ double squares(const Share<T> &s)
{
    constexpr int N = Share<T>::N;
    uint4 u[kPieces];
    s.load(u);
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
        if (!s.some(j)) continue;
        float v[N];
        values<T>(u[j], v);
        if (!s.whole(j)) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int64_t e = s.block(j) * N + i;
                if (e < s.head || e >= s.end) v[i] = 0.0f;
            }
            // (what stays is summed again below, from the same block)
        }
#pragma unroll
        for (int i = 0; i < N; ++i) sum = fmaf(v[i], v[i], sum);
    }
    if (sum <= 0x1p120f && sum >= 0x1p-80f) return double(sum);
    double wide = 0.0;
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
        if (!s.some(j) || (u[j].x | u[j].y | u[j].z | u[j].w) == 0) continue;
        float v[N];
        values<T>(u[j], v);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int64_t e = s.block(j) * N + i;
            if (e >= s.head && e < s.end) wide = fma(double(v[i]), double(v[i]), wide);
        }
    }
    return wide;
}

// Sums of a block in 64 bits, the same in all threads; `slot`: one entry per warp.
__device__ __forceinline__ double block_sum(double v, double *slot)
{
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    if ((threadIdx.x & 31) == 0) slot[threadIdx.x >> 5] = v;
    __syncthreads();
    double all = 0.0;
#pragma unroll
    for (int i = 0; i < kThreads / 32; ++i) all += slot[i];
    return all;
}

template <int MOST> __device__ __forceinline__ int tensor_of(const ClipTable<MOST> &c, int unit)
{
    int lo = 0, hi = c.count - 1;       // the last tensor that begins at or before the unit (empty ones begin where the next does)
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (c.begin[mid] <= unit) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

template <int MOST> __global__ void __launch_bounds__(kThreads, kBlocksPerSm) redist_squares_kernel(const __grid_constant__ ClipTable<MOST> c, double *sums)
{
    __shared__ double slot[kThreads / 32];
    let_next_start();
    wait_for_previous();
    const int units = c.begin[c.count];
    double sum = 0.0;
    for (int u = blockIdx.x; u < units; u += gridDim.x) {
        const int i = tensor_of(c, u);
        const int64_t unit = u - c.begin[i];
        if (c.type[i] == T_BF16) sum += squares(Share<__nv_bfloat16>(c.data[i], c.elements[i], unit));
        else if (c.type[i] == T_F16) sum += squares(Share<__half>(c.data[i], c.elements[i], unit));
        else sum += squares(Share<float>(c.data[i], c.elements[i], unit));
    }
    sum = block_sum(sum, slot);
    if (threadIdx.x == 0) sums[blockIdx.x] = sum;
}

template <typename T, typename F> __device__ __forceinline__ void scale(const void *data, void *out, int64_t elements, int64_t unit, F factor)
{
    constexpr int N = Share<T>::N;
    const Share<T> s(data, elements, unit);
    uint4 u[kPieces];
    s.load(u);
    T *to = static_cast<T *>(out) - s.head;
    const bool aligned = reinterpret_cast<uintptr_t>(to) % 16 == 0;
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
        if (!s.some(j)) continue;
        float v[N];
        values<T>(u[j], v);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = float(F(v[i]) * factor);
        const int64_t first = s.block(j) * N;
        if (aligned && s.whole(j)) {
            uint4 w;
            if constexpr (sizeof(T) == 4)
                w = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
            else
                w = make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
            *reinterpret_cast<uint4 *>(to + first) = w;
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (first + i >= s.head && first + i < s.end) to[first + i] = from_float<T>(v[i]);
        }
    }
}

template <int MOST, typename F> __device__ __forceinline__ void scale_all(const ClipTable<MOST> &c, F factor)
{
    for (int u = c.begin[c.count] - 1 - int(blockIdx.x); u >= 0; u -= gridDim.x) {
        const int i = tensor_of(c, u);
        if (factor == F(1) && c.out[i] == c.data[i]) continue;
        const int64_t unit = u - c.begin[i];
        if (c.type[i] == T_BF16) scale<__nv_bfloat16>(c.data[i], c.out[i], c.elements[i], unit, factor);
        else if (c.type[i] == T_F16) scale<__half>(c.data[i], c.out[i], c.elements[i], unit, factor);
        else scale<float>(c.data[i], c.out[i], c.elements[i], unit, factor);
    }
}

template <int MOST> __global__ void __launch_bounds__(kThreads, kBlocksPerSm) redist_clip_kernel(const __grid_constant__ ClipTable<MOST> c)
{
    __shared__ double slot[kThreads / 32];
    let_next_start();
    wait_for_previous();
    double sum = 0.0;
    for (int i = threadIdx.x; i < c.partials; i += kThreads) sum += c.sums[i];
    const double exact = sqrt(block_sum(sum, slot));
    const float norm = float(exact);
    if (c.norm && blockIdx.x == 0 && threadIdx.x == 0) *c.norm = norm;
    if (c.max_norm < 0.0f) return;
    float factor = c.max_norm / (norm + c.eps);
    if (!(factor >= 0x1p-100f) && exact <= 0x1p1000) {
        // a finite norm that 32 bits do not hold, or a quotient for which they have a few bits or none
        const double quotient = double(c.max_norm) / (exact + double(c.eps));
        if (quotient > 0.0 && quotient < 0x1p-100) return scale_all(c, quotient);
        factor = float(quotient);
    }
    if (factor > 1.0f) factor = 1.0f;                       // (a NaN stays)
    scale_all(c, factor);
}

// ---- host --------------------------------------------------------------------------------------------------

constexpr int kMostTensors = 1000;      // 32 bytes each; a launch takes 32764 bytes of arguments

int64_t units_of(const ClipTensor &t)
{
    if (t.elements == 0) return 0;
    const int64_t bytes = int64_t(uintptr_t(t.data) & 15) + t.elements * type_bytes(t.type);
    return (bytes + kUnit - 1) / kUnit;
}

// The tensors of one launch, from `at` on: how many there are, and how many units they have.
void portion(const ClipTensor *tensors, int64_t count, int64_t at, int64_t &n, int64_t &units)
{
    n = units = 0;
    for (; at + n < count && n < kMostTensors; ++n) {
        const int64_t u = units_of(tensors[at + n]);
        if (n > 0 && units + u > INT32_MAX / 2) return;
        units += u;
    }
}

int64_t blocks_for(int64_t units, int sms) { return std::max<int64_t>(1, std::min<int64_t>(units, int64_t(sms) * kBlocksPerSm)); }

template <typename... P, typename... A>
cudaError_t launch(void (*kernel)(P...), int64_t grid, const LaunchOptions &o, cudaStream_t stream, const A &...args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(grid));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = stream;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = o.pdl ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

struct Pass {
    float max_norm, eps;
    float *norm;
    double *sums;
    int64_t partials;                   // of all launches; 0: the first pass
};

template <int MOST>
cudaError_t launch_portion(const ClipTensor *tensors, int64_t n, const Pass &p, int64_t blocks, double *sums, const LaunchOptions &o, cudaStream_t stream)
{
    ClipTable<MOST> c;
    static_assert(sizeof(c) <= 32764 - 16, "arguments of a launch");
    std::memset(&c, 0, sizeof c);
    int64_t units = 0;
    for (int64_t i = 0; i < n; ++i) {
        c.data[i] = tensors[i].data;
        c.out[i] = tensors[i].out;
        c.elements[i] = tensors[i].elements;
        c.type[i] = uint8_t(tensors[i].type);
        c.begin[i] = int32_t(units);
        units += units_of(tensors[i]);
    }
    for (int64_t i = n; i <= MOST; ++i) c.begin[i] = int32_t(units);
    c.count = int32_t(n);
    if (p.partials == 0) return launch(redist_squares_kernel<MOST>, blocks, o, stream, c, sums);
    c.partials = int32_t(p.partials);
    c.sums = p.sums;
    c.norm = p.norm;
    c.max_norm = p.max_norm;
    c.eps = p.eps;
    return launch(redist_clip_kernel<MOST>, blocks, o, stream, c);
}

cudaError_t launch_any(const ClipTensor *tensors, int64_t n, const Pass &p, int64_t blocks, double *sums, const LaunchOptions &o, cudaStream_t stream)
{
    // (a few of them: fewer arguments to bring over)
    if (n <= 32) return launch_portion<32>(tensors, n, p, blocks, sums, o, stream);
    if (n <= 256) return launch_portion<256>(tensors, n, p, blocks, sums, o, stream);
    return launch_portion<kMostTensors>(tensors, n, p, blocks, sums, o, stream);
}

}  // namespace

int64_t clip_partials(const ClipTensor *tensors, int64_t count, int sms)
{
    int64_t all = 0, n = 0, units = 0;
    for (int64_t at = 0; at < count || at == 0; at += std::max<int64_t>(n, 1)) {
        portion(tensors, count, at, n, units);
        all += blocks_for(units, sms);
    }
    return all;
}

cudaError_t launch_clip(const ClipTensor *tensors, int64_t count, float max_norm, float eps, float *norm, double *partials, int sms,
                        const LaunchOptions &o, cudaStream_t stream)
{
    int64_t n = 0, units = 0, sums = 0;
    Pass p = {max_norm, eps, norm, partials, 0};
    for (int64_t at = 0; at < count || at == 0; at += std::max<int64_t>(n, 1)) {
        portion(tensors, count, at, n, units);
        if (units > INT32_MAX / 2) return cudaErrorInvalidValue;
        const int64_t blocks = blocks_for(units, sms);
        const cudaError_t ce = launch_any(tensors + at, n, p, blocks, partials + sums, o, stream);
        if (ce != cudaSuccess) return ce;
        sums += blocks;
    }
    p.partials = sums;
    for (int64_t at = 0; at < count || at == 0; at += std::max<int64_t>(n, 1)) {
        portion(tensors, count, at, n, units);
        if (max_norm < 0.0f) n = units = 0;                 // nothing is scaled: one block writes the norm
        const cudaError_t ce = launch_any(tensors + at, n, p, blocks_for(units, sms), nullptr, o, stream);
        if (ce != cudaSuccess || max_norm < 0.0f) return ce;
        p.norm = nullptr;                                   // written once
    }
    return cudaSuccess;
}

}  // namespace redist
