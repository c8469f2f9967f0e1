// The linear layer for a few rows: y = act(x w^T + b) + r with 1 to 16 rows.
//
// The time is that of reading w once, so nothing is staged: every lane loads 16 bytes (8 neighbours along the sum) of
// two rows of w at a time straight into the fragments of mma.m16n8k16 -- w's rows are the fragment's m, x's rows its n.
// The order of a sum is free, so the eight neighbours serve as columns (2t, 2t+1, 2t+8, 2t+9) of two products, and x is
// read in the same order.  The eight warps of a block take turns along the sum (256 bytes of every row each), and where w has few rows a cluster of blocks
// splits it further; the parts meet in (distributed) shared memory and are added in a fixed order.  One launch, no
// tensor memory, no tensor maps: what those take to set up is more than the small calls need altogether.
#include "product.h"

#include <algorithm>
#include <atomic>

#include "activation.cuh"
#include "elements.cuh"

namespace redist {

namespace {

constexpr int kWarps = 8, kUnroll = 4, kMostCluster = 8;

struct Few {
    int64_t n, k;               // rows of w, length of the sum
    int32_t rows;               // of x
    const void *x, *w;
    int64_t ld_x, ld_w;
    int64_t k_per_block;        // a multiple of 32
    Epilogue e;
};

template <typename T> __device__ __forceinline__ void mma16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma16<__nv_bfloat16>(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma16<__half>(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Eight neighbours of a row, zero beyond its end; w is read once and does not displace x in L1.
template <bool ALIGNED, bool STREAM, typename T> __device__ __forceinline__ uint4 eight(const T *row, int64_t at, int64_t end)
{
    const int64_t left = end - at;
    if (left <= 0) return make_uint4(0, 0, 0, 0);
    uint4 v;
    if (ALIGNED) {              // k is a multiple of 8: all eight or none
        if (STREAM)
            asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(row + at));
        else
            v = __ldg(reinterpret_cast<const uint4 *>(row + at));
        return v;
    }
    v = load16_any(row + at, int(left < 8 ? left : 8) * 2);
    if (left < 8) {
        uint32_t *w = &v.x;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (2 * i >= left) w[i] = 0;
            else if (2 * i + 1 >= left) w[i] &= 0xffffu;
        }
    }
    return v;
}

__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

__device__ __forceinline__ uint32_t cluster_size()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(r));
    return r;
}

// MT * 16 rows of w per block, NT * 8 rows of x.
template <typename T, int MT, int NT, bool ALIGNED>
__global__ void __launch_bounds__(32 * kWarps) redist_few_rows_kernel(const Few f)
{
    constexpr int kOut = MT * 16 * NT * 8;
    __shared__ float parts[kWarps][kOut];
    __shared__ float total[kOut];
    let_next_start();
    wait_for_previous();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const uint32_t splits = cluster_size(), rank = cluster_rank();
    const int64_t n0 = int64_t(blockIdx.x / splits) * MT * 16;
    const int64_t lo = int64_t(rank) * f.k_per_block, hi = min(f.k, lo + f.k_per_block);
    const T *x = static_cast<const T *>(f.x), *w = static_cast<const T *>(f.w);
    float acc[MT][NT][4] = {};
    for (int64_t at = lo + warp * 32 * kUnroll; at < hi; at += 32 * kUnroll * kWarps) {
        uint4 a[kUnroll][MT][2], b[kUnroll][NT];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int64_t c = at + u * 32 + t * 8;
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int64_t row = n0 + i * 16 + h * 8 + g;
                    a[u][i][h] = eight<ALIGNED, true>(w + row * f.ld_w, row < f.n ? c : hi, hi);
                }
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const int row = j * 8 + g;
                b[u][j] = eight<ALIGNED, false>(x + int64_t(row) * f.ld_x, row < f.rows ? c : hi, hi);
            }
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    mma16<T>(acc[i][j], a[u][i][0].x, a[u][i][1].x, a[u][i][0].y, a[u][i][1].y, b[u][j].x, b[u][j].y);
                    mma16<T>(acc[i][j], a[u][i][0].z, a[u][i][1].z, a[u][i][0].w, a[u][i][1].w, b[u][j].z, b[u][j].w);
                }
    }
    // parts[warp][row of x][row of w]
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) parts[warp][(j * 8 + 2 * t + (q & 1)) * MT * 16 + i * 16 + g + (q >> 1) * 8] = acc[i][j][q];
    __syncthreads();
    for (int o = threadIdx.x; o < kOut; o += 32 * kWarps) {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < kWarps; ++i) s += parts[i][o];
        total[o] = s;
    }
    if (splits > 1) {
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    } else {
        __syncthreads();
    }
    // each block of the cluster finishes its share of the outputs
    const Epilogue &e = f.e;
    for (int o = int(rank) * 32 * kWarps + threadIdx.x; o < kOut; o += int(splits) * 32 * kWarps) {
        const int row = o / (MT * 16);
        const int64_t col = n0 + o % (MT * 16);
        float v[8] = {};
        if (splits > 1) {
            const uint32_t here = uint32_t(__cvta_generic_to_shared(&total[o]));
            for (uint32_t s = 0; s < splits; ++s) {
                uint32_t there;
                float part;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(here), "r"(s));
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(part) : "r"(there) : "memory");
                v[0] += part;
            }
        } else {
            v[0] = total[o];
        }
        if (row >= f.rows || col >= f.n) continue;
        if (e.bias) v[0] += load_any(e.bias, e.bias_type, col);
        if (e.pre) static_cast<T *>(e.pre)[row * e.ld_pre + col] = from_float<T>(v[0]);
        activate8(v, e.activation);
        if (e.residual) v[0] += to_float(static_cast<const T *>(e.residual)[row * e.ld_residual + col]);
        static_cast<T *>(e.out)[row * e.ld_out + col] = from_float<T>(v[0]);
    }
    if (splits > 1) {                                     // the others read this block's shared memory
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
}

template <typename T, int MT, int NT, bool ALIGNED>
cudaError_t launch(Few f, int sms, const LaunchOptions &o, cudaStream_t stream)
{
    const int64_t groups = (f.n + MT * 16 - 1) / (MT * 16);
    // Blocks for two per SM, as long as a warp keeps 128 steps of the sum.
    int64_t splits = 1;
    while (splits < kMostCluster && groups * splits < 2 * sms && f.k >= splits * 2 * kWarps * 128) splits *= 2;
    f.k_per_block = (f.k + splits * 32 - 1) / (splits * 32) * 32;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(groups * splits));
    cfg.blockDim = dim3(32 * kWarps);
    cfg.stream = stream;
    cudaLaunchAttribute at[2];
    int n_at = 0;
    if (splits > 1) {
        at[n_at].id = cudaLaunchAttributeClusterDimension;
        at[n_at].val.clusterDim.x = unsigned(splits);
        at[n_at].val.clusterDim.y = 1;
        at[n_at].val.clusterDim.z = 1;
        ++n_at;
    }
    if (o.pdl) {
        at[n_at].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at[n_at].val.programmaticStreamSerializationAllowed = 1;
        ++n_at;
    }
    cfg.attrs = at;
    cfg.numAttrs = unsigned(n_at);
    return cudaLaunchKernelEx(&cfg, redist_few_rows_kernel<T, MT, NT, ALIGNED>, f);
}

template <typename T, bool ALIGNED> cudaError_t launch_rows(const Few &f, int sms, const LaunchOptions &o, cudaStream_t stream)
{
    if (f.rows <= 8) return launch<T, 1, 1, ALIGNED>(f, sms, o, stream);
    return launch<T, 1, 2, ALIGNED>(f, sms, o, stream);
}

}  // namespace

cudaError_t launch_few_rows(const Product &p, const LaunchOptions &o, cudaStream_t stream)
{
    int device = 0, sms = 0;
    const cudaError_t ce = current_device(&device, &sms);
    if (ce != cudaSuccess) return ce;
    Few f = {};
    f.n = p.n;
    f.k = p.k;
    f.rows = int32_t(p.m);
    f.x = p.a.data;
    f.w = p.b.data;
    f.ld_x = p.a.ld;
    f.ld_w = p.b.ld;
    f.e = p.e;
    const bool aligned = p.k % 8 == 0 && operand_fits(f.x, f.ld_x, 0, 1) && operand_fits(f.w, f.ld_w, 0, 1);
    if (p.type == T_BF16) return aligned ? launch_rows<__nv_bfloat16, true>(f, sms, o, stream) : launch_rows<__nv_bfloat16, false>(f, sms, o, stream);
    return aligned ? launch_rows<__half, true>(f, sms, o, stream) : launch_rows<__half, false>(f, sms, o, stream);
}

}  // namespace redist
