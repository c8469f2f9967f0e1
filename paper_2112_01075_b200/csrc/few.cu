// The linear layer for a few rows: y = act(x w^T + b) + r with 1 to 32 rows.
//
// The time is that of reading w once, so nothing is staged: every lane loads 32 bytes (16 neighbours along the sum) of
// two rows of w at a time straight into the fragments of mma.m16n8k16 -- w's rows are the fragment's m, x's rows its n.
// The order of a sum is free, so eight neighbours serve as columns (2t, 2t+1, 2t+8, 2t+9) of two products, and x is
// read in the same order.  Four lanes so read 128 bytes of a row with one instruction; with 16 bytes a lane the memory
// gave a sixth less (1 x 4096 -> 16384: 27.4 against 23.9 us with the same weight again, part of which L2 keeps; 16 rows
// 25.7).  With nothing in L2 that takes 26 us (134 MB take 20.5 at the measured copy rate), 1 x 4096 -> 4096 8.6 (5.1), of
// which two are the launch.  Latency of memory bounds it: what counts is the number of loads under way, thus few
// registers (four blocks per SM) and x fetched only while w is.  The eight warps of a block take turns along the sum (up to
// 256 bytes of every row each), and where w has few rows a cluster of blocks splits it further; the parts meet in
// (distributed) shared memory and are added in a fixed order.  One launch, no tensor memory, no tensor maps: what those
// take to set up is more than the small calls need altogether.
#include "product.h"

#include <algorithm>
#include <atomic>

#include "activation.cuh"
#include "elements.cuh"
#include "experts.h"

namespace redist {

namespace {

constexpr int kWarps = 8, kStep = 128, kMostCluster = 8;     // kStep: steps of the sum per turn of a warp (at most)

struct Few {
    int64_t n, k;               // rows of w, length of the sum
    int32_t rows;               // of x
    const void *x, *w;
    int64_t ld_x, ld_w;
    int64_t k_per_block;        // a multiple of 64
    Epilogue e;
    // rows by expert
    const int32_t *offsets;
    int32_t experts, by_row;
    int64_t w_batch, bias_stride;
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

// 16 neighbours of a row in two blocks, zero beyond its end.  ALIGN 32: rows start on 32-byte boundaries and their length
// is a multiple of 16 elements; 16: 16 bytes and 8 elements; 0: any.  STREAM: read once, not kept in L1.  Plain loads
// (ld.global.nc is for what nobody writes while a kernel runs, and the kernel before, which may have written x and w, is
// still running when this one has begun to wait for it).
template <int ALIGN, bool STREAM, typename T> __device__ __forceinline__ void sixteen(const T *row, int64_t at, int64_t end, uint4 &u, uint4 &v)
{
    u = v = make_uint4(0, 0, 0, 0);
    const int64_t left = end - at;
    if (left <= 0) return;
    if constexpr (ALIGN == 32 && STREAM) {
        asm volatile("ld.global.L1::no_allocate.v8.u32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w), "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(row + at));
    } else if constexpr (ALIGN == 32) {
        // (kept where it stands: loads of x that the compiler moved up together spilled, 16 x 4096 -> 16384 41 us for 37)
        asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "l"(row + at));
        asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(row + at + 8));
    } else if constexpr (ALIGN == 16) {
        u = *reinterpret_cast<const uint4 *>(row + at);
        if (left > 8) v = *(reinterpret_cast<const uint4 *>(row + at) + 1);
    } else {
        const int n = int(left < 16 ? left : 16);
        u = load16_any(row + at, min(n, 8) * 2);
        if (n > 8) v = load16_any(row + at + 8, (n - 8) * 2);
        if (n < 16) {
            uint32_t w[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (2 * i >= n) w[i] = 0;
                else if (2 * i + 1 >= n) w[i] &= 0xffffu;
            }
            u = make_uint4(w[0], w[1], w[2], w[3]);
            v = make_uint4(w[4], w[5], w[6], w[7]);
        }
    }
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

// An expert and its rows, of `rows`: expert `y` itself, or (by row: fewer rows than experts) the one whose first row is y; no rows
// where there is none.  Offsets that decrease count as the largest before them.
__device__ __forceinline__ int range_of(const int32_t *offsets, int experts, bool by_row, int y, int rows, int &lo, int &hi)
{
    const int lane = int(threadIdx.x) & 31;
    int e = y, most = 0;
    if (by_row) {
        uint32_t next = uint32_t(experts) + 1;              // the first offset beyond row y: where its expert ends
        for (int i = lane; i <= experts && next > uint32_t(experts); i += 32)
            if (offsets[i] > y) next = uint32_t(i);
        e = int(__reduce_min_sync(0xffffffffu, next)) - 1;
    }
    lo = hi = 0;
    if (e < 0 || e >= experts) return 0;
    for (int i = lane; i <= e; i += 32) most = max(most, offsets[i]);
    lo = min(__reduce_max_sync(0xffffffffu, most), rows);
    hi = max(lo, min(offsets[e + 1], rows));
    if (by_row && lo != y) lo = hi;
    return e;
}

// MT * 16 rows of w per block, NT * 8 rows of x at a time.  GROUPED: a weight (and bias) for each range of rows of x; the
// second dimension of the grid are the experts, or the rows.
template <typename T, int MT, int NT, int ALIGN, bool GROUPED>
__global__ void __launch_bounds__(32 * kWarps, NT > 2 || ALIGN == 0 ? 3 : 4) redist_few_rows_kernel(Few f)
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
    int from = 0, to = f.rows, expert = 0;
    if constexpr (GROUPED) {
        expert = range_of(f.offsets, f.experts, f.by_row, blockIdx.y, f.rows, from, to);
        if (from == to) return;                             // all blocks of a cluster
    }
#pragma unroll 1
    do {
        const int rows = GROUPED ? min(to - from, NT * 8) : f.rows;
        const T *x = static_cast<const T *>(f.x) + (GROUPED ? from * f.ld_x : 0), *w = static_cast<const T *>(f.w) + (GROUPED ? expert * f.w_batch : 0);
        float acc[MT][NT][4] = {};
        constexpr int kPairs = 2, kTurn = kPairs * 64;
#pragma unroll 1
        for (int64_t at = lo + warp * kTurn; at < hi; at += kTurn * kWarps) {
            uint4 a[kPairs][MT][2][2];
#pragma unroll
            for (int u = 0; u < kPairs; ++u) {
                const int64_t c = at + u * 64 + t * 16;
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int64_t row = n0 + i * 16 + h * 8 + g;
                        sixteen<ALIGN, true>(w + row * f.ld_w, row < f.n ? c : hi, hi, a[u][i][h][0], a[u][i][h][1]);
                    }
            }
            // x is in L1 or L2: it is fetched while w is under way, and does not take registers from that
#pragma unroll
            for (int u = 0; u < kPairs; ++u)
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    const int64_t c = at + u * 64 + t * 16;
                    const int row = j * 8 + g;
                    uint4 b[2];
                    sixteen<ALIGN, false>(x + int64_t(row) * f.ld_x, row < rows ? c : hi, hi, b[0], b[1]);
#pragma unroll
                    for (int q = 0; q < 2; ++q)
#pragma unroll
                        for (int i = 0; i < MT; ++i) {
                            const uint4 &a0 = a[u][i][0][q], &a1 = a[u][i][1][q];
                            mma16<T>(acc[i][j], a0.x, a1.x, a0.y, a1.y, b[q].x, b[q].y);
                            mma16<T>(acc[i][j], a0.z, a1.z, a0.w, a1.w, b[q].z, b[q].w);
                        }
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
            if (row >= rows || col >= f.n) continue;
            if (e.bias) v[0] += load_any(e.bias, e.bias_type, (GROUPED ? expert * f.bias_stride : 0) + col);
            const int64_t at = GROUPED ? from + row : row;
            if (e.pre) static_cast<T *>(e.pre)[at * e.ld_pre + col] = from_float<T>(v[0]);
            activate8(v, e.activation);
            if (!GROUPED && e.residual) v[0] += to_float(static_cast<const T *>(e.residual)[at * e.ld_residual + col]);
            static_cast<T *>(e.out)[at * e.ld_out + col] = from_float<T>(v[0]);
        }
        if (splits > 1) {                                     // the others read this block's shared memory
            asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
            asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        } else if (GROUPED) {
            __syncthreads();
        }
        from += NT * 8;
    } while (GROUPED && from < to);
}

template <typename T, int MT, int NT, int ALIGN, bool GROUPED>
cudaError_t launch(Few f, int sms, const LaunchOptions &o, cudaStream_t stream)
{
    const int64_t groups = (f.n + MT * 16 - 1) / (MT * 16), busy = std::min(f.experts, f.rows);
    // Blocks for two per SM, as long as a warp keeps two turns of the sum.
    int64_t splits = 1;
    while (splits < kMostCluster && groups * busy * splits < 2 * sms && f.k >= splits * 2 * kWarps * kStep) splits *= 2;
    f.k_per_block = (f.k + splits * 64 - 1) / (splits * 64) * 64;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(groups * splits), unsigned(busy));
    f.by_row = f.rows < f.experts;
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
    return cudaLaunchKernelEx(&cfg, redist_few_rows_kernel<T, MT, NT, ALIGN, GROUPED>, f);
}

template <typename T, int ALIGN, bool GROUPED> cudaError_t launch_rows(const Few &f, int sms, const LaunchOptions &o, cudaStream_t stream)
{
    // (by expert: the experts' rows in turns of eight, unless they have more on average)
    if (f.rows <= (GROUPED ? 8 * f.experts : 8)) return launch<T, 1, 1, ALIGN, GROUPED>(f, sms, o, stream);
    if (f.rows <= 16) return launch<T, 1, 2, ALIGN, GROUPED>(f, sms, o, stream);
    return launch<T, 1, 4, ALIGN, GROUPED>(f, sms, o, stream);
}

template <typename T, bool GROUPED> cudaError_t launch_typed(const Few &f, int sms, const LaunchOptions &o, cudaStream_t stream)
{
    const int matrices = std::min(f.experts, 2);
    const bool on16 = f.k % 8 == 0 && operand_fits(f.x, f.ld_x, 0, 1) && operand_fits(f.w, f.ld_w, f.w_batch, matrices);
    if (on16 && f.k % 16 == 0 && uintptr_t(f.w) % 32 == 0 && f.ld_w % 16 == 0 && (matrices == 1 || f.w_batch % 16 == 0))
        return launch_rows<T, 32, GROUPED>(f, sms, o, stream);
    return on16 ? launch_rows<T, 16, GROUPED>(f, sms, o, stream) : launch_rows<T, 0, GROUPED>(f, sms, o, stream);
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
    f.experts = 1;
    return p.type == T_BF16 ? launch_typed<__nv_bfloat16, false>(f, sms, o, stream) : launch_typed<__half, false>(f, sms, o, stream);
}

cudaError_t launch_few_grouped(const Grouped &g, const LaunchOptions &o, cudaStream_t stream)
{
    int device = 0, sms = 0;
    const cudaError_t ce = current_device(&device, &sms);
    if (ce != cudaSuccess) return ce;
    Few f = {};
    f.n = g.m;
    f.k = g.k;
    f.rows = int32_t(g.rows);
    f.x = g.b.data;
    f.w = g.a.data;
    f.ld_x = g.b.ld;
    f.ld_w = g.a.ld;
    f.w_batch = g.a.batch_stride;
    f.offsets = g.offsets;
    f.experts = g.experts;
    f.bias_stride = g.bias_stride;
    f.e.out = g.out;
    f.e.ld_out = g.ld_out;
    f.e.pre = g.pre;
    f.e.ld_pre = g.ld_pre;
    f.e.bias = g.bias;
    f.e.bias_type = g.bias_type;
    f.e.activation = g.activation;
    return g.type == T_BF16 ? launch_typed<__nv_bfloat16, true>(f, sms, o, stream) : launch_typed<__half, true>(f, sms, o, stream);
}

}  // namespace redist
