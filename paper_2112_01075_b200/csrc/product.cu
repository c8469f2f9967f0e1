// D = epilogue(A B^T): 16-bit operands, 32-bit accumulation on the tensor cores (tcgen05).
//
// One thread block (CG = 1) or a pair of them on two SMs (CG = 2) owns a tile of 128 CG x BN outputs at a time and
// walks over the sum in steps of 64: one thread brings the 128-byte wide slices of both operands into a ring of
// shared-memory stages by TMA (128-byte swizzle), one thread issues the tcgen05.mma that consume them, and four
// warps turn the finished accumulator of the previous tile into outputs while the next one runs: tensor memory holds
// two accumulators of BN columns.  Operands may be contiguous along the sum or along their rows (the gradients need
// both): only the boxes and the shared-memory descriptors differ.  Ragged sizes cost nothing extra: the TMA fills
// what lies outside an operand with zeros, and the epilogue stores what lies inside the result.
//
// Every wait on an mbarrier is bounded.  A role whose wait runs out leaves its loop, so the others' waits run out too;
// the block waits (bounded) for its own copies in flight, counts itself in g_product_timeouts, frees its tensor
// memory and returns without storing the tile.
#include "product.h"

#include <cuda.h>

#include <atomic>
#include <cstring>

#include "elements.cuh"

namespace redist {

namespace {

constexpr int kBK = 64;                 // elements of the sum per stage: 128 bytes, one swizzle row
constexpr int kThreads = 256;           // warp 0 loads, warp 1 multiplies, warp 2 owns tensor memory, warps 4-7 store
constexpr int kRing = 196608;           // bytes of the ring of stages
constexpr int kPitch = 36;              // words per row of a warp's 32 x 32 transpose buffer: 16-byte accesses of
                                        // eight lanes, by rows or by row groups, fall into distinct banks
constexpr int kEpiBytes = 4 * 32 * kPitch * 4;
constexpr int kBarBytes = 256;
constexpr int kSmem = 1024 + kRing + kEpiBytes + kBarBytes;
constexpr int kMaxStages = 12;

__device__ unsigned int g_product_timeouts = 0;

struct ProductParams {
    int32_t m, n, k_blocks, batch;
    int32_t tiles_m, tiles_n, tiles_per_matrix, tiles;
    int32_t symmetric, a_along_rows, b_along_rows;
    uint32_t idesc, wait_polls, test_extra_tx;
    int32_t vector_out;                 // every row of out (and residual, pre) starts on a 16-byte boundary
    Epilogue e;
};

// ---- shared memory, barriers, tensor memory -----------------------------------------------------

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return uint32_t(__cvta_generic_to_shared(p)); }

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}

__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, uint32_t polls)
{
    for (uint32_t i = 0; i < polls; ++i) {
        uint32_t done;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.b32 %0, 1, 0, p;\n\t}"
            : "=r"(done) : "r"(bar), "r"(parity) : "memory");
        if (done) return true;
    }
    return false;
}

__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}

__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

// The address, in the cluster's shared-memory window, of what lies at `addr` in the block of rank 0.
__device__ __forceinline__ uint32_t in_first(uint32_t addr)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
    return r;
}

__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// One box of an operand; `bar` is this block's own barrier (CG = 1) or the first block's (CG = 2).
template <int CG>
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap *map, uint32_t bar, int x, int y, int z)
{
    if constexpr (CG == 1)
        asm volatile(
            "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
            ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
            ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}

// Shared-memory descriptor of a 128-byte-swizzled operand slice.  Contiguous along the sum: eight rows of 128 bytes
// form a group, groups follow each other every 1024 bytes.  Contiguous along the rows: 64 rows x 8 sum steps form a
// group of 1024 bytes, the next eight steps follow at 1024 bytes, the next 64 rows after the whole box of 64 steps.
__device__ __forceinline__ uint64_t slice_desc(uint32_t addr, int along_rows)
{
    const uint64_t lead = along_rows ? (kBK * 128) >> 4 : 1, stride = 1024 >> 4;
    return uint64_t((addr & 0x3ffff) >> 4) | (lead << 16) | (stride << 32) | (uint64_t(1) << 46) | (uint64_t(2) << 61);
}

template <int CG>
__device__ __forceinline__ void mma(uint32_t acc, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add)
{
    if constexpr (CG == 1)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
            ::"r"(acc), "l"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
            ::"r"(acc), "l"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
}

// Arrive on `bar` (of both blocks, at the same place, for CG = 2) when all products issued so far are done.
template <int CG>
__device__ __forceinline__ void commit(uint32_t bar)
{
    if constexpr (CG == 1)
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
    else
        asm volatile(
            "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
            ::"r"(bar), "h"(uint16_t(3)) : "memory");
}

template <int CG> __device__ __forceinline__ void tmem_alloc(uint32_t where, uint32_t columns)
{
    if constexpr (CG == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(where), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    } else {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(where), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
}

template <int CG> __device__ __forceinline__ void tmem_free(uint32_t base, uint32_t columns)
{
    if constexpr (CG == 1)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns) : "memory");
    else
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns) : "memory");
}

__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 32 columns of this warp's 32 lanes of tensor memory: register j = column j of lane `lane`.
__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t (&v)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
          "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]),
          "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]),
          "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(addr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

// ---- tiles ---------------------------------------------------------------------------------------

struct Tile {
    int tm, tn, matrix;
};

// Tiles of a matrix in groups of eight tile rows, column after column within a group, so that the blocks at work at
// one time share slices of both operands in L2.  Symmetric: the lower triangle, row after row.
__device__ __forceinline__ Tile tile_at(const ProductParams &p, int t)
{
    Tile r;
    r.matrix = t / p.tiles_per_matrix;
    int q = t - r.matrix * p.tiles_per_matrix;
    if (p.symmetric) {
        int i = int((sqrtf(8.0f * float(q) + 1.0f) - 1.0f) * 0.5f);
        while (i * (i + 1) / 2 > q) --i;
        while ((i + 1) * (i + 2) / 2 <= q) ++i;
        r.tm = i;
        r.tn = q - i * (i + 1) / 2;
    } else {
        const int per_group = 8 * p.tiles_n, group = q / per_group;
        const int rows = min(8, p.tiles_m - group * 8);
        q -= group * per_group;
        r.tm = group * 8 + q % rows;
        r.tn = q / rows;
    }
    return r;
}

// ---- epilogue --------------------------------------------------------------------------------------

__device__ __forceinline__ float activate(float z, int act)
{
    if (act == ACT_RELU) return z < 0.0f ? 0.0f : z;                     // NaN stays
    if (act == ACT_GELU) return 0.5f * z * (1.0f + erff(z * 0.70710678118654752f));
    if (act == ACT_SILU) return __fdividef(z, 1.0f + __expf(-z));
    return z;
}

// `count` (1 to 8) neighbouring elements, from 16 bytes of packed ones.
__device__ __forceinline__ void store_some(void *p, const uint4 &v, int count)
{
    if (count >= 8) {
        *static_cast<uint4 *>(p) = v;
        return;
    }
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 7; ++i)
        if (i < count) static_cast<uint16_t *>(p)[i] = uint16_t(w[i >> 1] >> (16 * (i & 1)));
}

template <typename T> __device__ __forceinline__ uint4 pack8(const float (&v)[8])
{
    return make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
}

template <typename T> __device__ __forceinline__ void unpack8(const uint4 &u, float (&v)[8])
{
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = unpack2<T>(w[i]);
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}

// One 32 x 32 piece of the linear epilogue.  `buf` holds the accumulators, row by row; (row0, col0) is its place.
template <typename T>
__device__ __forceinline__ void linear_piece(const ProductParams &p, float *buf, int lane, int row0, int col0)
{
    const Epilogue &e = p.e;
    if (p.vector_out) {
        const int c = col0 + (lane & 3) * 8, count = p.n - c;
        if (count <= 0) return;
        float bias[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) bias[i] = e.bias && i < count ? load_any(e.bias, e.bias_type, c + i) : 0.0f;
#pragma unroll
        for (int it = 0; it < 4; ++it) {
            const int r = it * 8 + (lane >> 2), row = row0 + r;
            if (row >= p.m) break;
            const float4 *s = reinterpret_cast<const float4 *>(buf + r * kPitch + (lane & 3) * 8);
            const float4 x = s[0], y = s[1];
            float v[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += bias[i];
            if (e.pre) store_some(static_cast<T *>(e.pre) + int64_t(row) * e.ld_pre + c, pack8<T>(v), count);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = activate(v[i], e.activation);
            if (e.residual) {
                const T *q = static_cast<const T *>(e.residual) + int64_t(row) * e.ld_residual + c;
                float w[8];
                if (count >= 8) {
                    unpack8<T>(*reinterpret_cast<const uint4 *>(q), w);      // may be the output itself
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[i] = i < count ? to_float(q[i]) : 0.0f;
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] += w[i];
            }
            store_some(static_cast<T *>(e.out) + int64_t(row) * e.ld_out + c, pack8<T>(v), count);
        }
    } else {
        const int c = col0 + lane;
        if (c >= p.n) return;
        const float bias = e.bias ? load_any(e.bias, e.bias_type, c) : 0.0f;
        for (int r = 0; r < 32 && row0 + r < p.m; ++r) {
            const int64_t row = row0 + r;
            float v = buf[r * kPitch + lane] + bias;
            if (e.pre) static_cast<T *>(e.pre)[row * e.ld_pre + c] = from_float<T>(v);
            v = activate(v, e.activation);
            if (e.residual) v += to_float(static_cast<const T *>(e.residual)[row * e.ld_residual + c]);
            static_cast<T *>(e.out)[row * e.ld_out + c] = from_float<T>(v);
        }
    }
}

// One piece of the scaled epilogue.  hi, lo and f16 outputs lie in workspaces whose rows start on 16-byte boundaries
// and are padded to whole 16 bytes; only a bf16 output may be ragged.  f16 results leave their values in `buf`, from
// where a mirrored tile is stored along its columns.
__device__ __forceinline__ void scaled_piece(const ProductParams &p, float *buf, int lane, int row0, int col0, int matrix,
                                             float alpha, float beta, bool mirror)
{
    const Epilogue &e = p.e;
    const int c = col0 + (lane & 3) * 8, count = p.n - c;
    if (count > 0) {
#pragma unroll
        for (int it = 0; it < 4; ++it) {
            const int r = it * 8 + (lane >> 2), row = row0 + r;
            if (row >= p.m) break;
            float4 *s = reinterpret_cast<float4 *>(buf + r * kPitch + (lane & 3) * 8);
            const float4 x = s[0], y = s[1];
            float v[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= alpha;
            const int64_t at = int64_t(matrix) * e.add_batch + int64_t(row) * e.ld_add + c;
            if (e.hi) {
                float w[8];
                unpack8<__half>(*reinterpret_cast<const uint4 *>(static_cast<const __half *>(e.hi) + at), w);
                if (e.lo) {
                    float u[8];
                    unpack8<__half>(*reinterpret_cast<const uint4 *>(static_cast<const __half *>(e.lo) + at), u);
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[i] = fmaf(u[i], 1.0f / 2048.0f, w[i]);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = fmaf(beta, w[i], v[i]);
            }
            const int64_t to = int64_t(matrix) * e.out_batch + int64_t(row) * e.ld_out + c;
            if (e.out_type == T_BF16) {
                __nv_bfloat16 *q = static_cast<__nv_bfloat16 *>(e.out) + to;
                if (p.vector_out) {
                    store_some(q, pack8<__nv_bfloat16>(v), count);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (i < count) q[i] = __float2bfloat16_rn(v[i]);
                }
            } else {
                const uint4 h = pack8<__half>(v);
                *reinterpret_cast<uint4 *>(static_cast<__half *>(e.out) + to) = h;
                if (e.out_lo) {
                    float w[8];
                    unpack8<__half>(h, w);
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[i] = (v[i] - w[i]) * 2048.0f;
                    *reinterpret_cast<uint4 *>(static_cast<__half *>(e.out_lo) + at) = pack8<__half>(w);
                }
                if (mirror) {
                    s[0] = make_float4(v[0], v[1], v[2], v[3]);
                    s[1] = make_float4(v[4], v[5], v[6], v[7]);
                }
            }
        }
    }
    if (!mirror) return;
    __syncwarp();
    if (col0 + lane < p.n) {
        __half *q = static_cast<__half *>(e.out) + int64_t(matrix) * e.out_batch + int64_t(col0 + lane) * e.ld_out + row0;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            if (row0 + g * 8 >= p.m) break;
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = buf[(g * 8 + i) * kPitch + lane];
            *reinterpret_cast<uint4 *>(q + g * 8) = pack8<__half>(v);
        }
    }
}

// ---- the kernel ------------------------------------------------------------------------------------

template <int CG, int BN, int KIND>
__global__ void __launch_bounds__(kThreads, 1)
redist_product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                      const __grid_constant__ ProductParams p)
{
    constexpr int kRowsB = BN / CG;                         // rows of B that this block loads
    constexpr int kStageA = 128 * 128, kStageB = kRowsB * 128, kStage = kStageA + kStageB;
    constexpr int kStages = kRing / kStage < kMaxStages ? kRing / kStage : kMaxStages;
    constexpr uint32_t kColumns = 2 * BN < 32 ? 32 : 2 * BN;
    static_assert((kColumns & (kColumns - 1)) == 0 && kColumns <= 512, "tensor memory is allocated in powers of two");

    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_addr(raw) + 1023) & ~1023u;
    uint8_t *ring = raw + (base - smem_addr(raw));
    float *epi = reinterpret_cast<float *>(ring + kRing);
    const uint32_t bars = base + kRing + kEpiBytes;
    auto full = [&](int s) { return bars + 8 * s; };
    auto empty = [&](int s) { return bars + 8 * (kStages + s); };
    auto acc_full = [&](int b) { return bars + 8 * (2 * kStages + b); };
    auto acc_free = [&](int b) { return bars + 8 * (2 * kStages + 2 + b); };
    const uint32_t tmem_at = bars + 8 * (2 * kStages + 4), failed_at = tmem_at + 4;
    volatile uint32_t *tmem_word = reinterpret_cast<volatile uint32_t *>(ring + kRing + kEpiBytes + 8 * (2 * kStages + 4));
    volatile uint32_t *failed = tmem_word + 1;
    (void)failed_at;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = CG == 1 ? 0 : cluster_rank();
    const int first = blockIdx.x / CG, step = gridDim.x / CG;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            bar_init(full(s), 1);
            bar_init(empty(s), 1);
        }
        for (int b = 0; b < 2; ++b) {
            bar_init(acc_full(b), 1);
            bar_init(acc_free(b), 4 * CG);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        *failed = 0;
    }
    if (warp == 2) tmem_alloc<CG>(tmem_at, kColumns);
    fence_before();
    __syncthreads();
    if constexpr (CG == 2) cluster_sync();
    fence_after();
    const uint32_t tmem = *tmem_word;
    let_next_start();
    wait_for_previous();

    bool ok = true;
    if (warp == 0 && lane == 0) {
        // loads
        int stage = 0;
        uint32_t phase = 0, rounds = 0;
        for (int t = first; ok && t < p.tiles; t += step) {
            const Tile at = tile_at(p, t);
            const int row_a = (at.tm * CG + int(rank)) * 128, row_b = at.tn * BN + int(rank) * kRowsB;
            for (int kb = 0; kb < p.k_blocks; ++kb) {
                if (!bar_wait(empty(stage), phase ^ 1, p.wait_polls)) {
                    ok = false;
                    break;
                }
                const uint32_t to_a = base + stage * kStage, to_b = to_a + kStageA;
                const uint32_t bar = CG == 1 ? full(stage) : in_first(full(stage));
                if (rank == 0) bar_expect(full(stage), CG * kStage + p.test_extra_tx);
                if (p.a_along_rows) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) load_box<CG>(to_a + i * kBK * 128, &map_a, bar, row_a + 64 * i, kb * kBK, at.matrix);
                } else {
                    load_box<CG>(to_a, &map_a, bar, kb * kBK, row_a, at.matrix);
                }
                if (p.b_along_rows) {
#pragma unroll
                    for (int i = 0; i < kRowsB / 64; ++i) load_box<CG>(to_b + i * kBK * 128, &map_b, bar, row_b + 64 * i, kb * kBK, at.matrix);
                } else {
                    load_box<CG>(to_b, &map_b, bar, kb * kBK, row_b, at.matrix);
                }
                if (++stage == kStages) {
                    stage = 0;
                    phase ^= 1;
                    rounds = 1;
                }
            }
        }
        // every stage's last use has to be over before this block may end: its products read, its copies landed
        const int used = rounds ? kStages : stage;
        for (int i = 0; i < used; ++i) {
            const int s = rounds ? (stage + i) % kStages : i;
            const uint32_t last = s < stage ? phase : phase ^ 1;          // the phase of the stage's last use
            if (ok) {
                ok = bar_wait(empty(s), last, p.wait_polls);
            } else if (rank == 0) {
                bar_wait(full(s), last, p.wait_polls);
            }
        }
        if (!ok && rank != 0)                                             // its copies report to the first block: give
            for (int i = 0; i < 64; ++i) __nanosleep(1 << 15);            // them 2 ms to land in memory it still owns
    } else if (warp == 1 && lane == 0 && rank == 0) {
        // products
        int stage = 0;
        uint32_t phase = 0;
        int use = 0;
        for (int t = first; ok && t < p.tiles; t += step, ++use) {
            const int buf = use & 1;
            if (!bar_wait(acc_free(buf), ((use >> 1) & 1) ^ 1, p.wait_polls)) {
                ok = false;
                break;
            }
            fence_after();
            const uint32_t acc = tmem + buf * BN;
            for (int kb = 0; kb < p.k_blocks; ++kb) {
                if (!bar_wait(full(stage), phase, p.wait_polls)) {
                    ok = false;
                    break;
                }
                fence_after();
                const uint32_t at_a = base + stage * kStage, at_b = at_a + kStageA;
                const uint64_t da = slice_desc(at_a, p.a_along_rows), db = slice_desc(at_b, p.b_along_rows);
                const uint64_t da_step = p.a_along_rows ? 2048 >> 4 : 32 >> 4, db_step = p.b_along_rows ? 2048 >> 4 : 32 >> 4;
#pragma unroll
                for (int i = 0; i < kBK / 16; ++i) mma<CG>(acc, da + i * da_step, db + i * db_step, p.idesc, (kb | i) != 0);
                commit<CG>(empty(stage));
                if (++stage == kStages) {
                    stage = 0;
                    phase ^= 1;
                }
            }
            if (ok) commit<CG>(acc_full(buf));
        }
    } else if (warp >= 4) {
        // outputs
        const int quarter = warp & 3;
        float *buf = epi + quarter * 32 * kPitch;
        int use = 0;
        for (int t = first; t < p.tiles; t += step, ++use) {
            const int b = use & 1;
            if (!bar_wait(acc_full(b), (use >> 1) & 1, p.wait_polls)) {
                ok = false;
                break;
            }
            fence_after();
            const Tile at = tile_at(p, t);
            const int row0 = (at.tm * CG + int(rank)) * 128 + quarter * 32, col0 = at.tn * BN;
            float alpha = p.e.alpha, beta = p.e.beta;
            if (KIND == EPI_SCALED && p.e.scale) {
                const float s = p.e.scale[at.matrix];
                for (int i = 0; i < p.e.alpha_power; ++i) alpha *= s;
                for (int i = 0; i < p.e.beta_power; ++i) beta *= s;
            }
            const bool mirror = KIND == EPI_SCALED && p.symmetric && at.tm != at.tn;
#pragma unroll 1
            for (int c = 0; c < BN; c += 32) {
                if (col0 + c >= p.n || row0 >= p.m) break;
                uint32_t v[32];
                tmem_load32(tmem + (uint32_t(quarter * 32) << 16) + b * BN + c, v);
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    *reinterpret_cast<uint4 *>(buf + lane * kPitch + 4 * i) = make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
                __syncwarp();
                if constexpr (KIND == EPI_LINEAR) {
                    if (p.e.out_type == T_BF16) linear_piece<__nv_bfloat16>(p, buf, lane, row0, col0 + c);
                    else linear_piece<__half>(p, buf, lane, row0, col0 + c);
                } else {
                    scaled_piece(p, buf, lane, row0, col0 + c, at.matrix, alpha, beta, mirror);
                }
            }
            fence_before();
            __syncwarp();
            if (lane == 0) {
                if constexpr (CG == 1)
                    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(acc_free(b)) : "memory");
                else
                    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(in_first(acc_free(b))) : "memory");
            }
        }
    }
    if (!ok) *failed = 1;
    __syncwarp();
    fence_before();
    __syncthreads();
    if constexpr (CG == 2) cluster_sync();
    fence_after();
    if (threadIdx.x == 0 && *failed) atomicAdd(&g_product_timeouts, 1u);
    if (warp == 2) tmem_free<CG>(tmem, kColumns);
}

// ---- host --------------------------------------------------------------------------------------------

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                 const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled()
{
    static std::atomic<void *> known{nullptr};
    void *fn = known.load(std::memory_order_acquire);
    if (!fn) {
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            return nullptr;
        known.store(fn, std::memory_order_release);
    }
    return reinterpret_cast<EncodeTiled>(fn);
}

// Tensor map of an operand of `rows` x `cols` (cols: the sum).  The box is 128 bytes wide: 64 steps of the sum by
// `box_rows` rows, or 64 rows by 64 steps where the operand is contiguous along its rows.
bool make_map(CUtensorMap *map, const Operand &op, int64_t rows, int64_t cols, int batch, int box_rows)
{
    EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    const cuuint64_t dims[3] = {cuuint64_t(op.along_rows ? rows : cols), cuuint64_t(op.along_rows ? cols : rows), cuuint64_t(batch)};
    // a line's stride is never used where there is one line only: any legal value does
    const int64_t line = dims[1] > 1 ? op.ld : (int64_t(dims[0]) + 7) / 8 * 8;
    const int64_t plane = batch > 1 ? op.batch_stride : line;
    const cuuint64_t strides[2] = {cuuint64_t(line) * 2, cuuint64_t(plane) * 2};
    const cuuint32_t box[3] = {cuuint32_t(kBK), cuuint32_t(op.along_rows ? kBK : box_rows), 1};
    const cuuint32_t one[3] = {1, 1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 3, const_cast<void *>(op.data), dims, strides, box, one,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool on_16(const void *p, int64_t ld) { return p == nullptr || (uintptr_t(p) % 16 == 0 && ld % 8 == 0); }

template <int CG, int BN, int KIND>
cudaError_t launch(const Product &q, const LaunchOptions &o, int sms, cudaStream_t stream)
{
    ProductParams p;
    std::memset(&p, 0, sizeof p);
    p.m = int32_t(q.m);
    p.n = int32_t(q.n);
    p.k_blocks = int32_t((q.k + kBK - 1) / kBK);
    p.batch = q.batch;
    p.tiles_m = int32_t((q.m + 128 * CG - 1) / (128 * CG));
    p.tiles_n = int32_t((q.n + BN - 1) / BN);
    const int64_t per = q.symmetric ? int64_t(p.tiles_m) * (p.tiles_m + 1) / 2 : int64_t(p.tiles_m) * p.tiles_n;
    if (per * q.batch > INT32_MAX / 2) return cudaErrorInvalidValue;
    p.tiles_per_matrix = int32_t(per);
    p.tiles = int32_t(per * q.batch);
    p.symmetric = q.symmetric;
    p.a_along_rows = q.a.along_rows;
    p.b_along_rows = q.b.along_rows;
    const uint32_t format = q.type == T_BF16 ? 1 : 0;
    // 32-bit accumulators, operand types, operand orders, tile width / 8, tile height / 16
    p.idesc = (1u << 4) | (format << 7) | (format << 10) | (uint32_t(q.a.along_rows) << 15) | (uint32_t(q.b.along_rows) << 16) |
              (uint32_t(BN >> 3) << 17) | (uint32_t(128 * CG >> 4) << 24);
    p.wait_polls = o.wait_polls;
    p.test_extra_tx = o.test_extra_tx;
    p.e = q.e;
    const Epilogue &e = q.e;
    p.vector_out = on_16(e.out, e.ld_out) && (q.batch == 1 || e.out_batch % 8 == 0) && on_16(e.residual, e.ld_residual) && on_16(e.pre, e.ld_pre);
    CUtensorMap ma, mb;
    if (!make_map(&ma, q.a, q.m, q.k, q.batch, 128) || !make_map(&mb, q.b, q.n, q.k, q.batch, BN / CG)) return cudaErrorInvalidValue;

    auto *kernel = redist_product_kernel<CG, BN, KIND>;
    cudaError_t ce = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (ce != cudaSuccess) return ce;
    cudaLaunchConfig_t cfg = {};
    const int groups = sms / CG;
    cfg.gridDim = dim3(unsigned((p.tiles < groups ? p.tiles : groups) * CG));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmem;
    cfg.stream = stream;
    cudaLaunchAttribute at[2];
    int n_at = 0;
    if (CG > 1) {
        at[n_at].id = cudaLaunchAttributeClusterDimension;
        at[n_at].val.clusterDim.x = CG;
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
    return cudaLaunchKernelEx(&cfg, kernel, ma, mb, p);
}

}  // namespace

bool operand_fits(const void *data, int64_t ld, int64_t batch_stride, int batch)
{
    return uintptr_t(data) % 16 == 0 && ld % 8 == 0 && (batch == 1 || batch_stride % 8 == 0);
}

cudaError_t launch_product(const Product &p, const LaunchOptions &o, cudaStream_t stream)
{
    if (p.m == 0 || p.n == 0 || p.batch == 0) return cudaSuccess;
    int device = 0, sms = 0;
    cudaError_t ce = cudaGetDevice(&device);
    if (ce == cudaSuccess) ce = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
    if (ce != cudaSuccess) return ce;
    if (p.kind == EPI_LINEAR) return launch<1, 256, EPI_LINEAR>(p, o, sms, stream);
    if (p.symmetric) return launch<1, 128, EPI_SCALED>(p, o, sms, stream);
    return launch<1, 256, EPI_SCALED>(p, o, sms, stream);
}

cudaError_t read_product_timeouts(unsigned int *out) { return cudaMemcpyFromSymbol(out, g_product_timeouts, sizeof *out); }

}  // namespace redist
