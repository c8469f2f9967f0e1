// D = epilogue(A B^T): 16-bit operands, 32-bit accumulation on the tensor cores (tcgen05).
//
// One thread block (CG = 1) or a pair of them on two SMs (CG = 2) owns a tile of 128 CG x BN outputs at a time and
// walks over the sum in steps of 64 KB: two threads bring the 128-byte wide slices of the two operands into a ring of
// shared-memory stages by TMA (128-byte swizzle), one thread issues the tcgen05.mma that consume them, and eight
// warps turn the finished accumulator of the previous tile into outputs while the next one runs: tensor memory holds
// two accumulators of BN columns.  Operands may be contiguous along the sum or along their rows (the gradients need
// both): only the boxes and the shared-memory descriptors differ.  Ragged sizes cost nothing extra: the TMA fills
// what lies outside an operand with zeros, and the epilogue stores what lies inside the result.
//
// What bounds it: large products the tensor cores and, in long runs, the power they may draw -- 8192 x 4096 -> 8192 with
// GELU keeps their pipe busy 96 % of the cycles at 1.43 GHz; 16384 x 4096 -> 16384 takes 1370 us in a run of 50 ms and 1600
// in one of two seconds (1605 and 1372 TFLOP/s; a library product 1649 at its best and 1372 sustained), with bias and GELU
// 1385 and 1615.  A stack of 2048 x 2048 squares keeps the pipe busy 64-70 %: 32 stages of sum do not hide the last epilogue.  Small
// products: the 2 us of a launch, 1 us to the first operands, 0.1-0.15 us per 64 steps of the sum, 1-3 us for the last
// epilogue (512^3: 4.4 us, 1024^3: 6.0).  Rows of outputs or residuals off 16-byte boundaries cost about 20 us per
// 4096 x 4096 outputs in the epilogue's stores.
//
// Every wait on an mbarrier is bounded, the storing warps' by polls that grow with a tile's sum.  A role whose wait runs
// out leaves its loop, so the others' waits run out too; products already issued are awaited, as they are in a healthy
// run, and so are copies in flight (both with limits of their own, which wait_polls does not shorten); then the block
// counts itself in g_product_timeouts, frees its tensor memory and returns without storing the tile.
#include "product.h"

#include <cuda.h>

#include <algorithm>
#include <atomic>
#include <cstring>

#include "activation.cuh"
#include "elements.cuh"
#include "rows.h"

namespace redist {

namespace {

constexpr int kBK = 64;                 // elements of the sum per stage: 128 bytes, one swizzle row
constexpr int kThreads = 384;           // warps 0 and 3 load, warp 1 multiplies, warp 2 owns tensor memory, warps 4-11 store
constexpr int kRing = 196608;           // bytes of the ring of stages
constexpr int kPiece = 2048;            // a warp's 32 x 32 piece of 16-bit outputs: rows of 64 bytes, 64-byte swizzle
constexpr int kEpiBytes = 8 * 2 * kPiece;                   // two pieces per warp: one is filled while one is stored
constexpr int kBiasBytes = 8 * 32 * 4;
constexpr int kBarBytes = 256;
constexpr int kSmem = 1024 + kRing + kEpiBytes + kBiasBytes + kBarBytes;
constexpr int kMaxStages = 12;
// (a poll holds a thread for up to 4 us)
constexpr uint32_t kDrainPolls = 1 << 16;       // for products already issued, which always end
constexpr uint32_t kCopyPolls = 1 << 10;        // for a stage's copies once a wait has run out: 4 ms

__device__ unsigned int g_product_timeouts = 0;

struct ProductParams {
    int32_t m, n, k_blocks, batch;
    int32_t tiles_m, tiles_n, tiles_per_matrix, tiles;
    int32_t splits, k_per_split;        // parts of the sum, each a unit of work of its own (EPI_PARTIAL)
    int32_t symmetric, a_along_rows, b_along_rows;
    uint32_t idesc, wait_polls, test_extra_tx;
    int32_t aligned_out;                // every row of out and pre starts on a 16-byte boundary: pieces go out by TMA
    int32_t aligned_residual;
    Epilogue e;
};

// ---- shared memory, barriers, tensor memory -----------------------------------------------------

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return uint32_t(__cvta_generic_to_shared(p)); }

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}

// True when the phase is over, false when this lane's `polls` polls have not seen it end.  (The roles that act through one
// lane ask that lane; the storing warps ask all.)  The loop is hidden from the compiler: the loading and the multiplying
// warp stay convergent in its eyes, and the descriptors of what they issue in uniform registers (a k-step took 400 cycles to
// issue when they did not, more than the tensor cores need for it).
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, uint32_t polls)
{
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t.reg .u32 n;\n\tmov.u32 n, %3;\n"
        "POLL:\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "@p bra DONE;\n\t"
        "sub.u32 n, n, 1;\n\t"
        "setp.ne.u32 q, n, 0;\n\t"
        "@q bra POLL;\n"
        "DONE:\n\t"
        "selp.b32 %0, 1, 0, p;\n\t}"
        : "=r"(done) : "r"(bar), "r"(parity), "r"(polls) : "memory");
    return done != 0;
}

// One lane of a convergent warp, always the same.
__device__ __forceinline__ bool elected()
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
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

// ... in the block of rank 1.
__device__ __forceinline__ uint32_t in_second(uint32_t addr)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 1;" : "=r"(r) : "r"(addr));
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
    int tm, tn, matrix, k0, k1;         // k0 ... k1: its steps of the sum
};

// Tiles of a matrix in groups of eight tile rows, column after column within a group, so that the blocks at work at
// one time share slices of both operands in L2.  Symmetric: those that reach the lower triangle, row after row; R is a
// tile's height over its width (a whole number there), so that tile row i has R (i + 1) of them.
template <int R> __device__ __forceinline__ Tile tile_at(const ProductParams &p, int t)
{
    Tile r;
    r.k0 = 0;
    r.k1 = p.k_blocks;
    if (p.splits > 1) {
        const int part = t % p.splits;
        t /= p.splits;
        r.k0 = part * p.k_per_split;
        r.k1 = min(p.k_blocks, r.k0 + p.k_per_split);
    }
    r.matrix = t / p.tiles_per_matrix;
    int q = t - r.matrix * p.tiles_per_matrix;
    if (p.symmetric) {
        int i = int((sqrtf(8.0f / R * float(q) + 1.0f) - 1.0f) * 0.5f);
        while (R * (i * (i + 1) / 2) > q) --i;
        while (R * ((i + 1) * (i + 2) / 2) <= q) ++i;
        r.tm = i;
        r.tn = q - R * (i * (i + 1) / 2);
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

// A warp takes its quarter of the lanes (rows) and half of the columns of an accumulator, 32 x 32 values at a time: a
// lane holds 32 neighbours of one row, computes, rounds and writes them to a piece in shared memory, from where a TMA
// store takes it (or, where rows are not on 16-byte boundaries, the warp itself, row by row).  Everything 32-bit stays
// in registers: a 256 x 256 tile takes 2 us (GELU 2.3 more, SiLU 2, bias 0.8, residual 2.2, pre-activation 1), 12 when the
// 32-bit accumulators went through shared memory.  It hides behind the next tile's sum from about 1000 steps on.

// Where the 16 bytes of columns 8 j ... 8 j + 7 of row r of a piece lie (the TMA's 64-byte swizzle).
__device__ __forceinline__ uint32_t piece_at(int r, int j) { return uint32_t(r * 64 + ((j ^ ((r >> 1) & 3)) << 4)); }

// A warp's two pieces, used in turn.
struct Pieces {
    uint8_t *smem;
    uint32_t addr;
    int turn = 0;

    // the piece to fill next, free of the store that used it last
    __device__ __forceinline__ uint8_t *next(int lane)
    {
        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
        __syncwarp();
        return smem + turn * kPiece;
    }

    // Rows row0 ... and columns col0 ... of the output are in the piece: send them off.
    __device__ __forceinline__ void store(const CUtensorMap *map, int lane, int row0, int col0, int matrix)
    {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
            asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4}], [%1];"
                         ::"l"(map), "r"(addr + turn * kPiece), "r"(col0), "r"(row0), "r"(matrix) : "memory");
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        }
        turn ^= 1;
    }

    // ---- rows that start anywhere: the piece to fill, and what sends it off

    __device__ __forceinline__ uint8_t *plain() const { return smem; }

    // Stores `cnt` (up to 32) columns of up to `rows` rows from the piece, `to` the first of them.  A row's aligned blocks
    // of 16 bytes go out whole, four per row; what the last of them lacks of a piece waits in `carry` (0: out, 1: pre) for
    // the piece to its right.  Only a row's ends go out in smaller stores.
    __device__ __forceinline__ void store_any(uint16_t *to, int64_t ld, int lane, int rows, int cnt, bool first, bool last, int carry) const
    {
        uint8_t *kept = smem + 2 * kPiece - (2 - carry) * 512;
        auto word = [&](int r, int w) -> uint32_t {
            return *reinterpret_cast<const uint32_t *>(w >= 0 ? smem + piece_at(r, w >> 2) + (w & 3) * 4 : kept + r * 16 + (w + 4) * 4);
        };
        auto element = [&](int r, int e) -> uint16_t {
            return *reinterpret_cast<const uint16_t *>(e >= 0 ? smem + piece_at(r, e >> 3) + (e & 7) * 2 : kept + r * 16 + (e + 8) * 2);
        };
        auto two = [&](int r, int e) -> uint32_t { return element(r, e) | uint32_t(element(r, e + 1)) << 16; };
        __syncwarp();
#pragma unroll
        for (int it = 0; it < 4; ++it) {
            const int r = it * 8 + (lane >> 2);
            uint16_t *row = to + r * ld;
            const int s = 8 * (lane & 3) - int(reinterpret_cast<uintptr_t>(row) & 15) / 2;
            if (r < rows && (s >= 0 || !first) && s + 8 <= cnt) {
                const int w = s >> 1;                       // rounds down, below zero too
                uint4 u = make_uint4(word(r, w), word(r, w + 1), word(r, w + 2), word(r, w + 3));
                if (s & 1) {
                    const uint32_t end = word(r, w + 4);
                    u = make_uint4(__funnelshift_r(u.x, u.y, 16), __funnelshift_r(u.y, u.z, 16), __funnelshift_r(u.z, u.w, 16), __funnelshift_r(u.w, end, 16));
                }
                *reinterpret_cast<uint4 *>(row + s) = u;
            }
        }
        if ((first || last) && lane < rows) {
            uint16_t *row = to + lane * ld;
            const int p = int(reinterpret_cast<uintptr_t>(row) & 15) / 2, head = p ? 8 - p : 0;
            // in stores of two, four and eight bytes: a row's end begins (its beginning ends) on a 16-byte boundary
            if (first && cnt < head) {
                for (int e = 0; e < cnt; ++e) row[e] = element(lane, e);
            } else if (first) {
                int e = 0;
                if (head & 1) {
                    row[e] = element(lane, e);
                    e += 1;
                }
                if (head & 2) {
                    *reinterpret_cast<uint32_t *>(row + e) = two(lane, e);
                    e += 2;
                }
                if (head & 4) *reinterpret_cast<uint2 *>(row + e) = make_uint2(two(lane, e), two(lane, e + 2));
            }
            if (last) {
                const int whole = ((cnt + p) >> 3) * 8 - p;
                int e = first ? max(whole, head) : whole;
                const int left = cnt - e;
                if (left > 0) {
                    if (left & 4) {
                        *reinterpret_cast<uint2 *>(row + e) = make_uint2(two(lane, e), two(lane, e + 2));
                        e += 4;
                    }
                    if (left & 2) {
                        *reinterpret_cast<uint32_t *>(row + e) = two(lane, e);
                        e += 2;
                    }
                    if (left & 1) row[e] = element(lane, e);
                }
            }
        }
        __syncwarp();
        if (!last) *reinterpret_cast<uint4 *>(kept + lane * 16) = *reinterpret_cast<const uint4 *>(smem + piece_at(lane, 3));
        __syncwarp();
    }

    // Rows of a matrix whose rows start anywhere, 32 columns of 32 rows: `ask` loads the aligned blocks that hold them, lanes
    // along the rows; `take` hands every lane its row.
    static __device__ __forceinline__ void ask(const uint16_t *from, int64_t ld, int lane, int rows, int cnt, uint4 (&blocks)[4], uint4 &end)
    {
#pragma unroll
        for (int it = 0; it < 4; ++it) {
            const int r = it * 8 + (lane >> 2), b = lane & 3;
            const uintptr_t at = reinterpret_cast<uintptr_t>(from + r * ld);
            blocks[it] = make_uint4(0, 0, 0, 0);
            if (r < rows && 16 * b < int(at & 15) + 2 * cnt) blocks[it] = *reinterpret_cast<const uint4 *>((at & ~uintptr_t(15)) + 16 * b);
        }
        const uintptr_t at = reinterpret_cast<uintptr_t>(from + lane * ld);
        end = make_uint4(0, 0, 0, 0);
        if (lane < rows && 64 < int(at & 15) + 2 * cnt) end = *reinterpret_cast<const uint4 *>((at & ~uintptr_t(15)) + 64);
    }
    __device__ __forceinline__ void take(const uint16_t *from, int64_t ld, int lane, uint4 (&blocks)[4], const uint4 &end) const
    {
        __syncwarp();
#pragma unroll
        for (int it = 0; it < 4; ++it) *reinterpret_cast<uint4 *>(smem + (it * 8 + (lane >> 2)) * 80 + (lane & 3) * 16) = blocks[it];
        *reinterpret_cast<uint4 *>(smem + lane * 80 + 64) = end;
        __syncwarp();
        const int off = int(reinterpret_cast<uintptr_t>(from + lane * ld) & 15);
        const uint32_t *w = reinterpret_cast<const uint32_t *>(smem + lane * 80 + (off & ~3));
        uint32_t v[17];
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = w[i];
        v[16] = off & 2 ? w[16] : 0;
        if (off & 2)
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = __funnelshift_r(v[i], v[i + 1], 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) blocks[i] = make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
        __syncwarp();
    }
};

template <typename T> __device__ __forceinline__ void put_row(uint8_t *piece, int lane, const float (&v)[32])
{
#pragma unroll
    for (int j = 0; j < 4; ++j)
        *reinterpret_cast<uint4 *>(piece + piece_at(lane, j)) =
            make_uint4(pack2<T>(v[8 * j], v[8 * j + 1]), pack2<T>(v[8 * j + 2], v[8 * j + 3]), pack2<T>(v[8 * j + 4], v[8 * j + 5]),
                       pack2<T>(v[8 * j + 6], v[8 * j + 7]));
}

template <typename T> __device__ __forceinline__ void unpack8(const uint4 &u, float *v)
{
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = unpack2<T>(w[i]);
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}

// 32 x 32 values of the linear epilogue; `bias` holds the columns' biases, `ahead` the lane's row of the residual.
template <typename T>
__device__ __forceinline__ void linear_piece(const ProductParams &p, const CUtensorMap *map_out, const CUtensorMap *map_pre, Pieces &pieces,
                                             float (&v)[32], const float *bias, const uint4 (&ahead)[4], int lane, int row0, int col0,
                                             bool first, bool last)
{
    const Epilogue &e = p.e;
    if (e.bias) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float4 b = *reinterpret_cast<const float4 *>(bias + 4 * j);
            v[4 * j] += b.x;
            v[4 * j + 1] += b.y;
            v[4 * j + 2] += b.z;
            v[4 * j + 3] += b.w;
        }
    }
    if (e.pre) {
        if (p.aligned_out) {
            put_row<T>(pieces.next(lane), lane, v);
            pieces.store(map_pre, lane, row0, col0, 0);
        } else {
            put_row<T>(pieces.plain(), lane, v);
            pieces.store_any(static_cast<uint16_t *>(e.pre) + int64_t(row0) * e.ld_pre + col0, e.ld_pre, lane, p.m - row0, min(32, p.n - col0), first, last, 1);
        }
    }
    activate32(v, e.activation);
    if (e.residual) {
        float w[32];
#pragma unroll
        for (int j = 0; j < 4; ++j) unpack8<T>(ahead[j], w + 8 * j);
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] += w[i];
    }
    if (p.aligned_out) {
        put_row<T>(pieces.next(lane), lane, v);
        pieces.store(map_out, lane, row0, col0, 0);
    } else {
        put_row<T>(pieces.plain(), lane, v);
        pieces.store_any(static_cast<uint16_t *>(e.out) + int64_t(row0) * e.ld_out + col0, e.ld_out, lane, p.m - row0, min(32, p.n - col0), first, last, 0);
    }
}

// 32 x 32 values of the scaled epilogue; `hi` and `lo` hold the lane's row of what is added.  A mirrored piece is
// written a second time with rows and columns exchanged.
__device__ __forceinline__ void scaled_piece(const ProductParams &p, const CUtensorMap *map_out, const CUtensorMap *map_lo, Pieces &pieces,
                                             float (&v)[32], const uint4 (&hi)[4], const uint4 (&lo)[4], int lane, int row0, int col0,
                                             int matrix, float alpha, float beta, float center, bool mirror, bool first, bool last)
{
    const Epilogue &e = p.e;
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] *= alpha;
    if (e.hi) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float w[8], u[8];
            unpack8<__half>(hi[j], w);
            unpack8<__half>(lo[j], u);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[8 * j + i] = fmaf(beta, fmaf(u[i], 1.0f / 2048.0f, w[i]), v[8 * j + i]);
        }
    }
    if (e.diagonal && row0 == col0) {
#pragma unroll
        for (int i = 0; i < 32; ++i)
            if (i == lane) v[i] = fmaf(-center, e.on_diagonal, v[i]);
    }
    if (e.out_type == T_BF16 && !p.aligned_out) {
        put_row<__nv_bfloat16>(pieces.plain(), lane, v);
        pieces.store_any(static_cast<uint16_t *>(e.out) + int64_t(matrix) * e.out_batch + int64_t(row0) * e.ld_out + col0, e.ld_out, lane, p.m - row0,
                         min(32, p.n - col0), first, last, 0);
        return;
    }
    uint8_t *piece = pieces.next(lane);
    if (e.out_type == T_BF16) {
        put_row<__nv_bfloat16>(piece, lane, v);
        pieces.store(map_out, lane, row0, col0, matrix);
        return;
    }
    put_row<__half>(piece, lane, v);
    pieces.store(map_out, lane, row0, col0, matrix);
    if (e.out_lo) {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = (v[i] - __half2float(__float2half_rn(v[i]))) * 2048.0f;
        put_row<__half>(pieces.next(lane), lane, v);
        pieces.store(map_lo, lane, row0, col0, matrix);
    }
    if (mirror) {
        piece = pieces.next(lane);
#pragma unroll
        for (int i = 0; i < 32; ++i) *reinterpret_cast<__half *>(piece + piece_at(i, lane >> 3) + (lane & 7) * 2) = __float2half_rn(v[i]);
        pieces.store(map_out, lane, col0, row0, matrix);
    }
}

// The lane's row of 32 neighbours, 16 bytes at a time; what lies outside the matrix reads as zero (or as the padding of a
// workspace row: it is not stored).
__device__ __forceinline__ void get_row(const uint16_t *row, bool in, int left, uint4 (&v)[4])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        v[j] = make_uint4(0, 0, 0, 0);
        if (in && left > 8 * j) v[j] = *reinterpret_cast<const uint4 *>(row + 8 * j);
    }
}

// ---- the kernel ------------------------------------------------------------------------------------

template <int CG, int BN, int KB, int KIND>
__global__ void __launch_bounds__(kThreads, 1)
redist_product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                      const __grid_constant__ CUtensorMap map_out, const __grid_constant__ CUtensorMap map_more,
                      const __grid_constant__ ProductParams p)
{
    constexpr int kRowsB = BN / CG;                         // rows of B that this block loads
    constexpr int kSliceA = 128 * 128, kSliceB = kRowsB * 128, kStageA = KB * kSliceA, kStageB = KB * kSliceB, kStage = kStageA + kStageB;
    constexpr int kStages = kRing / kStage < kMaxStages ? kRing / kStage : kMaxStages;
    constexpr uint32_t kColumns = 2 * BN < 32 ? 32 : 2 * BN;
    constexpr int kShare = BN >= 64 ? BN / 2 : BN;          // columns of an accumulator that one warp stores
    constexpr int kStorers = 4 * (BN / kShare);
    static_assert(8 * (2 * kStages + 5) + 8 <= kBarBytes, "barriers, tensor memory's address and the flag");
    static_assert((kColumns & (kColumns - 1)) == 0 && kColumns <= 512, "tensor memory is allocated in powers of two");

    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_addr(raw) + 1023) & ~1023u;
    uint8_t *ring = raw + (base - smem_addr(raw));
    const uint32_t bars = base + kRing + kEpiBytes + kBiasBytes;
    auto full = [&](int s) { return bars + 8 * s; };
    auto empty = [&](int s) { return bars + 8 * (kStages + s); };
    auto acc_full = [&](int b) { return bars + 8 * (2 * kStages + b); };
    auto acc_free = [&](int b) { return bars + 8 * (2 * kStages + 2 + b); };
    const uint32_t drained = bars + 8 * (2 * kStages + 4);
    const uint32_t tmem_at = bars + 8 * (2 * kStages + 5);
    volatile uint32_t *tmem_word = reinterpret_cast<volatile uint32_t *>(ring + kRing + kEpiBytes + kBiasBytes + 8 * (2 * kStages + 5));
    volatile uint32_t *failed = tmem_word + 1;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = CG == 1 ? 0 : cluster_rank();
    const int first = blockIdx.x / CG, step = gridDim.x / CG;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            bar_init(full(s), 2);                           // both operands' bytes are announced
            bar_init(empty(s), 1);
        }
        for (int b = 0; b < 2; ++b) {
            bar_init(acc_full(b), 1);
            bar_init(acc_free(b), kStorers * CG);
        }
        bar_init(drained, 1);
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
    if (warp == 0 || warp == 3) {
        // Loads: warp 0 those of A, warp 3 those of B.  The whole warp walks along, one lane issues; after a wait that ran
        // out it only counts on to the end.
        const bool second = warp == 3;
        int stage = 0;
        uint32_t phase = 0, rounds = 0, polls = p.wait_polls;
        const CUtensorMap *map = second ? &map_b : &map_a;
        const int along_rows = second ? p.b_along_rows : p.a_along_rows;
        const uint32_t announced = CG * (second ? kStageB : kStageA + p.test_extra_tx);
        for (int t = first; t < p.tiles; t += step) {
            const Tile at = tile_at<CG * 128 / BN>(p, t);
            const int row = second ? at.tn * BN + int(rank) * kRowsB : (at.tm * CG + int(rank)) * 128;
            for (int kb = at.k0; kb < at.k1; ++kb) {
                if (!bar_wait(empty(stage), phase ^ 1, polls)) {
                    ok = false;
                    polls = 1;
                }
                if (elected() && ok) {
                    const uint32_t to = base + stage * kStage + (second ? kStageA : 0);
                    const uint32_t bar = CG == 1 ? full(stage) : in_first(full(stage));
                    if (rank == 0) bar_expect(full(stage), announced);
#pragma unroll
                    for (int k = 0; k < KB; ++k) {
                        const int x = (kb * KB + k) * kBK;
                        const uint32_t slice = to + k * (second ? kSliceB : kSliceA);
                        if (!along_rows) {
                            load_box<CG>(slice, map, bar, x, row, at.matrix);
                        } else {
                            const int boxes = second ? kRowsB / 64 : 2;
                            for (int i = 0; i < boxes; ++i) load_box<CG>(slice + i * kBK * 128, map, bar, row + 64 * i, x, at.matrix);
                        }
                    }
                }
                if (ok && ++stage == kStages) {
                    stage = 0;
                    phase ^= 1;
                    rounds = 1;
                }
            }
        }
        // every stage's last use has to be over before this block may end: its products read, its copies landed
        const int used = rounds ? kStages : stage;
        auto use = [&](int i) { return rounds ? (stage + i) % kStages : i; };
        auto last = [&](int s) { return s < stage ? phase : phase ^ 1; };   // the phase of the stage's last use
        for (int i = 0; i < used && ok; ++i) ok = bar_wait(empty(use(i)), last(use(i)), p.wait_polls);
        if (!ok && rank == 0)
            for (int i = 0; i < used; ++i) bar_wait(full(use(i)), last(use(i)), kCopyPolls);
        if (!ok && rank != 0)                                             // its copies report to the first block: give
            for (int i = 0; i < 128; ++i) __nanosleep(1 << 15);           // them 4 ms to land in memory it still owns
    } else if (warp == 1 && rank == 0) {
        // Products, in the same way.
        int stage = 0;
        uint32_t phase = 0, polls = p.wait_polls;
        int use = 0;
        const uint64_t desc_a = slice_desc(base, p.a_along_rows), desc_b = slice_desc(base + kStageA, p.b_along_rows);
        const uint64_t step_a = p.a_along_rows ? 2048 >> 4 : 32 >> 4, step_b = p.b_along_rows ? 2048 >> 4 : 32 >> 4;
        for (int t = first; t < p.tiles; t += step, ++use) {
            const int buf = use & 1;
            if (!bar_wait(acc_free(buf), ((use >> 1) & 1) ^ 1, polls)) {
                ok = false;
                polls = 1;
            }
            fence_after();
            const uint32_t acc = tmem + buf * BN;
            const Tile at = tile_at<CG * 128 / BN>(p, t);
            for (int kb = at.k0; kb < at.k1; ++kb) {
                if (!bar_wait(full(stage), phase, polls)) {
                    ok = false;
                    polls = 1;
                }
                fence_after();
                if (elected() && ok) {
                    const uint64_t da = desc_a + uint32_t(stage * (kStage >> 4)), db = desc_b + uint32_t(stage * (kStage >> 4));
#pragma unroll
                    for (int k = 0; k < KB; ++k)
#pragma unroll
                        for (int i = 0; i < kBK / 16; ++i)
                            mma<CG>(acc, da + k * (kSliceA >> 4) + i * step_a, db + k * (kSliceB >> 4) + i * step_b, p.idesc, kb > at.k0 || k + i > 0);
                    commit<CG>(empty(stage));
                    if (kb + 1 == at.k1) commit<CG>(acc_full(buf));
                }
                if (++stage == kStages) {
                    stage = 0;
                    phase ^= 1;
                }
            }
        }
        if (!ok) {
            *failed = 1;
            if constexpr (CG == 2)
                asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(in_second(tmem_at + 4)), "r"(1u) : "memory");
        }
        // whatever became of the waits: what was issued reads the stages and writes tensor memory, of both blocks of a pair
        if (elected()) commit<CG>(drained);
        ok = bar_wait(drained, 0, kDrainPolls) && ok;
    } else if (warp == 1) {
        ok = bar_wait(drained, 0, kDrainPolls);                           // reported by the first block
    } else if (warp >= 4 && warp < 4 + kStorers) {
        // outputs
        const int quarter = warp & 3, half = (warp - 4) >> 2;
        Pieces pieces{ring + kRing + (warp - 4) * 2 * kPiece, base + kRing + (warp - 4) * 2 * kPiece};
        float *bias = reinterpret_cast<float *>(ring + kRing + kEpiBytes) + (warp - 4) * 32;
        int use = 0, centred = -1;
        float center = 0.0f;
        for (int t = first; t < p.tiles; t += step, ++use) {
            const int b = use & 1;
            const Tile at = tile_at<CG * 128 / BN>(p, t);
            const int row0 = (at.tm * CG + int(rank)) * 128 + quarter * 32, col_at = at.tn * BN + half * kShare;
            const int64_t row = row0 + lane;
            const bool in = row < p.m;
            float alpha = p.e.alpha, beta = p.e.beta;
            if (KIND == EPI_SCALED && p.e.diagonal) {
                if (at.matrix != centred) {             // every warp for itself, all in the same order
                    const __half *d = static_cast<const __half *>(p.e.diagonal) + int64_t(at.matrix) * p.e.diagonal_batch;
                    float t = 0.0f;
#pragma unroll 4
                    for (int i = lane; i < p.e.diagonal_n; i += 32) t += __half2float(d[i * p.e.diagonal_step]);
#pragma unroll
                    for (int i = 16; i; i >>= 1) t += __shfl_xor_sync(0xffffffffu, t, i);
                    t *= p.e.mean_scale;
                    center = t >= 0.25f ? t * fmaf(t, p.e.center_2, p.e.center_1) : 0.0f;
                    centred = at.matrix;
                }
                beta = fmaf(center, p.e.to_beta, beta);
            }
            if (KIND == EPI_SCALED && p.e.scale) {
                const float s = p.e.scale[at.matrix];
                for (int i = 0; i < p.e.alpha_power; ++i) alpha *= s;
                for (int i = 0; i < p.e.beta_power; ++i) beta *= s;
            }
            // what a piece needs besides its accumulators is fetched before the wait (the first piece) or while the
            // piece before it is computed
            uint4 more[4], rest[4];
            float next_bias = 0.0f;
            auto fetch = [&](int col0) {
                const int left = p.n - col0;
                if constexpr (KIND == EPI_LINEAR) {
                    if (p.e.residual) {
                        const uint16_t *q = static_cast<const uint16_t *>(p.e.residual) + int64_t(row0) * p.e.ld_residual + col0;
                        if (p.aligned_residual) get_row(q + lane * p.e.ld_residual, in, left, more);
                        else Pieces::ask(q, p.e.ld_residual, lane, p.m - row0, min(32, left), more, rest[0]);
                    }
                    if (p.e.bias) next_bias = lane < left ? load_any(p.e.bias, p.e.bias_type, col0 + lane) : 0.0f;
                } else if (KIND == EPI_SCALED && p.e.hi) {
                    const int64_t q = int64_t(at.matrix) * p.e.add_batch + row * p.e.ld_add + col0;
                    get_row(static_cast<const uint16_t *>(p.e.hi) + q, in, left, more);
                    if (p.e.lo) get_row(static_cast<const uint16_t *>(p.e.lo) + q, in, left, rest);
                }
            };
#pragma unroll
            for (int i = 0; i < 4; ++i) more[i] = rest[i] = make_uint4(0, 0, 0, 0);
            if (col_at < p.n && row0 < p.m) fetch(col_at);
            // This wait is for a whole tile's sum: the polls again for every 512 stages of it (0.4 ms at most), unless the
            // multiplying warp has given up.  One answer for the warp: what follows is for all of its lanes.
            bool ready = false;
            for (int turns = 1 + (at.k1 - at.k0) / 512; turns > 0 && !ready; --turns) {
                ready = __all_sync(0xffffffffu, bar_wait(acc_full(b), (use >> 1) & 1, p.wait_polls));
                if (!ready && __any_sync(0xffffffffu, *failed)) break;
            }
            if (!ready) {
                ok = false;
                break;
            }
            fence_after();
#pragma unroll 1
            for (int c = 0; c < kShare; c += 32) {
                const int col0 = col_at + c;
                if (col0 >= p.n || row0 >= p.m) break;
                uint32_t u[32];
                tmem_load32(tmem + (uint32_t(quarter * 32) << 16) + b * BN + half * kShare + c, u);
                float v[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(u[i]);
                uint4 now[4], now_rest[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    now[i] = more[i];
                    now_rest[i] = rest[i];
                }
                if (KIND == EPI_LINEAR && p.e.bias) {
                    __syncwarp();
                    bias[lane] = next_bias;
                    __syncwarp();
                }
                const bool begins = c == 0, ends = c + 32 >= kShare || col0 + 32 >= p.n;
                if (!ends) fetch(col0 + 32);
                if (KIND == EPI_LINEAR && p.e.residual && !p.aligned_residual)
                    pieces.take(static_cast<const uint16_t *>(p.e.residual) + int64_t(row0) * p.e.ld_residual + col0, p.e.ld_residual, lane, now, now_rest[0]);
                if constexpr (KIND == EPI_PARTIAL) {
                    if (in) {
                        float4 *q = reinterpret_cast<float4 *>(static_cast<float *>(p.e.out) + (int64_t(t % p.splits) * p.m + row) * p.e.ld_out + col0);
#pragma unroll
                        for (int i = 0; i < 8; ++i) q[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
                    }
                } else if constexpr (KIND == EPI_LINEAR) {
                    if (p.e.out_type == T_BF16) linear_piece<__nv_bfloat16>(p, &map_out, &map_more, pieces, v, bias, now, lane, row0, col0, begins, ends);
                    else linear_piece<__half>(p, &map_out, &map_more, pieces, v, bias, now, lane, row0, col0, begins, ends);
                } else {
                    // above the diagonal only what no tile computes
                    const bool mirror = p.symmetric && row0 / BN > col0 / (128 * CG) * (128 * CG / BN) + (128 * CG / BN - 1);
                    scaled_piece(p, &map_out, &map_more, pieces, v, now, now_rest, lane, row0, col0, at.matrix, alpha, beta, center, mirror, begins, ends);
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
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
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

// Tensor map of a row-major output, stored in pieces of 32 x 32.
bool make_out_map(CUtensorMap *map, void *data, int64_t ld, int64_t batch_stride, int64_t m, int64_t n, int batch)
{
    EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    const cuuint64_t dims[3] = {cuuint64_t(n), cuuint64_t(m), cuuint64_t(batch)};
    const int64_t line = m > 1 ? ld : (n + 7) / 8 * 8;
    const cuuint64_t strides[2] = {cuuint64_t(line) * 2, cuuint64_t(batch > 1 ? batch_stride : line) * 2};
    const cuuint32_t box[3] = {32, 32, 1}, one[3] = {1, 1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 3, data, dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Tiles that reach the lower triangle: ratio (i + 1) in tile row i, but no more than there are columns.
int64_t symmetric_tiles(int64_t tiles_m, int64_t tiles_n, int64_t ratio)
{
    return ratio * (tiles_m * (tiles_m - 1) / 2) + std::min(tiles_n, ratio * tiles_m);
}

bool on_16(const void *p, int64_t ld) { return p == nullptr || (uintptr_t(p) % 16 == 0 && ld % 8 == 0); }

template <int CG, int BN, int KB, int KIND>
cudaError_t launch(const Product &q, int splits, const LaunchOptions &o, int device, int sms, cudaStream_t stream)
{
    ProductParams p;
    std::memset(&p, 0, sizeof p);
    p.m = int32_t(q.m);
    p.n = int32_t(q.n);
    p.k_blocks = int32_t((q.k + KB * kBK - 1) / (KB * kBK));
    p.batch = q.batch;
    p.tiles_m = int32_t((q.m + 128 * CG - 1) / (128 * CG));
    p.tiles_n = int32_t((q.n + BN - 1) / BN);
    const int64_t per = q.symmetric ? symmetric_tiles(p.tiles_m, p.tiles_n, 128 * CG / BN) : int64_t(p.tiles_m) * p.tiles_n;
    if (per * q.batch * splits > INT32_MAX / 2) return cudaErrorInvalidValue;
    p.tiles_per_matrix = int32_t(per);
    p.tiles = int32_t(per * q.batch * splits);
    p.splits = splits;
    p.k_per_split = (p.k_blocks + splits - 1) / splits;
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
    p.aligned_out = KIND != EPI_PARTIAL && on_16(e.out, e.ld_out) && (q.batch == 1 || e.out_batch % 8 == 0) && on_16(e.pre, e.ld_pre);
    p.aligned_residual = on_16(e.residual, e.ld_residual);
    p.aligned_out = p.aligned_out && p.aligned_residual;    // one way of using the pieces' memory per launch
    CUtensorMap ma, mb, mo, mm;
    if (!make_map(&ma, q.a, q.m, q.k, q.batch, 128) || !make_map(&mb, q.b, q.n, q.k, q.batch, BN / CG)) return cudaErrorInvalidValue;
    std::memset(&mo, 0, sizeof mo);
    std::memset(&mm, 0, sizeof mm);
    if (p.aligned_out) {
        void *more = KIND == EPI_LINEAR ? e.pre : e.out_lo;
        if (!make_out_map(&mo, e.out, e.ld_out, e.out_batch, q.m, q.n, q.batch)) return cudaErrorInvalidValue;
        if (more && !make_out_map(&mm, more, KIND == EPI_LINEAR ? e.ld_pre : e.ld_add, KIND == EPI_LINEAR ? 0 : e.add_batch, q.m, q.n, q.batch))
            return cudaErrorInvalidValue;
    }

    auto *kernel = redist_product_kernel<CG, BN, KB, KIND>;
    static std::atomic<uint64_t> ready{0};                  // devices on which this kernel may use its shared memory
    if (device >= 64 || !(ready.load(std::memory_order_relaxed) >> device & 1)) {
        const cudaError_t ce = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
        if (ce != cudaSuccess) return ce;
        if (device < 64) ready.fetch_or(uint64_t(1) << device, std::memory_order_relaxed);
    }
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
    return cudaLaunchKernelEx(&cfg, kernel, ma, mb, mo, mm, p);
}

}  // namespace

cudaError_t current_device(int *device, int *sms)
{
    static std::atomic<int> known[64];
    cudaError_t ce = cudaGetDevice(device);
    if (ce != cudaSuccess) return ce;
    *sms = *device < 64 ? known[*device].load(std::memory_order_relaxed) : 0;
    if (*sms) return cudaSuccess;
    ce = cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, *device);
    if (ce == cudaSuccess && *device < 64) known[*device].store(*sms, std::memory_order_relaxed);
    return ce;
}

bool operand_fits(const void *data, int64_t ld, int64_t batch_stride, int batch)
{
    return uintptr_t(data) % 16 == 0 && ld % 8 == 0 && (batch == 1 || batch_stride % 8 == 0);
}

namespace {

// The tile shapes, and how long they take: microseconds per 64 steps of the sum, where the tiles fit on the GPU at once
// and where they take several rounds, and per launch besides (start, the last accumulator's epilogue); fitted to timings
// of some twenty sizes from 64 x 64 x 1000 to 4096 x 4096 x 4096.  A pair of SMs on 256 x 256 reads half the operand
// bytes per product of one SM on 128 x 256, but fills the GPU from 74 tiles on; small tiles are bound by the 0.15 us in
// which the warps can issue 64 steps' copies and products, whatever their size (with two slices of 64 per stage; with
// one it was 0.22).
enum Shape { kPair256, kPair128, kOne256, kOne128, kOne64 };
struct ShapeCost {
    int rows, cols, per_unit, slices;       // slices: steps of 64 per stage
    double step, step_rounds, launch;
};
constexpr ShapeCost kCosts[] = {{256, 256, 2, 1, 0.32, 0.33, 5.5}, {256, 128, 2, 2, 0.166, 0.23, 4.5}, {128, 256, 1, 1, 0.34, 0.39, 4.0},
                                {128, 128, 1, 2, 0.21, 0.28, 4.2}, {128, 64, 1, 2, 0.15, 0.20, 3.6}};

struct Choice {
    Shape shape;
    int splits;
};

// The shape, and into how many parts the sum is split, with the least time by these figures.  Parts are summed by a second
// kernel (3 us, a chain of loads and the traffic of the 32-bit parts), so splitting is for results of few tiles and long sums:
// 256 x 256 results of 16384 steps took 80 us unsplit.
Choice choose(const Product &p, int sms, bool may_split, const LaunchOptions &o)
{
    if (o.test_shape && !(p.symmetric && kCosts[o.test_shape - 1].rows < kCosts[o.test_shape - 1].cols)) {
        const int stage = kBK * kCosts[o.test_shape - 1].slices, steps = int((p.k + stage - 1) / stage);
        const int k = may_split && o.test_parts ? std::min(o.test_parts, steps) : 1, per = (steps + k - 1) / k;
        return Choice{Shape(o.test_shape - 1), (steps + per - 1) / per};
    }
    Choice best{kPair256, 1};
    double least = 1e30;
    for (int s = 0; s < 5; ++s) {
        const ShapeCost &c = kCosts[s];
        const int steps = int((p.k + kBK * c.slices - 1) / (kBK * c.slices));
        if (p.symmetric && c.rows < c.cols) continue;
        const int64_t tm = (p.m + c.rows - 1) / c.rows, tn = (p.n + c.cols - 1) / c.cols;
        const int64_t tiles = (p.symmetric ? symmetric_tiles(tm, tn, c.rows / c.cols) : tm * tn) * p.batch, units = sms / c.per_unit;
        const int most = may_split && tiles < units ? int(std::min<int64_t>({units / tiles, steps * c.slices / 4, 16})) : 1;
        for (int k = 1; k <= std::max(most, 1); ++k) {
            const int per = (steps + k - 1) / k, parts = (steps + per - 1) / per;
            if (parts != k) continue;
            const int64_t waves = (tiles * k + units - 1) / units;
            double t = double(waves) * per * c.slices * (waves > 1 ? c.step_rounds : c.step) + c.launch;
            if (k > 1) t += 3.0 + 0.2 * k + double(p.m) * double(p.n) * k * 8e-6 / 4.0;
            if (t < least) {
                least = t;
                best = Choice{Shape(s), k};
            }
        }
    }
    return best;
}

template <int KIND> cudaError_t launch_shape(const Product &p, const Choice &c, const LaunchOptions &o, int device, int sms, cudaStream_t stream)
{
    switch (c.shape) {
    case kPair256: return launch<2, 256, 1, KIND>(p, c.splits, o, device, sms, stream);
    case kPair128: return launch<2, 128, 2, KIND>(p, c.splits, o, device, sms, stream);
    case kOne256: return launch<1, 256, 1, KIND>(p, c.splits, o, device, sms, stream);
    case kOne128: return launch<1, 128, 2, KIND>(p, c.splits, o, device, sms, stream);
    default: return launch<1, 64, 2, KIND>(p, c.splits, o, device, sms, stream);
    }
}

int64_t part_pitch(int64_t n) { return (n + 31) / 32 * 32; }

}  // namespace

int64_t product_scratch_bytes(const Product &p, const LaunchOptions &o)
{
    int device = 0, sms = 0;
    if (p.kind != EPI_LINEAR || p.m == 0 || p.n == 0 || current_device(&device, &sms) != cudaSuccess) return 0;
    const Choice c = choose(p, sms, true, o);
    return c.splits > 1 ? c.splits * p.m * part_pitch(p.n) * 4 : 0;
}

cudaError_t launch_product(const Product &p, void *scratch, const LaunchOptions &o, cudaStream_t stream)
{
    if (p.m == 0 || p.n == 0 || p.batch == 0) return cudaSuccess;
    int device = 0, sms = 0;
    const cudaError_t ce = current_device(&device, &sms);
    if (ce != cudaSuccess) return ce;
    if (p.kind == EPI_SCALED) return launch_shape<EPI_SCALED>(p, choose(p, sms, false, o), o, device, sms, stream);
    const Choice c = choose(p, sms, true, o);
    if (c.splits == 1) return launch_shape<EPI_LINEAR>(p, c, o, device, sms, stream);
    Product q = p;
    q.e = Epilogue{};
    q.e.out = scratch;
    q.e.ld_out = part_pitch(p.n);
    const cudaError_t parts = launch_shape<EPI_PARTIAL>(q, c, o, device, sms, stream);
    return parts != cudaSuccess ? parts : launch_join(p, static_cast<const float *>(scratch), q.e.ld_out, c.splits, o, stream);
}

cudaError_t read_product_timeouts(unsigned int *out) { return cudaMemcpyFromSymbol(out, g_product_timeouts, sizeof *out); }

}  // namespace redist
