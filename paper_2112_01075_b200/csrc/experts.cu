// Matrix products grouped by expert: ranges of rows, each with a weight of its own (out), or each summed into one (gradients).
//
// The weight's features are the tall side of a tile (128 of them per SM, on the lanes of tensor memory), an expert's rows the
// other (its columns): the tensor cores' time is proportional to the columns, so a range that ends inside a tile costs its
// own length, rounded up to 16 (32 for a pair of SMs), and a few rows read a weight no differently from many.  An expert's
// rows are cut into tiles of nearly equal width.  Blocks stay on their SM and take tiles in turn; every warp walks along the
// offsets by itself, 32 experts at a time.  The rest is that of the plain product (product.cu): TMA ring, two accumulators,
// eight storing warps, bounded waits.  Outputs leave tensor memory transposed: the fragments are turned by stmatrix.trans on
// their way to the pieces that the TMA stores; where a range ends within a piece, or a row within 16 bytes, the warp stores the
// piece itself, so neighbours' rows and elements are not touched.
// Sums over an expert's rows end in the middle of a box: every expert has tensor maps of its own, which end with its rows,
// so that what follows is read as zeros -- products with the neighbours' rows would not do: zero times their infinities.
//
// What bounds it: many rows the tensor cores and the power they may draw (32768 rows of 8 experts, 4096 -> 4096, GELU: 726 us, 1514
// TFLOP/s, pipe busy 90 % of the cycles; 857 us in runs of seconds), few rows the reading of the weights (256 rows of 64 experts, 2048
// -> 1024: 46 us, 5.8 TB/s), gradients of few rows their writing (64 of 1024 x 2048 over 256 rows: 53 us, 5.1 TB/s), and small ones
// the 6 us that a launch, the first loads and the last stores take.
#include "experts.h"

#include <cuda.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstring>

#include "activation.cuh"
#include "elements.cuh"
#include "rows.h"
#include "tensor_core.cuh"

namespace redist {

namespace {

constexpr int kThreads = 384;           // warps 0 and 3 load, warp 1 multiplies, warp 2 owns tensor memory, warps 4-11 store
constexpr int kRing = 196608;           // bytes of the ring of stages
constexpr int kPiece = 2048;            // 32 rows of 32 16-bit outputs: 64 bytes, 64-byte swizzle
constexpr int kEpiBytes = 8 * 2 * kPiece;
constexpr int kBarBytes = 256;
constexpr int kSmem = 1024 + kRing + kEpiBytes + kBarBytes;
constexpr int kMostStages = 12;
constexpr uint32_t kDrainPolls = 1 << 16, kCopyPolls = 1 << 10;         // as in the plain product

__device__ unsigned int g_grouped_timeouts = 0;

// Quotients of small numbers without a division, of which a warp's every tile would take four: a thousand cycles, in which
// neither products nor stores are under way.
struct Divider {
    uint32_t mul, shift;                // mul 0: by one
};
struct GroupedParams {
    int32_t rows, m, n, experts, k_blocks;
    int32_t tiles_m, tiles_n;           // tiles_n: SUMS only
    int32_t a_along_rows, b_along_rows;
    Divider by_group, by_matrix;        // 8 tiles_m; SUMS: tiles_m tiles_n
    uint32_t idesc, wait_polls, test_extra_tx;
    int32_t aligned_out, activation, type, run;      // run: SUMS: log2 of the tiles that a block takes one after the other
    const int32_t *offsets;
    const CUtensorMap *maps;            // SUMS: of a and b for every expert
    void *out, *pre;
    int64_t ld_out, out_batch, ld_pre, bias_stride;
    const void *bias;
    int32_t bias_type;
    ExpertSums columns;                 // computed in passing, by the warp that has nothing else to do
};

// (Plain loads: the offsets come from a kernel that may still be running when this one has begun to wait for it.)
__device__ __forceinline__ int offset_at(const GroupedParams &p, int e) { return min(max(p.offsets[e], 0), p.rows); }

// ---- tiles ---------------------------------------------------------------------------------------

// Rows of the boxes in which a tile that is not full is loaded.
template <int ROWS> constexpr int kPartRows = ROWS < 32 ? ROWS : 32;

struct GroupedTile {
    int expert, tm, row0, count, k0, steps;     // rows row0 ... row0 + count - 1 of the result (SUMS: its rows, and where its sum begins)
};

__device__ __forceinline__ int quotient(int n, const Divider &d) { return d.mul ? int(__umulhi(uint32_t(n), d.mul) >> d.shift) : n; }    // n >= 0
__device__ __forceinline__ int by_height(int n, int height)      // 1 to 8; n < 2^29
{
    if (height == 8) return n >> 3;
    if (height == 1) return n;
    return int(__umulhi(uint32_t(n), height == 2 ? 0x80000000u : height == 3 ? 0x55555556u : height == 4 ? 0x40000000u : height == 5 ? 0x33333334u
                                     : height == 6 ? 0x2aaaaaabu : 0x24924925u));
}

// A warp's walk along the tiles, in increasing order.  ROWS: lane i knows the range of expert chunk + i and how many tiles
// it has up to there.
template <int CG, int BN, int KB, bool SUMS> struct Walk {
    const GroupedParams &p;
    int chunk = -32, lane, first, step;
    int lo = 0, hi = 0, parts = 0, width = 0, through = 0, before = 0, all = 0, carry = 0;  // before: tiles of earlier chunks; all: of this one
    int expert = -1, k0 = 0, steps = 0;

    __device__ __forceinline__ Walk(const GroupedParams &params) : p(params), lane(int(threadIdx.x) & 31), first(blockIdx.x / CG), step(gridDim.x / CG) {}

    // The n-th tile of this block, if there is one; all lanes get the answer.
    __device__ __forceinline__ bool next_at(int n, GroupedTile &r)
    {
        if constexpr (SUMS) return at(((((n >> p.run) * step) + first) << p.run) + (n & ((1 << p.run) - 1)), r);
        else return at(first + n * step, r);
    }

    // The next 32 experts.  Offsets that decrease count as the largest before them.
    __device__ __forceinline__ void next()
    {
        before += all;
        chunk += 32;
        const int e = chunk + lane;
        int start = e < p.experts ? offset_at(p, e) : p.rows;
        const int end = e < p.experts ? offset_at(p, e + 1) : 0;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int up = __shfl_up_sync(0xffffffffu, start, d);
            if (lane >= d) start = max(start, up);
        }
        lo = max(start, carry);
        hi = max(lo, end);
        carry = __shfl_sync(0xffffffffu, hi, 31);
        parts = e < p.experts ? (hi - lo + BN - 1) / BN : 0;
        width = parts ? ((hi - lo + parts - 1) / parts + 16 * CG - 1) / (16 * CG) * (16 * CG) : 0;
        through = parts * p.tiles_m;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int up = __shfl_up_sync(0xffffffffu, through, d);
            if (lane >= d) through += up;
        }
        all = __shfl_sync(0xffffffffu, through, 31);
    }

    // Tile `t`, if there is one.  Tiles of an expert in groups of eight parts of the rows (SUMS: of the result's rows), so that the
    // blocks at work at one time share both operands in L2.
    __device__ __forceinline__ bool at(int t, GroupedTile &r)
    {
        if constexpr (SUMS) {
            r.expert = quotient(t, p.by_matrix);
            if (r.expert >= p.experts) return false;
            int q = t - r.expert * p.tiles_m * p.tiles_n;
            const int group = quotient(q, p.by_group), height = min(8, p.tiles_n - group * 8);
            q -= group * 8 * p.tiles_m;
            r.tm = by_height(q, height);
            r.row0 = (group * 8 + q - r.tm * height) * BN;
            r.count = min(BN, p.n - r.row0);
            if (r.expert != expert) {
                expert = r.expert;
                k0 = offset_at(p, expert);
                steps = (max(0, offset_at(p, expert + 1) - k0) + KB * kBK - 1) / (KB * kBK);
            }
            r.k0 = k0;
            r.steps = steps;
            return true;
        } else {
            while (t >= before + all) {
                if (chunk + 32 >= p.experts) return false;
                next();
            }
            const int which = __ffs(__ballot_sync(0xffffffffu, before + through > t)) - 1;
            const int from = __shfl_sync(0xffffffffu, lo, which), to = __shfl_sync(0xffffffffu, hi, which);
            const int tiles = __shfl_sync(0xffffffffu, parts, which), wide = __shfl_sync(0xffffffffu, width, which);
            int q = t - before - (__shfl_sync(0xffffffffu, through, which) - tiles * p.tiles_m);
            const int group = quotient(q, p.by_group), height = min(8, tiles - group * 8);
            q -= group * 8 * p.tiles_m;
            r.expert = chunk + which;
            r.tm = by_height(q, height);
            r.row0 = from + (group * 8 + q - r.tm * height) * wide;
            r.count = max(0, min(wide, to - r.row0));
            r.k0 = 0;
            r.steps = p.k_blocks;
            return true;
        }
    }
    // The columns that the tensor cores compute.
    static __device__ __forceinline__ int columns(const GroupedTile &r) { return max(16 * CG, (r.count + 16 * CG - 1) / (16 * CG) * (16 * CG)); }
};

// ---- epilogue --------------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t piece_at(int r, int j) { return uint32_t(r * 64 + ((j ^ ((r >> 1) & 3)) << 4)); }

// 16 lanes x 32 columns of tensor memory, as fragments: registers 4 i, 4 i + 1 are columns 8 i + 2 (lane % 4) and the next of
// row lane / 4, registers 4 i + 2, 4 i + 3 those of row lane / 4 + 8.
__device__ __forceinline__ void tmem_load_fragments(uint32_t addr, uint32_t *v)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
          "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(addr));
}
__device__ __forceinline__ void tmem_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

struct GroupedPieces {
    uint8_t *smem;
    uint32_t addr;
    int turn = 0;

    // Fills a piece -- rows are the result's rows, 32 of its columns each -- and sends it off.  v: the fragments of lanes 0-15
    // and 16-31.  `rows` of them are stored, at row0 on, or (`ends`) as many as the map has; `left`: columns up to the end of the
    // result.  The TMA writes whole 16 bytes: where a row ends within, what lies behind it would become zero (seen with 35 columns
    // 40 apart), so the warp stores such a piece itself.
    template <typename T>
    __device__ __forceinline__ void put(const float (&v)[32], const CUtensorMap *map, int aligned, bool ends, void *out, int64_t ld, int lane, int64_t row0,
                                        int rows, int col0, int left, int z, int64_t batch)
    {
        if (aligned) {
            if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
        }
        __syncwarp();
        const uint32_t to = addr + turn * kPiece;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t at = to + piece_at(8 * i + (lane & 7), lane >> 3);
            asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};"
                         ::"r"(at), "r"(pack2<T>(v[4 * i], v[4 * i + 1])), "r"(pack2<T>(v[4 * i + 2], v[4 * i + 3])),
                           "r"(pack2<T>(v[16 + 4 * i], v[16 + 4 * i + 1])), "r"(pack2<T>(v[16 + 4 * i + 2], v[16 + 4 * i + 3])) : "memory");
        }
        if (aligned && (ends || rows >= 32) && (left >= 32 || (left & 7) == 0)) {
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
                asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4}], [%1];"
                             ::"l"(map), "r"(to), "r"(col0), "r"(int(row0)), "r"(z) : "memory");
                asm volatile("cp.async.bulk.commit_group;" ::: "memory");
            }
            turn ^= 1;
            return;
        }
        __syncwarp();
        const uint8_t *piece = smem + turn * kPiece;
        T *first = static_cast<T *>(out) + z * batch + row0 * ld + col0;
        if (aligned) {
#pragma unroll
            for (int it = 0; it < 4; ++it) {
                const int r = it * 8 + (lane >> 2), j = lane & 3;
                if (r >= rows || 8 * j >= left) continue;
                const uint4 u = *reinterpret_cast<const uint4 *>(piece + piece_at(r, j));
                T *q = first + r * ld + 8 * j;
                if (8 * j + 8 <= left) {
                    *reinterpret_cast<uint4 *>(q) = u;
                } else {
                    for (int i = 0; 8 * j + i < left; ++i) q[i] = reinterpret_cast<const T *>(piece + piece_at(r, j))[i];
                }
            }
        } else {
            // Rows that start anywhere: one instruction per row, all values at hand before the first (55 gradients of 514 x 4849: 112
            // us, with a loop of loads and stores 203).  Whole blocks of 16 bytes and the rows' ends on their own are more requests
            // to L2 for the same bytes, and took longer, in pieces of 64 columns too.
            T *to = first + lane;
            if (lane < left && rows >= 32) {
                T held[32];
#pragma unroll
                for (int r = 0; r < 32; ++r) held[r] = *reinterpret_cast<const T *>(piece + piece_at(r, lane >> 3) + (lane & 7) * 2);
#pragma unroll
                for (int r = 0; r < 32; ++r, to += ld) *to = held[r];
            } else if (lane < left) {
#pragma unroll 4
                for (int r = 0; r < rows; ++r) to[r * ld] = *reinterpret_cast<const T *>(piece + piece_at(r, lane >> 3) + (lane & 7) * 2);
            }
        }
        __syncwarp();
    }
};

// The sums of the experts' rows from their parts, in the order of the rows: warp `first` of `warps`, a lane one column.
__device__ __forceinline__ void expert_sums(const ExpertSums &s, int64_t first, int64_t warps, int lane)
{
    const int64_t across = (s.cols + 31) / 32, all = across * s.experts;
    for (int64_t q = first; q < all; q += warps) {
        const int64_t e = q / across, c = (q - e * across) * 32 + lane;
        const int64_t from = min(max(int64_t(s.offsets[e]), int64_t(0)), s.rows), to = min(max(int64_t(s.offsets[e + 1]), int64_t(0)), s.rows);
        if (c >= s.cols) continue;
        float part[8] = {}, sum = 0.0f;                     // every eighth part: the order of the kernel for the sums alone
        if (from < to) {
            const int64_t last = (to - 1) / s.per + e;
            for (int64_t at = from / s.per + e; at <= last; at += 8)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (at + i <= last) part[i] += s.partials[(at + i) * s.cols + c];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += part[i];
        s.sums[e * s.cols + c] = sum;
    }
}

// ---- the kernel ------------------------------------------------------------------------------------

template <int CG, int BN, int KB, bool SUMS>
__global__ void __launch_bounds__(kThreads, 1)
redist_grouped_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_part,
                      const __grid_constant__ CUtensorMap map_out, const __grid_constant__ CUtensorMap map_pre, const __grid_constant__ GroupedParams p)
{
    constexpr int kRowsB = BN / CG, kPart = kPartRows<kRowsB>;
    constexpr int kSliceA = 128 * 128, kSliceB = kRowsB * 128, kStageA = KB * kSliceA, kStageB = KB * kSliceB, kStage = kStageA + kStageB;
    constexpr int kStages = kRing / kStage < kMostStages ? kRing / kStage : kMostStages;
    constexpr uint32_t kColumns = 2 * BN < 32 ? 32 : 2 * BN;
    static_assert(8 * (2 * kStages + 5) + 8 <= kBarBytes, "barriers, tensor memory's address and the flag");
    static_assert((kColumns & (kColumns - 1)) == 0 && kColumns <= 512, "tensor memory is allocated in powers of two");
    static_assert(!SUMS || kRowsB % 64 == 0, "operands along their rows come in boxes of 64");

    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_addr(raw) + 1023) & ~1023u;
    uint8_t *ring = raw + (base - smem_addr(raw));
    const uint32_t bars = base + kRing + kEpiBytes;
    auto full = [&](int s) { return bars + 8 * s; };
    auto empty = [&](int s) { return bars + 8 * (kStages + s); };
    auto acc_full = [&](int b) { return bars + 8 * (2 * kStages + b); };
    auto acc_free = [&](int b) { return bars + 8 * (2 * kStages + 2 + b); };
    const uint32_t drained = bars + 8 * (2 * kStages + 4);
    const uint32_t tmem_at = bars + 8 * (2 * kStages + 5);
    volatile uint32_t *tmem_word = reinterpret_cast<volatile uint32_t *>(ring + kRing + kEpiBytes + 8 * (2 * kStages + 5));
    volatile uint32_t *failed = tmem_word + 1;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = CG == 1 ? 0 : cluster_rank();

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            bar_init(full(s), 2);                           // both operands' bytes are announced
            bar_init(empty(s), 1);
        }
        for (int b = 0; b < 2; ++b) {
            bar_init(acc_full(b), 1);
            bar_init(acc_free(b), 8 * CG);
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

    using Tiles = Walk<CG, BN, KB, SUMS>;
    Tiles walk(p);
    GroupedTile at;
    bool ok = true;
    if (warp == 0 || warp == 3) {
        // Loads: warp 0 those of the features, warp 3 those of the rows.
        const bool second = warp == 3;
        int stage = 0;
        uint32_t phase = 0, rounds = 0, polls = p.wait_polls;
        const CUtensorMap *map = second ? &map_b : &map_a;
        const int along_rows = SUMS ? 1 : second ? p.b_along_rows : p.a_along_rows;
        int expert = -1;
        for (int n = 0; walk.next_at(n, at); ++n) {
            if (SUMS && at.expert != expert && at.steps) {
                expert = at.expert;
                map = p.maps + 2 * expert + second;
                asm volatile("fence.proxy.tensormap::generic.acquire.gpu [%0], 128;" ::"l"(map) : "memory");
                __syncwarp();
            }
            const int width = Tiles::columns(at) / CG, row = second ? at.row0 + int(rank) * width : (at.tm * CG + int(rank)) * 128;
            const int z = SUMS || second ? 0 : at.expert;
            // a tile that is not full takes its rows in boxes of kPart, as many as it has
            const bool part = !SUMS && second && kPart < kRowsB && width <= kRowsB - kPart;
            if (!SUMS && second) map = part ? &map_part : &map_b;
            const int boxes = along_rows ? (second ? (width + 63) / 64 : 2) : part ? (width + kPart - 1) / kPart : 1;
            const uint32_t size = along_rows ? kBK * 128 : !second ? kSliceA : part ? kPart * 128 : kSliceB;
            const uint32_t announced = CG * (KB * uint32_t(boxes) * size + (second ? 0 : p.test_extra_tx));
            for (int kb = 0; kb < at.steps; ++kb) {
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
                        const int x = at.k0 + (kb * KB + k) * kBK;
                        const uint32_t slice = to + k * (second ? kSliceB : kSliceA);
                        if (!along_rows)
                            for (int i = 0; i < boxes; ++i) load_box<CG>(slice + i * size, map, bar, x, row + i * kPart, z);
                        else
                            for (int i = 0; i < boxes; ++i) load_box<CG>(slice + i * size, map, bar, row + 64 * i, x, z);
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
        // Products.
        int stage = 0;
        uint32_t phase = 0, polls = p.wait_polls;
        int use = 0;
        const int a_along = SUMS ? 1 : p.a_along_rows, b_along = SUMS ? 1 : p.b_along_rows;
        const uint64_t desc_a = slice_desc(base, a_along), desc_b = slice_desc(base + kStageA, b_along);
        const uint64_t step_a = a_along ? 2048 >> 4 : 32 >> 4, step_b = b_along ? 2048 >> 4 : 32 >> 4;
        for (; walk.next_at(use, at); ++use) {
            const int buf = use & 1;
            if (!(CG == 1 ? bar_wait(acc_free(buf), ((use >> 1) & 1) ^ 1, polls) : bar_wait_order(acc_free(buf), ((use >> 1) & 1) ^ 1, polls))) {
                ok = false;
                polls = 1;
            }
            fence_after();
            const uint32_t acc = tmem + buf * BN, idesc = p.idesc | uint32_t(Tiles::columns(at) >> 3) << 17;
            for (int kb = 0; kb < at.steps; ++kb) {
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
                            mma<CG>(acc, da + k * (kSliceA >> 4) + i * step_a, db + k * (kSliceB >> 4) + i * step_b, idesc, kb > 0 || k + i > 0);
                    commit<CG>(empty(stage));
                    if (kb + 1 == at.steps) commit<CG>(acc_full(buf));
                }
                if (++stage == kStages) {
                    stage = 0;
                    phase ^= 1;
                }
            }
            if (at.steps == 0 && elected() && ok) commit<CG>(acc_full(buf));     // an expert without rows: zeros, not from here
        }
        if (!ok) {
            *failed = 1;
            if constexpr (CG == 2)
                asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(in_second(tmem_at + 4)), "r"(1u) : "memory");
        }
        // whatever became of the waits: what was issued reads the stages and writes tensor memory, of both blocks of a pair
        if (elected()) commit<CG>(drained);
        ok = bar_wait(drained, 0, kDrainPolls) && ok;
    } else if (warp == 2) {
        if (p.columns.sums) expert_sums(p.columns, blockIdx.x, gridDim.x, lane);
    } else if (warp >= 4) {
        // outputs: a warp has 32 features (lanes of tensor memory) and every second piece of 32 columns
        const int quarter = warp & 3, half = (warp - 4) >> 2;
        GroupedPieces pieces{ring + kRing + (warp - 4) * 2 * kPiece, base + kRing + (warp - 4) * 2 * kPiece};
        int use = 0;
        for (; walk.next_at(use, at); ++use) {
            const int b = use & 1;
            const int col0 = (at.tm * CG + int(rank)) * 128 + quarter * 32, left = p.m - col0;
            float bias[4] = {};
            if (!SUMS && p.bias) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int f = i * 8 + (lane >> 2);
                    if (f < left) bias[i] = load_any(p.bias, p.bias_type, at.expert * p.bias_stride + col0 + f);
                }
            }
            // This wait is for a whole tile's sum: the polls again for every 512 stages of it (0.4 ms at most), unless the
            // multiplying warp has given up.  One answer for the warp: what follows is for all of its lanes.
            bool ready = false;
            for (int turns = 1 + at.steps / 512; turns > 0 && !ready; --turns) {
                ready = __all_sync(0xffffffffu, bar_wait(acc_full(b), (use >> 1) & 1, p.wait_polls));
                if (!ready && __any_sync(0xffffffffu, *failed)) break;
            }
            if (!ready) {
                ok = false;
                break;
            }
            fence_after();
#pragma unroll 1
            for (int c = half * 32; c < at.count && left > 0; c += 64) {
                float v[32];
                if (at.steps) {
                    uint32_t u[32];
                    const uint32_t from = tmem + (uint32_t(quarter * 32) << 16) + b * BN + c;
                    tmem_load_fragments(from, u);
                    tmem_load_fragments(from + (16u << 16), u + 16);
                    tmem_load_wait();
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(u[i]);
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = 0.0f;
                }
                const int rows = at.count - c;
                const int64_t row0 = at.row0 + c;
                const int z = SUMS ? at.expert : 0;
                // (SUMS: a stack's map ends with each matrix, so whole boxes go out)
                auto store = [&](const CUtensorMap *map, void *out, int64_t ld) {
                    if (p.type == T_BF16) pieces.put<__nv_bfloat16>(v, map, p.aligned_out, SUMS, out, ld, lane, row0, rows, col0, left, z, p.out_batch);
                    else pieces.put<__half>(v, map, p.aligned_out, SUMS, out, ld, lane, row0, rows, col0, left, z, p.out_batch);
                };
                if constexpr (!SUMS) {
                    if (p.bias)
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] += bias[(i >> 4) * 2 + ((i >> 1) & 1)];
                    if (p.pre) store(&map_pre, p.pre, p.ld_pre);
                    activate32(v, p.activation);
                }
                store(&map_out, p.out, p.ld_out);
            }
            fence_before();
            __syncwarp();
            if (lane == 0) {
                // (relaxed: what is handed back is tensor memory, which this warp has read to the end -- see bar_wait_order.  A release to the
                // cluster waits for the stores to memory as well, 1450 cycles a tile: 64 gradients of 1024 x 1024 over 8192 rows 53 us for 38.)
                if constexpr (CG == 1)
                    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(acc_free(b)) : "memory");
                else
                    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(in_first(acc_free(b))) : "memory");
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
    // The end of the products is reported to both blocks of a pair, so the second one's memory has to last until then.  It asks now
    // that the first has seen that end: a wait from the beginning would have to be as long as all tiles together.
    const bool second = CG == 2 && rank != 0;
    bool late = false;
    if (second && warp == 1) late = !bar_wait(drained, 0, kDrainPolls);
    if (threadIdx.x == (second ? 32 : 0) && (late || *failed)) atomicAdd(&g_grouped_timeouts, 1u);
    if (warp == 2) tmem_free<CG>(tmem, kColumns);
}

// ---- before the products ----------------------------------------------------------------------------

struct PrepareParams {
    Prepare p;
    int64_t slope_per, slope_across;            // rows of a block, blocks side by side
    int64_t slope_blocks, lay_blocks[2], lay_share[2], map_blocks;      // lay_share: blocks of one matrix
    int32_t rows, experts;                      // of the maps
    const int32_t *offsets;
};

constexpr int kPrepareCols = 256;           // a warp's columns

__device__ __forceinline__ int64_t offset_in(const int32_t *offsets, int e, int64_t rows) { return min(max(int64_t(offsets[e]), int64_t(0)), rows); }

constexpr int kHeldOffsets = 512;           // of so many experts the offsets are looked up in shared memory

// A lane's eight neighbours of one row: asked for, and dz of them, stored, and as it is before it is rounded.
template <typename T, bool ALIGNED> struct SlopeRow {
    Blocks dy, z;
    __device__ __forceinline__ void load(const ExpertSlope &s, int64_t row, int64_t c, int count)
    {
        const T *from = static_cast<const T *>(s.dy) + row * s.ld_dy + c, *at = static_cast<const T *>(s.z) + row * s.ld_z + c;
        if (ALIGNED) {                                      // (the end of a row is in the same block)
            dy.a = *reinterpret_cast<const uint4 *>(from);
            if (s.z) z.a = *reinterpret_cast<const uint4 *>(at);
        } else {
            dy.load(from, count * 2);
            if (s.z) z.load(at, count * 2);
        }
    }
    __device__ __forceinline__ void take(const ExpertSlope &s, int64_t row, int64_t c, float (&v)[8]) const
    {
        uint4 u = ALIGNED ? dy.a : dy.get(static_cast<const T *>(s.dy) + row * s.ld_dy + c);
        const uint4 y = !s.z ? make_uint4(0, 0, 0, 0) : ALIGNED ? z.a : z.get(static_cast<const T *>(s.z) + row * s.ld_z + c);
        float at[8];
        const uint32_t wu[4] = {u.x, u.y, u.z, u.w}, wy[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = unpack2<T>(wu[i]), g = unpack2<T>(wy[i]);
            v[2 * i] = f.x;
            v[2 * i + 1] = f.y;
            at[2 * i] = g.x;
            at[2 * i + 1] = g.y;
        }
        if (s.z) {
            times_slope8(v, at, s.activation);
            // dz becomes an operand of two products: 16 bits, as the tensor cores take them (see the linear layer's)
            u = make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
        }
        if (s.dst) *reinterpret_cast<uint4 *>(static_cast<T *>(s.dst) + row * s.ld_dst + c) = u;
    }
};

// A block takes `per` rows by 256 columns, and within them one expert's rows after the other; a warp every eighth row, a lane
// eight neighbours.  Chunk c's sums for expert e are part c + e: both only grow, so no two share one.  SMALL: eight rows, a
// warp each, whatever their experts are (one expert after the other, each a latency of memory, 8 rows of 72 experts took 14 us).
template <typename T, bool SMALL, bool ALIGNED> __device__ __forceinline__ void slope_block(const ExpertSlope &s, int64_t chunk, int64_t column, int64_t per,
                                                                                           float (&all)[8][kPrepareCols], int32_t (&offsets)[kHeldOffsets + 1])
{
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int64_t c = column * kPrepareCols + lane * 8, lo = chunk * per, hi = min(s.rows, lo + per), cc = column * kPrepareCols + threadIdx.x;
    const int count = int(min(s.cols - c, int64_t(8)));
    const bool held = s.experts <= kHeldOffsets;            // (a chain of searches and steps: a latency of L2 each otherwise)
    if (held) {
        for (int i = threadIdx.x; i <= s.experts; i += 256) offsets[i] = int32_t(offset_in(s.offsets, i, s.rows));
        __syncthreads();
    }
    auto offset = [&](int i) { return held ? int64_t(offsets[i]) : offset_in(s.offsets, i, s.rows); };
    auto first_behind = [&](int64_t row) {                  // the first expert that ends behind it
        int e = 0;
        for (int above = s.experts; e < above;) {
            const int mid = (e + above) >> 1;
            if (offset(mid + 1) > row) above = mid;
            else e = mid + 1;
        }
        return e;
    };
    if constexpr (SMALL) {
        __shared__ int32_t owner[8];
        const int64_t row = lo + w;
        int e = row < hi ? first_behind(row) : s.experts;
        if (e < s.experts && offset(e) > row) e = s.experts;
        float v[8] = {};
        if (e < s.experts && count > 0) {
            SlopeRow<T, ALIGNED> one;
            one.load(s, row, c, count);
            one.take(s, row, c, v);
        }
        if (!s.partials) return;
#pragma unroll
        for (int i = 0; i < 8; ++i) all[w][lane * 8 + i] = v[i];
        if (lane == 0) owner[w] = e;
        __syncthreads();
        if (cc >= s.cols) return;
        float sum = 0.0f;
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            const int here = owner[r];
            sum += all[r][threadIdx.x];
            if (here < s.experts && (r == 7 || owner[r + 1] != here)) s.partials[(chunk + here) * s.cols + cc] = sum;
            if (r == 7 || owner[r + 1] != here) sum = 0.0f;
        }
        return;
    }
    for (int e = first_behind(lo); e < s.experts; ++e) {
        const int64_t begin = offset(e), from = max(lo, begin), to = min(hi, offset(e + 1));
        if (begin >= hi) break;
        if (from >= to) continue;
        float sums[8] = {};
        SlopeRow<T, ALIGNED> next;                          // a row ahead
        if (count > 0 && from + w < to) next.load(s, from + w, c, count);
        if (count > 0)
            for (int64_t row = from + w; row < to; row += 8) {
                float v[8];
                const SlopeRow<T, ALIGNED> now = next;
                if (row + 8 < to) next.load(s, row + 8, c, count);
                now.take(s, row, c, v);
#pragma unroll
                for (int i = 0; i < 8; ++i) sums[i] += v[i];
            }
        if (!s.partials) continue;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) all[w][lane * 8 + i] = sums[i];
        __syncthreads();
        if (cc < s.cols) {
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += all[i][threadIdx.x];
            s.partials[(chunk + e) * s.cols + cc] = sum;
        }
    }
}

// The matrix that a group of blocks lays out: of experts only those that have rows (-1: none).  By row, where rows are fewer than
// experts: the expert whose first row is `slot`, so that the idle ones need no blocks.
__device__ __forceinline__ int64_t matrix_of(const StackLay &l, int64_t slot)
{
    if (!l.offsets) return slot;
    if (!l.by_row) return l.offsets[slot + 1] > l.offsets[slot] ? slot : -1;
    const int lane = threadIdx.x & 31, experts = int(l.count);
    uint32_t next = uint32_t(experts) + 1;                  // the first offset beyond the row: where its expert ends
    for (int i = lane; i <= experts && next > uint32_t(experts); i += 32)
        if (l.offsets[i] > slot) next = uint32_t(i);
    const int e = int(__reduce_min_sync(0xffffffffu, next)) - 1;
    if (e < 0 || e >= experts) return -1;
    int most = 0;
    for (int i = lane; i <= e; i += 32) most = max(most, l.offsets[i]);
    return __reduce_max_sync(0xffffffffu, most) == slot ? e : -1;
}

// Lines of up to 256 columns: a warp takes as many as fill it, twice; longer ones one at a time, four stretches of 256 columns
// under way.
constexpr int kShortLines = 2;
__host__ __device__ __forceinline__ int lay_lanes(int64_t line)       // of a line of up to 256 columns
{
    int lanes = 32;
    while (lanes > 1 && (lanes / 2) * 8 >= line) lanes /= 2;
    return lanes;
}

// Block `block` of the `blocks` that share a matrix.
__device__ __forceinline__ void lay_block(const StackLay &l, int64_t matrix, int64_t block, int64_t blocks)
{
    if (matrix < 0) return;
    const uint16_t *from = static_cast<const uint16_t *>(l.src) + matrix * l.plane_src;
    uint16_t *to = static_cast<uint16_t *>(l.dst) + matrix * l.plane_dst;
    const int lane = threadIdx.x & 31;
    const int64_t first = block * 8 + (threadIdx.x >> 5), step = blocks * 8;
    if (l.line > kPrepareCols) {
        constexpr int kAhead = 4;
        for (int64_t line = first; line < l.lines; line += step) {
            const uint16_t *src = from + line * l.ld_src;
            uint16_t *dst = to + line * l.ld_dst;
            for (int64_t c = lane * 8; c < l.line; c += kAhead * kPrepareCols) {
                Blocks b[kAhead];
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {
                    const int64_t count = min(l.line - c - i * kPrepareCols, int64_t(8));
                    if (count > 0) b[i].load(src + c + i * kPrepareCols, int(count) * 2);
                }
#pragma unroll
                for (int i = 0; i < kAhead; ++i)
                    if (c + i * kPrepareCols < l.line) *reinterpret_cast<uint4 *>(dst + c + i * kPrepareCols) = b[i].get(src + c + i * kPrepareCols);
            }
        }
        return;
    }
    const int lanes = lay_lanes(l.line), group = 32 / lanes, c = lane % lanes * 8, turn = kShortLines * group;
    if (c >= l.line) return;
    for (int64_t line0 = first * turn + lane / lanes; line0 < l.lines; line0 += step * turn) {
        Blocks b[kShortLines];
#pragma unroll
        for (int i = 0; i < kShortLines; ++i)
            if (line0 + i * group < l.lines) b[i].load(from + (line0 + i * group) * l.ld_src + c, int(min(l.line - c, int64_t(8))) * 2);
#pragma unroll
        for (int i = 0; i < kShortLines; ++i)
            if (line0 + i * group < l.lines)
                *reinterpret_cast<uint4 *>(to + (line0 + i * group) * l.ld_dst + c) = b[i].get(from + (line0 + i * group) * l.ld_src + c);
    }
}

// The maps of every expert's rows: copies of two that end with its last row.  A warp makes one.
__device__ __forceinline__ void map_block(const PrepareParams &p, const CUtensorMap &map_a, const CUtensorMap &map_b, int64_t block)
{
    const int lane = int(threadIdx.x) & 31;
    const int64_t which = block * 8 + (threadIdx.x >> 5), e = which >> 1;
    if (e >= p.experts) return;
    const int64_t lo = offset_in(p.offsets, int(e), p.rows), hi = offset_in(p.offsets, int(e) + 1, p.rows);
    if (hi <= lo) return;                                   // never used
    CUtensorMap *to = static_cast<CUtensorMap *>(p.p.maps) + which;
    const uint32_t *from = reinterpret_cast<const uint32_t *>(which & 1 ? &map_b : &map_a);
    reinterpret_cast<uint32_t *>(to)[lane] = from[lane];
    __threadfence();
    __syncwarp();
    if (lane == 0) {
        asm volatile("tensormap.replace.tile.global_dim.global.b1024.b32 [%0], 1, %1;" ::"l"(to), "r"(int(hi)) : "memory");
        asm volatile("fence.proxy.tensormap::generic.release.gpu;" ::: "memory");
    }
}

// Each of the four has blocks of its own: what these small works cost is mostly a launch.
template <typename T, bool SMALL, bool ALIGNED> __global__ void __launch_bounds__(256, 4)
redist_expert_prepare_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ PrepareParams p)
{
    __shared__ float all[8][kPrepareCols];
    __shared__ int32_t offsets[kHeldOffsets + 1];
    let_next_start();
    wait_for_previous();
    int64_t b = blockIdx.x;
    if (b < p.slope_blocks) {
        slope_block<T, SMALL, ALIGNED>(p.p.slope, b / p.slope_across, b % p.slope_across, p.slope_per, all, offsets);
        return;
    }
    b -= p.slope_blocks;
    if (b < p.lay_blocks[0]) return lay_block(p.p.lay[0], matrix_of(p.p.lay[0], b / p.lay_share[0]), b % p.lay_share[0], p.lay_share[0]);
    b -= p.lay_blocks[0];
    if (b < p.lay_blocks[1]) return lay_block(p.p.lay[1], matrix_of(p.p.lay[1], b / p.lay_share[1]), b % p.lay_share[1], p.lay_share[1]);
    map_block(p, map_a, map_b, b - p.lay_blocks[1]);
}

// The sums on their own: eight warps share the parts of 32 columns.
__global__ void __launch_bounds__(256) redist_expert_sums_kernel(const ExpertSums s)
{
    __shared__ float all[8][32];
    let_next_start();
    wait_for_previous();
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, e = blockIdx.y;
    const int64_t c = int64_t(blockIdx.x) * 32 + lane, from = offset_in(s.offsets, e, s.rows), to = offset_in(s.offsets, e + 1, s.rows);
    float sum = 0.0f;
    if (from < to && c < s.cols) {
        const int64_t last = (to - 1) / s.per + e;
#pragma unroll 4
        for (int64_t part = from / s.per + e + w; part <= last; part += 8) sum += s.partials[part * s.cols + c];
    }
    all[w][lane] = sum;
    __syncthreads();
    if (w == 0 && c < s.cols) {
        sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += all[i][lane];
        s.sums[e * s.cols + c] = sum;
    }
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

// A map of `depth` arrays of `lines` lines of `line` 16-bit elements, taken in boxes of box_lines x box_line.
bool make_map(CUtensorMap *map, const void *data, int64_t line, int64_t lines, int64_t depth, int64_t ld, int64_t plane, int box_line, int box_lines,
              CUtensorMapSwizzle swizzle, CUtensorMapL2promotion promotion)
{
    EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    const cuuint64_t dims[3] = {cuuint64_t(line), cuuint64_t(lines), cuuint64_t(depth)};
    // strides that are never used: any legal value does
    const int64_t pitch = lines > 1 ? ld : (line + 7) / 8 * 8, apart = depth > 1 ? plane : pitch;
    const cuuint64_t strides[2] = {cuuint64_t(pitch) * 2, cuuint64_t(apart) * 2};
    const cuuint32_t box[3] = {cuuint32_t(box_line), cuuint32_t(box_lines), 1}, one[3] = {1, 1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 3, const_cast<void *>(data), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                  promotion, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool make_operand(CUtensorMap *map, const Operand &op, int64_t rows, int64_t cols, int64_t depth, int box_rows)
{
    return make_map(map, op.data, op.along_rows ? rows : cols, op.along_rows ? cols : rows, depth, op.ld, op.batch_stride, kBK, op.along_rows ? kBK : box_rows,
                    CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
}

bool make_result(CUtensorMap *map, void *data, int64_t rows, int64_t cols, int64_t depth, int64_t ld, int64_t plane)
{
    return make_map(map, data, cols, rows, depth, ld, plane, 32, 32, CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE);
}

bool on_16(const void *p, int64_t ld) { return p == nullptr || (uintptr_t(p) % 16 == 0 && ld % 8 == 0); }

template <typename... P, typename... A>
cudaError_t launch_any(void (*kernel)(P...), dim3 grid, int threads, int smem, int cluster, const LaunchOptions &o, cudaStream_t stream, const A &...args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(unsigned(threads));
    cfg.dynamicSmemBytes = size_t(smem);
    cfg.stream = stream;
    cudaLaunchAttribute at[2];
    int n_at = 0;
    if (cluster > 1) {
        at[n_at].id = cudaLaunchAttributeClusterDimension;
        at[n_at].val.clusterDim.x = unsigned(cluster);
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
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// The smallest power of two that makes the quotient exact for numerators below 2^31.
Divider divider(int64_t d)
{
    if (d <= 1) return Divider{0, 0};
    int lg = 0;
    while ((int64_t(1) << lg) < d) ++lg;
    return Divider{uint32_t(((uint64_t(1) << (31 + lg)) + uint64_t(d) - 1) / uint64_t(d)), uint32_t(lg - 1)};
}

template <int CG, int BN, int KB, bool SUMS>
cudaError_t launch(const Grouped &g, void *scratch, ExpertSums *columns, const LaunchOptions &o, int device, int sms, cudaStream_t stream)
{
    GroupedParams p;
    std::memset(&p, 0, sizeof p);
    p.rows = int32_t(g.rows);
    p.m = int32_t(g.m);
    p.n = int32_t(g.n);
    p.experts = g.experts;
    p.k_blocks = SUMS ? 0 : int32_t((g.k + KB * kBK - 1) / (KB * kBK));
    p.tiles_m = int32_t((g.m + 128 * CG - 1) / (128 * CG));
    p.tiles_n = SUMS ? int32_t((g.n + BN - 1) / BN) : 0;
    p.a_along_rows = g.a.along_rows;
    p.b_along_rows = g.b.along_rows;
    const uint32_t format = g.type == T_BF16 ? 1 : 0;
    // 32-bit accumulators, operand types, operand orders, tile height / 16; the kernel adds the tile's width / 8
    p.idesc = (1u << 4) | (format << 7) | (format << 10) | (uint32_t(g.a.along_rows) << 15) | (uint32_t(g.b.along_rows) << 16) |
              (uint32_t(128 * CG >> 4) << 24);
    p.wait_polls = o.wait_polls;
    p.test_extra_tx = o.test_extra_tx;
    p.activation = g.activation;
    p.type = g.type;
    p.offsets = g.offsets;
    p.maps = static_cast<const CUtensorMap *>(scratch);
    p.out = g.out;
    p.pre = g.pre;
    p.ld_out = g.ld_out;
    p.out_batch = g.out_batch;
    p.ld_pre = g.ld_pre;
    p.bias = g.bias;
    p.bias_type = g.bias_type;
    p.bias_stride = g.bias_stride;
    p.aligned_out = on_16(g.out, g.ld_out) && (!SUMS || g.experts == 1 || g.out_batch % 8 == 0) && on_16(g.pre, g.ld_pre);

    // a bound on the tiles: every expert with rows has at most one that is not full
    const int64_t parts = SUMS ? int64_t(p.tiles_n) * g.experts : std::min<int64_t>(g.experts, g.rows) + g.rows / BN;
    const int64_t tiles = parts * p.tiles_m;
    if (tiles > INT32_MAX / 8 || int64_t(p.tiles_m) * 8 >= INT32_MAX / 8) return cudaErrorInvalidValue;
    p.by_group = divider(int64_t(p.tiles_m) * 8);
    p.by_matrix = divider(int64_t(p.tiles_m) * std::max(p.tiles_n, 1));

    CUtensorMap ma, mb, ms, mo, mp;
    const int64_t features = SUMS ? g.n : g.rows, sum = SUMS ? g.rows : g.k;
    if (!make_operand(&ma, g.a, g.m, sum, SUMS ? 1 : g.experts, 128) || !make_operand(&mb, g.b, features, sum, 1, BN / CG) ||
        !make_operand(&ms, g.b, features, sum, 1, kPartRows<BN / CG>))
        return cudaErrorInvalidValue;
    std::memset(&mo, 0, sizeof mo);
    std::memset(&mp, 0, sizeof mp);
    if (p.aligned_out) {
        if (!make_result(&mo, g.out, features, g.m, SUMS ? g.experts : 1, g.ld_out, g.out_batch)) return cudaErrorInvalidValue;
        if (g.pre && !make_result(&mp, g.pre, features, g.m, 1, g.ld_pre, 0)) return cudaErrorInvalidValue;
    }
    auto *kernel = redist_grouped_kernel<CG, BN, KB, SUMS>;
    static std::atomic<uint64_t> ready{0};                  // devices on which this kernel may use its shared memory
    if (device >= 64 || !(ready.load(std::memory_order_relaxed) >> device & 1)) {
        const cudaError_t ce = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
        if (ce != cudaSuccess) return ce;
        if (device < 64) ready.fetch_or(uint64_t(1) << device, std::memory_order_relaxed);
    }
    const int64_t groups = sms / CG;
    const unsigned blocks = unsigned(std::min(tiles, groups) * CG);
    // The sums of 32 columns of an expert take two latencies of memory and one for every eight of its parts; a product computes them
    // in passing where that hides behind its tiles (8192 x 1024 -> 1024 of 64 experts with 14 such groups a block: 97 us, with a
    // launch for them 89; 832 x 96 <- 865 of 7 with 7 of them: 21 us for the product, 7 alone).
    const double share = columns ? std::ceil(double((columns->cols + 31) / 32) * columns->experts / blocks) : 0;
    const double rows = columns ? double(columns->rows) / std::min<int64_t>(columns->experts, columns->rows) : 0;
    const double passing = columns ? share * (1.2 + 0.6 * std::ceil(1.5 * rows / double(columns->per) / 8)) : 0;
    const double own = 4 + 0.2 * std::ceil(double(tiles) / double(groups)) * (SUMS ? std::ceil(rows / 64) : double(g.k) / 64);
    if (columns && columns->sums && passing <= own) {
        p.columns = *columns;
        columns->sums = nullptr;                            // done
    }
    // Every other expert costs the loading warps a fence and the fetch of a tensor map: where sums are short, blocks take a few
    // tiles of one expert after the other (64 gradients of 1024 x 2048 over 256 rows: 56 -> 53 us on pairs, 70 -> 65 on single SMs;
    // more of them leave SMs idle at the end).
    if (SUMS) {
        const int64_t steps = std::max<int64_t>(1, g.rows / g.experts / kBK);
        while (p.run < (CG == 2 ? 1 : 3) && (steps << p.run) < 4 && (groups << (p.run + 1)) <= tiles) ++p.run;
    }
    return launch_any(kernel, dim3(blocks), kThreads, kSmem, CG, o, stream, ma, mb, ms, mo, mp, p);
}

// The tile shapes, and what they take: microseconds per 64 steps of a sum, `step` + `column` per column computed (at least
// `least`; three quarters where all tiles fit on the GPU at once), but at least `tile` a tile (its stores), and per launch
// besides.  Fitted to timings of some twenty sizes from 500 x 512 -> 512 to 32768 x 4096 -> 4096.
enum GroupedShape { kPair256, kPair128, kOne32, kOne128, kOne64 };
struct GroupedCost {
    int rows, cols, per_unit;
    double step, column, least, tile, launch;
};
constexpr GroupedCost kGroupedCosts[] = {{256, 256, 2, 0.044, 0.00147, 0.18, 1.6, 5.5}, {256, 128, 2, 0.044, 0.00147, 0.18, 1.0, 4.5}, {128, 32, 1, 0.185, 0.00066, 0, 0.5, 3.4},
                                         {128, 128, 1, 0.185, 0.00066, 0, 1.05, 4.2}, {128, 64, 1, 0.185, 0.00066, 0, 0.75, 3.6}};

// The shape with the least time by these figures, or the one that computes least where memory sets the time.  How the rows
// are spread over the experts is not known here: what a busy expert has is taken as one and a half times the mean.
GroupedShape choose(const Grouped &g, int sms, const LaunchOptions &o)
{
    if (o.test_shape) return GroupedShape(o.test_shape - 1);
    const double busy = double(std::min<int64_t>(g.experts, g.rows)), rows = 1.5 * double(g.rows) / busy;
    const double bytes = 2.0 * (double(g.sums ? g.experts : busy) * double(g.m) * double(g.sums ? g.n : g.k) + double(g.rows) * double(g.m + (g.sums ? g.n : g.k)));
    GroupedShape best = kPair256;
    double least = 1e30;
    for (int i = 0; i < 5; ++i) {
        const GroupedCost &c = kGroupedCosts[i];
        if (g.sums && c.cols < 64) continue;
        const double features = std::ceil(double(g.m) / c.rows), cols = g.sums ? double(g.n) : rows, per = std::ceil(cols / c.cols);
        const double tiles = features * per * (g.sums ? g.experts : busy), units = double(sms / c.per_unit);
        const double steps = std::ceil((g.sums ? double(g.rows) / g.experts : double(g.k)) / 64), waves = tiles <= units ? 0.75 : tiles / units + 0.5;
        const double compute = waves * std::max(steps * std::max(c.least, c.step + c.column * cols / per), c.tile), time = c.launch + std::max(compute, bytes / 6.5e6) + 0.1 * compute;
        if (time < least) {
            least = time;
            best = GroupedShape(i);
        }
    }
    return best;
}

}  // namespace

int64_t grouped_maps_bytes(int experts) { return int64_t(experts) * 2 * int64_t(sizeof(CUtensorMap)); }

cudaError_t launch_grouped(const Grouped &g, void *scratch, ExpertSums *columns, const LaunchOptions &o, cudaStream_t stream)
{
    if (!g.sums && g.rows == 0) return cudaSuccess;
    int device = 0, sms = 0;
    const cudaError_t ce = current_device(&device, &sms);
    if (ce != cudaSuccess) return ce;
    if (g.sums) {
        switch (choose(g, sms, o)) {
        case kPair256: return launch<2, 256, 1, true>(g, scratch, columns, o, device, sms, stream);
        case kPair128: return launch<2, 128, 2, true>(g, scratch, columns, o, device, sms, stream);
        case kOne128: return launch<1, 128, 2, true>(g, scratch, columns, o, device, sms, stream);
        default: return launch<1, 64, 2, true>(g, scratch, columns, o, device, sms, stream);
        }
    }
    switch (choose(g, sms, o)) {
    case kPair256: return launch<2, 256, 1, false>(g, scratch, columns, o, device, sms, stream);
    case kPair128: return launch<2, 128, 2, false>(g, scratch, columns, o, device, sms, stream);
    case kOne32: return launch<1, 32, 2, false>(g, scratch, columns, o, device, sms, stream);
    case kOne128: return launch<1, 128, 2, false>(g, scratch, columns, o, device, sms, stream);
    default: return launch<1, 64, 2, false>(g, scratch, columns, o, device, sms, stream);
    }
}

cudaError_t launch_expert_sums(const ExpertSums &s, const LaunchOptions &o, cudaStream_t stream)
{
    return launch_any(redist_expert_sums_kernel, dim3(unsigned((s.cols + 31) / 32), unsigned(s.experts)), 256, 0, 1, o, stream, s);
}

// Rows of a block of the slope: as few as keep four blocks on each of 148 SMs (written here because scratch is asked for by
// sizes alone), 8 to 128, more where the grid would grow beyond its limit.
int64_t slope_rows(int64_t rows, int64_t cols)
{
    int64_t per = 128 * ((rows + 128 * 32768 - 1) / (128 * 32768));
    while (per > 8 && ((rows + per - 1) / per) * ((cols + kPrepareCols - 1) / kPrepareCols) < 4 * 148) per /= 2;
    return per;
}

int64_t expert_partial_bytes(int64_t rows, int64_t cols, int experts)
{
    const int64_t per = slope_rows(rows, cols);
    return ((rows + per - 1) / per + experts) * cols * 4;
}

cudaError_t launch_prepare(const Prepare &p, const LaunchOptions &o, cudaStream_t stream)
{
    PrepareParams q;
    std::memset(static_cast<void *>(&q), 0, sizeof q);
    q.p = p;
    if (p.slope.dy && p.slope.rows > 0) {
        q.slope_per = slope_rows(p.slope.rows, p.slope.cols);
        q.slope_across = (p.slope.cols + kPrepareCols - 1) / kPrepareCols;
        q.slope_blocks = (p.slope.rows + q.slope_per - 1) / q.slope_per * q.slope_across;
    }
    for (int i = 0; i < 2; ++i)
        if (p.lay[i].dst) {
            // a turn for each warp: there are more blocks than fit at once, and a warp's turn hides little
            StackLay &l = q.p.lay[i];
            const int64_t turn = l.line > kPrepareCols ? 1 : kShortLines * (32 / lay_lanes(l.line));
            l.by_row = l.offsets && l.rows < l.count && l.count <= 4096;        // (every block looks through the offsets then)
            const int64_t slots = l.by_row ? l.rows : l.count;
            q.lay_share[i] = std::max<int64_t>(1, std::min<int64_t>((l.lines + 8 * turn - 1) / (8 * turn), (int64_t(1) << 22) / slots));
            q.lay_blocks[i] = slots * q.lay_share[i];
        }
    CUtensorMap ma, mb;
    std::memset(&ma, 0, sizeof ma);
    std::memset(&mb, 0, sizeof mb);
    if (p.sums) {
        const Grouped &g = *p.sums;
        if (!make_operand(&ma, g.a, g.m, g.rows, 1, 128) || !make_operand(&mb, g.b, g.n, g.rows, 1, 128)) return cudaErrorInvalidValue;
        q.rows = int32_t(g.rows);
        q.experts = g.experts;
        q.offsets = g.offsets;
        q.map_blocks = (int64_t(g.experts) * 2 + 7) / 8;
    }
    const int64_t blocks = q.slope_blocks + q.lay_blocks[0] + q.lay_blocks[1] + q.map_blocks;
    if (blocks == 0) return cudaSuccess;
    if (blocks > INT32_MAX) return cudaErrorInvalidValue;
    const dim3 grid = dim3(unsigned(blocks));
    const bool aligned = on_16(p.slope.dy, p.slope.ld_dy) && on_16(p.slope.z, p.slope.ld_z), small = q.slope_per == 8;
    auto go = [&](auto t) {
        using T = decltype(t);
        if (small) return aligned ? launch_any(redist_expert_prepare_kernel<T, true, true>, grid, 256, 0, 1, o, stream, ma, mb, q)
                                  : launch_any(redist_expert_prepare_kernel<T, true, false>, grid, 256, 0, 1, o, stream, ma, mb, q);
        return aligned ? launch_any(redist_expert_prepare_kernel<T, false, true>, grid, 256, 0, 1, o, stream, ma, mb, q)
                       : launch_any(redist_expert_prepare_kernel<T, false, false>, grid, 256, 0, 1, o, stream, ma, mb, q);
    };
    return p.type == T_BF16 ? go(__nv_bfloat16()) : go(__half());
}

cudaError_t read_grouped_timeouts(unsigned int *out) { return cudaMemcpyFromSymbol(out, g_grouped_timeouts, sizeof *out); }

}  // namespace redist
