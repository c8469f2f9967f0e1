// Layer norm and the preparation of operands: kernels bound by the memory they stream over.
#include "rows.h"

#include <algorithm>
#include <type_traits>

#include "activation.cuh"
#include "elements.cuh"

namespace redist {

namespace {

// ---- helpers -----------------------------------------------------------------------------------------

template <typename T> constexpr int kVec = 16 / int(sizeof(T));          // neighbours in 16 bytes

template <typename T> __device__ __forceinline__ void unpack16(const uint4 &u, float *v)
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

template <typename T> __device__ __forceinline__ uint4 pack16(const float *v)
{
    if constexpr (sizeof(T) == 4)
        return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    else
        return make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
}

// Bytes 4 WORD (+ 2 with `half`) ... of two consecutive 16-byte blocks, 16 of them.
template <int WORD> __device__ __forceinline__ uint4 join16(const uint4 &a, const uint4 &b, bool half)
{
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    if (!half) return make_uint4(w[WORD], w[WORD + 1], w[WORD + 2], w[WORD + 3]);
    return make_uint4(__funnelshift_r(w[WORD], w[WORD + 1], 16), __funnelshift_r(w[WORD + 1], w[WORD + 2], 16),
                      __funnelshift_r(w[WORD + 2], w[WORD + 3], 16), __funnelshift_r(w[WORD + 3], w[WORD + 4], 16));
}

// NV pieces of 16 bytes of shared memory, `pitch` bytes apart, each from byte `off` (even, below 16) on.  All threads of a
// row have the same offset: the branches hardly ever diverge, and whole blocks are read, where single words would meet in
// the same banks.
template <int NV> __device__ __forceinline__ void read_any(const uint8_t *p, int pitch, uint32_t off, uint4 (&u)[NV])
{
    const bool half = off & 2;
    auto all = [&](auto word) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const uint4 *q = reinterpret_cast<const uint4 *>(p + j * pitch);
            u[j] = join16<decltype(word)::value>(q[0], q[1], half);
        }
    };
    if (off == 0) {
#pragma unroll
        for (int j = 0; j < NV; ++j) u[j] = *reinterpret_cast<const uint4 *>(p + j * pitch);
    } else if (off < 4) {
        all(std::integral_constant<int, 0>());
    } else if (off < 8) {
        all(std::integral_constant<int, 1>());
    } else if (off < 12) {
        all(std::integral_constant<int, 2>());
    } else {
        all(std::integral_constant<int, 3>());
    }
}

// L threads share a row; a thread holds NV pieces of 16 bytes of it.  The threads of a row that share a warp form a
// segment, which has NV x kSegment consecutive pieces; piece j of a thread is its segment's (j kSegment + at)-th.
template <typename T, int L, int NV> struct RowShape {
    static constexpr int VEC = kVec<T>;
    static constexpr int kThreads = L < 256 ? 256 : L;
    static constexpr int kRows = kThreads / L;              // rows a block holds at a time
    static constexpr int kSegment = L < 32 ? L : 32;
    static __device__ __forceinline__ int column(int j)     // where a thread's piece begins
    {
        const int t = int(threadIdx.x) % L;
        return ((t / kSegment * NV + j) * kSegment + t % kSegment) * VEC;
    }
};

// Rows on their way to the registers: every thread copies its own pieces of the next rows into shared memory
// (cp.async: no registers, no barrier) and takes them out again in turn.  SHIFT: rows start anywhere.  Then a thread copies
// the aligned blocks in which its pieces begin, the last one of a segment (or of the row) the block after that too, and
// pieces are read from shared memory at their own offset.  A slot that was taken also serves to shift a row of outputs.
template <typename T, int L, int NV, int TENSORS, bool SHIFT> struct Stream {
    using S = RowShape<T, L, NV>;
    static constexpr int VEC = S::VEC, SEGMENT = S::kSegment;
    static constexpr int kBlocks = S::kThreads / SEGMENT * (NV * SEGMENT + (SHIFT ? 1 : 0));     // of one row of one tensor
    // three rows ahead, or as many as leave room for two blocks per SM (one at least)
    static constexpr int kFit = 100 * 1024 / (TENSORS * kBlocks * 16), kSlots = kFit >= 4 ? 4 : kFit >= 3 ? 3 : 2, kAhead = kSlots - 1;
    static constexpr int kPad = SHIFT ? 128 : 0;            // the block before the first is read, though not used
    static constexpr int kSmem = kPad + kSlots * TENSORS * kBlocks * 16;
    uint8_t *mine;                  // this thread's first block in the first slot
    int put = 0, got = 0;
    bool last;

    __device__ __forceinline__ Stream(uint8_t *smem)
    {
        const int segment = int(threadIdx.x) / SEGMENT, at = int(threadIdx.x) % SEGMENT;
        mine = smem + kPad + (segment * (NV * SEGMENT + (SHIFT ? 1 : 0)) + at) * 16;
        last = at == SEGMENT - 1;
    }
    __device__ __forceinline__ uint8_t *place(int slot, int tensor, int piece) const
    {
        return mine + ((slot * TENSORS + tensor) * kBlocks + piece * SEGMENT) * 16;
    }

    // base[i]: this thread's first piece in tensor i's row; in == false: no such row
    __device__ __forceinline__ void send(const T *const (&base)[TENSORS], bool in, const int (&count)[NV])
    {
#pragma unroll
        for (int i = 0; i < TENSORS; ++i) {
            const uint32_t off = SHIFT ? uint32_t(reinterpret_cast<uintptr_t>(base[i]) & 15) : 0;
            const char *block = reinterpret_cast<const char *>(base[i]) - off;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                if (!in || count[j] <= 0) continue;
                const uint32_t to = uint32_t(__cvta_generic_to_shared(place(put, i, j)));
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(block + j * SEGMENT * 16) : "memory");
                if constexpr (SHIFT)        // the next block, if this piece reaches into it and nobody else brings it
                    if (((j == NV - 1 && last) || count[j] <= VEC) && off + uint32_t(min(count[j], VEC)) * uint32_t(sizeof(T)) > 16)
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + 16), "l"(block + j * SEGMENT * 16 + 16) : "memory");
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        put = put + 1 == kSlots ? 0 : put + 1;
    }

    // The oldest row sent for (kAhead more are under way); zero beyond the row's end.
    __device__ __forceinline__ void take(const T *const (&base)[TENSORS], const int (&count)[NV], float (&v)[TENSORS][NV][VEC])
    {
        asm volatile("cp.async.wait_group %0;" ::"n"(kAhead) : "memory");
        if constexpr (SHIFT) __syncwarp();
#pragma unroll
        for (int i = 0; i < TENSORS; ++i) {
            uint4 u[NV];
            read_any<NV>(place(got, i, 0), SEGMENT * 16, SHIFT ? uint32_t(reinterpret_cast<uintptr_t>(base[i]) & 15) : 0, u);
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                unpack16<T>(u[j], v[i][j]);
                if (count[j] < VEC)
#pragma unroll
                    for (int q = 0; q < VEC; ++q)
                        if (q >= count[j]) v[i][j][q] = 0.0f;
            }
        }
        if constexpr (SHIFT) __syncwarp();                  // the slot may be written again
        got = got + 1 == kSlots ? 0 : got + 1;
    }

    // Stores a row of outputs; `to`: this thread's first piece.  SHIFT: the pieces go through the slot just taken, from
    // which a thread reads the aligned block that ends in its piece, its beginning from the thread before; what no whole
    // block of a segment covers goes out one by one.
    __device__ __forceinline__ void store(T *to, bool in, const int (&count)[NV], const float (&v)[NV][VEC])
    {
        const int q = SHIFT ? int(reinterpret_cast<uintptr_t>(to) & 15) / int(sizeof(T)) : 0;
        const int slot = got == 0 ? kSlots - 1 : got - 1;
        uint4 blocks[NV];
        if constexpr (SHIFT) {
#pragma unroll
            for (int j = 0; j < NV; ++j) *reinterpret_cast<uint4 *>(place(slot, 0, j)) = pack16<T>(v[j]);
            __syncwarp();
            // (what a segment's first piece reads before itself it does not use)
            read_any<NV>(place(slot, 0, 0) - (q ? 16 : 0), SEGMENT * 16, q ? uint32_t(16 - q * int(sizeof(T))) : 0, blocks);
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            T *p = to + j * SEGMENT * VEC;
            if constexpr (!SHIFT) {
                if (!in) continue;
                if (count[j] >= VEC) {
                    *reinterpret_cast<uint4 *>(p) = pack16<T>(v[j]);
                } else {
#pragma unroll
                    for (int i = 0; i < VEC; ++i)
                        if (i < count[j]) p[i] = from_float<T>(v[j][i]);
                }
            } else {
                const bool head = j == 0 && int(threadIdx.x) % SEGMENT == 0, tail = j == NV - 1 && last;
                const uint8_t *at = place(slot, 0, j);
                const bool whole = in && (!head || q == 0) && count[j] >= VEC - q;
                if (whole) *reinterpret_cast<uint4 *>(p - q) = blocks[j];
                // one by one: my first VEC - q where there is no whole block, my last q where the next piece has none
                const uint32_t front = (1u << (VEC - q)) - 1, all = (1u << VEC) - 1;
                uint32_t rest = 0;
                if (in && count[j] > 0) {
                    rest = (whole ? 0 : front) | (tail || count[j] - VEC < VEC - q ? all & ~front : 0);
                    if (count[j] < VEC) rest &= (1u << count[j]) - 1;
                }
                if (rest) {
#pragma unroll
                    for (int i = 0; i < VEC; ++i)
                        if (rest >> i & 1) p[i] = reinterpret_cast<const T *>(at)[i];
                }
            }
        }
        if constexpr (SHIFT) __syncwarp();
    }
};

// Sums over the L threads that share a row; every thread gets them.  L > 32: `slot` has two entries per warp of the block
// and may be written again after one more barrier of the row's threads.
template <int L> __device__ __forceinline__ void row_barrier()
{
    if constexpr (L < 256) asm volatile("bar.sync %0, %1;" ::"r"(1 + (int(threadIdx.x) >> 5) / (L / 32)), "n"(L) : "memory");
    else __syncthreads();
}

template <int L> __device__ __forceinline__ float2 row_sums(float a, float b, float2 *slot)
{
#pragma unroll
    for (int d = (L < 32 ? L : 32) / 2; d; d >>= 1) {
        a += __shfl_xor_sync(0xffffffffu, a, d);
        b += __shfl_xor_sync(0xffffffffu, b, d);
    }
    if constexpr (L > 32) {
        const int warp = int(threadIdx.x) >> 5, first = warp & ~(L / 32 - 1);
        if ((threadIdx.x & 31) == 0) slot[warp] = make_float2(a, b);
        row_barrier<L>();
        Pair sum(0.0f, 0.0f);
#pragma unroll
        for (int i = 0; i < L / 32; i += 2) {
            const float4 two = *reinterpret_cast<const float4 *>(slot + first + i);
            sum = add2(add2(sum, Pair(two.x, two.y)), Pair(two.z, two.w));
        }
        sum.get(a, b);
    }
    return make_float2(a, b);
}

// One sum only.
template <int L> __device__ __forceinline__ float row_sum(float a, float2 *slot)
{
#pragma unroll
    for (int d = (L < 32 ? L : 32) / 2; d; d >>= 1) a += __shfl_xor_sync(0xffffffffu, a, d);
    if constexpr (L > 32) {
        float *one = reinterpret_cast<float *>(slot);
        const int warp = int(threadIdx.x) >> 5, first = warp & ~(L / 32 - 1);
        if ((threadIdx.x & 31) == 0) one[warp] = a;
        row_barrier<L>();
        a = 0.0f;
#pragma unroll
        for (int i = 0; i < L / 32; i += 2) {
            const float2 two = *reinterpret_cast<const float2 *>(one + first + i);
            a += two.x + two.y;
        }
    }
    return a;
}

// Rows too long for a block are shared by a cluster of CL blocks, each with its own columns: the blocks' sums meet in every
// block's shared memory and are added in the order of the blocks.  `meet` has CL entries per use and may be used again
// after one more such meeting.
__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

template <int L, int CL> __device__ __forceinline__ float2 row_sums(float a, float b, float2 *slot, float2 *meet, uint32_t rank)
{
    const float2 mine = row_sums<L>(a, b, slot);
    if constexpr (CL == 1) return mine;
    if (threadIdx.x < CL) {
        const uint32_t here = uint32_t(__cvta_generic_to_shared(meet + rank));
        uint32_t there;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(here), "r"(threadIdx.x));
        asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(there), "f"(mine.x), "f"(mine.y) : "memory");
    }
    __syncwarp();
    cluster_sync();
    float2 all = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < CL; ++i) {
        all.x += meet[i].x;
        all.y += meet[i].y;
    }
    return all;
}

// ---- layer norm, forward -------------------------------------------------------------------------------

// A row is read once and written once: 16384 x 4096 bf16 41 us at the measured copy rate, 50 here (f32: 82 and 88); what is
// missing is spent on instructions and on the two barriers per row (issue slots 64 % used, three blocks of 256 threads per
// SM; four where aligned 32-bit rows of 2049 to 4096 columns leave registers for them: 97 -> 87 us, but 48 -> 57 at 2048).
// Two barriers because the sum of squares waits for the mean: one pass with a shifted sum would save one, and lose digits
// where the shift is far from the mean.
// Mean first, then the differences d from it, sum of d^2 and sum of d: the latter is what rounding left in the mean, and
// corrects both (var = mean d^2 - (mean d)^2), so a mean far larger than the spread costs no digits.
template <typename T, int L, int NV, bool SHIFT, int CL>
__global__ void __launch_bounds__(RowShape<T, L, NV>::kThreads, L >= 512 ? 2 : sizeof(T) == 4 && !SHIFT && L == 256 ? 4 : 3) redist_layer_norm_kernel(const LayerNorm l)
{
    using S = RowShape<T, L, NV>;
    constexpr int VEC = S::VEC;
    __shared__ __align__(16) float2 slots[2][32], meet[2][CL];
    extern __shared__ __align__(16) uint8_t ring[];
    const uint32_t rank = CL > 1 ? cluster_rank() : 0;
    const int from = int(rank) * L * NV * VEC;              // this block's first column
    const int t = int(threadIdx.x) % L, group = int(threadIdx.x) / L, cols = int(l.cols) - from;
    let_next_start();
    wait_for_previous();
    int count[NV];
    float gamma[NV][VEC], beta[NV][VEC];
    Stream<T, L, NV, 1, SHIFT> rows(ring);
    const int64_t step = int64_t(gridDim.x / CL) * S::kRows;
    const int64_t start = int64_t(blockIdx.x / CL) * S::kRows + group;
#pragma unroll
    for (int j = 0; j < NV; ++j) count[j] = cols - S::column(j);
    auto at = [&](int64_t row) { return static_cast<const T *>(l.x) + row * l.ld_x + from + S::column(0); };
#pragma unroll
    for (int i = 0; i < rows.kAhead; ++i) {
        const T *const base[1] = {at(start + i * step)};
        rows.send(base, start + i * step < l.rows, count);
    }
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const int c = S::column(j) + i;
            gamma[j][i] = l.gamma && c < cols ? load_any(l.gamma, l.weight_type, from + c) : 1.0f;
            beta[j][i] = l.beta && c < cols ? load_any(l.beta, l.weight_type, from + c) : 0.0f;
        }
    const float over = 1.0f / float(l.cols);
    const int64_t turns = (l.rows - int64_t(blockIdx.x / CL) * S::kRows + step - 1) / step;       // the same for all rows of the block
    int64_t row = start;
    for (int64_t turn = 0; turn < turns; ++turn, row += step) {
        const T *const ahead[1] = {at(row + rows.kAhead * step)};
        rows.send(ahead, row + rows.kAhead * step < l.rows, count);
        const T *const base[1] = {at(row)};
        float all[1][NV][VEC];
        rows.take(base, count, all);
        float (&v)[NV][VEC] = all[0];
        Pair sums(0.0f, 0.0f), rests(0.0f, 0.0f), squares(0.0f, 0.0f);
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VEC; i += 2) sums = add2(sums, Pair(v[j][i], v[j][i + 1]));
        const float mean = (CL == 1 ? row_sum<L>(sums.sum(), slots[0]) : row_sums<L, CL>(sums.sum(), 0.0f, slots[0], meet[0], rank).x) * over;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
#pragma unroll
            for (int i = 0; i < VEC; i += 2) add2(Pair(v[j][i], v[j][i + 1]), Pair(-mean, -mean)).get(v[j][i], v[j][i + 1]);
            if (count[j] < VEC)
#pragma unroll
                for (int i = 0; i < VEC; ++i)
                    if (i >= count[j]) v[j][i] = 0.0f;
#pragma unroll
            for (int i = 0; i < VEC; i += 2) {
                const Pair d(v[j][i], v[j][i + 1]);
                rests = add2(rests, d);
                squares = fma2(d, d, squares);
            }
        }
        const float2 both = row_sums<L, CL>(rests.sum(), squares.sum(), slots[1], meet[1], rank);
        const float rest = both.x * over;
        float var = both.y * over - rest * rest;
        if (var < 0.0f) var = 0.0f;                         // by rounding alone; NaN stays
        const float rstd = rsqrtf(var + l.eps);
        const bool in = row < l.rows;
        const float less = -rest * rstd;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VEC; i += 2)
                fma2(fma2(Pair(v[j][i], v[j][i + 1]), Pair(rstd, rstd), Pair(less, less)), Pair(gamma[j][i], gamma[j][i + 1]),
                     Pair(beta[j][i], beta[j][i + 1]))
                    .get(v[j][i], v[j][i + 1]);
        rows.store(static_cast<T *>(l.y) + row * l.ld_y + from + S::column(0), in, count, v);
        if (t == 0 && in && rank == 0) {
            if (l.mean) l.mean[row] = mean + rest;
            if (l.rstd) l.rstd[row] = rstd;
        }
    }
    if constexpr (CL > 1) cluster_sync();                   // the others write into this block's shared memory
}

// Eight neighbours at any alignment from global memory; what is not wanted reads as zero.
template <typename T> __device__ __forceinline__ void load8(const T *p, int count, float (&v)[8])
{
    if constexpr (sizeof(T) == 2) {
        unpack16<T>(load16_any(p, min(count, 8) * 2), v);
    } else {
        unpack16<T>(load16_any(p, min(count, 4) * 4), v);
        uint4 b = make_uint4(0, 0, 0, 0);
        if (count > 4) b = load16_any(p + 4, (min(count, 8) - 4) * 4);
        unpack16<T>(b, v + 4);
    }
    if (count < 8)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i >= count) v[i] = 0.0f;
}

template <typename T> __device__ __forceinline__ void store8(T *p, const float (&v)[8], int count)
{
    if (count >= 8 && reinterpret_cast<uintptr_t>(p) % 16 == 0) {
#pragma unroll
        for (int i = 0; i < 8; i += kVec<T>) *reinterpret_cast<uint4 *>(p + i) = pack16<T>(v + i);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count) p[i] = from_float<T>(v[i]);
    }
}

// Rows that do not fit into the registers of a block: three passes over a row, which its first pass left in L2.
constexpr int kLong = 512;

template <typename T>
__global__ void __launch_bounds__(kLong) redist_layer_norm_long_kernel(const LayerNorm l)
{
    __shared__ __align__(16) float2 slots[2][32];
    let_next_start();
    wait_for_previous();
    const float over = 1.0f / float(l.cols);
    for (int64_t row = blockIdx.x; row < l.rows; row += gridDim.x) {
        const T *x = static_cast<const T *>(l.x) + row * l.ld_x;
        T *y = static_cast<T *>(l.y) + row * l.ld_y;
        float sum = 0.0f, rest = 0.0f, square = 0.0f;
#pragma unroll 2
        for (int64_t c = int64_t(threadIdx.x) * 8; c < l.cols; c += kLong * 8) {
            float v[8];
            load8<T>(x + c, int(min(l.cols - c, int64_t(8))), v);
            sum += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
        }
        const float mean = row_sum<kLong>(sum, slots[0]) * over;
#pragma unroll 2
        for (int64_t c = int64_t(threadIdx.x) * 8; c < l.cols; c += kLong * 8) {
            float v[8];
            const int count = int(min(l.cols - c, int64_t(8)));
            load8<T>(x + c, count, v);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < count) {
                    const float d = v[i] - mean;
                    rest += d;
                    square = fmaf(d, d, square);
                }
        }
        const float2 both = row_sums<kLong>(rest, square, slots[1]);
        rest = both.x * over;
        float var = both.y * over - rest * rest;
        if (var < 0.0f) var = 0.0f;
        const float rstd = rsqrtf(var + l.eps);
#pragma unroll 2
        for (int64_t c = int64_t(threadIdx.x) * 8; c < l.cols; c += kLong * 8) {
            float v[8];
            const int count = int(min(l.cols - c, int64_t(8)));
            load8<T>(x + c, count, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float g = l.gamma && i < count ? load_any(l.gamma, l.weight_type, c + i) : 1.0f;
                const float b = l.beta && i < count ? load_any(l.beta, l.weight_type, c + i) : 0.0f;
                v[i] = fmaf((v[i] - mean - rest) * rstd, g, b);
            }
            store8<T>(y + c, v, count);
        }
        if (threadIdx.x == 0) {
            if (l.mean) l.mean[row] = mean + rest;
            if (l.rstd) l.rstd[row] = rstd;
        }
    }
}

// ---- layer norm, backward ------------------------------------------------------------------------------

// With c = dy gamma and xh = (x - mean) rstd: dx = rstd (c - mean(c) - xh mean(c xh)).  A block walks over its rows
// and keeps the column sums of dy xh and dy in registers; partials holds them per block, gamma's before beta's, and a
// second kernel adds the blocks' in a fixed order (atomics would not).  16384 x 4096 bf16: 61 us at the measured copy rate,
// 79 here (with the second kernel's 4); 262144 x 256: 80.  The sums' registers allow two blocks per SM; what they have
// under way of the next rows lies in shared memory instead.
template <typename T, int L, int NV, bool SHIFT, int CL>
__global__ void __launch_bounds__(RowShape<T, L, NV>::kThreads, L <= 32 && NV == 1 ? 4 : L <= 256 ? 2 : 1) redist_layer_norm_grad_kernel(const LayerNorm l, float *partials)
{
    using S = RowShape<T, L, NV>;
    constexpr int VEC = S::VEC;
    __shared__ __align__(16) float2 slots[2][32], meet[2][CL];
    extern __shared__ __align__(16) uint8_t ring[];
    const uint32_t rank = CL > 1 ? cluster_rank() : 0;
    const int from = int(rank) * L * NV * VEC;              // this block's first column
    const int t = int(threadIdx.x) % L, group = int(threadIdx.x) / L, cols = int(l.cols) - from;
    let_next_start();
    wait_for_previous();
    int count[NV];
    float gamma[NV][VEC], dgamma[NV][VEC], dbeta[NV][VEC];
    Stream<T, L, NV, 2, SHIFT> rows(ring);
    const int64_t step = int64_t(gridDim.x / CL) * S::kRows;
    const int64_t start = int64_t(blockIdx.x / CL) * S::kRows + group;
#pragma unroll
    for (int j = 0; j < NV; ++j) count[j] = cols - S::column(j);
    auto at_x = [&](int64_t row) { return static_cast<const T *>(l.x) + row * l.ld_x + from + S::column(0); };
    auto at_dy = [&](int64_t row) { return static_cast<const T *>(l.dy) + row * l.ld_dy + from + S::column(0); };
#pragma unroll
    for (int i = 0; i < rows.kAhead; ++i) {
        const T *const base[2] = {at_x(start + i * step), at_dy(start + i * step)};
        rows.send(base, start + i * step < l.rows, count);
    }
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const int c = S::column(j) + i;
            gamma[j][i] = l.gamma && c < cols ? load_any(l.gamma, l.weight_type, from + c) : 1.0f;
            dgamma[j][i] = dbeta[j][i] = 0.0f;
        }
    const float over = 1.0f / float(l.cols);
    const int64_t turns = (l.rows - int64_t(blockIdx.x / CL) * S::kRows + step - 1) / step;
    int64_t row = start;
    float next_mean = row < l.rows ? l.mean[row] : 0.0f, next_rstd = row < l.rows ? l.rstd[row] : 0.0f;
    for (int64_t turn = 0; turn < turns; ++turn, row += step) {
        const T *const ahead[2] = {at_x(row + rows.kAhead * step), at_dy(row + rows.kAhead * step)};
        rows.send(ahead, row + rows.kAhead * step < l.rows, count);
        const bool in = row < l.rows;
        const float mean = next_mean, rstd = next_rstd;
        next_mean = next_rstd = 0.0f;
        if (row + step < l.rows) {
            next_mean = l.mean[row + step];
            next_rstd = l.rstd[row + step];
        }
        const T *const base[2] = {at_x(row), at_dy(row)};
        float both[2][NV][VEC];
        rows.take(base, count, both);
        float (&xh)[NV][VEC] = both[0], (&c1)[NV][VEC] = both[1];
        // (beyond the row's end dy is zero, and with it all that is summed; so it is in rows that are not there)
        const float by = in ? rstd : 0.0f;
        Pair s1(0.0f, 0.0f), s2(0.0f, 0.0f);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (!in)
#pragma unroll
                for (int i = 0; i < VEC; ++i) xh[j][i] = c1[j][i] = 0.0f;
#pragma unroll
            for (int i = 0; i < VEC; i += 2) {
                const Pair dy(c1[j][i], c1[j][i + 1]);
                const Pair h = mul2(add2(Pair(xh[j][i], xh[j][i + 1]), Pair(-mean, -mean)), Pair(by, by));
                fma2(dy, h, Pair(dgamma[j][i], dgamma[j][i + 1])).get(dgamma[j][i], dgamma[j][i + 1]);
                add2(dy, Pair(dbeta[j][i], dbeta[j][i + 1])).get(dbeta[j][i], dbeta[j][i + 1]);
                const Pair c = mul2(dy, Pair(gamma[j][i], gamma[j][i + 1]));
                s1 = add2(s1, c);
                s2 = fma2(c, h, s2);
                h.get(xh[j][i], xh[j][i + 1]);
                c.get(c1[j][i], c1[j][i + 1]);
            }
        }
        const float2 sums = row_sums<L, CL>(s1.sum(), s2.sum(), slots[turn & 1], meet[turn & 1], rank);
        const float m1 = -sums.x * over, m2 = -sums.y * over;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VEC; i += 2)
                mul2(add2(fma2(Pair(xh[j][i], xh[j][i + 1]), Pair(m2, m2), Pair(c1[j][i], c1[j][i + 1])), Pair(m1, m1)), Pair(by, by))
                    .get(c1[j][i], c1[j][i + 1]);
        rows.store(static_cast<T *>(l.dx) + row * l.ld_dx + from + S::column(0), in, count, c1);
    }
    if constexpr (CL > 1) cluster_sync();
    if (!partials) return;
    float *out = partials + int64_t(blockIdx.x / CL) * 2 * l.cols + from;
    if constexpr (S::kRows > 1) {
        // the block's groups hold sums of the same columns: added in the order of the groups
        asm volatile("cp.async.wait_all;" ::: "memory");
        float *all = reinterpret_cast<float *>(ring);       // [group][column of this piece]
        static_assert(Stream<T, L, NV, 2, SHIFT>::kSmem >= 256 * VEC * 4, "the ring holds one piece of every thread");
#pragma unroll
        for (int which = 0; which < 2; ++which)
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                __syncthreads();
#pragma unroll
                for (int i = 0; i < VEC; ++i) all[(group * VEC + i) * L + t] = which ? dbeta[j][i] : dgamma[j][i];
                __syncthreads();
                for (int q = int(threadIdx.x); q < L * VEC; q += S::kThreads) {
                    const int i = q / L, from = q % L;
                    float s = 0.0f;
#pragma unroll 8
                    for (int g = 0; g < S::kRows; ++g) s += all[(g * VEC + i) * L + from];
                    const int c = ((from / S::kSegment * NV + j) * S::kSegment + from % S::kSegment) * VEC + i;
                    if (c < cols) out[which * l.cols + c] = s;
                }
            }
    } else {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const int c = S::column(j) + i;
                if (c < cols) {
                    out[c] = dgamma[j][i];
                    out[l.cols + c] = dbeta[j][i];
                }
            }
    }
}

// Long rows: dx alone, with a second pass over a row that the first left in L2 ...
template <typename T>
__global__ void __launch_bounds__(kLong) redist_layer_norm_grad_long_kernel(const LayerNorm l)
{
    __shared__ __align__(16) float2 slots[2][32];
    let_next_start();
    wait_for_previous();
    const float over = 1.0f / float(l.cols);
    int turn = 0;
    for (int64_t row = blockIdx.x; row < l.rows; row += gridDim.x, turn ^= 1) {
        const T *x = static_cast<const T *>(l.x) + row * l.ld_x, *dy = static_cast<const T *>(l.dy) + row * l.ld_dy;
        T *dx = static_cast<T *>(l.dx) + row * l.ld_dx;
        const float mean = l.mean[row], rstd = l.rstd[row];
        float s1 = 0.0f, s2 = 0.0f;
        for (int64_t c = int64_t(threadIdx.x) * 8; c < l.cols; c += kLong * 8) {
            float v[8], d[8];
            const int count = int(min(l.cols - c, int64_t(8)));
            load8<T>(x + c, count, v);
            load8<T>(dy + c, count, d);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < count) {
                    const float g = d[i] * (l.gamma ? load_any(l.gamma, l.weight_type, c + i) : 1.0f);
                    s1 += g;
                    s2 = fmaf(g, (v[i] - mean) * rstd, s2);
                }
        }
        const float2 sums = row_sums<kLong>(s1, s2, slots[turn]);
        s1 = sums.x * over;
        s2 = sums.y * over;
        for (int64_t c = int64_t(threadIdx.x) * 8; c < l.cols; c += kLong * 8) {
            float v[8], d[8];
            const int count = int(min(l.cols - c, int64_t(8)));
            load8<T>(x + c, count, v);
            load8<T>(dy + c, count, d);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < count) v[i] = (d[i] * (l.gamma ? load_any(l.gamma, l.weight_type, c + i) : 1.0f) - s1 - (v[i] - mean) * rstd * s2) * rstd;
            store8<T>(dx + c, v, count);
        }
    }
}

// ... and the column sums on their own: a lane has eight columns, a warp every eighth row of the block's slice.
template <typename T>
__global__ void __launch_bounds__(256) redist_layer_norm_columns_kernel(const LayerNorm l, float *partials)
{
    __shared__ float all[2][8][256];
    let_next_start();
    wait_for_previous();
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int64_t c = int64_t(blockIdx.x) * 256 + lane * 8;
    const int count = int(min(l.cols - c, int64_t(8)));
    const int64_t per = (l.rows + gridDim.y - 1) / gridDim.y, lo = per * blockIdx.y, hi = min(l.rows, lo + per);
    float g[8] = {}, b[8] = {};
    if (count > 0)
#pragma unroll 2
        for (int64_t row = lo + w; row < hi; row += 8) {
            float v[8], d[8];
            load8<T>(static_cast<const T *>(l.x) + row * l.ld_x + c, count, v);
            load8<T>(static_cast<const T *>(l.dy) + row * l.ld_dy + c, count, d);
            const float mean = l.mean[row], rstd = l.rstd[row];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                g[i] = fmaf(d[i], (v[i] - mean) * rstd, g[i]);
                b[i] += d[i];
            }
        }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        all[0][w][lane * 8 + i] = g[i];
        all[1][w][lane * 8 + i] = b[i];
    }
    __syncthreads();
    const int64_t cc = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (cc >= l.cols) return;
    float *out = partials + int64_t(blockIdx.y) * 2 * l.cols;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s += all[which][i][threadIdx.x];
        out[which * l.cols + cc] = s;
    }
}

// out[c] = sum over the parts of partials[part][c], in the same order every time.
// A warp per 32nd of the parts: the loads of one thread are few and independent.
constexpr int kSumThreads = 1024;

__global__ void __launch_bounds__(kSumThreads) redist_column_sum_kernel(const float *partials, int parts, int64_t stride, int64_t cols,
                                                                       float *first, float *second)
{
    __shared__ float all[kSumThreads / 32][33];
    let_next_start();
    wait_for_previous();
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int64_t c = int64_t(blockIdx.x) * 32 + lane;
    const float *p = partials + (blockIdx.y ? cols : 0);
    float *out = blockIdx.y ? second : first;
    float s = 0.0f;
    if (out && c < cols)
#pragma unroll 8
        for (int q = w; q < parts; q += kSumThreads / 32) s += __ldg(p + q * stride + c);
    all[w][lane] = s;
    __syncthreads();
    // the warps' sums of column `w` of the block
    s = all[lane][w];
#pragma unroll
    for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    if (lane == 0 && out && int64_t(blockIdx.x) * 32 + w < cols) out[int64_t(blockIdx.x) * 32 + w] = s;
}

// ---- operands of a product -------------------------------------------------------------------------------

constexpr int kLayCols = 256;

// Rows of a block: 128, fewer where that leaves SMs without work (148 of them at four blocks each, written here because
// scratch is asked for by sizes alone), more where the grid would grow beyond its limit.
int64_t lay_rows(int64_t rows, int64_t cols)
{
    int64_t per = 128 * ((rows + 128 * 32768 - 1) / (128 * 32768));
    while (per > 8 && ((rows + per - 1) / per) * ((cols + kLayCols - 1) / kLayCols) < 4 * 148) per /= 2;
    return per;
}

struct Lays {
    Lay l[3];
    int64_t rows_per_block[3];
};

// Up to three matrices in one launch.  A block takes rows_per_block rows by 256 columns, a warp every eighth row, a lane
// eight neighbours.
template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(256, 4) redist_lay_kernel(const __grid_constant__ Lays lays)
{
    __shared__ float all[8][kLayCols];
    let_next_start();
    wait_for_previous();
    const Lay &l = lays.l[blockIdx.z];
    const int64_t rows_per_block = lays.rows_per_block[blockIdx.z];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int64_t c = int64_t(blockIdx.x) * kLayCols + lane * 8;
    const int64_t lo = int64_t(blockIdx.y) * rows_per_block, hi = min(l.rows, lo + rows_per_block);
    if (lo >= l.rows || int64_t(blockIdx.x) * kLayCols >= l.cols) return;
    const int count = int(min(l.cols - c, int64_t(8)));
    float sums[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    // One row at a time and many warps (four blocks per SM, for which GELU has to do with 64 registers): two or four rows'
    // loads under way per warp cost registers, thus warps, and were slower (4096 x 16384 with GELU: 80 us, with four 91; at
    // odd strides 120 and 203).  61 us at the measured copy rate without dz, which adds 20 of them.
    if (count > 0)
        for (int64_t row = lo + w; row < hi; row += 8) {
            const T *src = static_cast<const T *>(l.src) + row * l.ld_src + c, *z = static_cast<const T *>(l.z) + row * l.ld_z + c;
            uint4 u, y;
            if (ALIGNED && count >= 8) {
                u = *reinterpret_cast<const uint4 *>(src);
                if (l.z) y = *reinterpret_cast<const uint4 *>(z);
            } else {
                Blocks a, b = {};
                a.load(src, count * 2);
                if (l.z) b.load(z, count * 2);
                u = a.get(src);
                y = b.get(z);
            }
            if (l.z || l.sums) {
                float v[8];
                unpack16<T>(u, v);
                if (l.z) {
                    float at[8];
                    unpack16<T>(y, at);
                    times_slope8(v, at, l.activation);
                    // dz becomes an operand of two products: 16 bits, as the tensor cores take them with the other operand.
                    // (bf16 gradients are 2.3e-3 off with it, 1.7e-3 by their own rounding alone; dz in two halves would cost
                    // both products once more.)  The column sums below take the 32-bit values.
                    u = pack16<T>(v);
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
// Warps take rows (or pieces of 1024 columns of them) in turn, four loads under way per lane.
template <typename T, bool ALIGNED, typename F> __device__ __forceinline__ void along_rows(const Scaled &s, F f)
{
    constexpr int kRaw = int(sizeof(T)) / 2;                // 16-byte blocks in eight neighbours
    const T *x = static_cast<const T *>(s.x) + int64_t(blockIdx.y) * s.x_batch;
    const int lane = threadIdx.x & 31, cols = int(s.cols), per_row = (cols + 1023) / 1024;
    const int64_t warps = int64_t(gridDim.x) * 8, all = s.rows * per_row;
    for (int64_t q = int64_t(blockIdx.x) * 8 + (threadIdx.x >> 5); q < all; q += warps) {
        const int64_t row = per_row == 1 ? q : q / per_row;
        const int c0 = int(q - row * per_row) * 1024 + lane * 8;
        const T *p = x + row * s.ld_x + c0;
        if (ALIGNED && c0 + 776 <= cols) {                  // all four pieces are whole
            uint4 u[4][kRaw];
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int i = 0; i < kRaw; ++i) u[k][i] = __ldg(reinterpret_cast<const uint4 *>(p + k * 256) + i);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float v[8];
#pragma unroll
                for (int i = 0; i < kRaw; ++i) unpack16<T>(u[k][i], v + i * kVec<T>);
                f(row, c0 + k * 256, v);
            }
        } else {
            Blocks u[4][kRaw];
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int i = 0; i < kRaw; ++i) {
                    const int left = cols - c0 - k * 256 - i * kVec<T>;
                    if (left > 0) u[k][i].load(p + k * 256 + i * kVec<T>, min(left, kVec<T>) * int(sizeof(T)));
                }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int left = cols - c0 - k * 256;
                if (left <= 0) break;
                float v[8];
#pragma unroll
                for (int i = 0; i < kRaw; ++i) unpack16<T>(u[k][i].get(p + k * 256 + i * kVec<T>), v + i * kVec<T>);
                if (left < 8)
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (i >= left) v[i] = 0.0f;
                f(row, c0 + k * 256, v);
            }
        }
    }
}

template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(256) redist_norm_parts_kernel(const Scaled s)
{
    __shared__ double slots[8];
    let_next_start();
    wait_for_previous();
    double sum = 0.0, more = 0.0;
    along_rows<T, ALIGNED>(s, [&](int64_t, int, const float (&v)[8]) {
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            sum = fma(double(v[i]), double(v[i]), sum);
            more = fma(double(v[i + 1]), double(v[i + 1]), more);
        }
    });
    sum = block_sum(sum + more, slots);
    if (threadIdx.x == 0) s.partials[int64_t(blockIdx.y) * kNormParts + blockIdx.x] = sum;
}

template <typename T, bool ALIGNED>
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
    __half *hi = static_cast<__half *>(s.hi) + int64_t(blockIdx.y) * s.plane, *lo = s.lo ? static_cast<__half *>(s.lo) + int64_t(blockIdx.y) * s.plane : nullptr;
    along_rows<T, ALIGNED>(s, [&](int64_t row, int c, float (&v)[8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= power;
        const uint4 u = pack16<__half>(v);
        *reinterpret_cast<uint4 *>(hi + row * s.ld + c) = u;
        if (lo) {
            float h[8];
            unpack16<__half>(u, h);
#pragma unroll
            for (int i = 0; i < 8; ++i) h[i] = (v[i] - h[i]) * 2048.0f;
            *reinterpret_cast<uint4 *>(lo + row * s.ld + c) = pack16<__half>(h);
        }
    });
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
        unpack16<T>(load16_any(static_cast<const T *>(e.residual) + row * e.ld_residual + c, count * 2), w);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += w[i];
    }
    put(e.out, e.ld_out);
}

// ---- host ---------------------------------------------------------------------------------------------------

template <typename... P, typename... A>
cudaError_t launch_with(int smem, int cluster, void (*kernel)(P...), dim3 grid, int block, const LaunchOptions &o, cudaStream_t stream, A... args)
{
    cudaLaunchConfig_t cfg = {};
    if (smem > 48 * 1024) {
        const cudaError_t ce = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (ce != cudaSuccess) return ce;
    }
    cfg.dynamicSmemBytes = size_t(smem);
    cfg.gridDim = grid;
    cfg.blockDim = dim3(unsigned(block));
    cfg.stream = stream;
    cudaLaunchAttribute at[2];
    int n_at = 0;
    if (o.pdl) {
        at[n_at].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at[n_at].val.programmaticStreamSerializationAllowed = 1;
        ++n_at;
    }
    if (cluster > 1) {
        at[n_at].id = cudaLaunchAttributeClusterDimension;
        at[n_at].val.clusterDim.x = unsigned(cluster);
        at[n_at].val.clusterDim.y = 1;
        at[n_at].val.clusterDim.z = 1;
        ++n_at;
    }
    cfg.attrs = at;
    cfg.numAttrs = unsigned(n_at);
    return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}

template <typename... P, typename... A>
cudaError_t launch(void (*kernel)(P...), dim3 grid, int block, const LaunchOptions &o, cudaStream_t stream, A... args)
{
    return launch_with(0, 1, kernel, grid, block, o, stream, args...);
}

cudaError_t sm_count(int *sms)
{
    int device = 0;
    return current_device(&device, sms);
}

bool on_16(const void *p, int64_t ld, int64_t element) { return p == nullptr || (uintptr_t(p) % 16 == 0 && ld * element % 16 == 0); }

// Threads per row and pieces per thread by the row's length: up to 16 neighbours per thread (more would cost the registers
// that hold gamma and beta), within that the fewest threads; rows of fewer than 32 pieces share warps, rows of more than a
// block's 8192 (16-bit) or 4096 (32-bit) columns are shared by a cluster.
template <typename T, typename F> bool by_pieces(int64_t pieces, F f)
{
    using std::integral_constant;
    constexpr int MOST = 16 / kVec<T>;
#define TAKE(THREADS, NV, CL)                                                                   \
    if (pieces <= THREADS * NV * CL) {                                                          \
        f(integral_constant<int, THREADS>(), integral_constant<int, NV>(), integral_constant<int, CL>()); \
        return true;                                                                            \
    }
    TAKE(8, 1, 1)
    TAKE(16, 1, 1)
    TAKE(32, 1, 1)
    TAKE(32, 2, 1)
    TAKE(32, MOST, 1)
    TAKE(64, MOST, 1)
    TAKE(128, MOST, 1)
    TAKE(256, MOST, 1)
    TAKE(512, MOST, 1)
    TAKE(512, MOST, 2)
    TAKE(512, MOST, 4)
    TAKE(512, MOST, 8)
#undef TAKE
    return false;
}

unsigned row_blocks(const LayerNorm &l, int rows_per_block, int threads, int smem, int registers, int sms)
{
    const int64_t resident = std::max<int64_t>(1, std::min<int64_t>({2048 / threads, 65536 / (threads * registers), 220 * 1024 / std::max(smem + 1024, 1)}));
    return unsigned(std::min<int64_t>((l.rows + rows_per_block - 1) / rows_per_block, sms * resident));
}

template <typename T, bool SHIFT> cudaError_t forward_as(const LayerNorm &l, int sms, const LaunchOptions &o, cudaStream_t stream)
{
    cudaError_t ce = cudaSuccess;
    const bool held = by_pieces<T>((l.cols + kVec<T> - 1) / kVec<T>, [&](auto threads, auto pieces, auto cluster) {
        constexpr int L = decltype(threads)::value, NV = decltype(pieces)::value, CL = decltype(cluster)::value;
        using S = RowShape<T, L, NV>;
        constexpr int smem = Stream<T, L, NV, 1, SHIFT>::kSmem;
        ce = launch_with(smem, CL, redist_layer_norm_kernel<T, L, NV, SHIFT, CL>, dim3(row_blocks(l, S::kRows, S::kThreads, smem, L >= 512 || (sizeof(T) == 4 && !SHIFT && L == 256) ? 64 : NV == 1 ? 56 : 80, sms / CL) * CL),
                         S::kThreads, o, stream, l);
    });
    if (held) return ce;
    return launch(redist_layer_norm_long_kernel<T>, dim3(unsigned(std::min<int64_t>(l.rows, sms * 4))), kLong, o, stream, l);
}

// Slices of the rows for long rows' column sums, and blocks of the backward pass per SM at most: what the parts of the
// column sums need of scratch follows from these.
constexpr int kLongParts = 64;
constexpr int grad_per_sm(int64_t pieces) { return pieces <= 32 ? 4 : 2; }       // by the registers that hold the sums

template <typename T, bool SHIFT>
cudaError_t backward_as(const LayerNorm &l, float *partials, int sms, const LaunchOptions &o, cudaStream_t stream)
{
    int parts = 0;
    cudaError_t ce = cudaSuccess;
    const bool held = by_pieces<T>((l.cols + kVec<T> - 1) / kVec<T>, [&](auto threads, auto pieces, auto cluster) {
        constexpr int L = decltype(threads)::value, NV = decltype(pieces)::value, CL = decltype(cluster)::value;
        using S = RowShape<T, L, NV>;
        constexpr int smem = Stream<T, L, NV, 2, SHIFT>::kSmem;
        parts = int(std::min<unsigned>(row_blocks(l, S::kRows, S::kThreads, smem, L <= 32 && NV == 1 ? 64 : 128, sms / CL),
                                       unsigned(sms * grad_per_sm((l.cols + kVec<T> - 1) / kVec<T>))));
        ce = launch_with(smem, CL, redist_layer_norm_grad_kernel<T, L, NV, SHIFT, CL>, dim3(unsigned(parts * CL)), S::kThreads, o, stream, l, partials);
    });
    if (!held) {
        ce = launch(redist_layer_norm_grad_long_kernel<T>, dim3(unsigned(std::min<int64_t>(l.rows, sms * 4))), kLong, o, stream, l);
        if (ce != cudaSuccess || !partials) return ce;
        parts = int(std::min<int64_t>((l.rows + 7) / 8, kLongParts));
        ce = launch(redist_layer_norm_columns_kernel<T>, dim3(unsigned((l.cols + 255) / 256), unsigned(parts)), 256, o, stream, l, partials);
    }
    if (ce != cudaSuccess || !partials) return ce;
    return launch(redist_column_sum_kernel, dim3(unsigned((l.cols + 31) / 32), 2), kSumThreads, o, stream, static_cast<const float *>(partials), parts,
                  int64_t(2) * l.cols, l.cols, l.dgamma, l.dbeta);
}

template <typename F> cudaError_t by_type(int type, F f)
{
    if (type == T_BF16) return f(__nv_bfloat16());
    if (type == T_F16) return f(__half());
    return f(float());
}

}  // namespace

size_t layer_norm_backward_bytes(int64_t rows, int64_t cols, int type, int sms)
{
    const int64_t vec = 16 / type_bytes(type);
    const int64_t parts = std::min<int64_t>(rows, std::max(int64_t(sms) * grad_per_sm((cols + vec - 1) / vec), int64_t(kLongParts)));
    return size_t(parts * 2 * cols * 4);
}

cudaError_t launch_layer_norm_forward(const LayerNorm &l, const LaunchOptions &o, cudaStream_t stream)
{
    int sms = 0;
    cudaError_t ce = sm_count(&sms);
    if (ce != cudaSuccess || l.rows == 0) return ce;
    return by_type(l.type, [&](auto t) {
        using T = decltype(t);
        if (on_16(l.x, l.ld_x, sizeof(T)) && on_16(l.y, l.ld_y, sizeof(T))) return forward_as<T, false>(l, sms, o, stream);
        return forward_as<T, true>(l, sms, o, stream);
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
        if (on_16(l.x, l.ld_x, sizeof(T)) && on_16(l.dy, l.ld_dy, sizeof(T)) && on_16(l.dx, l.ld_dx, sizeof(T)))
            return backward_as<T, false>(l, partials, sms, o, stream);
        return backward_as<T, true>(l, partials, sms, o, stream);
    });
}

size_t column_partial_bytes(int64_t rows, int64_t cols)
{
    if (rows == 0) return 0;
    const int64_t per = lay_rows(rows, cols);
    return size_t((rows + per - 1) / per * cols * 4);
}

cudaError_t launch_lay(const Lay *l, int count, const LaunchOptions &o, cudaStream_t stream)
{
    Lays lays = {};
    int64_t x = 0, y = 0;
    for (int i = 0; i < count; ++i) {
        lays.l[i] = l[i];
        lays.rows_per_block[i] = lay_rows(l[i].rows, l[i].cols);
        x = std::max(x, (l[i].cols + kLayCols - 1) / kLayCols);
        y = std::max(y, (l[i].rows + lays.rows_per_block[i] - 1) / lays.rows_per_block[i]);
    }
    if (count == 0 || x == 0 || y == 0) return cudaSuccess;
    const dim3 grid{unsigned(x), unsigned(y), unsigned(count)};
    bool aligned = true;
    for (int i = 0; i < count; ++i) aligned = aligned && on_16(l[i].src, l[i].ld_src, 2) && on_16(l[i].z, l[i].ld_z, 2);
    cudaError_t ce;
    if (l[0].type == T_BF16)
        ce = aligned ? launch(redist_lay_kernel<__nv_bfloat16, true>, grid, 256, o, stream, lays) : launch(redist_lay_kernel<__nv_bfloat16, false>, grid, 256, o, stream, lays);
    else
        ce = aligned ? launch(redist_lay_kernel<__half, true>, grid, 256, o, stream, lays) : launch(redist_lay_kernel<__half, false>, grid, 256, o, stream, lays);
    for (int i = 0; i < count && ce == cudaSuccess; ++i)
        if (l[i].sums) {
            const int64_t per = lays.rows_per_block[i];
            ce = launch(redist_column_sum_kernel, dim3(unsigned((l[i].cols + 31) / 32), 1), kSumThreads, o, stream, static_cast<const float *>(l[i].partials),
                        int((l[i].rows + per - 1) / per), l[i].cols, l[i].cols, l[i].sums, static_cast<float *>(nullptr));
        }
    return ce;
}

cudaError_t launch_join(const Product &p, const float *parts, int64_t ld, int splits, const LaunchOptions &o, cudaStream_t stream)
{
    const dim3 grid(unsigned((p.m * (ld / 8) + 255) / 256));
    return p.type == T_BF16 ? launch(redist_join_kernel<__nv_bfloat16>, grid, 256, o, stream, p.e, parts, ld, splits, p.m, p.n)
                            : launch(redist_join_kernel<__half>, grid, 256, o, stream, p.e, parts, ld, splits, p.m, p.n);
}

cudaError_t launch_scaled(const Scaled &s, const LaunchOptions &o, cudaStream_t stream)
{
    const int64_t turns = s.rows * ((s.cols + 1023) / 1024);               // of a warp
    const int parts = int(std::min<int64_t>(kNormParts, (turns + 7) / 8));
    const int blocks = int(std::min<int64_t>(1024, (turns + 7) / 8));
    return by_type(s.type, [&](auto t) {
        using T = decltype(t);
        const bool aligned = on_16(s.x, s.ld_x, sizeof(T)) && s.x_batch * int64_t(sizeof(T)) % 16 == 0;
        const dim3 first{unsigned(parts), unsigned(s.batch)}, second{unsigned(blocks), unsigned(s.batch)};
        cudaError_t ce = aligned ? launch(redist_norm_parts_kernel<T, true>, first, 256, o, stream, s) : launch(redist_norm_parts_kernel<T, false>, first, 256, o, stream, s);
        if (ce != cudaSuccess) return ce;
        return aligned ? launch(redist_scaled_kernel<T, true>, second, 256, o, stream, s, parts) : launch(redist_scaled_kernel<T, false>, second, 256, o, stream, s, parts);
    });
}

}  // namespace redist
