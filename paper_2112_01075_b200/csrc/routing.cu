// The router of a block of experts, and the moves of tokens to their experts' rows and back: kernels bound by the memory they
// stream over, or by the latency of a launch.
#include "routing.h"

#include <algorithm>
#include <type_traits>

#include "elements.cuh"

namespace redist {

namespace {

constexpr int kRouteThreads = 1024, kRouteWarps = kRouteThreads / 32;
constexpr int kCounters = 8192;         // of a block: experts times the warps that count

// A logit as a number whose order is that of the choice: NaN first, minus infinity (and 0, for what has been chosen already)
// never.  Both zeros are one.
constexpr uint32_t kNever = 0x007fffffu;
__device__ __forceinline__ uint32_t order_of(float v)
{
    const uint32_t b = __float_as_uint(v + 0.0f);
    return v != v ? 0xffffffffu : b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key >> 31 ? key ^ 0x80000000u : ~key); }

// L lanes share a token.
template <int L> __device__ __forceinline__ float lane_sum(float v)
{
#pragma unroll
    for (int d = L / 2; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}
template <int L> __device__ __forceinline__ uint32_t lane_max(uint32_t v)
{
    if constexpr (L == 32) return __reduce_max_sync(0xffffffffu, v);
#pragma unroll
    for (int d = L / 2; d; d >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, d));
    return v;
}

struct RouteParams {
    Route r;
    int64_t per_block;                  // tokens
    int32_t *counts;                    // [block][expert]; null: one block, which places the rows itself
};

// Exclusive sums of `n` counters in shared memory, in place, by the first warp; the total goes to `total`.
__device__ __forceinline__ void scan_counts(int32_t *c, int n, int32_t *total)
{
    if (threadIdx.x >= 32) return;
    const int lane = threadIdx.x;
    int32_t carry = 0;
    for (int at = 0; at < n; at += 32) {
        const int32_t mine = at + lane < n ? c[at + lane] : 0;
        int32_t sum = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int32_t up = __shfl_up_sync(0xffffffffu, sum, d);
            if (lane >= d) sum += up;
        }
        if (at + lane < n) c[at + lane] = carry + sum - mine;
        carry += __shfl_sync(0xffffffffu, sum, 31);
    }
    if (lane == 0) *total = carry;
}

// The places of tokens lo ... hi - 1 are shared by warps that take a stretch of them each.
struct Stretch {
    int counting;                       // warps
    int64_t from, to;                   // this warp's places
    int32_t held[2];                    // the experts of the first two turns
    __device__ __forceinline__ Stretch(const Route &r, int64_t lo, int64_t hi)
    {
        const int warp = int(threadIdx.x) >> 5, lane = int(threadIdx.x) & 31;
        const int64_t first = lo * r.chosen, places = (hi - lo) * r.chosen;
        // two turns of a warp, where there are warps for that: every warp's counters make the chain of the counts longer
        counting = max(1, int(min(int64_t(min(kRouteWarps, kCounters / r.experts)), (places + 63) / 64)));
        const int64_t share = (places + counting - 1) / counting;
        from = first + min(places, warp * share);
        to = first + min(places, (warp + 1) * share);
#pragma unroll
        for (int i = 0; i < 2; ++i) held[i] = warp < counting && from + 32 * i + lane < to ? r.choice[from + 32 * i + lane] : -1;
    }
};
// Rows for the places, the next free row of expert e being base[e]: first the warps count the experts of their stretch, then they
// know where theirs begin.
__device__ __forceinline__ void place_rows(const Route &r, const Stretch &own, const int32_t *base, int32_t *counters)
{
    const int warp = int(threadIdx.x) >> 5, lane = int(threadIdx.x) & 31, experts = r.experts;
    const int counting = own.counting;
    const int64_t from = own.from, to = own.to;
    for (int i = threadIdx.x; i < counting * experts; i += kRouteThreads) counters[i] = 0;
    __syncthreads();
    int32_t *mine = counters + warp * experts;
    auto expert = [&](int64_t at) { return at == from ? own.held[0] : at == from + 32 ? own.held[1] : at + lane < to ? r.choice[at + lane] : -1; };
    if (warp < counting)
        for (int64_t at = from; at < to; at += 32) {
            const int32_t e = expert(at);
            if (e >= 0) atomicAdd(mine + e, 1);
        }
    __syncthreads();
    for (int e = threadIdx.x; e < experts; e += kRouteThreads) {
        int32_t next = base[e];
#pragma unroll 4
        for (int w = 0; w < counting; ++w) {
            const int32_t n = counters[w * experts + e];
            counters[w * experts + e] = next;
            next += n;
        }
    }
    __syncthreads();
    if (warp < counting)
        for (int64_t at = from; at < to; at += 32) {
            const int64_t i = at + lane;
            const int32_t e = expert(at);
            const uint32_t same = __match_any_sync(0xffffffffu, e);
            const int before = __popc(same & ((1u << lane) - 1));
            const int32_t start = e >= 0 ? mine[e] : 0;
            __syncwarp();
            if (e >= 0 && before == 0) mine[e] = start + __popc(same);
            __syncwarp();
            if (i < to) r.position[i] = e >= 0 ? start + before : -1;
        }
}

// A logit's place in the order of the choice, as the warp compares it.  The 16 bits of a 16-bit logit leave room for its
// index: one maximum over the lanes then gives both, where 32 bits take a second step.
template <typename T> struct Ranked {
    static constexpr bool kIndexed = sizeof(T) == 2;
    static __device__ __forceinline__ uint32_t of(T v, int index)
    {
        const uint32_t key = order_of(to_float(v));
        if constexpr (!kIndexed) return key;
        // (a bf16 is the upper half of its 32 bits; a f16 is ordered by its own)
        if constexpr (std::is_same_v<T, __half>) {
            const uint32_t b = __half_as_ushort(__hadd(v, __float2half_rn(0.0f)));
            const uint32_t h = __hisnan(v) ? 0xffffu : b >> 15 ? (~b & 0xffffu) : b | 0x8000u;
            return h << 16 | (0xffffu - uint32_t(index));
        }
        return (key & 0xffff0000u) | (0xffffu - uint32_t(index));
    }
    // What is never chosen: minus infinity and what has been taken.
    static __device__ __forceinline__ bool never(uint32_t r)
    {
        if constexpr (!kIndexed) return r <= kNever;
        else if constexpr (std::is_same_v<T, __half>) return r >> 16 <= 0x03ffu;
        else return r >> 16 <= kNever >> 16;
    }
    static __device__ __forceinline__ float value(uint32_t r)
    {
        if constexpr (!kIndexed) return value_of(r);
        const uint32_t h = r >> 16, b = h >> 15 ? h ^ 0x8000u : ~h & 0xffffu;
        if constexpr (std::is_same_v<T, __half>) return __half2float(__ushort_as_half(uint16_t(b)));
        return __uint_as_float(b << 16);
    }
};

// A lane's logits in descending order, each with its index where it does not hold it: what is taken is the first, and taking it
// moves the others up.  (Of equal ones the lower index comes first: neighbours only change places when they are out of order,
// and the pairs of the networks are ordered by index to begin with.)
template <bool INDEXED, int PER> struct Sorted {
    uint32_t key[PER];
    uint16_t index[INDEXED ? 1 : PER];
    __device__ __forceinline__ void order(int a, int b)     // a < b
    {
        bool swap = key[b] > key[a];
        if constexpr (!INDEXED) swap = swap || (key[b] == key[a] && index[b] < index[a]);
        const uint32_t k = swap ? key[b] : key[a];
        key[b] = swap ? key[a] : key[b];
        key[a] = k;
        if constexpr (!INDEXED) {
            const uint16_t i = swap ? index[b] : index[a];
            index[b] = swap ? index[a] : index[b];
            index[a] = i;
        }
    }
    __device__ __forceinline__ void sort()                  // odd-even merges
    {
#pragma unroll
        for (int p = 1; p < PER; p *= 2)
#pragma unroll
            for (int k = p; k >= 1; k /= 2)
#pragma unroll
                for (int j = k % p; j + k < PER; j += 2 * k)
#pragma unroll
                    for (int i = 0; i < k; ++i)
                        if ((i + j) / (2 * p) == (i + j + k) / (2 * p) && i + j + k < PER) order(i + j, i + j + k);
    }
    __device__ __forceinline__ void take(bool mine)
    {
#pragma unroll
        for (int j = 0; j + 1 < PER; ++j) {
            key[j] = mine ? key[j + 1] : key[j];
            if constexpr (!INDEXED) index[j] = mine ? index[j + 1] : index[j];
        }
        key[PER - 1] = mine ? 0 : key[PER - 1];
    }
};

// The choice: L lanes hold PER logits of a token each, and agree `chosen` times on the largest that is left.  Blocks count how
// many places each expert got among their tokens.  What bounds it is the number of instructions per token: 16384 tokens, 8 of
// 128 experts, 10.2 us, and 12.8 when the lane whose logit was taken looked through the others again, a dozen instructions with all
// lanes waiting.
template <typename T, int L, int PER>
__global__ void __launch_bounds__(kRouteThreads) redist_route_kernel(const RouteParams p)
{
    using R = Ranked<T>;
    constexpr int kTurn = kRouteThreads / L;                 // tokens of a block side by side
    constexpr bool kSorted = PER <= 8, kAhead = PER <= 8;    // (more of them do not fit into the registers, or take longer to sort)
    __shared__ int32_t counts[kMostExperts], counters[kCounters];
    const Route &r = p.r;
    const int lane = int(threadIdx.x) & 31, at = lane % L, group = int(threadIdx.x) / L;
    const uint32_t segment = L == 32 ? 0xffffffffu : ((1u << L) - 1) << (lane / L * L);
    for (int e = threadIdx.x; e < r.experts; e += kRouteThreads) counts[e] = 0;
    let_next_start();
    wait_for_previous();
    __syncthreads();
    const int64_t lo = int64_t(blockIdx.x) * p.per_block, hi = min(r.tokens, lo + p.per_block);
    T ahead[PER];
    auto load = [&](int64_t t) {
        const T *row = static_cast<const T *>(r.logits) + t * r.ld;
#pragma unroll
        for (int j = 0; j < PER; ++j)
            if (t < hi && at + 32 * j < r.experts) ahead[j] = row[at + 32 * j];
    };
    if (kAhead) load(lo + group);
    for (int64_t base = lo; base < hi; base += kTurn) {                       // all lanes of a warp walk along
        const int64_t t = base + group;
        const bool in = t < hi;
        if (!kAhead) load(t);
        Sorted<R::kIndexed, PER> mine;
        uint32_t best = 0, top = 0, own = 0;
        int32_t own_choice = -1;
        float every = 0.0f;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            mine.key[j] = in && at + 32 * j < r.experts ? R::of(ahead[j], at + 32 * j) : 0;
            if constexpr (!R::kIndexed) mine.index[j] = uint16_t(at + 32 * j);
            best = max(best, mine.key[j]);
        }
        if (kAhead) load(t + kTurn);
        if (!r.normalize) {
            top = lane_max<L>(best);
#pragma unroll
            for (int j = 0; j < PER; ++j)
                if (!R::never(mine.key[j])) every += expf(R::value(mine.key[j]) - R::value(top));
        }
        if constexpr (kSorted) mine.sort();
        for (int s = 0; s < r.chosen; ++s) {
            if constexpr (kSorted) best = mine.key[0];
            const uint32_t most = lane_max<L>(best);
            if (s == 0) top = most;
            if constexpr (R::kIndexed) {
                if (at == s) own = most;
                if constexpr (kSorted) {
                    mine.take(best == most);                                  // (its own lane, or all are taken)
                } else if (best == most) {
                    best = 0;
#pragma unroll
                    for (int j = 0; j < PER; ++j) {
                        if (mine.key[j] == most) mine.key[j] = 0;
                        best = max(best, mine.key[j]);
                    }
                }
            } else {
                int32_t which;
                if constexpr (PER == 1) {
                    which = __ffs(__ballot_sync(0xffffffffu, best == most) & segment) - 1 - lane / L * L;
                } else {
                    uint32_t index = 0xffffu;
                    if constexpr (kSorted) {
                        if (best == most) index = mine.index[0];
                    } else if (best == most) {
#pragma unroll
                        for (int j = PER - 1; j >= 0; --j)
                            if (mine.key[j] == most) index = uint32_t(at + 32 * j);
                    }
                    which = int32_t(__reduce_min_sync(0xffffffffu, index));
                }
                if (at == s) {
                    own = most;
                    own_choice = which;
                }
                if constexpr (kSorted) {
                    mine.take(which % 32 == at);
                } else if (which % 32 == at) {
                    best = 0;
#pragma unroll
                    for (int j = 0; j < PER; ++j) {
                        if (at + 32 * j == which) mine.key[j] = 0;
                        best = max(best, mine.key[j]);
                    }
                }
            }
        }
        if constexpr (R::kIndexed) own_choice = int32_t(0xffffu - (own & 0xffffu));
        if (R::never(own)) own_choice = -1;
        const float part = own_choice >= 0 ? expf(R::value(own) - R::value(top)) : 0.0f;
        const float total = lane_sum<L>(r.normalize ? part : every);
        if (in && at < r.chosen) {
            r.weights[t * r.chosen + at] = own_choice >= 0 ? part / total : 0.0f;
            r.choice[t * r.chosen + at] = own_choice;
            if (own_choice >= 0) atomicAdd(counts + own_choice, 1);           // whole numbers: any order
        }
    }
    __syncthreads();
    if (p.counts) {
        for (int e = threadIdx.x; e < r.experts; e += kRouteThreads) p.counts[int64_t(blockIdx.x) * r.experts + e] = counts[e];
        return;
    }
    __shared__ int32_t total;
    scan_counts(counts, r.experts, &total);
    __syncthreads();
    for (int e = threadIdx.x; e <= r.experts; e += kRouteThreads) r.offsets[e] = e < r.experts ? counts[e] : total;
    place_rows(r, Stretch(r, lo, hi), counts, counters);
}

// The second step where tokens are many: a block's rows of expert e follow those of lower experts and those of the blocks
// before it.  Two chains bound it, the blocks' counts (2 us) and the stretches' (3), at 16384 tokens with 8 of 128 experts.
__global__ void __launch_bounds__(kRouteThreads) redist_place_kernel(const RouteParams p)
{
    __shared__ int32_t base[kMostExperts], before[kMostExperts], counters[kCounters], total;
    const Route &r = p.r;
    let_next_start();
    wait_for_previous();
    const int64_t lo = int64_t(blockIdx.x) * p.per_block, hi = min(r.tokens, lo + p.per_block);
    const Stretch own(r, min(lo, hi), hi);                  // on its way while the counts are
    for (int e = threadIdx.x; e < r.experts; e += kRouteThreads) base[e] = before[e] = 0;
    __syncthreads();
    // the experts side by side, the blocks divided among the threads that are left
    const int across = (r.experts + 31) / 32 * 32, parts = max(1, kRouteThreads / across), part = int(threadIdx.x) / across;
    if (part < parts)
        for (int e = int(threadIdx.x) - part * across; e < r.experts; e += kRouteThreads) {
            int32_t sum = 0, early = 0;
#pragma unroll 8
            for (int b = part; b < int(gridDim.x); b += parts) {
                const int32_t n = p.counts[int64_t(b) * r.experts + e];
                sum += n;
                if (b < int(blockIdx.x)) early += n;
            }
            atomicAdd(base + e, sum);                       // whole numbers: any order
            atomicAdd(before + e, early);
        }
    __syncthreads();
    scan_counts(base, r.experts, &total);
    __syncthreads();
    if (blockIdx.x == 0)
        for (int e = threadIdx.x; e <= r.experts; e += kRouteThreads) r.offsets[e] = e < r.experts ? base[e] : total;
    __syncthreads();
    for (int e = threadIdx.x; e < r.experts; e += kRouteThreads) base[e] += before[e];
    __syncthreads();
    place_rows(r, own, base, counters);
}

// A warp per token.
template <typename T, int PER> __global__ void __launch_bounds__(256) redist_route_gradient_kernel(const Route r)
{
    const int lane = int(threadIdx.x) & 31;
    const int64_t t = int64_t(blockIdx.x) * 8 + (threadIdx.x >> 5);
    let_next_start();
    wait_for_previous();
    if (t >= r.tokens) return;
    float w = 0.0f, d = 0.0f;
    int32_t e = -1;
    if (lane < r.chosen) {
        e = r.choice[t * r.chosen + lane];
        if (e >= 0) {
            w = r.weights[t * r.chosen + lane];
            d = r.dweights[t * r.chosen + lane];
        }
    }
    const float mean = lane_sum<32>(w * d), own = r.normalize ? w * (d - mean) : w * d;
    float v[PER];
    if (r.normalize) {
#pragma unroll
        for (int j = 0; j < PER; ++j) v[j] = 0.0f;
    } else {
        const T *row = static_cast<const T *>(r.logits) + t * r.ld;
        uint32_t key[PER], top = 0;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            key[j] = lane + 32 * j < r.experts ? order_of(to_float(row[lane + 32 * j])) : 0;
            top = max(top, key[j]);
        }
        top = lane_max<32>(top);
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            v[j] = key[j] > kNever ? expf(value_of(key[j]) - value_of(top)) : 0.0f;
            sum += v[j];
        }
        const float scale = top > kNever ? -mean / lane_sum<32>(sum) : 0.0f;
#pragma unroll
        for (int j = 0; j < PER; ++j) v[j] *= scale;
    }
    for (int s = 0; s < r.chosen; ++s) {
        const int32_t to = __shfl_sync(0xffffffffu, e, s);
        const float g = __shfl_sync(0xffffffffu, own, s);
#pragma unroll
        for (int j = 0; j < PER; ++j)
            if (lane + 32 * j == to) v[j] += g;
    }
    T *out = static_cast<T *>(r.dlogits) + t * r.ld_dlogits;
#pragma unroll
    for (int j = 0; j < PER; ++j)
        if (lane + 32 * j < r.experts) out[lane + 32 * j] = from_float<T>(v[j]);
}

// ---- moves -----------------------------------------------------------------------------------------------

// All of them are bound by memory: 16384 tokens of 4096 bf16 to two rows each 57 us (7.0 TB/s), back with weights and a residual 85
// (6.3), their gradients 58 and 100 (6.7), against 6.56 for a plain copy.  Shorter rows share a warp; how many elements are
// accessed at once goes by what columns, addresses and strides have in common.

// N neighbours, loaded and stored at once.
template <typename T, int N> struct Some {
    static constexpr int kBytes = N * int(sizeof(T));
    union {
        T v[N];
        uint4 u4;
        uint2 u2;
        uint32_t u1;
        uint16_t uh;
    };
    __device__ __forceinline__ Some() {}
    __device__ __forceinline__ void load(const T *p)
    {
        if constexpr (kBytes == 16) u4 = *reinterpret_cast<const uint4 *>(p);
        else if constexpr (kBytes == 8) u2 = *reinterpret_cast<const uint2 *>(p);
        else if constexpr (kBytes == 4) u1 = *reinterpret_cast<const uint32_t *>(p);
        else uh = *reinterpret_cast<const uint16_t *>(p);
    }
    __device__ __forceinline__ void store(T *p) const
    {
        if constexpr (kBytes == 16) *reinterpret_cast<uint4 *>(p) = u4;
        else if constexpr (kBytes == 8) *reinterpret_cast<uint2 *>(p) = u2;
        else if constexpr (kBytes == 4) *reinterpret_cast<uint32_t *>(p) = u1;
        else *reinterpret_cast<uint16_t *>(p) = uh;
    }
};

__device__ __forceinline__ int32_t row_at(const Move &m, int64_t place)
{
    const int32_t p = m.position[place];
    return p >= 0 && p < m.rows ? p : -1;
}

constexpr int kMoveThreads = 256, kHeld = 4;        // pieces a thread holds at a time
constexpr int kGathered = 2;                        // ... of a row, where rows are read

// L threads take kHeld L pieces of a token (of its `pieces`): loaded once, stored to its rows.
template <typename T, int N, int L> __global__ void __launch_bounds__(kMoveThreads) redist_dispatch_kernel(const Move m, int pieces)
{
    const int64_t t = int64_t(blockIdx.x) * (kMoveThreads / L) + int(threadIdx.x) / L;
    const int first = int(blockIdx.y) * kHeld * L + int(threadIdx.x) % L;
    let_next_start();
    wait_for_previous();
    if (t >= m.tokens) return;
    const T *from = static_cast<const T *>(m.token) + t * m.ld_token;
    Some<T, N> v[kHeld];
#pragma unroll
    for (int j = 0; j < kHeld; ++j)
        if (first + j * L < pieces) v[j].load(from + int64_t(first + j * L) * N);
    for (int s = 0; s < m.chosen; ++s) {
        const int64_t row = row_at(m, t * m.chosen + s);
        if (row < 0) continue;
        T *to = static_cast<T *>(m.row) + row * m.ld_row;
#pragma unroll
        for (int j = 0; j < kHeld; ++j)
            if (first + j * L < pieces) v[j].store(to + int64_t(first + j * L) * N);
    }
}

// K places of a token: their rows and weights.
template <int K> struct Places {
    int32_t row[K];
    float weight[K];
    __device__ __forceinline__ void load(const Move &m, int64_t t, int from)
    {
#pragma unroll
        for (int i = 0; i < K; ++i) row[i] = t < m.tokens && from + i < m.chosen ? row_at(m, t * m.chosen + from + i) : -1;
#pragma unroll
        for (int i = 0; i < K; ++i) weight[i] = m.weights && t < m.tokens && from + i < m.chosen ? m.weights[t * m.chosen + from + i] : 1.0f;
    }
};

// The other way: a token's rows, weighted and added in the order of its places.  L threads share a token (or a stretch of it)
// and go on to others; K rows are on their way at a time, and the next token's places too, so that only one latency of
// memory stands between tokens.
template <typename T, int N, int L, int K> __global__ void __launch_bounds__(kMoveThreads, K > 2 ? 3 : 4) redist_combine_kernel(const Move m, int pieces)
{
    const int64_t step = int64_t(gridDim.x) * (kMoveThreads / L);
    const int first = int(blockIdx.y) * kGathered * L + int(threadIdx.x) % L;
    let_next_start();
    wait_for_previous();
    int64_t t = int64_t(blockIdx.x) * (kMoveThreads / L) + int(threadIdx.x) / L;
    Places<K> next;
    next.load(m, t, 0);
    for (; t < m.tokens; t += step) {
        float sum[kGathered][N] = {};
        Some<T, N> r[kGathered];
        if (m.residual) {
            const T *from = static_cast<const T *>(m.residual) + t * m.ld_residual;
#pragma unroll
            for (int j = 0; j < kGathered; ++j)
                if (first + j * L < pieces) r[j].load(from + int64_t(first + j * L) * N);
        }
        for (int s = 0; s < m.chosen; s += K) {
            const Places<K> now = next;
            Some<T, N> v[K][kGathered];
#pragma unroll
            for (int i = 0; i < K; ++i) {
                const T *from = static_cast<const T *>(m.row) + int64_t(now.row[i]) * m.ld_row;
#pragma unroll
                for (int j = 0; j < kGathered; ++j)
                    if (now.row[i] >= 0 && first + j * L < pieces) v[i][j].load(from + int64_t(first + j * L) * N);
            }
            if (s + K < m.chosen) next.load(m, t, s + K);
            else next.load(m, t + step, 0);
            if (s == 0 && m.residual)
#pragma unroll
                for (int j = 0; j < kGathered; ++j)
                    if (first + j * L < pieces)
#pragma unroll
                        for (int q = 0; q < N; ++q) sum[j][q] = to_float(r[j].v[q]);
#pragma unroll
            for (int i = 0; i < K; ++i)
#pragma unroll
                for (int j = 0; j < kGathered; ++j)
                    if (now.row[i] >= 0 && first + j * L < pieces)
#pragma unroll
                        for (int q = 0; q < N; ++q) sum[j][q] = fmaf(now.weight[i], to_float(v[i][j].v[q]), sum[j][q]);
        }
        T *to = static_cast<T *>(m.token) + t * m.ld_token;
#pragma unroll
        for (int j = 0; j < kGathered; ++j)
            if (first + j * L < pieces) {
                Some<T, N> out;
#pragma unroll
                for (int q = 0; q < N; ++q) out.v[q] = from_float<T>(sum[j][q]);
                out.store(to + int64_t(first + j * L) * N);
            }
    }
}

// The gradient of the latter: L threads take whole tokens, because dweights are sums over their columns.
template <typename T, int N, int L, int K> __global__ void __launch_bounds__(kMoveThreads, 3) redist_combine_gradient_kernel(const Move m, int pieces)
{
    constexpr int kLanes = L < 32 ? L : 32;                  // that add up a dot before it goes through shared memory
    __shared__ float dots[2][kMoveThreads / kLanes][kMostChosen];
    const int64_t step = int64_t(gridDim.x) * (kMoveThreads / L);
    const int group = int(threadIdx.x) / L, at = int(threadIdx.x) % L, slot = int(threadIdx.x) / kLanes, lane = int(threadIdx.x) % kLanes;
    let_next_start();
    wait_for_previous();
    int64_t t = int64_t(blockIdx.x) * (kMoveThreads / L) + group;
    Places<K> next;
    next.load(m, t, 0);
    int turn = 0;
    for (int64_t base = int64_t(blockIdx.x) * (kMoveThreads / L); base < m.tokens; base += step, t += step, turn ^= 1) {      // the block walks along
        const bool in = t < m.tokens;
        const T *dy = static_cast<const T *>(m.token) + (in ? t : 0) * m.ld_token;
        for (int s = 0; s < m.chosen; s += K) {
            const Places<K> now = next;
            float dot[K] = {};
            for (int first = at; first < pieces; first += kGathered * L) {
                Some<T, N> d[kGathered], v[K][kGathered];
#pragma unroll
                for (int j = 0; j < kGathered; ++j)
                    if (in && first + j * L < pieces) d[j].load(dy + int64_t(first + j * L) * N);
#pragma unroll
                for (int i = 0; i < K; ++i) {
                    const T *y = static_cast<const T *>(m.row) + int64_t(now.row[i]) * m.ld_row;
#pragma unroll
                    for (int j = 0; j < kGathered; ++j)
                        if (now.row[i] >= 0 && first + j * L < pieces) v[i][j].load(y + int64_t(first + j * L) * N);
                }
                if (first == at) {
                    if (s + K < m.chosen) next.load(m, t, s + K);
                    else next.load(m, t + step, 0);
                }
#pragma unroll
                for (int i = 0; i < K; ++i) {
                    T *to = static_cast<T *>(m.drow) + int64_t(now.row[i]) * m.ld_drow;
#pragma unroll
                    for (int j = 0; j < kGathered; ++j)
                        if (now.row[i] >= 0 && first + j * L < pieces) {
                            Some<T, N> out;
#pragma unroll
                            for (int q = 0; q < N; ++q) {
                                const float g = to_float(d[j].v[q]);
                                dot[i] = fmaf(g, to_float(v[i][j].v[q]), dot[i]);
                                out.v[q] = from_float<T>(now.weight[i] * g);
                            }
                            out.store(to + int64_t(first + j * L) * N);
                        }
                }
            }
            if (at >= pieces) {                             // (a thread without pieces has not asked)
                if (s + K < m.chosen) next.load(m, t, s + K);
                else next.load(m, t + step, 0);
            }
#pragma unroll
            for (int i = 0; i < K; ++i) {
                dot[i] = lane_sum<kLanes>(dot[i]);
                if (lane == 0 && s + i < m.chosen) dots[turn][slot][s + i] = dot[i];
            }
        }
        // the next token writes to the other half: one barrier for each
        if constexpr (L > 32) __syncthreads();
        else __syncwarp();
        for (int s = at; in && s < m.chosen; s += L) {
            float sum = 0.0f;
            for (int i = 0; i < L / kLanes; ++i) sum += dots[turn][group * (L / kLanes) + i][s];
            m.dweights[t * m.chosen + s] = sum;
        }
    }
}

// ---- moves of rows that start anywhere --------------------------------------------------------------------

// Where rows of 16-bit elements have no more in common than that: a row that is written is cut into the pieces that its own
// 16-byte boundaries make; what it is made of is loaded from any address and shifted.
template <typename T> struct Cut {
    static_assert(sizeof(T) == 2, "words are taken apart into halves");
    static constexpr int N = 8;
    int head, cols;                     // elements before the first boundary
    __device__ __forceinline__ Cut(const T *row, int64_t columns) : cols(int(columns))
    {
        head = min(int((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / int(sizeof(T)), cols);
    }
    // Piece p begins at element at(p) and has count(p) of them, none beyond the end.
    __device__ __forceinline__ int at(int p) const { return p == 0 ? 0 : head + (p - 1) * N; }
    __device__ __forceinline__ int count(int p) const { return p == 0 ? head : max(0, min(N, cols - at(p))); }
};
// Blocks together, shifted by an offset that all lanes of a warp share (a warp is at one row): one branch, then four
// instructions, where lanes with offsets of their own take thirty.
template <int WORD> __device__ __forceinline__ uint4 joined(const Blocks &b, bool half)
{
    const uint32_t w[8] = {b.a.x, b.a.y, b.a.z, b.a.w, b.b.x, b.b.y, b.b.z, b.b.w};
    if (!half) return make_uint4(w[WORD], w[WORD + 1], w[WORD + 2], w[WORD + 3]);
    return make_uint4(__funnelshift_r(w[WORD], w[WORD + 1], 16), __funnelshift_r(w[WORD + 1], w[WORD + 2], 16),
                      __funnelshift_r(w[WORD + 2], w[WORD + 3], 16), __funnelshift_r(w[WORD + 3], w[WORD + 4], 16));
}
__device__ __forceinline__ uint4 joined(const Blocks &b, const void *p)
{
    const uint32_t off = uint32_t(reinterpret_cast<uintptr_t>(p) & 15);
    if (off == 0) return b.a;
    if (off < 4) return joined<0>(b, off & 2);
    if (off < 8) return joined<1>(b, off & 2);
    if (off < 12) return joined<2>(b, off & 2);
    return joined<3>(b, off & 2);
}
template <typename T> __device__ __forceinline__ void floats(const uint4 &u, float (&v)[8])
{
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = unpack2<T>(w[i]);
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}
template <typename T> __device__ __forceinline__ uint4 rounded(const float (&v)[8])
{
    return make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
}
template <typename T> __device__ __forceinline__ void store_some(T *to, const uint4 &u, int count)
{
    if (count == 8) {
        *reinterpret_cast<uint4 *>(to) = u;
        return;
    }
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < count) reinterpret_cast<uint16_t *>(to)[i] = uint16_t(w[i >> 1] >> ((i & 1) * 16));
}

constexpr int kCut = 2;                 // pieces under way per thread

template <typename T, int L> __global__ void __launch_bounds__(kMoveThreads) redist_dispatch_any_kernel(const Move m)
{
    const int64_t t = int64_t(blockIdx.x) * (kMoveThreads / L) + int(threadIdx.x) / L;
    const int first = int(blockIdx.y) * kCut * L + int(threadIdx.x) % L;
    let_next_start();
    wait_for_previous();
    if (t >= m.tokens) return;
    const T *from = static_cast<const T *>(m.token) + t * m.ld_token;
    for (int s = 0; s < m.chosen; ++s) {
        const int64_t row = row_at(m, t * m.chosen + s);
        if (row < 0) continue;
        T *to = static_cast<T *>(m.row) + row * m.ld_row;
        const Cut<T> cut(to, m.cols);
        Blocks b[kCut];
#pragma unroll
        for (int j = 0; j < kCut; ++j)
            if (cut.count(first + j * L) > 0) b[j].load(from + cut.at(first + j * L), cut.count(first + j * L) * int(sizeof(T)));
#pragma unroll
        for (int j = 0; j < kCut; ++j)
            if (cut.count(first + j * L) > 0) store_some(to + cut.at(first + j * L), joined(b[j], from + cut.at(first + j * L)), cut.count(first + j * L));
    }
}

template <typename T, int L> __global__ void __launch_bounds__(kMoveThreads, 3) redist_combine_any_kernel(const Move m)
{
    constexpr int N = Cut<T>::N, K = 2;
    const int64_t step = int64_t(gridDim.x) * (kMoveThreads / L);
    const int first = int(blockIdx.y) * L + int(threadIdx.x) % L;
    let_next_start();
    wait_for_previous();
    int64_t t = int64_t(blockIdx.x) * (kMoveThreads / L) + int(threadIdx.x) / L;
    Places<K> next;
    next.load(m, t, 0);
    for (; t < m.tokens; t += step) {
        T *to = static_cast<T *>(m.token) + t * m.ld_token;
        const Cut<T> cut(to, m.cols);
        const int at = cut.at(first), count = cut.count(first), bytes = count * int(sizeof(T));
        const T *residual = static_cast<const T *>(m.residual) + t * m.ld_residual + at;
        Blocks r;
        if (m.residual && count > 0) r.load(residual, bytes);
        float sum[N] = {};
        for (int s = 0; s < m.chosen; s += K) {
            const Places<K> now = next;
            Blocks b[K];
#pragma unroll
            for (int i = 0; i < K; ++i)
                if (now.row[i] >= 0 && count > 0) b[i].load(static_cast<const T *>(m.row) + int64_t(now.row[i]) * m.ld_row + at, bytes);
            if (s + K < m.chosen) next.load(m, t, s + K);
            else next.load(m, t + step, 0);
            if (s == 0 && m.residual && count > 0) floats<T>(joined(r, residual), sum);
#pragma unroll
            for (int i = 0; i < K; ++i)
                if (now.row[i] >= 0 && count > 0) {
                    float v[N];
                    floats<T>(joined(b[i], static_cast<const T *>(m.row) + int64_t(now.row[i]) * m.ld_row + at), v);
#pragma unroll
                    for (int q = 0; q < N; ++q) sum[q] = fmaf(now.weight[i], v[q], sum[q]);
                }
        }
        if (count > 0) store_some(to + at, rounded<T>(sum), count);
    }
}

template <typename T, int L> __global__ void __launch_bounds__(kMoveThreads, 3) redist_combine_gradient_any_kernel(const Move m, int pieces)
{
    constexpr int N = Cut<T>::N;
    constexpr int kLanes = L < 32 ? L : 32;
    __shared__ float dots[2][kMoveThreads / kLanes][kMostChosen];
    const int64_t step = int64_t(gridDim.x) * (kMoveThreads / L);
    const int group = int(threadIdx.x) / L, lane_at = int(threadIdx.x) % L, slot = int(threadIdx.x) / kLanes, lane = int(threadIdx.x) % kLanes;
    let_next_start();
    wait_for_previous();
    int64_t t = int64_t(blockIdx.x) * (kMoveThreads / L) + group;
    int turn = 0;
    for (int64_t base = int64_t(blockIdx.x) * (kMoveThreads / L); base < m.tokens; base += step, t += step, turn ^= 1) {      // the block walks along
        const bool in = t < m.tokens;
        const T *dy = static_cast<const T *>(m.token) + (in ? t : 0) * m.ld_token;
#pragma unroll 1
        for (int s = 0; s < m.chosen; ++s) {
            const int64_t row = in ? row_at(m, t * m.chosen + s) : -1;
            float dot = 0.0f;
            if (row >= 0) {
                const float weight = m.weights[t * m.chosen + s];
                const T *y = static_cast<const T *>(m.row) + row * m.ld_row;
                T *to = static_cast<T *>(m.drow) + row * m.ld_drow;
                const Cut<T> cut(to, m.cols);
                for (int p = lane_at; p < pieces; p += kCut * L) {
                    Blocks d[kCut], v[kCut];
#pragma unroll
                    for (int j = 0; j < kCut; ++j) {
                        const int at = cut.at(p + j * L), bytes = cut.count(p + j * L) * int(sizeof(T));
                        if (bytes > 0) {
                            d[j].load(dy + at, bytes);
                            v[j].load(y + at, bytes);
                        }
                    }
#pragma unroll
                    for (int j = 0; j < kCut; ++j) {
                        const int at = cut.at(p + j * L), count = cut.count(p + j * L);
                        if (count <= 0) continue;
                        float g[N], x[N];
                        floats<T>(joined(d[j], dy + at), g);
                        floats<T>(joined(v[j], y + at), x);
#pragma unroll
                        for (int q = 0; q < N; ++q) {
                            if (q < count) dot = fmaf(g[q], x[q], dot);
                            g[q] *= weight;
                        }
                        store_some(to + at, rounded<T>(g), count);
                    }
                }
            }
            dot = lane_sum<kLanes>(dot);
            if (lane == 0) dots[turn][slot][s] = dot;
        }
        if constexpr (L > 32) __syncthreads();
        else __syncwarp();
        for (int s = lane_at; in && s < m.chosen; s += L) {
            float sum = 0.0f;
            for (int i = 0; i < L / kLanes; ++i) sum += dots[turn][group * (L / kLanes) + i][s];
            m.dweights[t * m.chosen + s] = sum;
        }
    }
}

// ---- host --------------------------------------------------------------------------------------------------

template <typename... P, typename... A>
cudaError_t launch(void (*kernel)(P...), dim3 grid, int threads, const LaunchOptions &o, cudaStream_t stream, A... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(unsigned(threads));
    cfg.stream = stream;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = o.pdl ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// Tokens of a block of the choice: those of one turn of its warps up to as many as are worth a second launch (the more the
// fewer the experts are), or one stretch per SM.
int64_t tokens_per_block(int64_t tokens, int experts, int sms)
{
    return std::max<int64_t>(experts <= 128 ? 128 : experts <= 256 ? 64 : 32, (tokens + sms - 1) / sms);
}

template <typename T> cudaError_t launch_route_typed(const RouteParams &p, int64_t blocks, const LaunchOptions &o, cudaStream_t stream)
{
    const dim3 grid = dim3(unsigned(blocks));
    const int e = p.r.experts;
    if (e <= 8) return launch(redist_route_kernel<T, 8, 1>, grid, kRouteThreads, o, stream, p);
    if (e <= 32) return launch(redist_route_kernel<T, 32, 1>, grid, kRouteThreads, o, stream, p);
    if (e <= 64) return launch(redist_route_kernel<T, 32, 2>, grid, kRouteThreads, o, stream, p);
    if (e <= 128) return launch(redist_route_kernel<T, 32, 4>, grid, kRouteThreads, o, stream, p);
    if (e <= 256) return launch(redist_route_kernel<T, 32, 8>, grid, kRouteThreads, o, stream, p);
    if (e <= 512) return launch(redist_route_kernel<T, 32, 16>, grid, kRouteThreads, o, stream, p);
    return launch(redist_route_kernel<T, 32, 32>, grid, kRouteThreads, o, stream, p);
}

template <typename T> cudaError_t launch_route_gradient_typed(const Route &r, const LaunchOptions &o, cudaStream_t stream)
{
    const dim3 grid = dim3(unsigned((r.tokens + 7) / 8));
    const int e = r.experts;
    if (e <= 32) return launch(redist_route_gradient_kernel<T, 1>, grid, 256, o, stream, r);
    if (e <= 128) return launch(redist_route_gradient_kernel<T, 4>, grid, 256, o, stream, r);
    if (e <= 256) return launch(redist_route_gradient_kernel<T, 8>, grid, 256, o, stream, r);
    if (e <= 512) return launch(redist_route_gradient_kernel<T, 16>, grid, 256, o, stream, r);
    return launch(redist_route_gradient_kernel<T, 32>, grid, 256, o, stream, r);
}

// How many neighbours can be accessed at once: what the columns, the addresses and the strides are all multiples of.
int together(int64_t cols, int type, std::initializer_list<std::pair<const void *, int64_t>> arrays)
{
    const int size = int(type_bytes(type));
    uint64_t all = 16 | uint64_t(cols * size);
    for (const auto &a : arrays)
        if (a.first) all |= uint64_t(uintptr_t(a.first)) | uint64_t(a.second * size);
    return int(all & (~all + 1)) / size;
}

enum Which { kDispatch, kCombine, kGradient };

// Blocks that walk along the tokens: as many as fit on the GPU.
unsigned walkers(int64_t tokens, int64_t tokens_per, unsigned across, int resident)
{
    return unsigned(std::max<int64_t>(1, std::min<int64_t>((tokens + tokens_per - 1) / tokens_per, (int64_t(resident) + across - 1) / across)));
}

template <Which W, typename T, int N, int L> cudaError_t launch_move_width(const Move &m, int pieces, int sms, const LaunchOptions &o, cudaStream_t stream)
{
    constexpr int kTokens = kMoveThreads / L;
    if constexpr (W == kDispatch) {
        const dim3 grid(unsigned((m.tokens + kTokens - 1) / kTokens), unsigned((pieces + kHeld * L - 1) / (kHeld * L)));
        if (grid.y > 65535) return cudaErrorInvalidValue;
        return launch(redist_dispatch_kernel<T, N, L>, grid, kMoveThreads, o, stream, m, pieces);
    } else if constexpr (W == kCombine) {
        const unsigned y = unsigned((pieces + kGathered * L - 1) / (kGathered * L));
        if (y > 65535) return cudaErrorInvalidValue;
        const dim3 grid(walkers(m.tokens, kTokens, y, sms * (m.chosen <= 2 ? 4 : 3)), y);
        if (m.chosen <= 2) return launch(redist_combine_kernel<T, N, L, 2>, grid, kMoveThreads, o, stream, m, pieces);
        return launch(redist_combine_kernel<T, N, L, 4>, grid, kMoveThreads, o, stream, m, pieces);
    } else {
        const dim3 grid(walkers(m.tokens, kTokens, 1, sms * 3));
        return launch(redist_combine_gradient_kernel<T, N, L, 2>, grid, kMoveThreads, o, stream, m, pieces);
    }
}

template <Which W, typename T, int N> cudaError_t launch_move_lanes(const Move &m, const LaunchOptions &o, cudaStream_t stream)
{
    const int64_t pieces = (m.cols + N - 1) / N;
    if (pieces > INT32_MAX / 2) return cudaErrorInvalidValue;
    int device = 0, sms = 0;
    const cudaError_t ce = current_device(&device, &sms);
    if (ce != cudaSuccess) return ce;
    // eight or sixteen lanes per token for the shortest rows, a warp (per stretch) for short ones, a block for longer ones
    // (single elements of 16 bits: rows of up to 15 only, see launch_move_typed)
    if constexpr (N * sizeof(T) > 2) {
        if (pieces > 32 * kHeld) return launch_move_width<W, T, N, kMoveThreads>(m, int(pieces), sms, o, stream);
        if (pieces > 16 && pieces <= 32) return launch_move_width<W, T, N, 16>(m, int(pieces), sms, o, stream);
        if (pieces > 16) return launch_move_width<W, T, N, 32>(m, int(pieces), sms, o, stream);
    }
    return launch_move_width<W, T, N, 8>(m, int(pieces), sms, o, stream);
}

template <Which W, typename T, int L> cudaError_t launch_move_any(const Move &m, const LaunchOptions &o, cudaStream_t stream)
{
    constexpr int kTokens = kMoveThreads / L;
    int device = 0, sms = 0;
    const cudaError_t ce = current_device(&device, &sms);
    if (ce != cudaSuccess) return ce;
    const int64_t pieces = 1 + (m.cols + Cut<T>::N - 1) / Cut<T>::N;        // at most
    const int64_t y = W == kGradient ? 1 : (pieces + L * (W == kDispatch ? kCut : 1) - 1) / (L * (W == kDispatch ? kCut : 1));
    if (y > 65535) return cudaErrorInvalidValue;
    if constexpr (W == kDispatch)
        return launch(redist_dispatch_any_kernel<T, L>, dim3(unsigned((m.tokens + kTokens - 1) / kTokens), unsigned(y)), kMoveThreads, o, stream, m);
    else if constexpr (W == kCombine)
        return launch(redist_combine_any_kernel<T, L>, dim3(walkers(m.tokens, kTokens, unsigned(y), sms * 3), unsigned(y)), kMoveThreads, o, stream, m);
    else
        return launch(redist_combine_gradient_any_kernel<T, L>, dim3(walkers(m.tokens, kTokens, 1, sms * 3)), kMoveThreads, o, stream, m, int(pieces));
}

template <Which W, typename T> cudaError_t launch_move_typed(const Move &m, int n, const LaunchOptions &o, cudaStream_t stream)
{
    constexpr int kMost = 16 / int(sizeof(T));
    // 8000 x 4095, two rows each, forward and backward: 295 us cut and shifted, 441 by single elements; but with two elements of
    // 16 bits or one of 32 at a time the latter take less (4094: 280 against 289; 1021 of 32 bits: 207 against 261)
    if constexpr (sizeof(T) == 2)
        if (n == 1 && m.cols >= 2 * kMost)
            return m.cols > 32 * kHeld * kMost ? launch_move_any<W, T, kMoveThreads>(m, o, stream)
                   : m.cols > 31 * kMost       ? launch_move_any<W, T, 32>(m, o, stream)
                   : m.cols > 15 * kMost       ? launch_move_any<W, T, 16>(m, o, stream)
                                               : launch_move_any<W, T, 8>(m, o, stream);
    if (n >= kMost) return launch_move_lanes<W, T, kMost>(m, o, stream);
    if (n >= kMost / 2) return launch_move_lanes<W, T, kMost / 2>(m, o, stream);
    if constexpr (kMost == 8)
        if (n >= 2) return launch_move_lanes<W, T, 2>(m, o, stream);
    return launch_move_lanes<W, T, 1>(m, o, stream);
}

template <Which W> cudaError_t launch_move(const Move &m, const LaunchOptions &o, cudaStream_t stream)
{
    if (m.tokens == 0) return cudaSuccess;
    const int n = together(m.cols, m.type, {{m.token, m.ld_token}, {m.row, m.ld_row}, {m.drow, m.ld_drow}, {m.residual, m.ld_residual}});
    switch (m.type) {
    case T_BF16: return launch_move_typed<W, __nv_bfloat16>(m, n, o, stream);
    case T_F16: return launch_move_typed<W, __half>(m, n, o, stream);
    default: return launch_move_typed<W, float>(m, n, o, stream);
    }
}

}  // namespace

int64_t route_scratch_bytes(int64_t tokens, int experts, int sms)
{
    const int64_t per = tokens_per_block(tokens, experts, sms), blocks = (tokens + per - 1) / per;
    return blocks > 1 ? blocks * experts * 4 : 0;
}

cudaError_t launch_route(const Route &r, void *scratch, int sms, const LaunchOptions &o, cudaStream_t stream)
{
    RouteParams p = {};
    p.r = r;
    p.per_block = tokens_per_block(r.tokens, r.experts, sms);
    const int64_t blocks = std::max<int64_t>(1, (r.tokens + p.per_block - 1) / p.per_block);
    p.counts = blocks > 1 ? static_cast<int32_t *>(scratch) : nullptr;
    const cudaError_t ce = r.type == T_BF16  ? launch_route_typed<__nv_bfloat16>(p, blocks, o, stream)
                           : r.type == T_F16 ? launch_route_typed<__half>(p, blocks, o, stream)
                                             : launch_route_typed<float>(p, blocks, o, stream);
    if (ce != cudaSuccess || blocks == 1) return ce;
    return launch(redist_place_kernel, dim3(unsigned(blocks)), kRouteThreads, o, stream, p);
}

cudaError_t launch_route_gradient(const Route &r, const LaunchOptions &o, cudaStream_t stream)
{
    if (r.tokens == 0) return cudaSuccess;
    switch (r.type) {
    case T_BF16: return launch_route_gradient_typed<__nv_bfloat16>(r, o, stream);
    case T_F16: return launch_route_gradient_typed<__half>(r, o, stream);
    default: return launch_route_gradient_typed<float>(r, o, stream);
    }
}

cudaError_t launch_dispatch(const Move &m, const LaunchOptions &o, cudaStream_t stream) { return launch_move<kDispatch>(m, o, stream); }
cudaError_t launch_combine(const Move &m, const LaunchOptions &o, cudaStream_t stream) { return launch_move<kCombine>(m, o, stream); }
cudaError_t launch_combine_gradient(const Move &m, const LaunchOptions &o, cudaStream_t stream) { return launch_move<kGradient>(m, o, stream); }

}  // namespace redist
