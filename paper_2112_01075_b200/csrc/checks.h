// What the C entry points of the operators share: checks of arguments, scratch handed out in pieces, operands laid out anew.
#pragma once

#include <cuda_runtime.h>

#include <algorithm>

#include "plan.hpp"
#include "product.h"
#include "redist.h"
#include "rows.h"

namespace redist {

extern thread_local int tl_cuda_error;

constexpr i64 kMostSize = (i64(1) << 31) - 512;      // tile coordinates are 32-bit

#define TRY(call)                          \
    do {                                   \
        redist_status rc_ = (call);        \
        if (rc_ != REDIST_OK) return rc_;  \
    } while (0)

inline redist_status cuda(cudaError_t ce)
{
    if (ce == cudaSuccess) return REDIST_OK;
    tl_cuda_error = int(ce);
    return REDIST_ECUDA;
}

inline LaunchOptions options()
{
    const Tuning t = current_tuning();
    return LaunchOptions{int32_t(t.pdl), uint32_t(t.wait_polls), uint32_t(t.test_extra_tx), int32_t(t.test_product_shape), int32_t(t.test_product_parts)};
}

inline i64 round_up(i64 v, i64 to) { return (v + to - 1) / to * to; }

// Hands out the caller's scratch piece by piece; with base 0 it only counts.
struct Pieces {
    uintptr_t base;
    i64 used = 0;
    void *take(i64 bytes)
    {
        const i64 at = used;
        used += round_up(bytes, 256);
        return reinterpret_cast<void *>(base + uintptr_t(at));
    }
};

// ---- matrices -----------------------------------------------------------------------------------------

inline bool row_major(const redist_matrix &m, i64 rows, i64 cols)
{
    return (m.col_stride == 1 || cols <= 1) && (m.row_stride >= cols || rows <= 1) && m.row_stride >= 0;
}

inline bool column_major(const redist_matrix &m, i64 rows, i64 cols)
{
    return (m.row_stride == 1 || rows <= 1) && (m.col_stride >= rows || cols <= 1) && m.col_stride >= 0;
}

// Bytes of a matrix in memory: where it begins and ends, and how its lines lie within.
struct Extent {
    uintptr_t lo, hi;
    i64 line, pitch;        // bytes of a line, bytes from line to line
};

inline Extent extent(const redist_matrix &m, i64 rows, i64 cols, i64 element, i64 batch = 1, i64 batch_stride = 0)
{
    const uintptr_t lo = uintptr_t(m.data);
    if (rows == 0 || cols == 0 || batch == 0) return Extent{lo, lo, 0, 1};
    const bool by_rows = row_major(m, rows, cols);
    const i64 lines = by_rows ? rows : cols, line = by_rows ? cols : rows;
    const i64 pitch = lines > 1 ? (by_rows ? m.row_stride : m.col_stride) : line;
    const i64 last = (lines - 1) * pitch + line + (batch > 1 ? (batch - 1) * batch_stride : 0);
    return Extent{lo, lo + uintptr_t(last * element), line * element, batch > 1 ? 1 : pitch * element};
}

inline Extent extent(const void *p, i64 bytes) { return Extent{uintptr_t(p), uintptr_t(p) + uintptr_t(p ? bytes : 0), bytes, 1}; }

// Whether two ranges share a byte.  Column blocks of one wider matrix interleave without doing so: with the same
// pitch, what counts is where the lines lie within it.
inline bool overlap(const Extent &a, const Extent &b)
{
    if (a.lo >= a.hi || b.lo >= b.hi || a.hi <= b.lo || b.hi <= a.lo) return false;
    if (a.pitch != b.pitch || a.pitch <= 1) return true;
    const uintptr_t pitch = uintptr_t(a.pitch);
    const i64 at = b.lo >= a.lo ? i64((b.lo - a.lo) % pitch) : i64((pitch - (a.lo - b.lo) % pitch) % pitch);
    return at < a.line || a.pitch - at < b.line;
}

// `outs` may overlap neither one another nor any of `ins`.
inline redist_status apart(const Extent *outs, int n_outs, const Extent *ins, int n_ins)
{
    for (int i = 0; i < n_outs; ++i) {
        for (int j = 0; j < i; ++j)
            if (overlap(outs[i], outs[j])) return REDIST_EOVERLAP;
        for (int j = 0; j < n_ins; ++j)
            if (overlap(outs[i], ins[j])) return REDIST_EOVERLAP;
    }
    return REDIST_OK;
}

inline redist_status check_out(const redist_matrix &m, i64 rows, i64 cols, i64 element)
{
    if (!m.data || !row_major(m, rows, cols)) return REDIST_EINVAL;
    return uintptr_t(m.data) % uintptr_t(element) ? REDIST_EALIGN : REDIST_OK;
}

inline redist_status check_in(const redist_matrix &m, i64 rows, i64 cols, i64 element)
{
    if (!m.data || !(row_major(m, rows, cols) || column_major(m, rows, cols))) return REDIST_EINVAL;
    return uintptr_t(m.data) % uintptr_t(element) ? REDIST_EALIGN : REDIST_OK;
}

inline redist_status check_scratch(const void *scratch, size_t have, i64 need)
{
    if (need == 0) return REDIST_OK;
    if (!scratch || have < size_t(need)) return REDIST_ESCRATCH;
    return uintptr_t(scratch) & 255 ? REDIST_EALIGN : REDIST_OK;
}

// The lines of a matrix: row-major by preference.
struct Lines {
    const void *data;
    i64 lines, line, ld;
    bool by_rows;
};

inline Lines lines_of(const redist_matrix &m, i64 rows, i64 cols)
{
    if (row_major(m, rows, cols)) return Lines{m.data, rows, cols, rows > 1 ? m.row_stride : round_up(cols, 8), true};
    return Lines{m.data, cols, rows, cols > 1 ? m.col_stride : round_up(rows, 8), false};
}

// A matrix as an operand: as it lies, or (fits == false) laid out anew in scratch, line by line.
struct Placed {
    Lines from;
    bool fits;
    void *copy = nullptr;
    i64 ld;
    Placed(const redist_matrix &m, i64 rows, i64 cols, Pieces &pieces) : from(lines_of(m, rows, cols))
    {
        fits = operand_fits(from.data, from.ld, 0, 1);
        ld = fits ? from.ld : round_up(from.line, 64);
        if (!fits) copy = pieces.take(from.lines * ld * 2);
    }
    // Adds what lays it anew to a list of such.
    void lay(int type, Lay *list, int &count) const
    {
        if (fits) return;
        Lay l = {};
        l.rows = from.lines;
        l.cols = from.line;
        l.type = type;
        l.src = from.data;
        l.ld_src = from.ld;
        l.dst = copy;
        l.ld_dst = ld;
        list[count++] = l;
    }
    // `rows_survive`: the product sums over this matrix's columns (else over its rows)
    Operand operand(bool rows_survive) const { return Operand{fits ? from.data : copy, ld, 0, from.by_rows == rows_survive ? 0 : 1}; }
};

}  // namespace redist
