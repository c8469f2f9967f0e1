// The C boundary of the block of experts and of the bound on the gradients: argument checks, scratch layout, launches.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <vector>

#include "checks.h"
#include "clip.h"
#include "experts.h"
#include "redist.h"
#include "routing.h"

using namespace redist;

namespace {

int sm_count()
{
    int device = 0, sms = 0;
    return current_device(&device, &sms) == cudaSuccess ? sms : 148;
}

bool on(const void *p, int bytes) { return uintptr_t(p) % uintptr_t(bytes) == 0; }

i64 row_stride(const redist_matrix &m, i64 rows, i64 cols) { return rows > 1 ? m.row_stride : round_up(cols, 8); }

// ---- the router ------------------------------------------------------------------------------------------

redist_status check_route(const redist_route &q)
{
    if (q.tokens < 0 || q.experts < 1 || q.chosen < 1 || q.chosen > q.experts || q.normalize < 0 || q.normalize > 1) return REDIST_EINVAL;
    if (q.type < REDIST_BF16 || q.type > REDIST_F32) return REDIST_EINVAL;
    if (q.experts > kMostExperts || q.chosen > kMostChosen || q.tokens > ((i64(1) << 31) - 1) / q.chosen) return REDIST_EUNSUPPORTED;
    return REDIST_OK;
}

redist_status check_route_forward(const redist_route &q)
{
    TRY(check_route(q));
    if (!q.offsets) return REDIST_EINVAL;
    if (!on(q.offsets, 4) || !on(q.weights, 4) || !on(q.choice, 4) || !on(q.position, 4)) return REDIST_EALIGN;
    if (q.tokens == 0) return REDIST_OK;
    if (!q.weights || !q.choice || !q.position) return REDIST_EINVAL;
    return check_out(q.logits, q.tokens, q.experts, type_bytes(q.type));
}

Route route_of(const redist_route &q)
{
    Route r = {};
    r.tokens = q.tokens;
    r.experts = q.experts;
    r.chosen = q.chosen;
    r.type = q.type;
    r.normalize = q.normalize;
    r.logits = q.logits.data;
    r.ld = row_stride(q.logits, q.tokens, q.experts);
    r.weights = q.weights;
    r.choice = q.choice;
    r.position = q.position;
    r.offsets = q.offsets;
    return r;
}

// ---- moves -----------------------------------------------------------------------------------------------

constexpr i64 kMostColumns = i64(65535) * 512;      // a grid's second dimension, where single elements are moved

redist_status check_move(const redist_move &q, bool weights)
{
    if (q.tokens < 0 || q.rows < 0 || q.cols < 1 || q.chosen < 1) return REDIST_EINVAL;
    if (q.type < REDIST_BF16 || q.type > REDIST_F32) return REDIST_EINVAL;
    if (q.tokens > kMostSize || q.rows > kMostSize || q.cols > kMostColumns || q.chosen > kMostChosen) return REDIST_EUNSUPPORTED;
    if (!on(q.position, 4) || !on(q.weights, 4) || !on(q.dweights, 4)) return REDIST_EALIGN;
    if (q.tokens == 0) return REDIST_OK;
    if (!q.position || (weights && !q.weights)) return REDIST_EINVAL;
    const i64 e = type_bytes(q.type);
    TRY(check_out(q.token, q.tokens, q.cols, e));
    if (q.rows > 0) TRY(check_out(q.row, q.rows, q.cols, e));
    return REDIST_OK;
}

Move move_of(const redist_move &q)
{
    Move m = {};
    m.tokens = q.tokens;
    m.rows = q.rows;
    m.cols = q.cols;
    m.type = q.type;
    m.chosen = q.chosen;
    m.token = q.token.data;
    m.ld_token = row_stride(q.token, q.tokens, q.cols);
    m.row = q.rows ? q.row.data : nullptr;
    m.ld_row = row_stride(q.row, q.rows, q.cols);
    m.position = q.position;
    return m;
}

struct MoveExtents {
    Extent token, row, residual, drow, position, weights, dweights;
    explicit MoveExtents(const redist_move &q)
        : token(extent(q.token, q.tokens, q.cols, type_bytes(q.type))), row(extent(q.row, q.rows, q.cols, type_bytes(q.type))),
          residual(extent(q.residual, q.residual.data ? q.tokens : 0, q.cols, type_bytes(q.type))),
          drow(extent(q.drow, q.rows, q.cols, type_bytes(q.type))), position(extent(q.position, q.tokens * q.chosen * 4)),
          weights(extent(q.weights, q.tokens * q.chosen * 4)), dweights(extent(q.dweights, q.tokens * q.chosen * 4))
    {
    }
};

// ---- experts ---------------------------------------------------------------------------------------------

redist_status check_experts(const redist_experts &q)
{
    if (q.rows < 0 || q.in_features < 1 || q.out_features < 1 || q.experts < 1) return REDIST_EINVAL;
    if (q.type != REDIST_BF16 && q.type != REDIST_F16) return REDIST_EINVAL;
    if (q.activation < REDIST_ACT_NONE || q.activation > REDIST_ACT_SILU) return REDIST_EINVAL;
    if (q.rows > kMostSize || q.in_features > kMostSize || q.out_features > kMostSize || q.experts > 65535) return REDIST_EUNSUPPORTED;
    if (q.rows > 0 && !q.offsets) return REDIST_EINVAL;
    return on(q.offsets, 4) ? REDIST_OK : REDIST_EALIGN;
}

// A stack of matrices, all row-major or all column-major, none overlapping the next.
redist_status check_stack(const redist_matrix &m, i64 rows, i64 cols, i64 count, i64 stride)
{
    TRY(check_in(m, rows, cols, 2));
    if (count > 1) {
        const Extent one = extent(m, rows, cols, 1);
        if (stride < i64(one.hi - one.lo)) return REDIST_EINVAL;
    }
    return REDIST_OK;
}

redist_status check_experts_forward(const redist_experts &q)
{
    TRY(check_experts(q));
    if (q.rows == 0) return REDIST_OK;
    TRY(check_out(q.x, q.rows, q.in_features, 2));
    TRY(check_stack(q.w, q.out_features, q.in_features, q.experts, q.w_stride));
    TRY(check_out(q.out, q.rows, q.out_features, 2));
    if (q.pre.data) TRY(check_out(q.pre, q.rows, q.out_features, 2));
    if (q.bias) {
        if (q.bias_type < REDIST_BF16 || q.bias_type > REDIST_F32 || q.bias_stride < 0) return REDIST_EINVAL;
        if (!on(q.bias, int(type_bytes(q.bias_type)))) return REDIST_EALIGN;
    }
    return REDIST_OK;
}

redist_status check_experts_backward(const redist_experts &q, const redist_experts_grads &g)
{
    TRY(check_experts(q));
    if (q.rows > 0) {
        TRY(check_out(g.dy, q.rows, q.out_features, 2));
        if (q.activation != REDIST_ACT_NONE) TRY(check_out(q.pre, q.rows, q.out_features, 2));
        if (g.dx.data) {
            TRY(check_stack(q.w, q.out_features, q.in_features, q.experts, q.w_stride));
            TRY(check_out(g.dx, q.rows, q.in_features, 2));
        }
        if (g.dw.data) TRY(check_out(q.x, q.rows, q.in_features, 2));
    }
    if (g.dw.data) {
        TRY(check_out(g.dw, q.out_features, q.in_features, 2));
        TRY(check_stack(g.dw, q.out_features, q.in_features, q.experts, g.dw_stride));
    }
    return on(g.dbias, 4) ? REDIST_OK : REDIST_EALIGN;
}

// A stack as an operand: as it lies, or laid out anew in scratch.
struct PlacedStack {
    Lines from;
    i64 count, stride, ld, plane;
    bool fits;
    void *copy = nullptr;
    PlacedStack(const redist_matrix &m, i64 rows, i64 cols, i64 n, i64 apart, Pieces &pieces) : from(lines_of(m, rows, cols)), count(n), stride(apart)
    {
        fits = !m.data || operand_fits(from.data, from.ld, stride, int(std::min<i64>(n, 2)));
        ld = fits ? from.ld : round_up(from.line, 64);
        plane = fits ? stride : from.lines * ld;
        if (!fits) copy = pieces.take(count * plane * 2);
    }
    StackLay lay(const int32_t *offsets, i64 rows) const
    {
        return StackLay{from.data, copy, count, from.lines, from.line, from.ld, stride, ld, plane, offsets, rows, 0};
    }
    Operand operand(bool rows_survive) const { return Operand{fits ? from.data : copy, ld, plane, from.by_rows == rows_survive ? 0 : 1}; }
};

const redist_matrix kAbsent = {nullptr, 1, 1};

// A forward call of a few rows reads its operands as they lie and needs no scratch: up to eight rows, where its blocks are more
// than the tiles and start sooner (2 rows of 8 experts, 4096 -> 4096: 15.4 us against 18; 6 rows of 128, 1024 -> 1024: 6.4 and 9.2;
// 4 of 8, 81 -> 153: 6.7 and 8.6), and up to 32 where the weights they meet are small or sums long, of which a tile takes one step
// after the other (32 rows of 4, 512 -> 512: 4.3 and 5.4; 20 of 2, 2576 -> 90: 6.1 and 10.2; but 9 of 2, 256 -> 6795: 7.4 and 6.2, and 32
// of 8, 4096 -> 4096: 52 and 49).  Off 16-byte boundaries shifting costs more, so only with a few rows for each expert or very long
// sums with few results (26 rows of 16, 555 -> 121: 6.9 and 8.5; 32 of 40, 5619 -> 73: 24 and 31; but 26 of one, 1037 -> 68: 16 and 10).
bool few_expert_rows(const redist_experts &q, const LaunchOptions &o)
{
    if (o.test_shape || q.rows > kFewRows || !row_major(q.x, q.rows, q.in_features) || !row_major(q.w, q.out_features, q.in_features)) return false;
    if (q.rows <= 8) return true;
    const i64 busy = std::min<i64>(q.rows, q.experts);
    const double met = double(busy) * double(q.in_features) * double(q.out_features);
    if (operand_fits(q.x.data, row_stride(q.x, q.rows, q.in_features), 0, 1) &&
        operand_fits(q.w.data, row_stride(q.w, q.out_features, q.in_features), q.w_stride, int(std::min<i64>(q.experts, 2))))
        return met <= double(q.in_features >= 2048 ? 1 << 22 : 1 << 20);
    return (met <= double(1 << 20) && q.rows <= 4 * busy) || (q.in_features >= 4096 && q.out_features <= 256);
}

struct ExpertsForward {
    PlacedStack x, w;
    ExpertsForward(const redist_experts &q, Pieces &p)
        : x(q.x, q.rows, q.in_features, 1, 0, p), w(q.w, q.out_features, q.in_features, q.experts, q.w_stride, p)
    {
    }
};

struct ExpertsBackward {
    bool fresh;             // dz is computed (or laid out) into scratch; else dy itself is the operand
    i64 ld_dz;
    void *dz = nullptr, *maps = nullptr;
    float *partials = nullptr;
    PlacedStack x, w;
    ExpertsBackward(const redist_experts &q, const redist_experts_grads &g, Pieces &p)
        : fresh((g.dx.data || g.dw.data) && (q.activation != REDIST_ACT_NONE || !operand_fits(g.dy.data, lines_of(g.dy, q.rows, q.out_features).ld, 0, 1))),
          x(g.dw.data ? q.x : kAbsent, g.dw.data ? q.rows : 0, g.dw.data ? q.in_features : 0, 1, 0, p),
          w(g.dx.data ? q.w : kAbsent, g.dx.data ? q.out_features : 0, g.dx.data ? q.in_features : 0, g.dx.data ? q.experts : 1, g.dx.data ? q.w_stride : 0, p)
    {
        ld_dz = fresh ? round_up(q.out_features, 64) : lines_of(g.dy, q.rows, q.out_features).ld;
        if (fresh) dz = p.take(q.rows * ld_dz * 2);
        if (g.dbias) partials = static_cast<float *>(p.take(expert_partial_bytes(q.rows, q.out_features, q.experts)));
        if (g.dw.data) maps = p.take(grouped_maps_bytes(q.experts));
    }
};

// ---- the bound on the gradients --------------------------------------------------------------------------

redist_status check_clip(const redist_clip_op &q)
{
    if (q.count < 0 || (q.count > 0 && !q.tensors) || !(q.eps >= 0.0f) || !std::isfinite(q.eps) || std::isnan(q.max_norm)) return REDIST_EINVAL;
    for (i64 i = 0; i < q.count; ++i) {
        const redist_tensor &t = q.tensors[i];
        if (t.elements < 0 || t.type < REDIST_BF16 || t.type > REDIST_F32 || t.reserved != 0 || (t.elements > 0 && !t.data)) return REDIST_EINVAL;
        if (t.elements > i64(1) << 40) return REDIST_EUNSUPPORTED;
        if (!on(t.data, int(type_bytes(t.type))) || !on(t.out, int(type_bytes(t.type)))) return REDIST_EALIGN;
    }
    return on(q.norm, 4) ? REDIST_OK : REDIST_EALIGN;
}

std::vector<ClipTensor> clip_tensors(const redist_clip_op &q)
{
    std::vector<ClipTensor> all;
    all.reserve(size_t(q.count));
    for (i64 i = 0; i < q.count; ++i) {
        const redist_tensor &t = q.tensors[i];
        if (t.elements > 0) all.push_back(ClipTensor{t.data, t.out ? t.out : t.data, t.elements, t.type});
    }
    return all;
}

// What is written may overlap neither anything else that is written nor anything that is read, but a tensor itself.
redist_status check_clip_overlap(const std::vector<ClipTensor> &tensors, const redist_clip_op &q, const void *scratch, i64 scratch_bytes)
{
    struct Range {
        uintptr_t lo, hi;
        i64 owner;
    };
    std::vector<Range> outs;
    outs.reserve(tensors.size() + 2);
    if (q.max_norm >= 0.0f)
        for (size_t i = 0; i < tensors.size(); ++i) {
            const uintptr_t lo = uintptr_t(tensors[i].out);
            outs.push_back(Range{lo, lo + uintptr_t(tensors[i].elements * type_bytes(tensors[i].type)), i64(i)});
        }
    if (q.norm) outs.push_back(Range{uintptr_t(q.norm), uintptr_t(q.norm) + 4, -1});
    if (scratch) outs.push_back(Range{uintptr_t(scratch), uintptr_t(scratch) + uintptr_t(scratch_bytes), -1});
    std::sort(outs.begin(), outs.end(), [](const Range &a, const Range &b) { return a.lo < b.lo; });
    for (size_t i = 1; i < outs.size(); ++i)
        if (outs[i].lo < outs[i - 1].hi) return REDIST_EOVERLAP;
    for (size_t i = 0; i < tensors.size(); ++i) {
        const uintptr_t lo = uintptr_t(tensors[i].data), hi = lo + uintptr_t(tensors[i].elements * type_bytes(tensors[i].type));
        // the outputs are disjoint, so their ends are in order too: the first that ends behind lo
        const auto at = std::partition_point(outs.begin(), outs.end(), [&](const Range &r) { return r.hi <= lo; });
        if (at == outs.end() || at->lo >= hi) continue;
        if (at->owner != i64(i) || at->lo != lo) return REDIST_EOVERLAP;
    }
    return REDIST_OK;
}

}  // namespace

extern "C" {

size_t redist_route_scratch_bytes(const redist_route *op)
{
    return op && check_route(*op) == REDIST_OK ? size_t(route_scratch_bytes(op->tokens, op->experts, sm_count())) : 0;
}

redist_status redist_route_forward(const redist_route *op, void *scratch, size_t scratch_bytes, void *cuda_stream)
{
    try {
        if (!op) return REDIST_EINVAL;
        const redist_route &q = *op;
        TRY(check_route_forward(q));
        const int sms = sm_count();
        const i64 places = q.tokens * q.chosen * 4, need = route_scratch_bytes(q.tokens, q.experts, sms);
        const Extent outs[5] = {extent(q.weights, places), extent(q.choice, places), extent(q.position, places), extent(q.offsets, i64(q.experts + 1) * 4),
                                extent(scratch, need)};
        const Extent ins[1] = {extent(q.logits, q.tokens, q.experts, type_bytes(q.type))};
        TRY(apart(outs, 5, ins, 1));
        TRY(check_scratch(scratch, scratch_bytes, need));
        return cuda(launch_route(route_of(q), scratch, sms, options(), static_cast<cudaStream_t>(cuda_stream)));
    } catch (...) {
        return REDIST_EINTERNAL;
    }
}

redist_status redist_route_backward(const redist_route *op, const float *dweights, const redist_matrix *dlogits, void *cuda_stream)
{
    try {
        if (!op || !dlogits) return REDIST_EINVAL;
        const redist_route &q = *op;
        TRY(check_route(q));
        if (q.tokens == 0) return REDIST_OK;
        if (!q.weights || !q.choice || !dweights) return REDIST_EINVAL;
        if (!on(q.weights, 4) || !on(q.choice, 4) || !on(dweights, 4)) return REDIST_EALIGN;
        const i64 e = type_bytes(q.type), places = q.tokens * q.chosen * 4;
        TRY(check_out(*dlogits, q.tokens, q.experts, e));
        if (!q.normalize) TRY(check_out(q.logits, q.tokens, q.experts, e));
        const Extent outs[1] = {extent(*dlogits, q.tokens, q.experts, e)};
        const Extent ins[4] = {extent(q.logits, q.normalize ? 0 : q.tokens, q.experts, e), extent(q.weights, places), extent(q.choice, places), extent(dweights, places)};
        TRY(apart(outs, 1, ins, 4));
        Route r = route_of(q);
        r.dweights = dweights;
        r.dlogits = dlogits->data;
        r.ld_dlogits = row_stride(*dlogits, q.tokens, q.experts);
        return cuda(launch_route_gradient(r, options(), static_cast<cudaStream_t>(cuda_stream)));
    } catch (...) {
        return REDIST_EINTERNAL;
    }
}

redist_status redist_dispatch_forward(const redist_move *op, void *cuda_stream)
{
    try {
        if (!op) return REDIST_EINVAL;
        TRY(check_move(*op, false));
        const MoveExtents x(*op);
        const Extent outs[1] = {x.row}, ins[2] = {x.token, x.position};
        TRY(apart(outs, 1, ins, 2));
        return cuda(launch_dispatch(move_of(*op), options(), static_cast<cudaStream_t>(cuda_stream)));
    } catch (...) {
        return REDIST_EINTERNAL;
    }
}

redist_status redist_dispatch_backward(const redist_move *op, void *cuda_stream)
{
    try {
        if (!op) return REDIST_EINVAL;
        TRY(check_move(*op, false));
        const MoveExtents x(*op);
        const Extent outs[1] = {x.token}, ins[2] = {x.row, x.position};
        TRY(apart(outs, 1, ins, 2));
        return cuda(launch_combine(move_of(*op), options(), static_cast<cudaStream_t>(cuda_stream)));
    } catch (...) {
        return REDIST_EINTERNAL;
    }
}

redist_status redist_combine_forward(const redist_move *op, void *cuda_stream)
{
    try {
        if (!op) return REDIST_EINVAL;
        const redist_move &q = *op;
        TRY(check_move(q, false));
        const bool residual = q.tokens > 0 && q.residual.data;
        if (residual) TRY(check_out(q.residual, q.tokens, q.cols, type_bytes(q.type)));
        Move m = move_of(q);
        m.weights = q.weights;
        if (residual) {
            m.residual = q.residual.data;
            m.ld_residual = row_stride(q.residual, q.tokens, q.cols);
        }
        MoveExtents x(q);
        if (residual && m.residual == m.token && m.ld_residual == m.ld_token) x.residual = extent(nullptr, 0);       // in place
        const Extent outs[1] = {x.token}, ins[4] = {x.row, x.position, x.weights, x.residual};
        TRY(apart(outs, 1, ins, 4));
        return cuda(launch_combine(m, options(), static_cast<cudaStream_t>(cuda_stream)));
    } catch (...) {
        return REDIST_EINTERNAL;
    }
}

redist_status redist_combine_backward(const redist_move *op, void *cuda_stream)
{
    try {
        if (!op) return REDIST_EINVAL;
        const redist_move &q = *op;
        TRY(check_move(q, true));
        if (q.tokens > 0 && !q.dweights) return REDIST_EINVAL;
        if (q.tokens > 0 && q.rows > 0) TRY(check_out(q.drow, q.rows, q.cols, type_bytes(q.type)));
        const MoveExtents x(q);
        const Extent outs[2] = {x.drow, x.dweights}, ins[4] = {x.token, x.row, x.position, x.weights};
        TRY(apart(outs, 2, ins, 4));
        Move m = move_of(q);
        m.weights = q.weights;
        m.dweights = q.dweights;
        m.drow = q.rows ? q.drow.data : nullptr;
        m.ld_drow = row_stride(q.drow, q.rows, q.cols);
        return cuda(launch_combine_gradient(m, options(), static_cast<cudaStream_t>(cuda_stream)));
    } catch (...) {
        return REDIST_EINTERNAL;
    }
}

size_t redist_experts_scratch_bytes(const redist_experts *op, const redist_experts_grads *grads)
{
    if (!op) return 0;
    Pieces p{0};
    if (!grads) {
        if (check_experts_forward(*op) != REDIST_OK || op->rows == 0 || few_expert_rows(*op, options())) return 0;
        ExpertsForward f(*op, p);
    } else {
        if (check_experts_backward(*op, *grads) != REDIST_OK || op->rows == 0) return 0;
        ExpertsBackward b(*op, *grads, p);
    }
    return size_t(p.used);
}

redist_status redist_experts_forward(const redist_experts *op, void *scratch, size_t scratch_bytes, void *cuda_stream)
{
    try {
        if (!op) return REDIST_EINVAL;
        const redist_experts &q = *op;
        TRY(check_experts_forward(q));
        if (q.rows == 0) return REDIST_OK;
        const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
        const LaunchOptions o = options();
        Pieces p{uintptr_t(scratch)};
        const bool few = few_expert_rows(q, o);
        Pieces none{0};
        const ExpertsForward f(q, few ? none : p);
        const Extent outs[3] = {extent(q.out, q.rows, q.out_features, 2), extent(q.pre, q.pre.data ? q.rows : 0, q.out_features, 2), extent(scratch, p.used)};
        const Extent ins[4] = {extent(q.x, q.rows, q.in_features, 2), extent(q.w, q.out_features, q.in_features, 2, q.experts, q.w_stride),
                               extent(q.bias, ((q.experts - 1) * q.bias_stride + q.out_features) * type_bytes(q.bias_type)), extent(q.offsets, i64(q.experts + 1) * 4)};
        TRY(apart(outs, 3, ins, 4));
        TRY(check_scratch(scratch, scratch_bytes, p.used));
        Grouped g = {};
        g.rows = q.rows;
        g.m = q.out_features;
        g.k = q.in_features;
        g.experts = q.experts;
        g.type = q.type;
        g.offsets = q.offsets;
        g.out = q.out.data;
        g.ld_out = row_stride(q.out, q.rows, q.out_features);
        g.pre = q.pre.data;
        g.ld_pre = q.pre.data ? row_stride(q.pre, q.rows, q.out_features) : 0;
        g.bias = q.bias;
        g.bias_type = q.bias_type;
        g.bias_stride = q.bias_stride;
        g.activation = q.activation;
        if (few) {
            g.a = Operand{f.w.from.data, f.w.from.ld, q.w_stride, 0};
            g.b = Operand{f.x.from.data, f.x.from.ld, 0, 0};
            return cuda(launch_few_grouped(g, o, stream));
        }
        Prepare before = {};
        before.type = q.type;
        before.lay[0] = f.w.lay(q.offsets, q.rows);
        before.lay[1] = f.x.lay(nullptr, 0);
        TRY(cuda(launch_prepare(before, o, stream)));
        g.a = f.w.operand(true);
        g.b = f.x.operand(true);
        return cuda(launch_grouped(g, nullptr, nullptr, o, stream));
    } catch (...) {
        return REDIST_EINTERNAL;
    }
}

redist_status redist_experts_backward(const redist_experts *op, const redist_experts_grads *grads, void *scratch, size_t scratch_bytes,
                                      void *cuda_stream)
{
    try {
        if (!op || !grads) return REDIST_EINVAL;
        const redist_experts &q = *op;
        const redist_experts_grads &g = *grads;
        TRY(check_experts_backward(q, g));
        const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
        const Extent dw = extent(g.dw, g.dw.data ? q.out_features : 0, q.in_features, 2, q.experts, g.dw_stride);
        const Extent dbias = extent(g.dbias, i64(q.experts) * q.out_features * 4);
        if (q.rows == 0) {
            const Extent outs[2] = {dw, dbias};
            TRY(apart(outs, 2, nullptr, 0));
            if (g.dw.data)
                for (i64 e = 0; e < q.experts; ++e)
                    TRY(cuda(cudaMemset2DAsync(static_cast<char *>(g.dw.data) + e * g.dw_stride * 2, size_t(lines_of(g.dw, q.out_features, q.in_features).ld) * 2, 0,
                                               size_t(q.in_features) * 2, size_t(q.out_features), stream)));
            return g.dbias ? cuda(cudaMemsetAsync(g.dbias, 0, size_t(q.experts) * size_t(q.out_features) * 4, stream)) : REDIST_OK;
        }
        const LaunchOptions o = options();
        Pieces p{uintptr_t(scratch)};
        const ExpertsBackward b(q, g, p);
        const Extent outs[4] = {extent(g.dx, g.dx.data ? q.rows : 0, q.in_features, 2), dw, dbias, extent(scratch, p.used)};
        const Extent ins[5] = {extent(g.dy, q.rows, q.out_features, 2), extent(q.pre, q.activation != REDIST_ACT_NONE ? q.rows : 0, q.out_features, 2),
                               extent(q.w, g.dx.data ? q.out_features : 0, q.in_features, 2, q.experts, q.w_stride),
                               extent(q.x, g.dw.data ? q.rows : 0, q.in_features, 2), extent(q.offsets, i64(q.experts + 1) * 4)};
        TRY(apart(outs, 4, ins, 5));
        TRY(check_scratch(scratch, scratch_bytes, p.used));
        const void *dz = b.fresh ? b.dz : g.dy.data;
        Grouped x = {};
        x.rows = q.rows;
        x.experts = q.experts;
        x.type = q.type;
        x.offsets = q.offsets;
        x.activation = ACT_NONE;
        Grouped w = x;
        x.m = q.in_features;
        x.k = q.out_features;
        x.a = b.w.operand(false);
        x.b = Operand{dz, b.ld_dz, 0, 0};
        x.out = g.dx.data;
        x.ld_out = row_stride(g.dx, q.rows, q.in_features);
        w.sums = 1;
        w.m = q.in_features;
        w.n = q.out_features;
        w.a = b.x.operand(false);
        w.b = Operand{dz, b.ld_dz, 0, 1};
        w.out = g.dw.data;
        w.ld_out = row_stride(g.dw, q.out_features, q.in_features);
        w.out_batch = g.dw_stride;

        Prepare before = {};
        before.type = q.type;
        if (b.fresh || g.dbias) {
            ExpertSlope &s = before.slope;
            s.rows = q.rows;
            s.cols = q.out_features;
            s.experts = q.experts;
            s.activation = q.activation;
            s.offsets = q.offsets;
            s.dy = g.dy.data;
            s.ld_dy = row_stride(g.dy, q.rows, q.out_features);
            if (q.activation != REDIST_ACT_NONE) {
                s.z = q.pre.data;
                s.ld_z = row_stride(q.pre, q.rows, q.out_features);
            }
            s.dst = b.dz;
            s.ld_dst = b.ld_dz;
            s.partials = b.partials;
        }
        before.lay[0] = b.w.lay(q.offsets, q.rows);
        before.lay[1] = b.x.lay(nullptr, 0);
        if (g.dw.data) before.sums = &w;
        before.maps = b.maps;
        TRY(cuda(launch_prepare(before, o, stream)));
        ExpertSums sums = {};
        sums.rows = q.rows;
        sums.cols = q.out_features;
        sums.per = slope_rows(q.rows, q.out_features);
        sums.experts = q.experts;
        sums.offsets = q.offsets;
        sums.partials = b.partials;
        sums.sums = g.dbias;
        if (g.dx.data) TRY(cuda(launch_grouped(x, nullptr, &sums, o, stream)));
        if (g.dw.data) TRY(cuda(launch_grouped(w, b.maps, &sums, o, stream)));
        if (sums.sums) TRY(cuda(launch_expert_sums(sums, o, stream)));
        return REDIST_OK;
    } catch (...) {
        return REDIST_EINTERNAL;
    }
}

size_t redist_clip_scratch_bytes(const redist_clip_op *op)
{
    try {
        if (!op || check_clip(*op) != REDIST_OK) return 0;
        const std::vector<ClipTensor> tensors = clip_tensors(*op);
        return size_t(round_up(clip_partials(tensors.data(), i64(tensors.size()), sm_count()) * 8, 256));
    } catch (...) {
        return 0;
    }
}

redist_status redist_clip(const redist_clip_op *op, void *scratch, size_t scratch_bytes, void *cuda_stream)
{
    try {
        if (!op) return REDIST_EINVAL;
        TRY(check_clip(*op));
        const int sms = sm_count();
        const std::vector<ClipTensor> tensors = clip_tensors(*op);
        const i64 need = clip_partials(tensors.data(), i64(tensors.size()), sms) * 8;
        TRY(check_scratch(scratch, scratch_bytes, need));
        TRY(check_clip_overlap(tensors, *op, scratch, need));
        return cuda(launch_clip(tensors.data(), i64(tensors.size()), op->max_norm, op->eps, op->norm, static_cast<double *>(scratch), sms, options(),
                                static_cast<cudaStream_t>(cuda_stream)));
    } catch (...) {
        return REDIST_EINTERNAL;
    }
}

}  // extern "C"
