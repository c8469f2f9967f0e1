// The C boundary of the operators: argument checks, scratch layout, and the launches each call is made of.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "checks.h"
#include "experts.h"
#include "plan.hpp"
#include "product.h"
#include "redist.h"
#include "rows.h"

using namespace redist;

namespace {

// ---- linear ----------------------------------------------------------------------------------------------

redist_status check_linear(const redist_linear &q)
{
    if (q.rows < 0 || q.in_features < 1 || q.out_features < 1) return REDIST_EINVAL;
    if (q.type != REDIST_BF16 && q.type != REDIST_F16) return REDIST_EINVAL;
    if (q.activation < REDIST_ACT_NONE || q.activation > REDIST_ACT_SILU || q.reserved != 0) return REDIST_EINVAL;
    if (q.rows > kMostSize || q.in_features > kMostSize || q.out_features > kMostSize) return REDIST_EUNSUPPORTED;
    return REDIST_OK;
}

redist_status check_forward(const redist_linear &q)
{
    TRY(check_linear(q));
    if (q.rows == 0) return REDIST_OK;
    TRY(check_in(q.x, q.rows, q.in_features, 2));
    TRY(check_in(q.w, q.out_features, q.in_features, 2));
    TRY(check_out(q.out, q.rows, q.out_features, 2));
    if (q.residual.data) TRY(check_out(q.residual, q.rows, q.out_features, 2));
    if (q.pre.data) TRY(check_out(q.pre, q.rows, q.out_features, 2));
    if (q.bias) {
        if (q.bias_type < REDIST_BF16 || q.bias_type > REDIST_F32) return REDIST_EINVAL;
        if (uintptr_t(q.bias) % uintptr_t(type_bytes(q.bias_type))) return REDIST_EALIGN;
    }
    return REDIST_OK;
}

redist_status check_backward(const redist_linear &q, const redist_linear_grads &g)
{
    TRY(check_linear(q));
    if (q.rows > 0) {
        TRY(check_out(g.dy, q.rows, q.out_features, 2));
        if (q.activation != REDIST_ACT_NONE) TRY(check_out(q.pre, q.rows, q.out_features, 2));
        if (g.dx.data) TRY(check_in(q.w, q.out_features, q.in_features, 2));
        if (g.dw.data) TRY(check_in(q.x, q.rows, q.in_features, 2));
        if (g.dx.data) TRY(check_out(g.dx, q.rows, q.in_features, 2));
    }
    if (g.dw.data) TRY(check_out(g.dw, q.out_features, q.in_features, 2));
    return uintptr_t(g.dbias) % 4 ? REDIST_EALIGN : REDIST_OK;
}

// Scratch of a product whose sum may be split.
void *parts_of(i64 m, i64 n, i64 k, const LaunchOptions &o, Pieces &pieces)
{
    Product p = {};
    p.m = m;
    p.n = n;
    p.k = k;
    p.batch = 1;
    p.kind = EPI_LINEAR;
    const i64 bytes = product_scratch_bytes(p, o);
    return bytes ? pieces.take(bytes) : nullptr;
}

// A forward call of a few rows reads its operands as they lie and needs no scratch.  Up to 16 rows that is the faster way
// at any size; from 17 on x's fragments take registers from the loads of w, and only a small w (whose call is over before
// the other kernel has set up its tensor memory) is read faster: 24 rows through 1024 -> 1024 4.3 us against 5.9, 4096 ->
// 130 4.2 against 8.2, but 4096 -> 4096 18 against 12, 16384 -> 1000 19 against 14 and 4096 -> 16384 41 against 27 (the same
// weight again and again, so that L2 has what fits).
bool few_rows(const redist_linear &q, const LaunchOptions &o)
{
    return !o.test_shape && q.rows <= kFewRows && (q.rows <= 16 || q.in_features * q.out_features <= (i64(1) << 22)) &&
           row_major(q.x, q.rows, q.in_features) && row_major(q.w, q.out_features, q.in_features);
}

// Everything another forward call takes from scratch.
struct Forward {
    Placed x, w;
    void *parts;
    Forward(const redist_linear &q, const LaunchOptions &o, Pieces &p)
        : x(q.x, q.rows, q.in_features, p), w(q.w, q.out_features, q.in_features, p), parts(parts_of(q.rows, q.out_features, q.in_features, o, p))
    {
    }
};

// What a backward call takes from scratch, in the order in which it is laid out.
struct Backward {
    bool fresh;             // dz is computed (or laid out) into scratch; else dy itself is the operand
    i64 ld_dz = 0;
    void *dz = nullptr;
    float *partials = nullptr;
    void *parts_dx = nullptr, *parts_dw = nullptr;
    Placed w, x;
    Backward(const redist_linear &q, const redist_linear_grads &g, const LaunchOptions &o, Pieces &p)
        : fresh((g.dx.data || g.dw.data) && (q.activation != REDIST_ACT_NONE || !operand_fits(g.dy.data, lines_of(g.dy, q.rows, q.out_features).ld, 0, 1))),
          w(g.dx.data ? q.w : redist_matrix{nullptr, 1, 1}, g.dx.data ? q.out_features : 0, g.dx.data ? q.in_features : 0, p),
          x(g.dw.data ? q.x : redist_matrix{nullptr, 1, 1}, g.dw.data ? q.rows : 0, g.dw.data ? q.in_features : 0, p)
    {
        ld_dz = fresh ? round_up(q.out_features, 64) : lines_of(g.dy, q.rows, q.out_features).ld;
        if (fresh) dz = p.take(q.rows * ld_dz * 2);
        if (g.dx.data) parts_dx = parts_of(q.rows, q.in_features, q.out_features, o, p);
        if (g.dw.data) parts_dw = parts_of(q.out_features, q.in_features, q.rows, o, p);
        if (g.dbias) partials = static_cast<float *>(p.take(i64(column_partial_bytes(q.rows, q.out_features))));
    }
};

Product product_of(i64 m, i64 n, i64 k, int type, const Operand &a, const Operand &b, const redist_matrix &out, i64 rows, i64 cols)
{
    Product p = {};
    p.m = m;
    p.n = n;
    p.k = k;
    p.batch = 1;
    p.type = type;
    p.kind = EPI_LINEAR;
    p.a = a;
    p.b = b;
    p.e.out = out.data;
    p.e.ld_out = lines_of(out, rows, cols).ld;
    p.e.out_type = type;
    return p;
}

// ---- layer norm --------------------------------------------------------------------------------------------

redist_status check_norm(const redist_layer_norm &q)
{
    if (q.rows < 0 || q.cols < 1 || !(q.eps >= 0.0f) || q.reserved != 0) return REDIST_EINVAL;
    if (q.type < REDIST_BF16 || q.type > REDIST_F32) return REDIST_EINVAL;
    if (q.rows > kMostSize || q.cols > kMostSize) return REDIST_EUNSUPPORTED;
    if (q.gamma || q.beta) {
        if (q.weight_type < REDIST_BF16 || q.weight_type > REDIST_F32) return REDIST_EINVAL;
        if ((uintptr_t(q.gamma) | uintptr_t(q.beta)) % uintptr_t(type_bytes(q.weight_type))) return REDIST_EALIGN;
    }
    if ((uintptr_t(q.mean) | uintptr_t(q.rstd)) % 4) return REDIST_EALIGN;
    if (q.rows > 0) {
        if (!q.x.data || !row_major(q.x, q.rows, q.cols)) return REDIST_EINVAL;
        if (uintptr_t(q.x.data) % uintptr_t(type_bytes(q.type))) return REDIST_EALIGN;
    }
    return REDIST_OK;
}

LayerNorm norm_of(const redist_layer_norm &q)
{
    LayerNorm l = {};
    l.rows = q.rows;
    l.cols = q.cols;
    l.type = q.type;
    l.weight_type = q.weight_type;
    l.eps = q.eps;
    l.x = q.x.data;
    l.ld_x = q.x.row_stride;
    l.gamma = q.gamma;
    l.beta = q.beta;
    l.mean = q.mean;
    l.rstd = q.rstd;
    if (q.rows == 1) l.ld_x = round_up(q.cols, 8);
    return l;
}

redist_status check_norm_grads(const redist_layer_norm &q, const redist_layer_norm_grads &g)
{
    TRY(check_norm(q));
    if (q.rows > 0) {
        if (!q.mean || !q.rstd) return REDIST_EINVAL;
        TRY(check_out(g.dy, q.rows, q.cols, type_bytes(q.type)));
        TRY(check_out(g.dx, q.rows, q.cols, type_bytes(q.type)));
    }
    return (uintptr_t(g.dgamma) | uintptr_t(g.dbeta)) % 4 ? REDIST_EALIGN : REDIST_OK;
}

int sm_count()
{
    int device = 0, sms = 0;
    return current_device(&device, &sms) == cudaSuccess ? sms : 148;
}

// ---- orthogonalisation ---------------------------------------------------------------------------------------

constexpr int kMostSteps = 64;

// The tensor cores cut every sum of 16 products more off to 24 bits, so A's sums of k squares come out small by up to k 2^-28:
// 8 x 2^19 results are 0.4 % off, 2^20 0.6 %, 2^22 2.3 %, 2^24 8 %.
constexpr i64 kMostLength = i64(1) << 22;

// The largest power of two that keeps a value of up to `most` at or below 2^14.
double room(double most) { return most > 0 ? std::ldexp(1.0, 14 - int(std::ceil(std::log2(most)))) : 1.0; }

// Powers of two by which a step's X, A and B are multiplied to use the range of f16: entries are bounded by the
// largest singular value, and that by the polynomial's largest value on the previous step's range (sampled; a margin
// of 1/512 a step is for what sampling and rounding miss -- more would let the range run away from itself where the
// polynomial grows quickly beyond it -- and f16 has a further factor of four above 2^14).
struct Steps {
    double x[kMostSteps + 1], a[kMostSteps], b[kMostSteps];
    bool ok;
    Steps(const float *abc, int steps)
    {
        double reach = 1 + 1.0 / 512;
        ok = true;
        x[0] = 0;                                   // found on the device, from the norm
        for (int s = 0; s < steps; ++s) {
            const double ca = abc[3 * s], cb = abc[3 * s + 1], cc = abc[3 * s + 2];
            double next = 0, most = 0;
            for (int i = 0; i <= 2048; ++i) {
                const double v = reach * i / 2048, l = v * v;
                const double f = std::fabs(v * (ca + cb * l + cc * l * l)), g = std::fabs(cb * l + cc * l * l);
                if (!(f <= 1e6) || !(g <= 1e12)) ok = false;
                next = std::max(next, f);
                most = std::max(most, g);
            }
            a[s] = room(reach * reach);
            b[s] = room(2 * most);                      // twice: B's mean is taken off its diagonal
            reach = std::max(next * (1 + 1.0 / 512), 1e-3);
            if (reach > 256) ok = false;
            if (!ok) return;
            x[s + 1] = room(reach);
        }
    }
};

struct Orthogonal {
    bool tall;
    i64 small, ld, plane, ld_gram, gram_plane;
    void *hi[2], *lo, *a, *b;
    float *scale;
    double *partials;
    Orthogonal(const redist_orthogonal &q, Pieces &p)
    {
        tall = q.rows > q.cols;
        small = std::min(q.rows, q.cols);
        ld = round_up(q.cols, 64);
        plane = q.rows * ld;
        ld_gram = round_up(small, 64);
        gram_plane = small * ld_gram;
        for (void *&h : hi) h = p.take(q.batch * plane * 2);
        lo = p.take(q.batch * plane * 2);
        a = p.take(q.batch * gram_plane * 2);
        b = p.take(q.batch * gram_plane * 2);
        scale = static_cast<float *>(p.take(q.batch * 4));
        partials = static_cast<double *>(p.take(q.batch * kNormParts * 8));
    }
};

redist_status check_orthogonal(const redist_orthogonal &q)
{
    if (q.batch < 1 || q.rows < 1 || q.cols < 1 || q.steps < 1 || q.steps > kMostSteps || q.reserved != 0) return REDIST_EINVAL;
    if (q.type < REDIST_BF16 || q.type > REDIST_F32 || !(q.eps >= 1e-30) || !std::isfinite(q.eps) || !std::isfinite(q.scale)) return REDIST_EINVAL;
    if (q.rows > kMostLength || q.cols > kMostLength || q.batch > 65535) return REDIST_EUNSUPPORTED;
    if (!q.coefficients || !q.x.data || !row_major(q.x, q.rows, q.cols)) return REDIST_EINVAL;
    TRY(check_out(q.out, q.rows, q.cols, 2));
    if (uintptr_t(q.x.data) % uintptr_t(type_bytes(q.type))) return REDIST_EALIGN;
    if (q.batch > 1) {
        if (q.x_batch_stride < 0) return REDIST_EINVAL;
        const i64 last = (q.rows - 1) * (q.rows > 1 ? q.out.row_stride : 0) + q.cols;
        if (q.out_batch_stride < last) return REDIST_EINVAL;
    }
    for (int i = 0; i < 3 * q.steps; ++i)
        if (!std::isfinite(q.coefficients[i])) return REDIST_EINVAL;
    return REDIST_OK;
}

}  // namespace

extern "C" {

size_t redist_linear_scratch_bytes(const redist_linear *op, const redist_linear_grads *grads)
{
    if (!op) return 0;
    Pieces p{0};
    const LaunchOptions o = options();
    if (!grads) {
        if (check_forward(*op) != REDIST_OK || op->rows == 0 || few_rows(*op, o)) return 0;
        Forward f(*op, o, p);
    } else {
        if (check_backward(*op, *grads) != REDIST_OK || op->rows == 0) return 0;
        Backward b(*op, *grads, o, p);
    }
    return size_t(p.used);
}

redist_status redist_linear_forward(const redist_linear *op, void *scratch, size_t scratch_bytes, void *cuda_stream)
{
    try {
        if (!op) return REDIST_EINVAL;
        const redist_linear &q = *op;
        TRY(check_forward(q));
        if (q.rows == 0) return REDIST_OK;
        const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
        const LaunchOptions o = options();
        const bool few = few_rows(q, o), in_place = q.residual.data == q.out.data &&
                                                 lines_of(q.residual, q.rows, q.out_features).ld == lines_of(q.out, q.rows, q.out_features).ld;
        Pieces p{uintptr_t(scratch)}, none{0};
        const Forward f(q, o, few ? none : p);
        const Extent outs[3] = {extent(q.out, q.rows, q.out_features, 2), extent(q.pre, q.pre.data ? q.rows : 0, q.out_features, 2), extent(scratch, p.used)};
        const Extent ins[4] = {extent(q.x, q.rows, q.in_features, 2), extent(q.w, q.out_features, q.in_features, 2),
                               extent(q.bias, q.out_features * type_bytes(q.bias_type)),
                               extent(q.residual, q.residual.data && !in_place ? q.rows : 0, q.out_features, 2)};
        TRY(apart(outs, 3, ins, 4));
        TRY(check_scratch(scratch, scratch_bytes, p.used));
        Product d = product_of(q.rows, q.out_features, q.in_features, q.type, f.x.operand(true), f.w.operand(true), q.out, q.rows, q.out_features);
        d.e.bias = q.bias;
        d.e.bias_type = q.bias_type;
        d.e.activation = q.activation;
        d.e.residual = q.residual.data;
        if (q.residual.data) d.e.ld_residual = lines_of(q.residual, q.rows, q.out_features).ld;
        d.e.pre = q.pre.data;
        if (q.pre.data) d.e.ld_pre = lines_of(q.pre, q.rows, q.out_features).ld;
        if (few) {
            d.a = Operand{f.x.from.data, f.x.from.ld, 0, 0};
            d.b = Operand{f.w.from.data, f.w.from.ld, 0, 0};
            return cuda(launch_few_rows(d, o, stream));
        }
        Lay list[2];
        int lays = 0;
        f.x.lay(q.type, list, lays);
        f.w.lay(q.type, list, lays);
        TRY(cuda(launch_lay(list, lays, o, stream)));
        return cuda(launch_product(d, f.parts, o, stream));
    } catch (...) {
        return REDIST_EINTERNAL;
    }
}

redist_status redist_linear_backward(const redist_linear *op, const redist_linear_grads *grads, void *scratch, size_t scratch_bytes,
                                     void *cuda_stream)
{
    try {
        if (!op || !grads) return REDIST_EINVAL;
        const redist_linear &q = *op;
        const redist_linear_grads &g = *grads;
        TRY(check_backward(q, g));
        const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
        if (q.rows == 0) {
            if (g.dw.data)
                TRY(cuda(cudaMemset2DAsync(g.dw.data, size_t(lines_of(g.dw, q.out_features, q.in_features).ld) * 2, 0, size_t(q.in_features) * 2,
                                           size_t(q.out_features), stream)));
            return g.dbias ? cuda(cudaMemsetAsync(g.dbias, 0, size_t(q.out_features) * 4, stream)) : REDIST_OK;
        }
        const LaunchOptions o = options();
        Pieces p{uintptr_t(scratch)};
        Backward b(q, g, o, p);
        const Extent outs[4] = {extent(g.dx, g.dx.data ? q.rows : 0, q.in_features, 2), extent(g.dw, g.dw.data ? q.out_features : 0, q.in_features, 2),
                                extent(g.dbias, q.out_features * 4), extent(scratch, p.used)};
        const Extent ins[4] = {extent(g.dy, q.rows, q.out_features, 2), extent(q.pre, q.activation != REDIST_ACT_NONE ? q.rows : 0, q.out_features, 2),
                               extent(q.w, g.dx.data ? q.out_features : 0, q.in_features, 2), extent(q.x, g.dw.data ? q.rows : 0, q.in_features, 2)};
        TRY(apart(outs, 4, ins, 4));
        TRY(check_scratch(scratch, scratch_bytes, p.used));
        const Lines dy = lines_of(g.dy, q.rows, q.out_features);
        Lay list[3];
        int lays = 0;
        if (b.fresh || g.dbias) {
            Lay l = {};
            l.rows = q.rows;
            l.cols = q.out_features;
            l.type = q.type;
            l.activation = q.activation;
            l.src = g.dy.data;
            l.ld_src = dy.ld;
            if (q.activation != REDIST_ACT_NONE) {
                l.z = q.pre.data;
                l.ld_z = lines_of(q.pre, q.rows, q.out_features).ld;
            }
            l.dst = b.dz;
            l.ld_dst = b.ld_dz;
            l.sums = g.dbias;
            l.partials = b.partials;
            list[lays++] = l;
        }
        if (g.dx.data) b.w.lay(q.type, list, lays);
        if (g.dw.data) b.x.lay(q.type, list, lays);
        TRY(cuda(launch_lay(list, lays, o, stream)));
        const void *dz = b.fresh ? b.dz : g.dy.data;
        if (g.dx.data) {
            TRY(cuda(launch_product(product_of(q.rows, q.in_features, q.out_features, q.type, Operand{dz, b.ld_dz, 0, 0}, b.w.operand(false), g.dx,
                                               q.rows, q.in_features), b.parts_dx, o, stream)));
        }
        if (g.dw.data) {
            TRY(cuda(launch_product(product_of(q.out_features, q.in_features, q.rows, q.type, Operand{dz, b.ld_dz, 0, 1}, b.x.operand(false), g.dw,
                                               q.out_features, q.in_features), b.parts_dw, o, stream)));
        }
        return REDIST_OK;
    } catch (...) {
        return REDIST_EINTERNAL;
    }
}

redist_status redist_layer_norm_forward(const redist_layer_norm *op, void *cuda_stream)
{
    try {
        if (!op) return REDIST_EINVAL;
        const redist_layer_norm &q = *op;
        TRY(check_norm(q));
        if (q.rows == 0) return REDIST_OK;
        const i64 e = type_bytes(q.type);
        TRY(check_out(q.y, q.rows, q.cols, e));
        const Extent outs[3] = {extent(q.y, q.rows, q.cols, e), extent(q.mean, q.rows * 4), extent(q.rstd, q.rows * 4)};
        const Extent ins[3] = {extent(q.x, q.rows, q.cols, e), extent(q.gamma, q.cols * type_bytes(q.weight_type)), extent(q.beta, q.cols * type_bytes(q.weight_type))};
        TRY(apart(outs, 3, ins, 3));
        LayerNorm l = norm_of(q);
        l.y = q.y.data;
        l.ld_y = q.rows == 1 ? round_up(q.cols, 8) : q.y.row_stride;
        return cuda(launch_layer_norm_forward(l, options(), static_cast<cudaStream_t>(cuda_stream)));
    } catch (...) {
        return REDIST_EINTERNAL;
    }
}

size_t redist_layer_norm_scratch_bytes(const redist_layer_norm *op, const redist_layer_norm_grads *grads)
{
    if (!op || !grads || check_norm_grads(*op, *grads) != REDIST_OK || op->rows == 0 || (!grads->dgamma && !grads->dbeta)) return 0;
    return layer_norm_backward_bytes(op->rows, op->cols, op->type, sm_count());
}

redist_status redist_layer_norm_backward(const redist_layer_norm *op, const redist_layer_norm_grads *grads, void *scratch, size_t scratch_bytes,
                                         void *cuda_stream)
{
    try {
        if (!op || !grads) return REDIST_EINVAL;
        const redist_layer_norm &q = *op;
        const redist_layer_norm_grads &g = *grads;
        TRY(check_norm_grads(q, g));
        const i64 e = type_bytes(q.type), need = i64(redist_layer_norm_scratch_bytes(op, grads));
        const Extent outs[4] = {extent(g.dx, q.rows, q.cols, e), extent(g.dgamma, q.cols * 4), extent(g.dbeta, q.cols * 4), extent(scratch, need)};
        const Extent ins[5] = {extent(q.x, q.rows, q.cols, e), extent(g.dy, q.rows, q.cols, e), extent(q.gamma, q.cols * type_bytes(q.weight_type)),
                               extent(q.mean, q.rows * 4), extent(q.rstd, q.rows * 4)};
        TRY(apart(outs, 4, ins, 5));
        TRY(check_scratch(scratch, scratch_bytes, need));
        LayerNorm l = norm_of(q);
        l.dy = g.dy.data;
        l.dx = g.dx.data;
        l.ld_dy = q.rows == 1 ? round_up(q.cols, 8) : g.dy.row_stride;
        l.ld_dx = q.rows == 1 ? round_up(q.cols, 8) : g.dx.row_stride;
        l.dgamma = g.dgamma;
        l.dbeta = g.dbeta;
        return cuda(launch_layer_norm_backward(l, scratch, options(), static_cast<cudaStream_t>(cuda_stream)));
    } catch (...) {
        return REDIST_EINTERNAL;
    }
}

size_t redist_orthogonalize_scratch_bytes(const redist_orthogonal *op)
{
    if (!op || check_orthogonal(*op) != REDIST_OK) return 0;
    Pieces p{0};
    Orthogonal w(*op, p);
    return size_t(p.used);
}

redist_status redist_orthogonalize(const redist_orthogonal *op, void *scratch, size_t scratch_bytes, void *cuda_stream)
{
    try {
        if (!op) return REDIST_EINVAL;
        const redist_orthogonal &q = *op;
        TRY(check_orthogonal(q));
        const Steps steps(q.coefficients, q.steps);
        if (!steps.ok) return REDIST_EINVAL;
        const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
        Pieces pieces{uintptr_t(scratch)};
        const Orthogonal w(q, pieces);
        const Extent outs[2] = {extent(q.out, q.rows, q.cols, 2, q.batch, q.out_batch_stride), extent(scratch, pieces.used)};
        const Extent ins[1] = {extent(q.x, q.rows, q.cols, type_bytes(q.type), q.batch, q.x_batch_stride)};
        TRY(apart(outs, 2, ins, 1));
        TRY(check_scratch(scratch, scratch_bytes, pieces.used));
        const LaunchOptions o = options();

        Scaled s = {};
        s.rows = q.rows;
        s.cols = q.cols;
        s.batch = int32_t(q.batch);
        s.type = q.type;
        s.x = q.x.data;
        s.ld_x = q.rows > 1 ? q.x.row_stride : q.cols;
        s.x_batch = q.batch > 1 ? q.x_batch_stride : 0;
        s.hi = w.hi[0];
        s.lo = q.type == REDIST_F32 ? w.lo : nullptr;      // a 16-bit input fits into f16 (but for what is below 2^-27 of the norm)
        s.ld = w.ld;
        s.plane = w.plane;
        s.scale = w.scale;
        s.partials = w.partials;
        s.eps = q.eps;
        TRY(cuda(launch_scaled(s, o, stream)));

        Product d = {};
        d.batch = int32_t(q.batch);
        d.type = T_F16;
        d.kind = EPI_SCALED;
        for (int k = 0; k < q.steps; ++k) {
            const float *abc = q.coefficients + 3 * k;
            const bool first = k == 0, last = k + 1 == q.steps, square = abc[2] != 0.0f;
            const double x = first ? 1.0 : 1.0 / steps.x[k];          // what undoes X's scale (the rest of it is on the device)
            const void *hi = w.hi[k & 1];
            // A = X X^T, or X^T X for a tall X
            Product g = d;
            g.m = g.n = w.small;
            g.k = std::max(q.rows, q.cols);
            g.symmetric = 1;
            g.a = g.b = Operand{hi, w.ld, w.plane, w.tall ? 1 : 0};
            g.e.out = w.a;
            g.e.ld_out = w.ld_gram;
            g.e.out_batch = w.gram_plane;
            g.e.out_type = T_F16;
            g.e.alpha = float(steps.a[k] * x * x);
            g.e.scale = first ? w.scale : nullptr;
            g.e.alpha_power = 2;
            TRY(cuda(launch_product(g, nullptr, o, stream)));
            // B = b A + c A A - z (A alone where c is zero: its factor goes into the update), and a + z for a below.  z = b t +
            // c t^2, with t the mean of (128 samples of) A's diagonal, is about the mean of B's, and the larger part of B
            // where A is near a multiple of one; what is left rounds to less.  But z X brings the rounding of X's strong
            // directions, which B alone would have kept out, into those that have yet to grow, and every later step
            // multiplies it by its a.  So only where the later steps grow by no more than 4 in all (the last two steps of the
            // Muon coefficients), and for t >= 1/4.  The error there, on Gaussian input, against none and against centring
            // wherever t >= 1/4: 128 x 128 2.0e-3 (2.4e-3, 1.9e-3), 32 x 64 2.6e-3 (3.0e-3, 2.1e-3); with half of the
            // directions strong over a noise of 1e-3, 128 x 256: 2.2e-3 (2.2e-3, 5.7e-3); 1.7e-3 of each is the output's rounding.
            double later = 1;
            for (int j = k + 1; j < q.steps; ++j) later *= std::max(1.0, std::fabs(double(q.coefficients[3 * j])));
            const bool centred = square && later <= 4;
            auto centre = [&](Epilogue &e) {
                const i64 samples = std::min<i64>(w.small, 128), apart = w.small / samples;
                e.diagonal = w.a;
                e.diagonal_step = apart * (w.ld_gram + 1);
                e.diagonal_batch = w.gram_plane;
                e.diagonal_n = int32_t(samples);
                e.mean_scale = float(1.0 / (steps.a[k] * double(samples)));
                e.center_1 = abc[1];
                e.center_2 = abc[2];
            };
            double factor = double(abc[1]) / steps.a[k];
            const void *poly = w.a;
            if (square) {
                g.k = w.small;
                g.a = g.b = Operand{w.a, w.ld_gram, w.gram_plane, 0};
                g.e.out = w.b;
                g.e.alpha = float(double(abc[2]) * steps.b[k] / (steps.a[k] * steps.a[k]));
                g.e.beta = float(double(abc[1]) * steps.b[k] / steps.a[k]);
                g.e.hi = w.a;
                g.e.ld_add = w.ld_gram;
                g.e.add_batch = w.gram_plane;
                g.e.scale = nullptr;
                if (centred) {
                    centre(g.e);
                    g.e.on_diagonal = float(steps.b[k]);
                }
                TRY(cuda(launch_product(g, nullptr, o, stream)));
                factor = 1.0 / steps.b[k];
                poly = w.b;
            }
            // X <- a X + B X, or a X + X B for a tall X
            const double to = last ? double(q.scale) : steps.x[k + 1];
            Product u = d;
            const Operand px{hi, w.ld, w.plane, w.tall ? 0 : 1}, pb{poly, w.ld_gram, w.gram_plane, 0};
            u.m = q.rows;
            u.n = q.cols;
            u.k = w.small;
            u.a = w.tall ? px : pb;
            u.b = w.tall ? pb : px;
            u.e.out = last ? q.out.data : w.hi[(k + 1) & 1];
            u.e.ld_out = last ? (q.rows > 1 ? q.out.row_stride : round_up(q.cols, 8)) : w.ld;
            u.e.out_batch = last ? (q.batch > 1 ? q.out_batch_stride : 0) : w.plane;
            u.e.out_type = last ? T_BF16 : T_F16;
            u.e.out_lo = last ? nullptr : w.lo;
            u.e.hi = hi;
            u.e.lo = first && q.type != REDIST_F32 ? nullptr : w.lo;
            u.e.ld_add = w.ld;
            u.e.add_batch = w.plane;
            u.e.alpha = float(to * factor * x);
            u.e.beta = float(double(abc[0]) * to * x);
            u.e.scale = first ? w.scale : nullptr;
            u.e.alpha_power = u.e.beta_power = 1;
            if (centred) {
                centre(u.e);
                u.e.to_beta = float(to * x);
            }
            TRY(cuda(launch_product(u, nullptr, o, stream)));
        }
        return REDIST_OK;
    } catch (...) {
        return REDIST_EINTERNAL;
    }
}

int64_t redist_product_timeouts(void)
{
    unsigned int n = 0, grouped = 0;
    return cuda(read_product_timeouts(&n)) == REDIST_OK && cuda(read_grouped_timeouts(&grouped)) == REDIST_OK ? int64_t(n) + grouped : -1;
}

}  // extern "C"
