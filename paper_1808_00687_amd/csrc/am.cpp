// Entry points of the acoustic-model operators: the argument checks (before
// any device call), then one launcher each.
#include <cmath>
#include <cstddef>
#include <cstdint>
#include <exception>
#include <vector>

#include "am.h"
#include "am_places.h"
#include "internal.h"

using namespace wfd;

namespace {

// A call's checks: the first one that fails sets the message.
struct Checks {
    const char *who;
    bool ok = true;

    bool fail(const char *what)
    {
        if (ok) set_error("%s: %s", who, what);
        return ok = false;
    }
    bool need(bool good, const char *what) { return good || fail(what); }

    // m is a matrix of rows x cols of one of the types in the bit mask
    bool matrix(const wfst_matrix &m, const char *name, int64_t rows, int64_t cols, uint32_t types)
    {
        if (!ok) return false;
        const char *bad = nullptr;
        if (m.type < 0 || m.type > 3 || !((types >> m.type) & 1)) bad = "has a type that is not taken here";
        else if (m.rows != rows || m.cols != cols) bad = "has another shape than the other operands ask for";
        else if (m.row_stride < m.cols) bad = "has a row stride below its columns";
        else if (rows > 0 && m.row_stride > (int64_t{1} << 56) / rows) bad = "is larger than an address space";
        else if (!m.data && rows > 0) bad = "is NULL";
        else if (reinterpret_cast<uintptr_t>(m.data) % am_type_bytes(m.type)) bad = "is not aligned to its type";
        if (!bad) return true;
        set_error("%s: %s %s", who, name, bad);
        return ok = false;
    }
    bool dims(int64_t rows, int64_t cols)
    {
        return need(rows >= 0 && rows <= INT32_MAX && cols >= 1 && cols <= INT32_MAX,
                    "rows must be in [0, 2^31) and columns in [1, 2^31)");
    }
    // of a product: rows and columns of tiles past the end, and the tiles' number, stay in 31 bits
    bool product_dims(int64_t rows, int64_t cols)
    {
        constexpr int64_t kMost = int64_t{1} << 30, kValues = int64_t{1} << 40;
        return dims(rows, cols) && need(rows <= kMost && cols <= kMost, "rows and columns of a product must be at most 2^30") &&
               need(rows * cols <= kValues, "a matrix of a product must have at most 2^40 elements");
    }
    bool vector(const void *p, const char *name, bool wanted)
    {
        if (!ok) return false;
        if ((wanted && !p) || reinterpret_cast<uintptr_t>(p) % 4) {
            set_error("%s: %s is %s", who, name, p ? "not aligned" : "NULL");
            return ok = false;
        }
        return true;
    }
    bool apart(Range a, Range b, const char *what)
    {
        return disjoint(a, b) || fail(what);
    }
};

Range range_of(const wfst_matrix &m)
{
    if (!m.data || m.rows < 1) return {0, 0};
    const uintptr_t p = reinterpret_cast<uintptr_t>(m.data), size = static_cast<uintptr_t>(am_type_bytes(m.type));
    const uintptr_t stride = static_cast<uintptr_t>(m.row_stride) * size, width = static_cast<uintptr_t>(m.cols) * size;
    return {p, p + static_cast<uintptr_t>(m.rows - 1) * stride + width, m.rows > 1 ? stride : 0, width};
}

Range range_of(const void *p, int64_t bytes)
{
    const uintptr_t b = reinterpret_cast<uintptr_t>(p);
    return p && bytes > 0 ? Range{b, b + static_cast<uintptr_t>(bytes)} : Range{0, 0};
}

// the same matrix in place: every element at the same address
bool same_place(const wfst_matrix &a, const wfst_matrix &b)
{
    return a.data == b.data && a.type == b.type && (a.row_stride == b.row_stride || a.rows <= 1);
}

bool apart_or_same(Checks &c, const wfst_matrix &out, const wfst_matrix &in, const char *what)
{
    return same_place(out, in) || c.apart(range_of(out), range_of(in), what);
}

constexpr uint32_t kFloats = 1u << WFST_F32 | 1u << WFST_F16 | 1u << WFST_BF16;
constexpr uint32_t kHalves = 1u << WFST_F16 | 1u << WFST_BF16;
constexpr const char *kOverlap = "an output overlaps an input or another output";

int launched(hipError_t e, const char *who)
{
    if (e == hipSuccess) return WFST_OK;
    set_error("%s: %s", who, hipGetErrorString(e));
    return e == hipErrorOutOfMemory ? WFST_ENOMEM : WFST_EDEVICE;
}

hipStream_t stream_of(void *s) { return static_cast<hipStream_t>(s); }

bool good_activation(int32_t a) { return a >= WFST_ACT_NONE && a <= WFST_ACT_GELU; }

bool check(Checks &c, const wfst_am_linear_args &a)
{
    const int64_t M = a.x.rows, K = a.x.cols, N = a.w.rows;
    const bool f8 = a.x.type == WFST_F8E4M3;
    if (!c.product_dims(M, K) || !c.product_dims(M, N) || !c.product_dims(N, K)) return false;
    if (!c.need(good_activation(a.activation), "unknown activation")) return false;
    if (!c.matrix(a.x, "x", M, K, kHalves | 1u << WFST_F8E4M3)) return false;
    if (!c.matrix(a.w, "w", N, K, 1u << a.x.type)) return false;
    if (!c.matrix(a.y, "y", M, N, kFloats)) return false;
    if (a.residual.data && !c.matrix(a.residual, "residual", M, N, 1u << a.y.type)) return false;
    if (a.pre.data && !c.matrix(a.pre, "pre", M, N, 1u << a.y.type)) return false;
    if (!c.need(f8 || (!a.x_scale && !a.w_scale), "scales are for 8-bit operands")) return false;
    if (!c.vector(a.x_scale, "x_scale", f8 && M > 0) || !c.vector(a.w_scale, "w_scale", f8)) return false;
    if (!c.vector(a.bias, "bias", false)) return false;
    const Range in[] = {range_of(a.x), range_of(a.w), range_of(a.x_scale, 4 * M), range_of(a.w_scale, 4 * N),
                        range_of(a.bias, 4 * N)};
    const Range y = range_of(a.y), pre = range_of(a.pre);
    for (const Range &r : in)
        if (!c.apart(y, r, kOverlap) || !c.apart(pre, r, kOverlap)) return false;
    return c.apart(y, pre, kOverlap) && c.apart(pre, range_of(a.residual), kOverlap) &&
           (!a.residual.data || apart_or_same(c, a.y, a.residual, kOverlap));
}

// everything but the pointers: what the workspace depends on
bool check_sizes(Checks &c, const wfst_am_linear_backward_args &a)
{
    const int64_t M = a.dy.rows, N = a.dy.cols;
    if (!c.product_dims(M, N) || !c.need(good_activation(a.activation), "unknown activation")) return false;
    if (!c.need(a.round_dz == 0 || a.round_dz == 1, "round_dz must be 0 or 1")) return false;
    if (!c.need(a.dy.type == WFST_F16 || a.dy.type == WFST_BF16, "dy has a type that is not taken here")) return false;
    if (a.dx.data && !c.product_dims(M, a.dx.cols)) return false;
    return !a.dw.data || c.product_dims(N, a.dw.cols);
}

bool check(Checks &c, const wfst_am_linear_backward_args &a)
{
    if (!check_sizes(c, a)) return false;
    const int64_t M = a.dy.rows, N = a.dy.cols;
    const uint32_t type = 1u << a.dy.type;
    const bool act = a.activation != WFST_ACT_NONE;
    if (!c.matrix(a.dy, "dy", M, N, type)) return false;
    if (act && !c.matrix(a.pre, "pre", M, N, type)) return false;
    if (a.dx.data && (!c.matrix(a.dx, "dx", M, a.dx.cols, kFloats) || !c.matrix(a.w, "w", N, a.dx.cols, type)))
        return false;
    if (a.dw.data && (!c.matrix(a.dw, "dw", N, a.dw.cols, kFloats) || !c.matrix(a.x, "x", M, a.dw.cols, type)))
        return false;
    if (!c.vector(a.dbias, "dbias", false)) return false;
    const int64_t need = am_linear_backward_bytes(a);
    if (!c.need(need == 0 || (a.workspace && a.workspace_bytes >= need), "the workspace is too small")) return false;
    if (!c.need(reinterpret_cast<uintptr_t>(a.workspace) % 256 == 0, "the workspace is not aligned")) return false;
    const Range none{0, 0};
    const Range in[] = {range_of(a.dy), act ? range_of(a.pre) : none, a.dw.data ? range_of(a.x) : none,
                        a.dx.data ? range_of(a.w) : none};
    const Range out[] = {range_of(a.dx), range_of(a.dw), range_of(a.dbias, 4 * N), range_of(a.workspace, need)};
    for (int i = 0; i < 4; i++) {
        for (const Range &r : in)
            if (!c.apart(out[i], r, kOverlap)) return false;
        for (int j = 0; j < i; j++)
            if (!c.apart(out[i], out[j], kOverlap)) return false;
    }
    return true;
}

bool check(Checks &c, const wfst_am_gated_args &a)
{
    const int64_t M = a.x.rows, K = a.x.cols, N = a.y.cols;
    const bool f8 = a.x.type == WFST_F8E4M3;
    if (!c.need(N >= 1 && N <= INT32_MAX, "y must have 1 to 2^31 - 1 columns")) return false;
    if (!c.product_dims(M, K) || !c.product_dims(M, 2 * N) || !c.product_dims(2 * N, K)) return false;
    if (!c.need(good_activation(a.activation), "unknown activation")) return false;
    if (!c.matrix(a.x, "x", M, K, kHalves | 1u << WFST_F8E4M3)) return false;
    if (!c.matrix(a.w, "w", 2 * N, K, 1u << a.x.type)) return false;
    if (!c.matrix(a.y, "y", M, N, kFloats)) return false;
    if (a.pre.data && !c.matrix(a.pre, "pre", M, 2 * N, 1u << a.y.type)) return false;
    if (!c.need(f8 || (!a.x_scale && !a.w_scale), "scales are for 8-bit operands")) return false;
    if (!c.vector(a.x_scale, "x_scale", f8 && M > 0) || !c.vector(a.w_scale, "w_scale", f8)) return false;
    if (!c.vector(a.bias, "bias", false)) return false;
    const Range in[] = {range_of(a.x), range_of(a.w), range_of(a.x_scale, 4 * M), range_of(a.w_scale, 8 * N),
                        range_of(a.bias, 8 * N)};
    const Range y = range_of(a.y), pre = range_of(a.pre);
    for (const Range &r : in)
        if (!c.apart(y, r, kOverlap) || !c.apart(pre, r, kOverlap)) return false;
    return c.apart(y, pre, kOverlap);
}

// everything but the pointers: what the workspace depends on
bool check_sizes(Checks &c, const wfst_am_gated_backward_args &a)
{
    const int64_t M = a.dy.rows, N = a.dy.cols;
    if (!c.need(N >= 1 && N <= INT32_MAX, "dy must have 1 to 2^31 - 1 columns") || !c.product_dims(M, 2 * N)) return false;
    if (!c.need(good_activation(a.activation), "unknown activation")) return false;
    if (!c.need(a.round_dz == 0 || a.round_dz == 1, "round_dz must be 0 or 1")) return false;
    if (!c.need(a.dy.type == WFST_F16 || a.dy.type == WFST_BF16, "dy has a type that is not taken here")) return false;
    if (a.dx.data && (!c.product_dims(M, a.dx.cols) || !c.product_dims(2 * N, a.dx.cols))) return false;
    return !a.dw.data || (c.product_dims(2 * N, a.dw.cols) && c.product_dims(M, a.dw.cols));
}

bool check(Checks &c, const wfst_am_gated_backward_args &a)
{
    if (!check_sizes(c, a)) return false;
    const int64_t M = a.dy.rows, N = a.dy.cols;
    const uint32_t type = 1u << a.dy.type;
    if (!c.matrix(a.dy, "dy", M, N, type) || !c.matrix(a.pre, "pre", M, 2 * N, type)) return false;
    if (a.dx.data && (!c.matrix(a.dx, "dx", M, a.dx.cols, kFloats) || !c.matrix(a.w, "w", 2 * N, a.dx.cols, type)))
        return false;
    if (a.dw.data && (!c.matrix(a.dw, "dw", 2 * N, a.dw.cols, kFloats) || !c.matrix(a.x, "x", M, a.dw.cols, type)))
        return false;
    if (!c.vector(a.dbias, "dbias", false)) return false;
    const int64_t need = am_gated_backward_bytes(a);
    if (!c.need(need == 0 || (a.workspace && a.workspace_bytes >= need), "the workspace is too small")) return false;
    if (!c.need(reinterpret_cast<uintptr_t>(a.workspace) % 256 == 0, "the workspace is not aligned")) return false;
    const Range none{0, 0};
    const Range in[] = {range_of(a.dy), range_of(a.pre), a.dw.data ? range_of(a.x) : none, a.dx.data ? range_of(a.w) : none};
    const Range out[] = {range_of(a.dx), range_of(a.dw), range_of(a.dbias, 8 * N), range_of(a.workspace, need)};
    for (int i = 0; i < 4; i++) {
        for (const Range &r : in)
            if (!c.apart(out[i], r, kOverlap)) return false;
        for (int j = 0; j < i; j++)
            if (!c.apart(out[i], out[j], kOverlap)) return false;
    }
    return true;
}

bool good_eps(float eps) { return std::isfinite(eps) && eps > 0.0f; }

bool check(Checks &c, const wfst_am_norm_args &a)
{
    const int64_t M = a.x.rows, D = a.x.cols;
    const bool f8 = a.y.type == WFST_F8E4M3;
    if (!c.dims(M, D) || !c.need(good_eps(a.eps), "eps must be positive and finite")) return false;
    if (!c.matrix(a.x, "x", M, D, kFloats)) return false;
    if (a.residual.data && !c.matrix(a.residual, "residual", M, D, 1u << a.x.type)) return false;
    if (a.sum.data && !c.matrix(a.sum, "sum", M, D, 1u << a.x.type)) return false;
    if (!c.matrix(a.y, "y", M, D, kFloats | 1u << WFST_F8E4M3)) return false;
    if (!c.need(f8 || !a.y_scale, "y_scale is for an 8-bit y")) return false;
    if (!c.vector(a.y_scale, "y_scale", f8 && M > 0) || !c.vector(a.gain, "gain", false)) return false;
    const Range y = range_of(a.y), sum = range_of(a.sum), scale = range_of(a.y_scale, 4 * M);
    const Range in[] = {range_of(a.x), range_of(a.residual), range_of(a.gain, 4 * D)};
    for (const Range &r : in)
        if (!c.apart(y, r, kOverlap) || !c.apart(scale, r, kOverlap)) return false;
    if (!c.apart(y, sum, kOverlap) || !c.apart(y, scale, kOverlap) || !c.apart(sum, scale, kOverlap) ||
        !c.apart(sum, in[2], kOverlap))
        return false;
    return !a.sum.data || (apart_or_same(c, a.sum, a.x, kOverlap) &&
                           (!a.residual.data || apart_or_same(c, a.sum, a.residual, kOverlap)));
}

bool check_sizes(Checks &c, const wfst_am_norm_backward_args &a) { return c.dims(a.s.rows, a.s.cols); }

bool check(Checks &c, const wfst_am_norm_backward_args &a)
{
    const int64_t M = a.s.rows, D = a.s.cols;
    if (!check_sizes(c, a) || !c.need(good_eps(a.eps), "eps must be positive and finite")) return false;
    if (!c.matrix(a.s, "s", M, D, kFloats) || !c.matrix(a.dy, "dy", M, D, 1u << a.s.type)) return false;
    if (a.dsum.data && !c.matrix(a.dsum, "dsum", M, D, 1u << a.s.type)) return false;
    if (a.dx.data && !c.matrix(a.dx, "dx", M, D, 1u << a.s.type)) return false;
    if (!c.vector(a.gain, "gain", false) || !c.vector(a.dgain, "dgain", false)) return false;
    const int64_t need = am_norm_backward_bytes(a);
    if (!c.need(need == 0 || (a.workspace && a.workspace_bytes >= need), "the workspace is too small")) return false;
    if (!c.need(reinterpret_cast<uintptr_t>(a.workspace) % 256 == 0, "the workspace is not aligned")) return false;
    const Range in[] = {range_of(a.gain, 4 * D), range_of(a.s), range_of(a.dy), range_of(a.dsum)};
    const Range out[] = {range_of(a.dx), range_of(a.dgain, 4 * D), range_of(a.workspace, need)};
    for (int i = 0; i < 3; i++) {
        for (int j = 0; j < (i ? 4 : 2); j++)
            if (!c.apart(out[i], in[j], kOverlap)) return false;
        for (int j = 0; j < i; j++)
            if (!c.apart(out[i], out[j], kOverlap)) return false;
    }
    return !a.dx.data || (apart_or_same(c, a.dx, a.dy, kOverlap) &&
                          (!a.dsum.data || apart_or_same(c, a.dx, a.dsum, kOverlap)));
}

bool check(Checks &c, const wfst_am_layer_norm_args &a)
{
    const int64_t M = a.x.rows, D = a.x.cols;
    const bool f8 = a.y.type == WFST_F8E4M3;
    if (!c.dims(M, D) || !c.need(good_eps(a.eps), "eps must be positive and finite")) return false;
    if (!c.matrix(a.x, "x", M, D, kFloats)) return false;
    if (a.residual.data && !c.matrix(a.residual, "residual", M, D, 1u << a.x.type)) return false;
    if (a.sum.data && !c.matrix(a.sum, "sum", M, D, 1u << a.x.type)) return false;
    if (!c.matrix(a.y, "y", M, D, kFloats | 1u << WFST_F8E4M3)) return false;
    if (!c.need(f8 || !a.y_scale, "y_scale is for an 8-bit y")) return false;
    if (!c.vector(a.y_scale, "y_scale", f8 && M > 0) || !c.vector(a.gain, "gain", false) || !c.vector(a.bias, "bias", false))
        return false;
    const Range y = range_of(a.y), sum = range_of(a.sum), scale = range_of(a.y_scale, 4 * M);
    const Range in[] = {range_of(a.x), range_of(a.residual), range_of(a.gain, 4 * D), range_of(a.bias, 4 * D)};
    for (const Range &r : in)
        if (!c.apart(y, r, kOverlap) || !c.apart(scale, r, kOverlap)) return false;
    if (!c.apart(y, sum, kOverlap) || !c.apart(y, scale, kOverlap) || !c.apart(sum, scale, kOverlap) ||
        !c.apart(sum, in[2], kOverlap) || !c.apart(sum, in[3], kOverlap))
        return false;
    return !a.sum.data || (apart_or_same(c, a.sum, a.x, kOverlap) &&
                           (!a.residual.data || apart_or_same(c, a.sum, a.residual, kOverlap)));
}

bool check_sizes(Checks &c, const wfst_am_layer_norm_backward_args &a) { return c.dims(a.s.rows, a.s.cols); }

bool check(Checks &c, const wfst_am_layer_norm_backward_args &a)
{
    const int64_t M = a.s.rows, D = a.s.cols;
    if (!check_sizes(c, a) || !c.need(good_eps(a.eps), "eps must be positive and finite")) return false;
    if (!c.matrix(a.s, "s", M, D, kFloats) || !c.matrix(a.dy, "dy", M, D, 1u << a.s.type)) return false;
    if (a.dsum.data && !c.matrix(a.dsum, "dsum", M, D, 1u << a.s.type)) return false;
    if (a.dx.data && !c.matrix(a.dx, "dx", M, D, 1u << a.s.type)) return false;
    if (!c.vector(a.gain, "gain", false) || !c.vector(a.dgain, "dgain", false) || !c.vector(a.dbias, "dbias", false)) return false;
    const int64_t need = am_layer_norm_backward_bytes(a);
    if (!c.need(need == 0 || (a.workspace && a.workspace_bytes >= need), "the workspace is too small")) return false;
    if (!c.need(reinterpret_cast<uintptr_t>(a.workspace) % 256 == 0, "the workspace is not aligned")) return false;
    const Range in[] = {range_of(a.gain, 4 * D), range_of(a.s), range_of(a.dy), range_of(a.dsum)};
    const Range out[] = {range_of(a.dx), range_of(a.dgain, 4 * D), range_of(a.dbias, 4 * D), range_of(a.workspace, need)};
    for (int i = 0; i < 4; i++) {
        for (int j = 0; j < (i ? 4 : 2); j++)
            if (!c.apart(out[i], in[j], kOverlap)) return false;
        for (int j = 0; j < i; j++)
            if (!c.apart(out[i], out[j], kOverlap)) return false;
    }
    return !a.dx.data || (apart_or_same(c, a.dx, a.dy, kOverlap) &&
                          (!a.dsum.data || apart_or_same(c, a.dx, a.dsum, kOverlap)));
}

bool check(Checks &c, const wfst_am_distill_args &a, bool backward)
{
    const int64_t M = a.logits.rows, L = a.logits.cols, k = a.top_logit.cols;
    if (!c.dims(M, L)) return false;
    // (the reciprocal of a subnormal one is no float32)
    if (!c.need(std::isnormal(a.temperature) && a.temperature > 0.0f, "temperature must be positive, finite and normal")) return false;
    if (!c.need(k >= 1 && k <= WFST_AM_MAX_TOP, "the teacher's entries must be 1 to 256 a row")) return false;
    if (!c.matrix(a.logits, "logits", M, L, kFloats) || !c.matrix(a.top_logit, "top_logit", M, k, kFloats)) return false;
    if ((backward || a.dlogits.data) && !c.matrix(a.dlogits, "dlogits", M, L, 1u << a.logits.type)) return false;
    if (!c.vector(a.top_index, "top_index", M > 0) || !c.vector(a.weight, "weight", false)) return false;
    if (!c.vector(a.loss, "loss", false) || !c.vector(a.lse, "lse", backward && M > 0)) return false;
    const Range d = range_of(a.dlogits), lse = range_of(a.lse, 4 * M);
    const Range loss = backward ? Range{0, 0} : range_of(a.loss, 4 * M);
    const Range in[] = {range_of(a.top_logit), range_of(a.top_index, 4 * M * k), range_of(a.weight, 4 * M)};
    for (const Range &r : in)
        if (!c.apart(d, r, kOverlap) || !c.apart(loss, r, kOverlap) || (!backward && !c.apart(lse, r, kOverlap)))
            return false;
    const Range x = range_of(a.logits);
    if (!c.apart(d, loss, kOverlap) || !c.apart(d, lse, kOverlap) || !c.apart(loss, lse, kOverlap) ||
        !c.apart(loss, x, kOverlap) || (!backward && !c.apart(lse, x, kOverlap)))
        return false;
    return !a.dlogits.data || apart_or_same(c, a.dlogits, a.logits, kOverlap);
}

bool check_sizes(Checks &c, const wfst_am_clip_args &a)
{
    return c.need(a.count >= 0 && a.count <= WFST_AM_MAX_TENSORS, "the tensors must be 0 to 65536");
}

// Outputs lie apart from one another and from all other grads.
bool check_places(Checks &c, const wfst_am_clip_args &a, Range norm, Range workspace)
{
    std::vector<Span> spans;
    spans.reserve(static_cast<size_t>(a.count) * 2 + 2);
    for (int64_t i = 0; i < a.count; i++) {
        spans.push_back({range_of(a.outs ? a.outs[i] : a.grads[i]), true});
        if (a.outs && !same_place(a.outs[i], a.grads[i])) spans.push_back({range_of(a.grads[i]), false});
    }
    spans.push_back({norm, true});
    spans.push_back({workspace, true});
    return c.need(spans_apart(spans), kOverlap);
}

bool check(Checks &c, const wfst_am_clip_args &a)
{
    if (!check_sizes(c, a)) return false;
    if (!c.need(a.max_norm > 0.0, "max_norm must be positive")) return false;
    if (!c.need(a.grads || a.count == 0, "grads is NULL") || !c.vector(a.norm, "norm", true)) return false;
    for (int64_t i = 0; i < a.count; i++) {
        const wfst_matrix &g = a.grads[i];
        if (!c.dims(g.rows, g.cols) || !c.matrix(g, "a grad", g.rows, g.cols, kFloats)) return false;
        if (a.outs && !c.matrix(a.outs[i], "an output", g.rows, g.cols, 1u << g.type)) return false;
    }
    const int64_t need = am_clip_bytes(a);
    if (!c.need(a.workspace && a.workspace_bytes >= need, "the workspace is too small")) return false;
    if (!c.need(reinterpret_cast<uintptr_t>(a.workspace) % 256 == 0, "the workspace is not aligned")) return false;
    return check_places(c, a, range_of(a.norm, 4), range_of(a.workspace, need));
}

bool check(Checks &c, const wfst_am_loglikes_args &a)
{
    const int64_t M = a.logits.rows, L = a.logits.cols;
    if (!c.dims(M, L)) return false;
    if (!c.need(std::isfinite(a.scale) && a.scale > 0.0f, "scale must be positive and finite")) return false;
    if (!c.matrix(a.logits, "logits", M, L, kFloats) || !c.matrix(a.ll, "ll", M, L, 1u << WFST_F32)) return false;
    return c.vector(a.log_prior, "log_prior", false) && c.apart(range_of(a.ll), range_of(a.logits), kOverlap) &&
           c.apart(range_of(a.ll), range_of(a.log_prior, 4 * L), kOverlap);
}

int no_args(const char *who)
{
    set_error("%s: NULL argument", who);
    return WFST_EINVAL;
}

}  // namespace

extern "C" int wfst_am_linear(const wfst_am_linear_args *args, void *hip_stream)
{
    clear_error();
    if (!args) return no_args("wfst_am_linear");
    Checks c{"wfst_am_linear"};
    if (!check(c, *args)) return WFST_EINVAL;
    return args->x.rows ? launched(am_launch_linear(*args, stream_of(hip_stream)), c.who) : WFST_OK;
}

extern "C" int wfst_am_linear_backward_workspace(const wfst_am_linear_backward_args *args, int64_t *bytes)
{
    clear_error();
    if (!args || !bytes) return no_args("wfst_am_linear_backward_workspace");
    Checks c{"wfst_am_linear_backward_workspace"};
    if (!check_sizes(c, *args)) return WFST_EINVAL;
    *bytes = am_linear_backward_bytes(*args);
    return WFST_OK;
}

extern "C" int wfst_am_linear_backward(const wfst_am_linear_backward_args *args, void *hip_stream)
{
    clear_error();
    if (!args) return no_args("wfst_am_linear_backward");
    Checks c{"wfst_am_linear_backward"};
    if (!check(c, *args)) return WFST_EINVAL;
    return launched(am_launch_linear_backward(*args, stream_of(hip_stream)), c.who);
}

extern "C" int wfst_am_gated(const wfst_am_gated_args *args, void *hip_stream)
{
    clear_error();
    if (!args) return no_args("wfst_am_gated");
    Checks c{"wfst_am_gated"};
    if (!check(c, *args)) return WFST_EINVAL;
    return args->x.rows ? launched(am_launch_gated(*args, stream_of(hip_stream)), c.who) : WFST_OK;
}

extern "C" int wfst_am_gated_backward_workspace(const wfst_am_gated_backward_args *args, int64_t *bytes)
{
    clear_error();
    if (!args || !bytes) return no_args("wfst_am_gated_backward_workspace");
    Checks c{"wfst_am_gated_backward_workspace"};
    if (!check_sizes(c, *args)) return WFST_EINVAL;
    *bytes = am_gated_backward_bytes(*args);
    return WFST_OK;
}

extern "C" int wfst_am_gated_backward(const wfst_am_gated_backward_args *args, void *hip_stream)
{
    clear_error();
    if (!args) return no_args("wfst_am_gated_backward");
    Checks c{"wfst_am_gated_backward"};
    if (!check(c, *args)) return WFST_EINVAL;
    return launched(am_launch_gated_backward(*args, stream_of(hip_stream)), c.who);
}

extern "C" int wfst_am_norm(const wfst_am_norm_args *args, void *hip_stream)
{
    clear_error();
    if (!args) return no_args("wfst_am_norm");
    Checks c{"wfst_am_norm"};
    if (!check(c, *args)) return WFST_EINVAL;
    return args->x.rows ? launched(am_launch_norm(*args, stream_of(hip_stream)), c.who) : WFST_OK;
}

extern "C" int wfst_am_norm_backward_workspace(const wfst_am_norm_backward_args *args, int64_t *bytes)
{
    clear_error();
    if (!args || !bytes) return no_args("wfst_am_norm_backward_workspace");
    Checks c{"wfst_am_norm_backward_workspace"};
    if (!check_sizes(c, *args)) return WFST_EINVAL;
    *bytes = am_norm_backward_bytes(*args);
    return WFST_OK;
}

extern "C" int wfst_am_norm_backward(const wfst_am_norm_backward_args *args, void *hip_stream)
{
    clear_error();
    if (!args) return no_args("wfst_am_norm_backward");
    Checks c{"wfst_am_norm_backward"};
    if (!check(c, *args)) return WFST_EINVAL;
    return launched(am_launch_norm_backward(*args, stream_of(hip_stream)), c.who);
}

extern "C" int wfst_am_layer_norm(const wfst_am_layer_norm_args *args, void *hip_stream)
{
    clear_error();
    if (!args) return no_args("wfst_am_layer_norm");
    Checks c{"wfst_am_layer_norm"};
    if (!check(c, *args)) return WFST_EINVAL;
    return args->x.rows ? launched(am_launch_layer_norm(*args, stream_of(hip_stream)), c.who) : WFST_OK;
}

extern "C" int wfst_am_layer_norm_backward_workspace(const wfst_am_layer_norm_backward_args *args, int64_t *bytes)
{
    clear_error();
    if (!args || !bytes) return no_args("wfst_am_layer_norm_backward_workspace");
    Checks c{"wfst_am_layer_norm_backward_workspace"};
    if (!check_sizes(c, *args)) return WFST_EINVAL;
    *bytes = am_layer_norm_backward_bytes(*args);
    return WFST_OK;
}

extern "C" int wfst_am_layer_norm_backward(const wfst_am_layer_norm_backward_args *args, void *hip_stream)
{
    clear_error();
    if (!args) return no_args("wfst_am_layer_norm_backward");
    Checks c{"wfst_am_layer_norm_backward"};
    if (!check(c, *args)) return WFST_EINVAL;
    return launched(am_launch_layer_norm_backward(*args, stream_of(hip_stream)), c.who);
}

extern "C" int wfst_am_distill(const wfst_am_distill_args *args, void *hip_stream)
{
    clear_error();
    if (!args) return no_args("wfst_am_distill");
    Checks c{"wfst_am_distill"};
    if (!check(c, *args, false)) return WFST_EINVAL;
    return args->logits.rows ? launched(am_launch_distill(*args, false, stream_of(hip_stream)), c.who) : WFST_OK;
}

extern "C" int wfst_am_distill_backward(const wfst_am_distill_args *args, void *hip_stream)
{
    clear_error();
    if (!args) return no_args("wfst_am_distill_backward");
    Checks c{"wfst_am_distill_backward"};
    if (!check(c, *args, true)) return WFST_EINVAL;
    return args->logits.rows ? launched(am_launch_distill(*args, true, stream_of(hip_stream)), c.who) : WFST_OK;
}

extern "C" int wfst_am_clip_workspace(const wfst_am_clip_args *args, int64_t *bytes)
{
    clear_error();
    if (!args || !bytes) return no_args("wfst_am_clip_workspace");
    Checks c{"wfst_am_clip_workspace"};
    if (!check_sizes(c, *args)) return WFST_EINVAL;
    *bytes = am_clip_bytes(*args);
    return WFST_OK;
}

extern "C" int wfst_am_clip(const wfst_am_clip_args *args, void *hip_stream)
{
    clear_error();
    if (!args) return no_args("wfst_am_clip");
    Checks c{"wfst_am_clip"};
    try {
        if (!check(c, *args)) return WFST_EINVAL;
    } catch (const std::exception &) {   // no memory for the list of places
        set_error("%s: out of host memory", c.who);
        return WFST_ENOMEM;
    }
    return launched(am_launch_clip(*args, stream_of(hip_stream)), c.who);
}

extern "C" int wfst_am_loglikes(const wfst_am_loglikes_args *args, void *hip_stream)
{
    clear_error();
    if (!args) return no_args("wfst_am_loglikes");
    Checks c{"wfst_am_loglikes"};
    if (!check(c, *args)) return WFST_EINVAL;
    return args->logits.rows ? launched(am_launch_loglikes(*args, stream_of(hip_stream)), c.who) : WFST_OK;
}
