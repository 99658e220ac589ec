// What the files of the acoustic model's matrix products share.
#pragma once

#include "am_tile.h"

namespace wfd {

// out = a b^T, both k-contiguous; tile 0: without tiles (am_thin.h) (am_linear_f16.hip, am_linear_bf16.hip, am_linear_f8.hip)
template <typename E>
void am_product_forward(const AmProduct &p, int32_t tile, hipStream_t st);
// out = act(a gates^T) * (a values^T); tile 0: without tiles (am_gated_f16.hip, am_gated_bf16.hip, am_gated_f8.hip)
template <typename E>
void am_product_gated(const AmProduct &p, int32_t tile, hipStream_t st);
// dx[m][k] = sum_n dz[m][n] w[n][k]: w is k-major
template <typename E>
void am_product_dx(const AmProduct &p, int32_t tile, hipStream_t st);
// dw[n][k] = sum_m dz[m][n] x[m][k]: both are k-major
template <typename E>
void am_product_dw(const AmProduct &p, int32_t tile, hipStream_t st);

// row stride of dz in the workspace: rows on 16 bytes
constexpr int64_t am_dz_stride(int64_t n) { return (n + 7) & ~int64_t{7}; }

// Is dz held in two 16-bit parts?  One holds all of dy times a slope of 0 or 1.
inline bool am_dz_in_parts(const wfst_am_linear_backward_args &a)
{
    return !a.round_dz && (a.activation == WFST_ACT_SILU || a.activation == WFST_ACT_GELU);
}

// The workspace: dz (where the activation has a slope; the low parts behind the
// high ones), then room that the column sums and each product's parts use one
// after the other.
struct BackwardPlan {
    int64_t dz_bytes;   // of one part
    int32_t dz_parts;
    int64_t partial_bytes;
    AmPlan dx, dw;
    int32_t across;   // threads side by side in the pass over dy
    int64_t strips;   // of rows, in that pass
};

// in_workspace: is dz written there (it is dy else)?  parts: of dz.  across_cols: columns that the pass over dy has side by
// side; rows: of a thread in that pass, at least
inline BackwardPlan am_backward_plan(const wfst_am_linear_backward_args &a, bool in_workspace, int32_t parts, int64_t across_cols, int64_t rows)
{
    const int64_t M = a.dy.rows, N = a.dy.cols;
    BackwardPlan p{0, parts, 0, {64, 1}, {64, 1}, 1, 1};
    while (p.across < 64 && p.across * 8 < across_cols) p.across *= 2;
    // about 1,024 workgroups at most
    const int64_t wide = (across_cols + p.across * 8 - 1) / (p.across * 8), tall = M * p.across / (256 * rows), most = 1024 / wide;
    p.strips = tall < most ? tall : most;
    if (p.strips < 1) p.strips = 1;
    if (a.dbias && p.strips > 1) p.partial_bytes = (p.strips * N * 4 + 255) & ~int64_t{255};
    if (in_workspace && (a.dx.data || a.dw.data)) p.dz_bytes = (M * am_dz_stride(N) * 2 + 255) & ~int64_t{255};
    // dz in the workspace is aligned whatever its address
    const AmOperand dz = p.dz_bytes ? AmOperand{nullptr, am_dz_stride(N) * 2, 0}
                                    : AmOperand{static_cast<const char *>(a.dy.data), a.dy.row_stride * 2, 0};
    const auto rows_of = [](AmOperand o, int64_t extent) { return AmOperand{o.data, o.ld, static_cast<int32_t>(extent)}; };
    const auto other = [](const wfst_matrix &m, int64_t cols) {
        return AmOperand{static_cast<const char *>(m.data), m.row_stride * 2, static_cast<int32_t>(cols)};
    };
    if (a.dx.data) {
        p.dx = am_plan(rows_of(dz, M), false, other(a.w, a.dx.cols), true, N, 2, p.dz_parts, true);
        const int64_t b = am_most_partial_bytes(M, a.dx.cols, N * p.dz_parts);
        p.partial_bytes = b > p.partial_bytes ? b : p.partial_bytes;
    }
    if (a.dw.data) {
        p.dw = am_plan(rows_of(dz, N), true, other(a.x, a.dw.cols), true, M, 2, p.dz_parts, true);
        const int64_t b = am_most_partial_bytes(N, a.dw.cols, M * p.dz_parts);
        p.partial_bytes = b > p.partial_bytes ? b : p.partial_bytes;
    }
    return p;
}

inline BackwardPlan am_backward_plan(const wfst_am_linear_backward_args &a)
{
    return am_backward_plan(a, a.activation != WFST_ACT_NONE, am_dz_in_parts(a) ? 2 : 1, a.dy.cols, 4);
}

// act'(z), and act(z) where it is asked for
__device__ __forceinline__ float am_slope(float z, int32_t kind, float *value = nullptr)
{
    if (kind == WFST_ACT_NONE) {
        if (value) *value = z;
        return 1.0f;
    }
    if (kind == WFST_ACT_RELU) {
        if (value) *value = z < 0.0f ? 0.0f : z;   // a NaN stays one
        return z > 0.0f ? 1.0f : 0.0f;
    }
    if (kind == WFST_ACT_SILU) {
        const float s = __builtin_amdgcn_rcpf(1.0f + am_exp(-z));
        if (value) *value = z * s;
        return s * (1.0f + z * (1.0f - s));
    }
    float bell;
    const float n = am_normal(z, bell);
    if (value) *value = z * n;
    return fmaf(z * 0.39894228f, bell, n);
}

// 8 float32 values as T, or as two values of it where `low` is not NULL (AmParts); n of them exist
template <typename T>
__device__ __forceinline__ void am_store_dz(T *high, T *low, int64_t n, const float (&g)[8])
{
    if (!low) return store_floats(high, n, g);
    float h[8], l[8];
#pragma unroll
    for (int e = 0; e < 8; e++) {
        h[e] = g[e] * (1.0f / AmParts<T>::kHigh);
        const float held = static_cast<float>(static_cast<T>(h[e])) * AmParts<T>::kHigh;
        l[e] = fabsf(held) < INFINITY ? (g[e] - held) * (1.0f / AmParts<T>::kLow) : 0.0f;
    }
    store_floats(high, n, h);
    store_floats(low, n, l);
}

// dx and dw of a.w and a.x from dz, whose rows lie `ld` bytes apart (a.dy's place is not looked at)
template <typename T>
void am_launch_gradient_products(const wfst_am_linear_backward_args &a, const BackwardPlan &plan, const char *dz, const char *dz_low,
                                 int64_t ld, float *partial, hipStream_t st)
{
    const int64_t M = a.dy.rows, N = a.dy.cols;
    if (a.dx.data && M > 0) {
        AmProduct p{};
        p.a = {dz, ld, static_cast<int32_t>(M)};
        p.a_low = dz_low;
        p.b = {static_cast<const char *>(a.w.data), a.w.row_stride * 2, static_cast<int32_t>(a.dx.cols)};
        p.inner = static_cast<int32_t>(N);
        p.splits = plan.dx.splits;
        p.partial = partial;
        p.out = a.dx;
        am_product_dx<T>(p, plan.dx.tile, st);
    }
    if (a.dw.data) {
        AmProduct p{};
        p.a = {dz, ld, static_cast<int32_t>(N)};
        p.a_low = dz_low;
        p.b = {static_cast<const char *>(a.x.data), a.x.row_stride * 2, static_cast<int32_t>(a.dw.cols)};
        p.inner = static_cast<int32_t>(M);
        p.splits = plan.dw.splits;
        p.partial = partial;   // the other product's parts are joined by now
        p.out = a.dw;
        am_product_dw<T>(p, plan.dw.tile, st);
    }
}

}  // namespace wfd
