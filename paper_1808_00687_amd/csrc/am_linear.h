// What the files of the acoustic model's matrix products share.
#pragma once

#include "am_tile.h"

namespace wfd {

// out = a b^T, both k-contiguous; tile 0: without tiles (am_thin.h) (am_linear_f16.hip, am_linear_bf16.hip, am_linear_f8.hip)
template <typename E>
void am_product_forward(const AmProduct &p, int32_t tile, hipStream_t st);
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

inline BackwardPlan am_backward_plan(const wfst_am_linear_backward_args &a)
{
    const int64_t M = a.dy.rows, N = a.dy.cols;
    BackwardPlan p{0, am_dz_in_parts(a) ? 2 : 1, 0, {64, 1}, {64, 1}, 1, 1};
    while (p.across < 64 && p.across * 8 < N) p.across *= 2;
    // 4 rows a thread at least, about 1,024 workgroups at most
    const int64_t wide = (N + p.across * 8 - 1) / (p.across * 8), tall = M * p.across / 1024, most = 1024 / wide;
    p.strips = tall < most ? tall : most;
    if (p.strips < 1) p.strips = 1;
    if (a.dbias && p.strips > 1) p.partial_bytes = (p.strips * N * 4 + 255) & ~int64_t{255};
    if (a.activation != WFST_ACT_NONE && (a.dx.data || a.dw.data)) p.dz_bytes = (M * am_dz_stride(N) * 2 + 255) & ~int64_t{255};
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

}  // namespace wfd
