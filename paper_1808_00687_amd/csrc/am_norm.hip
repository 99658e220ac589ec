// Root-mean-square norm of rows: forward (residual's addition, 8-bit output)
// and backward.
//
// Both are bound by memory: a row is read once into registers, its statistics
// are reduced over a wave (rows of up to 2,048), and it is written from there.
// A workgroup takes several rows in turn, so the gain stays in registers and in
// the backward pass the gain's gradient is summed there over the rows of a
// workgroup; workgroups' sums are joined by a second small kernel in a fixed order.
#include "am_rows.h"

namespace wfd {
namespace {

template <typename T>
__device__ __forceinline__ const T *row(const wfst_matrix &m, int64_t r)
{
    return static_cast<const T *>(m.data) + r * m.row_stride;
}

template <typename T>
__device__ __forceinline__ T *row_out(const wfst_matrix &m, int64_t r)
{
    return static_cast<T *>(m.data) + r * m.row_stride;
}

__device__ __forceinline__ void load_gain(const float *gain, int64_t c, int64_t left, float (&g)[8])
{
    if (gain) {
        load8(gain + c, left, g);
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; e++) g[e] = 1.0f;
}

template <typename T, typename S, bool k8Bits>
__global__ __launch_bounds__(S::kThreads) void norm_kernel(wfst_am_norm_args a)
{
    __shared__ RowScratch scratch;
    int turn = 0;
    const int64_t M = a.x.rows, D = a.x.cols;
    const int t = threadIdx.x % S::kTpr;
    RowPart<S> gain;
    const auto load_g = [&](int64_t c, int64_t left, float (&g)[8]) { load_gain(a.gain, c, left, g); };
    gain.hold(D, t, load_g);
    for (int64_t m = static_cast<int64_t>(blockIdx.x) * S::kRows + threadIdx.x / S::kTpr; m < M;
         m += static_cast<int64_t>(gridDim.x) * S::kRows) {
        const T *x = row<T>(a.x, m), *r = a.residual.data ? row<T>(a.residual, m) : nullptr;
        const auto load_s = [&](int64_t c, int64_t left, float (&v)[8]) {
            load8(x + c, left, v);
            if (!r) return;
            float w[8];
            load8(r + c, left, w);
#pragma unroll
            for (int e = 0; e < 8; e++) v[e] += w[e];
        };
        RowPart<S> s;
        s.hold(D, t, load_s);
        float ss = 0.0f;
        s.each(load_s, [&](int64_t, int64_t, float (&v)[8]) {
#pragma unroll
            for (int e = 0; e < 8; e++) ss = fmaf(v[e], v[e], ss);
        });
        const float rho = 1.0f / sqrtf(row_sum<S>(ss, scratch, turn) / static_cast<float>(D) + a.eps);
        int v_at = 0;   // the chunk's place among the held ones
        const auto gain_of = [&](int64_t c, int64_t left, float (&g)[8]) {
            if constexpr (S::kNv > 0) {
#pragma unroll
                for (int e = 0; e < 8; e++) g[e] = gain.x[v_at][e];
                v_at++;
            } else {
                load_gain(a.gain, c, left, g);
            }
        };
        float inv = 1.0f;
        if constexpr (k8Bits) {
            uint32_t top = 0;
            v_at = 0;
            s.each(load_s, [&](int64_t c, int64_t left, float (&v)[8]) {
                float g[8];
                gain_of(c, left, g);
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const uint32_t b = e < left ? __float_as_uint(v[e] * rho * g[e]) & 0x7FFFFFFFu : 0;
                    top = top > b ? top : b;
                }
            });
            float scale = __uint_as_float(row_max_u32<S>(top, scratch, turn)) / kE4m3Max;
            scale = scale < 1.17549435e-38f ? 1.17549435e-38f : scale;   // a NaN stays one
            inv = 1.0f / scale;
            if (t == 0) a.y_scale[m] = scale;
        }
        T *sum = a.sum.data ? row_out<T>(a.sum, m) : nullptr;
        v_at = 0;
        s.each(load_s, [&](int64_t c, int64_t left, float (&v)[8]) {
            float g[8];
            gain_of(c, left, g);
            if (sum) store8(sum + c, left, v);
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; e++) y[e] = v[e] * rho * g[e] * inv;
            if constexpr (k8Bits) store8(row_out<f8>(a.y, m) + c, left, y);
            else if (a.y.type == WFST_BF16) store8(row_out<bf16>(a.y, m) + c, left, y);
            else if (a.y.type == WFST_F16) store8(row_out<f16>(a.y, m) + c, left, y);
            else store8(row_out<float>(a.y, m) + c, left, y);
        });
    }
}

// dx, and in `partial` the workgroup's sums of dy s rho (held rows only; else
// rho of each row goes to `rhos` and a second kernel sums)
template <typename T, typename S>
__global__ __launch_bounds__(S::kThreads) void norm_backward_kernel(wfst_am_norm_backward_args a, float *partial, float *rhos)
{
    __shared__ RowScratch scratch;
    int turn = 0;
    const int64_t M = a.s.rows, D = a.s.cols;
    const int t = threadIdx.x % S::kTpr;
    constexpr int kHeld = RowPart<S>::kHeld;
    float dg[kHeld][8] = {};
    for (int64_t m = static_cast<int64_t>(blockIdx.x) * S::kRows + threadIdx.x / S::kTpr; m < M;
         m += static_cast<int64_t>(gridDim.x) * S::kRows) {
        const T *s_row = row<T>(a.s, m), *dy_row = row<T>(a.dy, m);
        const T *ds_row = a.dsum.data ? row<T>(a.dsum, m) : nullptr;
        T *dx = a.dx.data ? row_out<T>(a.dx, m) : nullptr;
        const auto load_s = [&](int64_t c, int64_t left, float (&v)[8]) { load8(s_row + c, left, v); };
        const auto load_dy = [&](int64_t c, int64_t left, float (&v)[8]) { load8(dy_row + c, left, v); };
        RowPart<S> s, dy;
        s.hold(D, t, load_s);
        dy.hold(D, t, load_dy);
        float ss = 0.0f, us = 0.0f;
        int v_at = 0;
        s.each(load_s, [&](int64_t c, int64_t left, float (&v)[8]) {
            float g[8];
            load_gain(a.gain, c, left, g);
            if constexpr (S::kNv == 0) load_dy(c, left, dy.x[0]);
            const float(&w)[8] = dy.x[S::kNv > 0 ? v_at : 0];
#pragma unroll
            for (int e = 0; e < 8; e++) {
                ss = fmaf(v[e], v[e], ss);
                us = fmaf(w[e] * g[e], v[e], us);
            }
            v_at++;
        });
        row_sums<S>(ss, us, scratch, turn);
        const float rho = 1.0f / sqrtf(ss / static_cast<float>(D) + a.eps);
        const float c0 = rho * rho * (us / static_cast<float>(D));
        if (S::kNv == 0 && rhos && t == 0) rhos[m] = rho;
        if (S::kNv == 0 && !dx) continue;
        v_at = 0;
        s.each(load_s, [&](int64_t c, int64_t left, float (&v)[8]) {
            if constexpr (S::kNv == 0) load_dy(c, left, dy.x[0]);
            const float(&w)[8] = dy.x[S::kNv > 0 ? v_at : 0];
            if constexpr (S::kNv > 0)
#pragma unroll
                for (int e = 0; e < 8; e++) dg[v_at][e] = fmaf(w[e] * rho, v[e], dg[v_at][e]);
            v_at++;
            if (!dx) return;
            float g[8], d[8] = {};
            load_gain(a.gain, c, left, g);
            if (ds_row) load8(ds_row + c, left, d);
#pragma unroll
            for (int e = 0; e < 8; e++) d[e] += rho * (w[e] * g[e] - v[e] * c0);
            store8(dx + c, left, d);
        });
    }
    if (S::kNv == 0 || !partial) return;
    // the rows' sums of a workgroup side by side in `partial`
    float *o = partial + (static_cast<int64_t>(blockIdx.x) * S::kRows + threadIdx.x / S::kTpr) * D;
#pragma unroll
    for (int v = 0; v < kHeld; v++) {
        const int64_t c = (static_cast<int64_t>(v) * S::kTpr + t) * 8;
        if (c < D) store8(o + c, D - c, dg[v]);
    }
}

// the gain's gradient of rows too long to hold, one thread a column
template <typename T>
__global__ __launch_bounds__(256) void norm_dgain_kernel(wfst_am_norm_backward_args a, const float *rhos)
{
    const int64_t M = a.s.rows, D = a.s.cols;
    const int64_t d = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (d >= D) return;
    float t = 0.0f;
    for (int64_t m = 0; m < M; m++) t = fmaf(to_f32(row<T>(a.dy, m)[d]) * rhos[m], to_f32(row<T>(a.s, m)[d]), t);
    a.dgain[d] = t;
}

// 32 columns a workgroup, 8 threads a column
__global__ __launch_bounds__(256) void column_join_kernel(const float *partial, int64_t strips, int64_t n, float *out)
{
    __shared__ float part[8][32];
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const int64_t c = static_cast<int64_t>(blockIdx.x) * 32 + x;
    float t = 0.0f;
    if (c < n)
        for (int64_t s = y; s < strips; s += 8) t += partial[s * n + c];
    part[y][x] = t;
    __syncthreads();
    if (y != 0 || c >= n) return;
    for (int i = 1; i < 8; i++) t += part[i][x];
    out[c] = t;
}

constexpr int64_t kForwardBlocks = 256 * 16;
constexpr int64_t kBackwardBlocks = 256 * 2;

// strips of rows whose sums of the gain's gradient are joined
int64_t dgain_strips(int64_t M, int64_t D)
{
    int64_t n = 0;
    am_row_shape(D, [&](auto shape) {
        using S = decltype(shape);
        n = S::kNv > 0 ? static_cast<int64_t>(am_row_blocks<S>(M, kBackwardBlocks)) * S::kRows : 0;
    });
    return n;
}

template <typename T>
void launch_norm(const wfst_am_norm_args &a, hipStream_t st)
{
    am_row_shape(a.x.cols, [&](auto shape) {
        using S = decltype(shape);
        const unsigned g = am_row_blocks<S>(a.x.rows, kForwardBlocks);
        if (a.y.type == WFST_F8E4M3) norm_kernel<T, S, true><<<g, S::kThreads, 0, st>>>(a);
        else norm_kernel<T, S, false><<<g, S::kThreads, 0, st>>>(a);
    });
}

template <typename T>
void launch_norm_backward(const wfst_am_norm_backward_args &a, hipStream_t st)
{
    const int64_t M = a.s.rows, D = a.s.cols;
    float *work = static_cast<float *>(a.workspace);
    am_row_shape(D, [&](auto shape) {
        using S = decltype(shape);
        const unsigned g = M ? am_row_blocks<S>(M, kBackwardBlocks) : 0;
        if constexpr (S::kNv > 0) {
            if (M) norm_backward_kernel<T, S><<<g, S::kThreads, 0, st>>>(a, a.dgain ? work : nullptr, nullptr);
            if (a.dgain) am_launch_column_join(work, static_cast<int64_t>(g) * S::kRows, D, a.dgain, st);
        } else {
            // the gain's gradient before dx may overwrite dy
            wfst_am_norm_backward_args b = a;
            b.dx.data = nullptr;
            if (a.dgain) {
                if (M) norm_backward_kernel<T, S><<<g, S::kThreads, 0, st>>>(b, nullptr, work);
                norm_dgain_kernel<T><<<static_cast<unsigned>((D + 255) / 256), 256, 0, st>>>(a, work);
            }
            if (M && a.dx.data) norm_backward_kernel<T, S><<<g, S::kThreads, 0, st>>>(a, nullptr, nullptr);
        }
    });
}

}  // namespace

void am_launch_column_join(const float *partial, int64_t strips, int64_t n, float *out, hipStream_t st)
{
    column_join_kernel<<<static_cast<unsigned>((n + 31) / 32), 256, 0, st>>>(partial, strips, n, out);
}

hipError_t am_launch_norm(const wfst_am_norm_args &a, hipStream_t st)
{
    if (a.x.type == WFST_F32) launch_norm<float>(a, st);
    else if (a.x.type == WFST_F16) launch_norm<f16>(a, st);
    else launch_norm<bf16>(a, st);
    return hipGetLastError();
}

int64_t am_norm_backward_bytes(const wfst_am_norm_backward_args &a)
{
    if (!a.dgain) return 0;
    const int64_t strips = dgain_strips(a.s.rows, a.s.cols);
    return ((strips ? strips * a.s.cols : a.s.rows) * 4 + 255) & ~int64_t{255};
}

hipError_t am_launch_norm_backward(const wfst_am_norm_backward_args &a, hipStream_t st)
{
    if (a.s.type == WFST_F32) launch_norm_backward<float>(a, st);
    else if (a.s.type == WFST_F16) launch_norm_backward<f16>(a, st);
    else launch_norm_backward<bf16>(a, st);
    return hipGetLastError();
}

}  // namespace wfd
