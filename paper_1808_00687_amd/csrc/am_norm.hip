// Root-mean-square norm of rows: forward (residual's addition, 8-bit output)
// and backward.
//
// Both are bound by memory: a row is read once into registers, its statistics
// are reduced over a wave (rows of up to 2,048), and it is written from there.
// A workgroup takes several rows in turn, so the gain stays in registers and in
// the backward pass the gain's gradient is summed there over the rows of a
// workgroup; workgroups' sums are joined by a second small kernel in a fixed order.
//
// (53274, 1024) bf16 with the residual to e4m3: 72 us, 382 MB, 5.3 TB/s (a large
// copy reaches 5.1); backward of (16384, 2048) bf16 with dsum: 57 us, 268 MB,
// 4.7 TB/s, 5 of it the join.
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

// chunks where a matrix has 32-bit elements are half as long (the result's type is looked at below)
template <typename T>
constexpr int kChunk = sizeof(T) == 4 ? 4 : 8;

template <typename T, typename S, bool k8Bits>
__global__ __launch_bounds__(S::kThreads) void norm_kernel(wfst_am_norm_args a)
{
    __shared__ RowScratch scratch;
    int turn = 0;
    const int64_t M = a.x.rows, D = a.x.cols, step = static_cast<int64_t>(gridDim.x) * S::kRows;
    const int t = threadIdx.x % S::kTpr;
    RowPart<S, float> gain;
    if (a.gain) gain.hold(a.gain, D, t);
    RowPart<S, T> x, r, x_next, r_next;
    const auto hold = [&](int64_t m) {
        if (m >= M) return;
        x_next.hold(row<T>(a.x, m), D, t);
        if (a.residual.data) r_next.hold(row<T>(a.residual, m), D, t);
    };
    int64_t m = static_cast<int64_t>(blockIdx.x) * S::kRows + threadIdx.x / S::kTpr;
    hold(m);
    for (; m < M; m += step) {
        x = x_next, r = r_next;
        hold(m + step);   // the next row is on its way while this one is worked on
        const auto sum_of = [&](int v, int64_t c, int64_t left, float (&s)[S::kC]) {
            x.get(v, c, left, s);
            if (!a.residual.data) return;
            float w[S::kC];
            r.get(v, c, left, w);
#pragma unroll
            for (int e = 0; e < S::kC; e++) s[e] += w[e];
        };
        const auto times_gain = [&](int v, int64_t c, int64_t left, float (&s)[S::kC]) {
            if (!a.gain) return;
            float g[S::kC];
            gain.get(v, c, left, g);
#pragma unroll
            for (int e = 0; e < S::kC; e++) s[e] *= g[e];
        };
        float ss = 0.0f;
        S::each(D, t, [&](int v, int64_t c, int64_t left) {
            float s[S::kC];
            sum_of(v, c, left, s);
#pragma unroll
            for (int e = 0; e < S::kC; e++) ss = fmaf(s[e], s[e], ss);
        });
        const float rho = 1.0f / sqrtf(row_sum<S>(ss, scratch, turn) / static_cast<float>(D) + a.eps);
        float scale = 1.0f, inv = 1.0f;
        bool whole = false;   // is a quotient formed by a division?
        if constexpr (k8Bits) {
            uint32_t top = 0;
            S::each(D, t, [&](int v, int64_t c, int64_t left) {
                float s[S::kC];
                sum_of(v, c, left, s);
#pragma unroll
                for (int e = 0; e < S::kC; e++) s[e] *= rho;
                times_gain(v, c, left, s);
#pragma unroll
                for (int e = 0; e < S::kC; e++) {
                    const uint32_t b = __float_as_uint(s[e]) & 0x7FFFFFFFu;
                    top = e < left && b > top ? b : top;
                }
            });
            scale = __uint_as_float(row_max_u32<S>(top, scratch, turn)) / kE4m3Max;
            scale = scale < 1.17549435e-38f ? 1.17549435e-38f : scale;   // a NaN stays one
            // A product with the rounded reciprocal, corrected once, is the rounded quotient
            // (Markstein 1990) unless the divisor's bits are all ones or something leaves the
            // range; 72.8 us for (53274, 1024) bf16, 74.5 with divisions.
            inv = 1.0f / scale;
            whole = __builtin_amdgcn_readfirstlane(!(scale >= 0x1p-90f && scale <= 0x1p90f) || (__float_as_uint(scale) & 0x7FFFFFu) == 0x7FFFFFu) != 0;
            if (t == 0) a.y_scale[m] = scale;
        }
        S::each(D, t, [&](int v, int64_t c, int64_t left) {
            float s[S::kC];
            sum_of(v, c, left, s);
            if (a.sum.data) store_floats(row_out<T>(a.sum, m) + c, left, s);
#pragma unroll
            for (int e = 0; e < S::kC; e++) s[e] *= rho;
            times_gain(v, c, left, s);
            if constexpr (k8Bits) {
                if (whole)
#pragma unroll
                    for (int e = 0; e < S::kC; e++) s[e] /= scale;
                else
#pragma unroll
                    for (int e = 0; e < S::kC; e++) {
                        const float q = s[e] * inv;   // alone it would move ties of e4m3
                        s[e] = fmaf(fmaf(-q, scale, s[e]), inv, q);
                    }
                store_floats(row_out<f8>(a.y, m) + c, left, s);
            } else if (a.y.type == WFST_BF16) {
                store_floats(row_out<bf16>(a.y, m) + c, left, s);
            } else if (a.y.type == WFST_F16) {
                store_floats(row_out<f16>(a.y, m) + c, left, s);
            } else {
                store_floats(row_out<float>(a.y, m) + c, left, s);
            }
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
    const int64_t M = a.s.rows, D = a.s.cols, step = static_cast<int64_t>(gridDim.x) * S::kRows;
    const int t = threadIdx.x % S::kTpr;
    RowPart<S, float> gain;
    if (a.gain) gain.hold(a.gain, D, t);
    float dg[S::kHeld][S::kC] = {};
    RowPart<S, T> s, dy, ds, s_next, dy_next;
    const auto hold = [&](int64_t m) {
        if (m >= M) return;
        s_next.hold(row<T>(a.s, m), D, t);
        dy_next.hold(row<T>(a.dy, m), D, t);
    };
    int64_t m = static_cast<int64_t>(blockIdx.x) * S::kRows + threadIdx.x / S::kTpr;
    hold(m);
    for (; m < M; m += step) {
        s = s_next, dy = dy_next;
        if (a.dsum.data) ds.hold(row<T>(a.dsum, m), D, t);
        hold(m + step);
        const auto u_of = [&](int v, int64_t c, int64_t left, const float (&w)[S::kC], float (&u)[S::kC]) {
#pragma unroll
            for (int e = 0; e < S::kC; e++) u[e] = w[e];
            if (!a.gain) return;
            float g[S::kC];
            gain.get(v, c, left, g);
#pragma unroll
            for (int e = 0; e < S::kC; e++) u[e] *= g[e];
        };
        float ss = 0.0f, us = 0.0f;
        S::each(D, t, [&](int v, int64_t c, int64_t left) {
            float x[S::kC], w[S::kC], u[S::kC];
            s.get(v, c, left, x);
            dy.get(v, c, left, w);
            u_of(v, c, left, w, u);
#pragma unroll
            for (int e = 0; e < S::kC; e++) {
                ss = fmaf(x[e], x[e], ss);
                us = fmaf(u[e], x[e], us);
            }
        });
        row_sums<S>(ss, us, scratch, turn);
        const float rho = 1.0f / sqrtf(ss / static_cast<float>(D) + a.eps);
        const float c0 = rho * rho * (us / static_cast<float>(D));
        if (S::kNv == 0 && rhos && t == 0) rhos[m] = rho;
        if (S::kNv == 0 && !a.dx.data) continue;
        S::each(D, t, [&](int v, int64_t c, int64_t left) {
            float x[S::kC], w[S::kC], u[S::kC];
            s.get(v, c, left, x);
            dy.get(v, c, left, w);
            u_of(v, c, left, w, u);
            if constexpr (S::kNv > 0)
#pragma unroll
                for (int e = 0; e < S::kC; e++) dg[v][e] = fmaf(w[e] * rho, x[e], dg[v][e]);
            if (!a.dx.data) return;
            float d[S::kC];
#pragma unroll
            for (int e = 0; e < S::kC; e++) d[e] = rho * (u[e] - x[e] * c0);
            if (a.dsum.data) {
                ds.get(v, c, left, u);
#pragma unroll
                for (int e = 0; e < S::kC; e++) d[e] += u[e];
            }
            store_floats(row_out<T>(a.dx, m) + c, left, d);
        });
    }
    if (S::kNv == 0 || !partial) return;
    if constexpr (S::kRows == 1) {
        S::each(D, t, [&](int v, int64_t c, int64_t left) { store_floats(partial + blockIdx.x * D + c, left, dg[v]); });
    } else {
        // the workgroup's rows' sums, one after the other
        __shared__ float total[S::kHeld * S::kTpr * S::kC];
        for (int w = 0; w < S::kRows; w++) {
            __syncthreads();
            if (static_cast<int>(threadIdx.x) / S::kTpr != w) continue;
#pragma unroll
            for (int v = 0; v < S::kHeld; v++)
#pragma unroll
                for (int e = 0; e < S::kC; e++) {
                    float &o = total[(v * S::kC + e) * S::kTpr + t];
                    o = w ? o + dg[v][e] : dg[v][e];
                    dg[v][e] = o;
                }
        }
        if (threadIdx.x / S::kTpr == S::kRows - 1)
            S::each(D, t, [&](int v, int64_t c, int64_t left) { store_floats(partial + blockIdx.x * D + c, left, dg[v]); });
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

// 32 columns a workgroup, 32 threads a column, 4 strips of a thread on their way at a time
__global__ __launch_bounds__(1024) void column_join_kernel(const float *partial, int64_t strips, int64_t n, float *out)
{
    __shared__ float part[32][33];
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const int64_t c = static_cast<int64_t>(blockIdx.x) * 32 + x;
    float t = 0.0f;
    if (c < n) {
        int64_t s = y;
        for (; s + 96 < strips; s += 128) {
            float v[4];
#pragma unroll
            for (int i = 0; i < 4; i++) v[i] = partial[(s + i * 32) * n + c];
            t += (v[0] + v[1]) + (v[2] + v[3]);
        }
        for (; s < strips; s += 32) t += partial[s * n + c];
    }
    part[y][x] = t;
    __syncthreads();
    if (y != 0 || c >= n) return;
    for (int i = 1; i < 32; i++) t += part[i][x];
    out[c] = t;
}

// Workgroups at most.  Forward, (53274, 1024) to 8 bits: 2, 4, 8, 16, 32 and 64 a CU take 74,
// 80, 75, 70, 68 and 66 us, (53274, 96) 45, 35, 31, 27, 27 and 29.  Backward, whose workgroups'
// sums are joined, (16384, 2048): 2, 3, 4, 6 and 8 take 57, 52, 49, 52 and 60, (53274, 256) 53,
// 42, 38, 35 and 38, (16000, 5000) with 3 133 and with 4 170.
constexpr int64_t kForwardBlocks = 256 * 16;
constexpr int64_t kBackwardBlocks = 256 * 3;

// strips of rows whose sums of the gain's gradient are joined
int64_t dgain_strips(int64_t M, int64_t D)
{
    int64_t n = 0;
    am_row_shape_lean<8>(D, [&](auto shape) {   // the same for shorter chunks
        using S = decltype(shape);
        n = S::kNv > 0 ? static_cast<int64_t>(am_row_blocks<S>(M, kBackwardBlocks)) : 0;
    });
    return n;
}

template <typename T>
void launch_norm(const wfst_am_norm_args &a, hipStream_t st)
{
    if constexpr (kChunk<T> > 4)
        if (a.y.type == WFST_F32) {
            // (53274, 1024) bf16 to f32: 60 us, with chunks of 8 71; with the residual 101 and 107
            am_row_shape_norm<4>(a.x.cols, [&](auto shape) {
                using S = decltype(shape);
                norm_kernel<T, S, false><<<am_row_blocks<S>(a.x.rows, kForwardBlocks), S::kThreads, 0, st>>>(a);
            });
            return;
        }
    am_row_shape_norm<kChunk<T>>(a.x.cols, [&](auto shape) {
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
    am_row_shape_lean<kChunk<T>>(D, [&](auto shape) {
        using S = decltype(shape);
        const unsigned g = M ? am_row_blocks<S>(M, kBackwardBlocks) : 0;
        if constexpr (S::kNv > 0) {
            if (M) norm_backward_kernel<T, S><<<g, S::kThreads, 0, st>>>(a, a.dgain ? work : nullptr, nullptr);
            if (a.dgain) am_launch_column_join(work, g, D, a.dgain, st);
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
    column_join_kernel<<<static_cast<unsigned>((n + 31) / 32), 1024, 0, st>>>(partial, strips, n, out);
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
