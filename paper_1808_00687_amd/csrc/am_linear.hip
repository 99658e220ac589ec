// Matrix products of the acoustic model with what follows them in the same
// kernel: scales, bias, activation, residual.
#include "am_device.h"

namespace wfd {
namespace {

__device__ __forceinline__ float activate(float z, int32_t kind)
{
    switch (kind) {
    case WFST_ACT_RELU: return z < 0.0f ? 0.0f : z;   // a NaN stays one
    case WFST_ACT_SILU: return z / (1.0f + expf(-z));
    case WFST_ACT_GELU: return 0.5f * z * (1.0f + erff(z * 0.70710678f));
    default: return z;
    }
}

__device__ __forceinline__ float slope(float z, int32_t kind)
{
    switch (kind) {
    case WFST_ACT_RELU: return z > 0.0f ? 1.0f : 0.0f;
    case WFST_ACT_SILU: {
        const float s = 1.0f / (1.0f + expf(-z));
        return s * (1.0f + z * (1.0f - s));
    }
    case WFST_ACT_GELU:
        return 0.5f * (1.0f + erff(z * 0.70710678f)) + z * expf(-0.5f * z * z) * 0.39894228f;
    default: return 1.0f;
    }
}

__device__ __forceinline__ void store_any(const wfst_matrix &m, int64_t at, float v)
{
    if (m.type == WFST_F32) static_cast<float *>(m.data)[at] = v;
    else if (m.type == WFST_F16) static_cast<f16 *>(m.data)[at] = from_f32<f16>(v);
    else static_cast<bf16 *>(m.data)[at] = from_f32<bf16>(v);
}

__device__ __forceinline__ float load_any(const wfst_matrix &m, int64_t at)
{
    return m.type == WFST_F32   ? static_cast<const float *>(m.data)[at]
           : m.type == WFST_F16 ? to_f32(static_cast<const f16 *>(m.data)[at])
                                : to_f32(static_cast<const bf16 *>(m.data)[at]);
}

// An operand: element (i, k) at data[i * row + k * step].
struct Operand {
    const void *data;
    int64_t row, step;
};

struct Product {
    Operand a, b;            // out[i][j] = sum_k a[i][k] b[j][k]
    int64_t rows, cols, inner;
    const float *a_scale, *b_scale, *bias;
    wfst_matrix residual, pre, out;
    int32_t activation;
};

constexpr int kTile = 16;

template <typename T>
__global__ __launch_bounds__(kTile *kTile) void product_kernel(Product p)
{
    __shared__ float as[kTile][kTile + 1], bs[kTile][kTile + 1];
    const int tx = threadIdx.x % kTile, ty = threadIdx.x / kTile;
    const int64_t across = (p.cols + kTile - 1) / kTile, tiles = across * ((p.rows + kTile - 1) / kTile);
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t i0 = tile / across * kTile, j0 = tile % across * kTile;
        float acc = 0.0f;
        for (int64_t k0 = 0; k0 < p.inner; k0 += kTile) {
            const int64_t k = k0 + tx;
            as[ty][tx] = i0 + ty < p.rows && k < p.inner
                             ? to_f32(static_cast<const T *>(p.a.data)[(i0 + ty) * p.a.row + k * p.a.step]) : 0.0f;
            bs[ty][tx] = j0 + ty < p.cols && k < p.inner
                             ? to_f32(static_cast<const T *>(p.b.data)[(j0 + ty) * p.b.row + k * p.b.step]) : 0.0f;
            __syncthreads();
            for (int i = 0; i < kTile; i++) acc = fmaf(as[ty][i], bs[tx][i], acc);
            __syncthreads();
        }
        const int64_t i = i0 + ty, j = j0 + tx;
        if (i >= p.rows || j >= p.cols) continue;
        if (p.a_scale) acc *= p.a_scale[i] * p.b_scale[j];
        if (p.bias) acc += p.bias[j];
        if (p.pre.data) store_any(p.pre, i * p.pre.row_stride + j, acc);
        float y = activate(acc, p.activation);
        if (p.residual.data) y += load_any(p.residual, i * p.residual.row_stride + j);
        store_any(p.out, i * p.out.row_stride + j, y);
    }
}

template <typename T>
void launch_product(const Product &p, hipStream_t st)
{
    const int64_t tiles = ((p.cols + kTile - 1) / kTile) * ((p.rows + kTile - 1) / kTile);
    product_kernel<T><<<static_cast<unsigned>(tiles < (1 << 22) ? tiles : 1 << 22), kTile * kTile, 0, st>>>(p);
}

constexpr int kColumns = 256;

// dz = dy * act'(pre) in the operands' type, and the column sums of the unrounded dz
template <typename T>
__global__ __launch_bounds__(kColumns) void slope_kernel(wfst_am_linear_backward_args a, T *dz)
{
    const int64_t M = a.dy.rows, N = a.dy.cols;
    const int64_t n = static_cast<int64_t>(blockIdx.x) * kColumns + threadIdx.x;
    if (n >= N) return;
    float sum = 0.0f;
    for (int64_t m = 0; m < M; m++) {
        float g = to_f32(static_cast<const T *>(a.dy.data)[m * a.dy.row_stride + n]);
        if (a.activation != WFST_ACT_NONE) {
            g *= slope(to_f32(static_cast<const T *>(a.pre.data)[m * a.pre.row_stride + n]), a.activation);
            if (dz) dz[m * N + n] = from_f32<T>(g);
        }
        sum += g;
    }
    if (a.dbias) a.dbias[n] = sum;
}

template <typename T>
void launch_backward(const wfst_am_linear_backward_args &a, hipStream_t st)
{
    const int64_t M = a.dy.rows, N = a.dy.cols;
    const bool act = a.activation != WFST_ACT_NONE, products = a.dx.data || a.dw.data;
    T *dz = act && products ? static_cast<T *>(a.workspace) : nullptr;
    if (a.dbias || dz)
        slope_kernel<T><<<static_cast<unsigned>((N + kColumns - 1) / kColumns), kColumns, 0, st>>>(a, dz);
    const void *g = dz ? dz : a.dy.data;
    const int64_t ld = dz ? N : a.dy.row_stride;
    Product p{};
    if (a.dx.data && M > 0) {
        p.a = {g, ld, 1};
        p.b = {a.w.data, 1, a.w.row_stride};
        p.rows = M, p.cols = a.dx.cols, p.inner = N;
        p.out = a.dx;
        launch_product<T>(p, st);
    }
    if (a.dw.data) {
        p.a = {g, 1, ld};
        p.b = {a.x.data, 1, a.x.row_stride};
        p.rows = N, p.cols = a.dw.cols, p.inner = M;
        p.out = a.dw;
        launch_product<T>(p, st);
    }
}

}  // namespace

hipError_t am_launch_linear(const wfst_am_linear_args &a, hipStream_t st)
{
    Product p{};
    p.a = {a.x.data, a.x.row_stride, 1};
    p.b = {a.w.data, a.w.row_stride, 1};
    p.rows = a.x.rows, p.cols = a.w.rows, p.inner = a.x.cols;
    p.a_scale = a.x_scale, p.b_scale = a.w_scale, p.bias = a.bias;
    p.residual = a.residual, p.pre = a.pre, p.out = a.y;
    p.activation = a.activation;
    if (a.x.type == WFST_F16) launch_product<f16>(p, st);
    else if (a.x.type == WFST_BF16) launch_product<bf16>(p, st);
    else launch_product<f8>(p, st);
    return hipGetLastError();
}

int64_t am_linear_backward_bytes(const wfst_am_linear_backward_args &a)
{
    const bool dz = a.activation != WFST_ACT_NONE && (a.dx.data || a.dw.data);
    return dz ? (a.dy.rows * a.dy.cols * 2 + 255) & ~int64_t{255} : 0;
}

hipError_t am_launch_linear_backward(const wfst_am_linear_backward_args &a, hipStream_t st)
{
    if (a.dy.type == WFST_F16) launch_backward<f16>(a, st);
    else launch_backward<bf16>(a, st);
    return hipGetLastError();
}

}  // namespace wfd
