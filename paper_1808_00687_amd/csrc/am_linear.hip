// The acoustic model's layers: wfst_am_linear and its gradients.
#include "am_linear.h"
#include "am_rows.h"

namespace wfd {
namespace {

// Sums the parts of a split product and finishes them.
__global__ __launch_bounds__(256) void join_kernel(AmProduct p)
{
    const int64_t n = static_cast<int64_t>(p.a.extent) * p.b.extent;
    for (int64_t at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; at < n; at += static_cast<int64_t>(gridDim.x) * 256) {
        float v[1] = {0.0f}, b_scale[1], bias[1];
        int s = 0;
        for (; s + 4 <= p.splits; s += 4) {   // 4 loads under way, added in order
            float u[4];
#pragma unroll
            for (int e = 0; e < 4; e++) u[e] = p.partial[(s + e) * n + at];
            v[0] = v[0] + u[0] + u[1] + u[2] + u[3];
        }
        for (; s < p.splits; s++) v[0] += p.partial[s * n + at];
        const int64_t i = at / p.b.extent, j = at % p.b.extent;
        am_columns(p, j, b_scale, bias);
        am_finish(p, i, j, v, b_scale, bias);
    }
}

// dz = dy * act'(pre) in the operands' type, or in two values of it (dz_low is
// not NULL), and sums of the unrounded dz over a strip of rows.  8 columns a thread; `across` threads (a power of two) side
// by side, 256 / across rows at a time.  sums: [strips][N].  Bound by memory:
// (16384, 4096) bf16 85 us, 403 MB, 4.7 TB/s; dz in two values 98 us, 537 MB.
template <typename T>
__global__ __launch_bounds__(256) void slope_kernel(wfst_am_linear_backward_args a, T *dz, T *dz_low, float *sums, int across)
{
    __shared__ float part[256][9];
    const int64_t M = a.dy.rows, N = a.dy.cols, ld = am_dz_stride(N);
    const int down = 256 / across, x = threadIdx.x % across, y = threadIdx.x / across;
    const int64_t n = (static_cast<int64_t>(blockIdx.x) * across + x) * 8;
    const int64_t first = M * blockIdx.y / gridDim.y, last = M * (blockIdx.y + 1) / gridDim.y;
    float sum[8] = {};
    if (n < N)
        for (int64_t m = first + y; m < last; m += down) {
            float g[8];
            load_floats(static_cast<const T *>(a.dy.data) + m * a.dy.row_stride + n, N - n, g);
            if (a.activation != WFST_ACT_NONE) {
                float z[8];
                load_floats(static_cast<const T *>(a.pre.data) + m * a.pre.row_stride + n, N - n, z);
#pragma unroll
                for (int e = 0; e < 8; e++) g[e] *= am_slope(z[e], a.activation);
                if (dz) am_store_dz(dz + m * ld + n, dz_low ? dz_low + m * ld + n : nullptr, N - n, g);
            }
#pragma unroll
            for (int e = 0; e < 8; e++) sum[e] += g[e];
        }
    if (!sums) return;
#pragma unroll
    for (int e = 0; e < 8; e++) part[threadIdx.x][e] = sum[e];
    __syncthreads();
    for (int c = threadIdx.x; c < across * 8; c += 256) {
        const int64_t col = static_cast<int64_t>(blockIdx.x) * across * 8 + c;
        if (col >= N) break;
        float t = 0.0f;
        for (int r = 0; r < down; r++) t += part[r * across + c / 8][c % 8];
        sums[blockIdx.y * N + col] = t;
    }
}

template <typename T>
void launch_backward(const wfst_am_linear_backward_args &a, hipStream_t st)
{
    const int64_t N = a.dy.cols;
    const BackwardPlan plan = am_backward_plan(a);
    char *work = static_cast<char *>(a.workspace);
    T *dz = plan.dz_bytes ? reinterpret_cast<T *>(work) : nullptr;
    T *dz_low = dz && plan.dz_parts > 1 ? reinterpret_cast<T *>(work + plan.dz_bytes) : nullptr;
    work += plan.dz_bytes * plan.dz_parts;
    float *sums = a.dbias ? plan.strips > 1 ? reinterpret_cast<float *>(work) : a.dbias : nullptr;
    if (a.dbias || dz) {
        const dim3 grid(static_cast<unsigned>((N + plan.across * 8 - 1) / (plan.across * 8)), static_cast<unsigned>(plan.strips));
        slope_kernel<T><<<grid, 256, 0, st>>>(a, dz, dz_low, sums, plan.across);
        if (sums && plan.strips > 1) am_launch_column_join(sums, plan.strips, N, a.dbias, nullptr, st);
    }
    const char *g = dz ? reinterpret_cast<const char *>(dz) : static_cast<const char *>(a.dy.data);
    const int64_t ld = (dz ? am_dz_stride(N) : a.dy.row_stride) * static_cast<int64_t>(sizeof(T));
    // the column sums are joined before the products' parts take their place
    am_launch_gradient_products<T>(a, plan, g, reinterpret_cast<const char *>(dz_low), ld, reinterpret_cast<float *>(work), st);
}

}  // namespace

void am_launch_join(const AmProduct &p, hipStream_t st)
{
    const int64_t n = (static_cast<int64_t>(p.a.extent) * p.b.extent + 255) / 256;
    join_kernel<<<static_cast<unsigned>(n < 4096 ? n : 4096), 256, 0, st>>>(p);
}

hipError_t am_launch_linear(const wfst_am_linear_args &a, hipStream_t st)
{
    const int64_t el = am_type_bytes(a.x.type);
    AmProduct p{};
    p.a = {static_cast<const char *>(a.x.data), a.x.row_stride * el, static_cast<int32_t>(a.x.rows)};
    p.b = {static_cast<const char *>(a.w.data), a.w.row_stride * el, static_cast<int32_t>(a.w.rows)};
    p.inner = static_cast<int32_t>(a.x.cols);
    p.splits = 1;
    p.a_scale = a.x_scale, p.b_scale = a.w_scale, p.bias = a.bias;
    p.residual = a.residual, p.pre = a.pre, p.out = a.y;
    p.activation = a.activation;
    // Few rows, or tiles for less than half of the chip: a tile waits for memory once a
    // stage, the thin kernel hardly at all ((1, 1024, 6000): 5.1 us against 10.0, (400, 1024, 1024),
    // 112 tiles: 8.8 against 11.1); with more it reads too much ((1500, 512, 640), 240 tiles: 8.8 against 7.7)
    const bool thin = a.x.rows <= 32 || am_tiles(a.x.rows, a.w.rows, 64, 64) <= kComputeUnits / 2;
    const int32_t tile = thin ? 0 : am_plan(p.a, false, p.b, false, p.inner, static_cast<int>(el), 1, false).tile;
    if (a.x.type == WFST_F16) am_product_forward<f16>(p, tile, st);
    else if (a.x.type == WFST_BF16) am_product_forward<bf16>(p, tile, st);
    else am_product_forward<f8>(p, tile, st);
    return hipGetLastError();
}

int64_t am_linear_backward_bytes(const wfst_am_linear_backward_args &a)
{
    const BackwardPlan plan = am_backward_plan(a);
    return plan.dz_bytes * plan.dz_parts + plan.partial_bytes;
}

hipError_t am_launch_linear_backward(const wfst_am_linear_backward_args &a, hipStream_t st)
{
    if (a.dy.type == WFST_F16) launch_backward<f16>(a, st);
    else launch_backward<bf16>(a, st);
    return hipGetLastError();
}

}  // namespace wfd
