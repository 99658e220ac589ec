// Gated layers: y = act(gate) * value, both projections of the same rows, and their gradients.
//
// Forward: one product over the gates' and the values' rows of w, whose epilogue has
// a result's gate and value in one lane (am_tile.h, am_thin.h).
// Backward: dgate = dy * value * act'(gate) and dvalue = dy * act(gate) go to the
// workspace as the rows [dgate dvalue]; dx and dw are then those of one layer with 2 N
// outputs (am_linear.h).
#include "am_linear.h"
#include "am_rows.h"

namespace wfd {
namespace {

// dz = [dgate dvalue] in the operands' type, or in two values of it (dz_low is not
// NULL), and sums of the unrounded dz over a strip of rows.  8 columns of either a
// thread; `across` threads (a power of two) side by side, 256 / across rows at a
// time.  sums: [strips][2 N].  Bound by memory: (16384, 2048) bf16 to two values 86 us, 470 MB, 5.5 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void gated_slope_kernel(wfst_am_gated_backward_args a, T *dz, T *dz_low, float *sums, int across)
{
    __shared__ float part[256][17];
    const int64_t M = a.dy.rows, N = a.dy.cols, ld = am_dz_stride(2 * N);
    const int down = 256 / across, x = threadIdx.x % across, y = threadIdx.x / across;
    const int64_t n = (static_cast<int64_t>(blockIdx.x) * across + x) * 8;
    const int64_t first = M * blockIdx.y / gridDim.y, last = M * (blockIdx.y + 1) / gridDim.y;
    float sum[16] = {};
    if (n < N)
        for (int64_t m = first + y; m < last; m += down) {
            float g[8], z[8], u[8];
            const T *pre = static_cast<const T *>(a.pre.data) + m * a.pre.row_stride + n;
            load_floats(static_cast<const T *>(a.dy.data) + m * a.dy.row_stride + n, N - n, g);
            load_floats(pre, N - n, z);
            load_floats(pre + N, N - n, u);
#pragma unroll
            for (int e = 0; e < 8; e++) {
                float act;
                const float slope = am_slope(z[e], a.activation, &act);
                // the slope (at most 1.13) takes bf16's larger factor: dy * value may be no float32 where dz is one
                const bool by_value = __is_same(T, bf16) && fabsf(u[e]) > fabsf(g[e]);
                u[e] = (by_value ? u[e] : g[e]) * slope * (by_value ? g[e] : u[e]);
                z[e] = g[e] * act;
                sum[e] += u[e];
                sum[8 + e] += z[e];
            }
            if (dz) {
                am_store_dz(dz + m * ld + n, dz_low ? dz_low + m * ld + n : nullptr, N - n, u);
                am_store_dz(dz + m * ld + N + n, dz_low ? dz_low + m * ld + N + n : nullptr, N - n, z);
            }
        }
    if (!sums) return;
#pragma unroll
    for (int e = 0; e < 16; e++) part[threadIdx.x][e] = sum[e];
    __syncthreads();
    for (int c = threadIdx.x; c < across * 16; c += 256) {
        const int half = c / (across * 8), at = c % (across * 8);
        const int64_t col = static_cast<int64_t>(blockIdx.x) * across * 8 + at;
        if (col >= N) continue;
        float t = 0.0f;
        for (int r = 0; r < down; r++) t += part[r * across + at / 8][half * 8 + at % 8];
        sums[blockIdx.y * 2 * N + half * N + col] = t;
    }
}

// the products' arguments: a layer of 2 N outputs
wfst_am_linear_backward_args as_layer(const wfst_am_gated_backward_args &a)
{
    wfst_am_linear_backward_args b{};
    b.dy = {nullptr, a.dy.rows, 2 * a.dy.cols, 2 * a.dy.cols, a.dy.type, 0};
    b.x = a.x, b.w = a.w, b.dx = a.dx, b.dw = a.dw, b.dbias = a.dbias;
    return b;
}

// A row a thread where there are few: its loads, activation and stores are a chain of about 2 us ((833, 1280) with dbias
// and a small dx 26 us, with four 30; 50 rows of 512 18 and 23).
BackwardPlan plan_of(const wfst_am_gated_backward_args &a) { return am_backward_plan(as_layer(a), true, a.round_dz ? 1 : 2, a.dy.cols, 1); }

template <typename T>
void launch_backward(const wfst_am_gated_backward_args &a, hipStream_t st)
{
    const int64_t N = a.dy.cols;
    const BackwardPlan plan = plan_of(a);
    char *work = static_cast<char *>(a.workspace);
    T *dz = plan.dz_bytes ? reinterpret_cast<T *>(work) : nullptr;
    T *dz_low = dz && plan.dz_parts > 1 ? reinterpret_cast<T *>(work + plan.dz_bytes) : nullptr;
    work += plan.dz_bytes * plan.dz_parts;
    float *sums = a.dbias ? plan.strips > 1 ? reinterpret_cast<float *>(work) : a.dbias : nullptr;
    if (a.dbias || dz) {
        const dim3 grid(static_cast<unsigned>((N + plan.across * 8 - 1) / (plan.across * 8)), static_cast<unsigned>(plan.strips));
        gated_slope_kernel<T><<<grid, 256, 0, st>>>(a, dz, dz_low, sums, plan.across);
        if (sums && plan.strips > 1) am_launch_column_join(sums, plan.strips, 2 * N, a.dbias, nullptr, st);
    }
    // the column sums are joined before the products' parts take their place
    am_launch_gradient_products<T>(as_layer(a), plan, reinterpret_cast<const char *>(dz), reinterpret_cast<const char *>(dz_low),
                                   am_dz_stride(2 * N) * static_cast<int64_t>(sizeof(T)), reinterpret_cast<float *>(work), st);
}

}  // namespace

hipError_t am_launch_gated(const wfst_am_gated_args &a, hipStream_t st)
{
    const int64_t el = am_type_bytes(a.x.type), M = a.x.rows, N = a.y.cols;
    AmProduct p{};
    p.a = {static_cast<const char *>(a.x.data), a.x.row_stride * el, static_cast<int32_t>(M)};
    p.b = {static_cast<const char *>(a.w.data), a.w.row_stride * el, static_cast<int32_t>(N)};
    p.inner = static_cast<int32_t>(a.x.cols);
    p.splits = 1;
    p.a_scale = a.x_scale, p.b_scale = a.w_scale, p.bias = a.bias;
    p.out = a.y;
    p.pre = a.pre;
    if (a.pre.data) {
        p.pre.cols = N;
        p.value_pre = p.pre;
        p.value_pre.data = static_cast<char *>(a.pre.data) + N * am_type_bytes(a.pre.type);
    }
    p.activation = a.activation;
    // as a layer's products (am_linear.hip), of 2 N outputs
    const bool thin = M <= 32 || am_tiles(M, 2 * N, 64, 64) <= kComputeUnits / 2;
    const int32_t tile = thin ? 0 : am_plan(M, 2 * N, p.inner, false, am_gated_direct(p.a, p.b, p.inner, static_cast<int>(el)), true).tile;
    if (a.x.type == WFST_F16) am_product_gated<f16>(p, tile, st);
    else if (a.x.type == WFST_BF16) am_product_gated<bf16>(p, tile, st);
    else am_product_gated<f8>(p, tile, st);
    return hipGetLastError();
}

int64_t am_gated_backward_bytes(const wfst_am_gated_backward_args &a)
{
    const BackwardPlan plan = plan_of(a);
    return plan.dz_bytes * plan.dz_parts + plan.partial_bytes;
}

hipError_t am_launch_gated_backward(const wfst_am_gated_backward_args &a, hipStream_t st)
{
    if (a.dy.type == WFST_F16) launch_backward<f16>(a, st);
    else launch_backward<bf16>(a, st);
    return hipGetLastError();
}

}  // namespace wfd
