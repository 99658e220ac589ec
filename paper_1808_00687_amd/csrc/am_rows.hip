// Row operators of the acoustic model: root-mean-square norm (forward and
// backward), distillation loss, log-likelihood rows.  One workgroup a row.
#include "am_device.h"

namespace wfd {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

// Reductions over the workgroup, in a fixed order; every thread gets the result.
__device__ float block_sum(float v)
{
    __shared__ float part[kWaves];
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    float t = part[0];
    for (int i = 1; i < kWaves; i++) t += part[i];
    return t;
}

__device__ float block_max(float v)
{
    __shared__ float part[kWaves];
    v = wave_max(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    float t = part[0];
    for (int i = 1; i < kWaves; i++) t = fmaxf(t, part[i]);
    return t;
}

__device__ uint32_t block_max_u32(uint32_t v)
{
    __shared__ uint32_t part[kWaves];
    v = wave_max_u32(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    uint32_t t = part[0];
    for (int i = 1; i < kWaves; i++) t = max(t, part[i]);
    return t;
}

// --------------------------------------------------------------------------
// norm
// --------------------------------------------------------------------------

template <typename T, typename Y>
__global__ __launch_bounds__(kThreads) void norm_kernel(wfst_am_norm_args a)
{
    const int64_t M = a.x.rows, D = a.x.cols;
    for (int64_t m = blockIdx.x; m < M; m += gridDim.x) {
        const T *x = static_cast<const T *>(a.x.data) + m * a.x.row_stride;
        const T *r = a.residual.data ? static_cast<const T *>(a.residual.data) + m * a.residual.row_stride : nullptr;
        T *s = a.sum.data ? static_cast<T *>(a.sum.data) + m * a.sum.row_stride : nullptr;
        Y *y = static_cast<Y *>(a.y.data) + m * a.y.row_stride;
        float ss = 0.0f;
        for (int64_t d = threadIdx.x; d < D; d += kThreads) {
            float v = to_f32(x[d]) + (r ? to_f32(r[d]) : 0.0f);
            ss = fmaf(v, v, ss);
        }
        const float rho = 1.0f / sqrtf(block_sum(ss) / static_cast<float>(D) + a.eps);
        float inv = 1.0f;
        if constexpr (sizeof(Y) == 1) {
            // the largest magnitude by its bits: a NaN counts as larger than an infinity
            uint32_t top = 0;
            for (int64_t d = threadIdx.x; d < D; d += kThreads) {
                float v = (to_f32(x[d]) + (r ? to_f32(r[d]) : 0.0f)) * rho * (a.gain ? a.gain[d] : 1.0f);
                top = max(top, __float_as_uint(v) & 0x7FFFFFFFu);
            }
            float scale = __uint_as_float(block_max_u32(top)) / kE4m3Max;
            scale = scale < 1.17549435e-38f ? 1.17549435e-38f : scale;
            inv = 1.0f / scale;
            if (threadIdx.x == 0) a.y_scale[m] = scale;
        }
        for (int64_t d = threadIdx.x; d < D; d += kThreads) {
            float v = to_f32(x[d]) + (r ? to_f32(r[d]) : 0.0f);
            if (s) s[d] = from_f32<T>(v);
            y[d] = from_f32<Y>(v * rho * (a.gain ? a.gain[d] : 1.0f) * inv);
        }
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void norm_backward_kernel(wfst_am_norm_backward_args a)
{
    const int64_t M = a.s.rows, D = a.s.cols;
    float *rhos = static_cast<float *>(a.workspace);
    for (int64_t m = blockIdx.x; m < M; m += gridDim.x) {
        const T *s = static_cast<const T *>(a.s.data) + m * a.s.row_stride;
        const T *dy = static_cast<const T *>(a.dy.data) + m * a.dy.row_stride;
        float ss = 0.0f, us = 0.0f;
        for (int64_t d = threadIdx.x; d < D; d += kThreads) {
            float v = to_f32(s[d]);
            ss = fmaf(v, v, ss);
            us = fmaf(to_f32(dy[d]) * (a.gain ? a.gain[d] : 1.0f), v, us);
        }
        const float rho = 1.0f / sqrtf(block_sum(ss) / static_cast<float>(D) + a.eps);
        const float c = rho * rho * (block_sum(us) / static_cast<float>(D));
        if (threadIdx.x == 0) rhos[m] = rho;
        if (!a.dx.data) continue;
        const T *ds = a.dsum.data ? static_cast<const T *>(a.dsum.data) + m * a.dsum.row_stride : nullptr;
        T *dx = static_cast<T *>(a.dx.data) + m * a.dx.row_stride;
        for (int64_t d = threadIdx.x; d < D; d += kThreads) {
            float u = to_f32(dy[d]) * (a.gain ? a.gain[d] : 1.0f);
            float g = rho * (u - to_f32(s[d]) * c);
            dx[d] = from_f32<T>(g + (ds ? to_f32(ds[d]) : 0.0f));
        }
    }
}

// gradient of the gain, one thread a column; runs before dx may overwrite dy
template <typename T>
__global__ __launch_bounds__(kThreads) void norm_dgain_kernel(wfst_am_norm_backward_args a)
{
    const int64_t M = a.s.rows, D = a.s.cols;
    const int64_t d = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    if (d >= D) return;
    const float *rhos = static_cast<const float *>(a.workspace);
    const T *s = static_cast<const T *>(a.s.data) + d;
    const T *dy = static_cast<const T *>(a.dy.data) + d;
    float t = 0.0f;
    for (int64_t m = 0; m < M; m++)
        t += to_f32(dy[m * a.dy.row_stride]) * to_f32(s[m * a.s.row_stride]) * rhos[m];
    a.dgain[d] = t;
}

// --------------------------------------------------------------------------
// softmax statistics of a row
// --------------------------------------------------------------------------

// log sum exp of x / temperature
template <typename T>
__device__ float row_lse(const T *x, int64_t L, float inv_t)
{
    float top = -INFINITY;
    for (int64_t i = threadIdx.x; i < L; i += kThreads) top = fmaxf(top, to_f32(x[i]) * inv_t);
    top = block_max(top);
    const float shift = top == -INFINITY ? 0.0f : top;
    float t = 0.0f;
    for (int64_t i = threadIdx.x; i < L; i += kThreads) t += expf(to_f32(x[i]) * inv_t - shift);
    return shift + logf(block_sum(t));
}

template <typename T>
__global__ __launch_bounds__(kThreads) void loglikes_kernel(wfst_am_loglikes_args a)
{
    const int64_t M = a.logits.rows, L = a.logits.cols;
    for (int64_t m = blockIdx.x; m < M; m += gridDim.x) {
        const T *x = static_cast<const T *>(a.logits.data) + m * a.logits.row_stride;
        float *ll = static_cast<float *>(a.ll.data) + m * a.ll.row_stride;
        const float lse = row_lse(x, L, 1.0f);
        for (int64_t i = threadIdx.x; i < L; i += kThreads) {
            float v = to_f32(x[i]), p = a.log_prior ? a.log_prior[i] : 0.0f;
            ll[i] = v == -INFINITY || p == -INFINITY ? -INFINITY : a.scale * ((v - lse) - p);
        }
    }
}

// --------------------------------------------------------------------------
// distillation
// --------------------------------------------------------------------------

__device__ __forceinline__ float load_any(const wfst_matrix &m, int64_t r, int64_t c)
{
    const int64_t at = r * m.row_stride + c;
    return m.type == WFST_F32   ? static_cast<const float *>(m.data)[at]
           : m.type == WFST_F16 ? to_f32(static_cast<const f16 *>(m.data)[at])
                                : to_f32(static_cast<const bf16 *>(m.data)[at]);
}

template <typename T, bool kBackward>
__global__ __launch_bounds__(kThreads) void distill_kernel(wfst_am_distill_args a)
{
    __shared__ int32_t unit[WFST_AM_MAX_TOP];   // -1: not used
    __shared__ float share[WFST_AM_MAX_TOP];
    const int64_t M = a.logits.rows, L = a.logits.cols;
    const int k = static_cast<int>(a.top_logit.cols), j = threadIdx.x;
    const float t = a.temperature, inv_t = 1.0f / t;
    for (int64_t m = blockIdx.x; m < M; m += gridDim.x) {
        const T *x = static_cast<const T *>(a.logits.data) + m * a.logits.row_stride;
        T *d = a.dlogits.data ? static_cast<T *>(a.dlogits.data) + m * a.dlogits.row_stride : nullptr;
        const float w = a.weight ? a.weight[m] : 1.0f;
        int32_t u = -1;
        float top = -INFINITY;
        if (j < k) {
            u = a.top_index[m * k + j];
            top = load_any(a.top_logit, m, j) * inv_t;
            if (u < 0 || u >= L || top == -INFINITY) u = -1, top = -INFINITY;
        }
        const float best = block_max(top);
        const float e = u >= 0 ? expf(top - best) : 0.0f;
        const float z = block_sum(e);
        const bool used = block_max(u >= 0 ? 1.0f : 0.0f) > 0.0f;
        float lse = 0.0f;
        if constexpr (kBackward) lse = a.lse[m];
        else if ((w != 0.0f && used) || a.lse) lse = row_lse(x, L, inv_t);
        if (!kBackward && a.lse && j == 0) a.lse[m] = lse;
        if (w == 0.0f || !used) {
            if (!kBackward && a.loss && j == 0) a.loss[m] = 0.0f;
            if (d)
                for (int64_t i = j; i < L; i += kThreads) d[i] = from_f32<T>(0.0f);
            continue;
        }
        const float p = u >= 0 ? e / z : 0.0f;
        const float log_q = u >= 0 ? to_f32(x[u]) * inv_t - lse : 0.0f;
        if (!kBackward && a.loss) {
            // a masked unit whose share has underflowed is worth nothing
            const float term = p == 0.0f ? 0.0f : p * ((top - best - logf(z)) - log_q);
            const float sum = block_sum(term);
            if (j == 0) a.loss[m] = w * t * t * sum;
        }
        if (!d) continue;
        unit[j] = u;
        share[j] = p;
        __syncthreads();   // also: every x[u] is read before dlogits may overwrite it
        for (int64_t i = j; i < L; i += kThreads) d[i] = from_f32<T>(w * t * expf(to_f32(x[i]) * inv_t - lse));
        __syncthreads();
        bool first = u >= 0;
        float mass = 0.0f;
        for (int i = 0; i < k && u >= 0; i++)
            if (unit[i] == u) {
                if (i < j) first = false;
                mass += share[i];
            }
        if (first) d[u] = from_f32<T>(w * t * (expf(log_q) - mass));
        __syncthreads();
    }
}

// workgroups for M rows
unsigned blocks_for(int64_t M) { return static_cast<unsigned>(M < (1 << 20) ? M : 1 << 20); }

template <typename T>
void launch_norm(const wfst_am_norm_args &a, hipStream_t st)
{
    const unsigned g = blocks_for(a.x.rows);
    if (a.y.type == WFST_F32) norm_kernel<T, float><<<g, kThreads, 0, st>>>(a);
    else if (a.y.type == WFST_F16) norm_kernel<T, f16><<<g, kThreads, 0, st>>>(a);
    else if (a.y.type == WFST_BF16) norm_kernel<T, bf16><<<g, kThreads, 0, st>>>(a);
    else norm_kernel<T, f8><<<g, kThreads, 0, st>>>(a);
}

template <typename T>
void launch_norm_backward(wfst_am_norm_backward_args a, hipStream_t st)
{
    const wfst_matrix dx = a.dx;
    if (a.dgain) {
        a.dx.data = nullptr;
        if (a.s.rows) norm_backward_kernel<T><<<blocks_for(a.s.rows), kThreads, 0, st>>>(a);
        norm_dgain_kernel<T><<<static_cast<unsigned>((a.s.cols + kThreads - 1) / kThreads), kThreads, 0, st>>>(a);
        a.dx = dx;
    }
    if (dx.data && a.s.rows) norm_backward_kernel<T><<<blocks_for(a.s.rows), kThreads, 0, st>>>(a);
}

template <typename T>
void launch_distill(const wfst_am_distill_args &a, bool backward, hipStream_t st)
{
    const unsigned g = blocks_for(a.logits.rows);
    if (backward) distill_kernel<T, true><<<g, kThreads, 0, st>>>(a);
    else distill_kernel<T, false><<<g, kThreads, 0, st>>>(a);
}

}  // namespace

hipError_t am_launch_norm(const wfst_am_norm_args &a, hipStream_t st)
{
    if (a.x.type == WFST_F32) launch_norm<float>(a, st);
    else if (a.x.type == WFST_F16) launch_norm<f16>(a, st);
    else launch_norm<bf16>(a, st);
    return hipGetLastError();
}

int64_t am_norm_backward_bytes(const wfst_am_norm_backward_args &a)
{
    return ((a.s.rows * 4 + 255) & ~int64_t{255});
}

hipError_t am_launch_norm_backward(const wfst_am_norm_backward_args &a, hipStream_t st)
{
    if (a.s.type == WFST_F32) launch_norm_backward<float>(a, st);
    else if (a.s.type == WFST_F16) launch_norm_backward<f16>(a, st);
    else launch_norm_backward<bf16>(a, st);
    return hipGetLastError();
}

hipError_t am_launch_distill(const wfst_am_distill_args &a, bool backward, hipStream_t st)
{
    if (a.logits.type == WFST_F32) launch_distill<float>(a, backward, st);
    else if (a.logits.type == WFST_F16) launch_distill<f16>(a, backward, st);
    else launch_distill<bf16>(a, backward, st);
    return hipGetLastError();
}

hipError_t am_launch_loglikes(const wfst_am_loglikes_args &a, hipStream_t st)
{
    const unsigned g = blocks_for(a.logits.rows);
    if (a.logits.type == WFST_F32) loglikes_kernel<float><<<g, kThreads, 0, st>>>(a);
    else if (a.logits.type == WFST_F16) loglikes_kernel<f16><<<g, kThreads, 0, st>>>(a);
    else loglikes_kernel<bf16><<<g, kThreads, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace wfd
