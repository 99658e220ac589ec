// Softmax statistics of a row, for the operators over units.
#pragma once

#include "am_rows.h"

namespace wfd {

template <typename T>
__device__ __forceinline__ const T *row(const wfst_matrix &m, int64_t r)
{
    return static_cast<const T *>(m.data) + r * m.row_stride;
}

constexpr float kLog2e = 1.44269504f;
constexpr float kFloatMax = 3.40282347e38f;

// A row's softmax statistics.  The maximum is subtracted before anything is scaled,
// so they do not change with an offset of the row, however large: its exponent is 0.
struct RowStat {
    float top;    // largest x; 0 for a row of -inf
    float own;    // largest x of the thread's wave, likewise: what `keep` got is relative to it
    float sum;    // of e^((x - top) / temperature)
};

// get(v, column, left, x): a chunk, -inf beyond the row.  c: log2(e) / temperature.
// keep(v, e): e^((x - own) / temperature) of the chunk.
template <typename S, typename G, typename K>
__device__ __forceinline__ RowStat row_stat(int64_t cols, int t, float c, G get, K keep, RowScratch &r, int &turn)
{
    float top = -INFINITY;
    S::each(cols, t, [&](int v, int64_t at, int64_t left) {
        float x[S::kC];
        get(v, at, left, x);
#pragma unroll
        for (int e = 0; e < S::kC; e++) top = fmaxf(top, x[e]);
    });
    top = wave_max(top);
    RowStat o;
    o.own = top == -INFINITY ? 0.0f : top;
    float s = 0.0f;
    S::each(cols, t, [&](int v, int64_t at, int64_t left) {
        float x[S::kC];
        get(v, at, left, x);
#pragma unroll
        for (int e = 0; e < S::kC; e++) {
            x[e] = __builtin_amdgcn_exp2f((x[e] - o.own) * c);
            s += x[e];
        }
        keep(v, x);
    });
    s = wave_sum(s);
    if constexpr (S::kWaves > 1) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) r.a[turn][wave] = top, r.b[turn][wave] = s;
        __syncthreads();
        top = r.a[turn][0];
#pragma unroll
        for (int i = 1; i < S::kWaves; i++) top = fmaxf(top, r.a[turn][i]);
        o.top = top == -INFINITY ? 0.0f : top;
        s = 0.0f;
#pragma unroll
        for (int i = 0; i < S::kWaves; i++)   // a wave of -inf has sum 0
            s += r.a[turn][i] == -INFINITY ? r.b[turn][i] : r.b[turn][i] * __builtin_amdgcn_exp2f((r.a[turn][i] - o.top) * c);
        turn ^= 1;
    } else {
        o.top = o.own;
    }
    o.sum = s;
    return o;
}

// x / temperature; of a finite x never an infinity (a mask's lowest value, a temperature below 1)
__device__ __forceinline__ float tempered(float x, float inv_t)
{
    const float y = x * inv_t;
    return fabsf(x) <= kFloatMax ? fminf(fmaxf(y, -kFloatMax), kFloatMax) : y;
}

// log sum exp of x / temperature; -inf for a row of -inf
__device__ __forceinline__ float lse_of(const RowStat &s, float inv_t) { return tempered(s.top, inv_t) + logf(s.sum); }

// Workgroups at most.  Loss and gradient of (16384, 6000): 2, 3, 4, 5, 6 and 8 a CU take 151,
// 117, 99, 127, 116 and 101 us; log-likelihoods of (53274, 6000): 2, 4, 8 and 16 359, 376, 376
// and 370, of (4000, 20000) 113, 117, 122 and 138.  Short rows would rather have more (loss and
// gradient of (53274, 80): 4 71, 16 59).
constexpr int64_t kSoftmaxBlocks = 256 * 4;

}  // namespace wfd
