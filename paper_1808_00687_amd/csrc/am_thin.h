// Matrix products with few rows or few tiles (k-contiguous operands), where a
// tile would wait for memory once a stage: nothing is staged.
//
// A workgroup of eight waves computes TI x TJ fragments of 16 x 16; the waves
// take consecutive parts of k, load their fragments from memory straight into
// matrix-core operands with many loads under way, and their sums are added
// through LDS, in the order of the waves.  Loads need no alignment.  b is read
// once for every TI * 16 rows of a, which is once where there are no more.
//
// Bound by latency and by what a CU takes in.  (1, 1024, 6000) bf16: 5.2 us, 12.3 MB
// (2.4 us at the copy's rate); (200, 2048, 512): 7.9 us, in 64 x 64 tiles 18.
#pragma once

#include "am_tile.h"

namespace wfd {

constexpr int kThinWaves = 8;

// 16 bytes of row `row` of o from value k on, zeros from `end` on
template <typename E>
__device__ __forceinline__ i32x4 am_thin_load(const AmOperand &o, int64_t row, int32_t k, int32_t end)
{
    constexpr int kEl = sizeof(E), kWide = 16 / kEl;
    const AM_GLOBAL char *p = (const AM_GLOBAL char *)o.data + row * o.ld + static_cast<int64_t>(k) * kEl;
    if (k + kWide <= end) return *(const AM_GLOBAL i32x4_any *)p;
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < kWide; e++)
        if (k + e < end) {
            uint32_t t;
            if constexpr (kEl == 2) t = ((const AM_GLOBAL uint16_t *)p)[e];
            else t = ((const AM_GLOBAL uint8_t *)p)[e];
            w[e * kEl / 4] |= t << (e * kEl % 4 * 8);
        }
    return i32x4{static_cast<int>(w[0]), static_cast<int>(w[1]), static_cast<int>(w[2]), static_cast<int>(w[3])};
}

template <typename E, int TI, int TJ>
__global__ __launch_bounds__(kThinWaves * 64, 2) void am_thin_kernel(AmProduct p)
{
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int kWide = 16 / static_cast<int>(sizeof(E)), kStep = 4 * kWide;   // values of k in a fragment's row
    constexpr int kUnroll = TI + TJ <= 2 ? 8 : TI + TJ <= 3 ? 4 : 2;           // steps under way
    constexpr int kCols = TJ * 16, kRows = TI * 16, kValues = kRows * kCols;
    constexpr int kOwn = kValues <= kThinWaves * 64 ? 1 : kValues / (kThinWaves * 64);   // results a thread finishes
    __shared__ float part[kThinWaves][kRows][kCols + 4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, s = lane & 15;
    const int64_t tiles_j = (static_cast<int64_t>(p.b.extent) + kCols - 1) / kCols;
    const int64_t block = p.first + blockIdx.x, i0 = block / tiles_j * kRows, j0 = block % tiles_j * kCols;

    int64_t row_a[TI], row_b[TJ];   // past the end: the last row again, whose results are not stored
    am_each<TI>([&](auto f) { row_a[f] = i0 + f * 16 + s < p.a.extent ? i0 + f * 16 + s : p.a.extent - 1; });
    am_each<TJ>([&](auto f) { row_b[f] = j0 + f * 16 + s < p.b.extent ? j0 + f * 16 + s : p.b.extent - 1; });
    const int32_t steps = (p.inner + kStep - 1) / kStep;
    const int32_t s_first = static_cast<int32_t>(static_cast<int64_t>(steps) * wave / kThinWaves);
    const int32_t s_last = static_cast<int32_t>(static_cast<int64_t>(steps) * (wave + 1) / kThinWaves);

    using C = std::conditional_t<sizeof(E) == 1, bf16, E>;
    f32x4 acc[TI][TJ];
    am_each<TI>([&](auto f) { am_each<TJ>([&](auto h) { acc[f][h] = f32x4{0.0f, 0.0f, 0.0f, 0.0f}; }); });
    for (int32_t t = s_first; t < s_last; t += kUnroll) {
        i32x4 x[kUnroll][TI], y[kUnroll][TJ];
        am_each<kUnroll>([&](auto u) {
            const int32_t k = (t + u) * kStep + g * kWide;
            if (t + u < s_last) {
                am_each<TJ>([&](auto h) { y[u][h] = am_thin_load<E>(p.b, row_b[h], k, p.inner); });
                am_each<TI>([&](auto f) { x[u][f] = am_thin_load<E>(p.a, row_a[f], k, p.inner); });
            } else {   // past the wave's part
                am_each<TJ>([&](auto h) { y[u][h] = i32x4{0, 0, 0, 0}; });
                am_each<TI>([&](auto f) { x[u][f] = i32x4{0, 0, 0, 0}; });
            }
        });
        am_each<kUnroll>([&](auto u) {
            if constexpr (sizeof(E) == 1) {
                i32x4 y_lo[TJ], y_hi[TJ];
                am_each<TJ>([&](auto h) { am_widen(y[u][h], y_lo[h], y_hi[h]); });
                am_each<TI>([&](auto f) {
                    i32x4 lo, hi;
                    am_widen(x[u][f], lo, hi);
                    am_each<TJ>([&](auto h) {
                        acc[f][h] = am_mfma<C>(y_lo[h], lo, acc[f][h]);
                        acc[f][h] = am_mfma<C>(y_hi[h], hi, acc[f][h]);
                    });
                });
            } else {
                am_each<TI>([&](auto f) { am_each<TJ>([&](auto h) { acc[f][h] = am_mfma<C>(y[u][h], x[u][f], acc[f][h]); }); });
            }
        });
    }
    am_each<TI>([&](auto f) {
        am_each<TJ>([&](auto h) { *reinterpret_cast<f32x4 *>(&part[wave][f * 16 + s][h * 16 + g * 4]) = acc[f][h]; });
    });
    __syncthreads();
    const int at = threadIdx.x * kOwn, ri = at / kCols, rj = at % kCols;
    const int64_t i = i0 + ri, j = j0 + rj;
    if (at >= kValues || i >= p.a.extent || j >= p.b.extent) return;
    float v[kOwn], b_scale[kOwn], bias[kOwn];
    am_columns(p, j, b_scale, bias);
#pragma unroll
    for (int e = 0; e < kOwn; e++) {
        v[e] = part[0][ri][rj + e];
#pragma unroll
        for (int w = 1; w < kThinWaves; w++) v[e] += part[w][ri][rj + e];
    }
    am_finish(p, i, j, v, b_scale, bias);
#endif
}

template <typename E, int TI, int TJ>
void am_launch_thin(const AmProduct &p, hipStream_t st)
{
    am_in_launches(am_tiles(p.a.extent, p.b.extent, TI * 16, TJ * 16), [&](uint32_t first, uint32_t blocks) {
        AmProduct part = p;
        part.first = first;
        am_thin_kernel<E, TI, TJ><<<blocks, kThinWaves * 64, 0, st>>>(part);
    });
}

// The fragments of a workgroup: a CU takes in about 45 bytes a nanosecond
// whatever the shape (measured), so the best shape is the one whose busiest CU has
// the fewest rows of k to read.  (833, 2048, 80): 4 x 2 on 42 CUs 14.0 us, 2 x 1
// on 135 8.1.
template <typename E>
void am_thin(const AmProduct &p, hipStream_t st)
{
    const auto rows = [&](int ti, int tj) {
        return (am_tiles(p.a.extent, p.b.extent, ti * 16, tj * 16) + kComputeUnits - 1) / kComputeUnits * (ti + tj);
    };
    const int64_t r11 = rows(1, 1), r21 = rows(2, 1), r22 = rows(2, 2), r42 = rows(4, 2);
    if (r42 <= r22 && r42 <= r21 && r42 <= r11) am_launch_thin<E, 4, 2>(p, st);
    else if (r22 <= r21 && r22 <= r11) am_launch_thin<E, 2, 2>(p, st);
    else if (r21 <= r11) am_launch_thin<E, 2, 1>(p, st);
    else am_launch_thin<E, 1, 1>(p, st);
}

}  // namespace wfd
