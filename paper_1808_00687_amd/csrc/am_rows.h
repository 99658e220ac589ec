// Rows of the acoustic model's row operators: who reads which part, and the
// reductions over a row.
//
// A row belongs to TPR threads (a wave, 256 or 1024), C consecutive columns at
// a time: chunk c is thread c % TPR's.  C is 8 where every matrix has at most 16-bit
// elements and 4 where one has 32-bit ones, so that no access to a matrix is wider
// than 16 bytes and neighbouring lanes' accesses touch.  (Vectors are 32-bit in
// either case; a workgroup reads them once.)  With NV > 0 a thread holds its
// NV chunks in registers, as they are in memory, so a row is read once; with
// NV = 0 the row is too long for that and every pass reads it again.
#pragma once

#include "am_device.h"

namespace wfd {

constexpr int64_t kRowHeld = 32768;   // longest row held in registers

template <int TPR, int NV, int C>
struct RowShape {
    static constexpr int kThreads = TPR < 256 ? 256 : TPR;
    static constexpr int kRows = kThreads / TPR;           // rows a workgroup works on
    static constexpr int kWaves = TPR / 64;                // waves a row
    static constexpr int kTpr = TPR, kNv = NV, kC = C;
    static constexpr int kHeld = NV > 0 ? NV : 1;

    // use(v, column, left) for each of thread t's chunks with a column below cols: `left` columns are left there
    template <typename F>
    __device__ __forceinline__ static void each(int64_t cols, int t, F use)
    {
        if constexpr (NV > 0) {
#pragma unroll
            for (int v = 0; v < NV; v++) {
                const int64_t c = (static_cast<int64_t>(v) * TPR + t) * C;
                if (c < cols) use(v, c, cols - c);
            }
        } else {
            for (int64_t c = static_cast<int64_t>(t) * C; c < cols; c += TPR * C) use(0, c, cols - c);
        }
    }
};

// Calls go(shape) with the shape for rows of D columns.  Its bounds, in us for 8e7
// bf16 values (norm to 8 bits with a residual / loss with gradient / log-likelihoods):
//   1,024 columns: a wave 73 / 85 / 60, 256 threads 87 / 180 / 110
//   2,048: a wave 106 / 109 / 94, 256 threads 112 / 147 / 92
//   4,096: 256 threads 110 / 95 / 93, 1,024 threads 137 / 277 / 156
//   6,000: 256 threads in three chunks 117 / 86 / 94, in four 130 / 142 / 96
//   8,192: 256 threads 108 / 106 / 94, 1,024 threads 112 / 160 / 95
//   16,384: 1,024 threads in two chunks 137 / 101 / 94, in four 300 / 110 / 122
//   20,000: held in four chunks 369 / 97 / 115, read again in each pass 178 / 130 / 136
template <int C, typename F>
void am_row_shape(int64_t D, F go)
{
    constexpr int k = 8 / C;
    if (D <= 512) go(RowShape<64, 1 * k, C>{});
    else if (D <= 1024) go(RowShape<64, 2 * k, C>{});
    else if (D <= 2048) go(RowShape<64, 4 * k, C>{});
    else if (D <= 4096) go(RowShape<256, 2 * k, C>{});
    else if (D <= 6144) go(RowShape<256, 3 * k, C>{});
    else if (D <= 8192) go(RowShape<256, 4 * k, C>{});
    else if (D <= 16384) go(RowShape<1024, 2 * k, C>{});
    else if (D <= kRowHeld) go(RowShape<1024, 4 * k, C>{});
    else go(RowShape<1024, 0, C>{});
}

// The same for the norm's gradients, which hold three matrices and sums besides: a
// chunk a thread (2,048 columns 124 us, a wave 140; 8,192 136, 256 threads 145) but where
// many threads would have none (5,000 bf16 223, 256 threads 131, float32 255 and 273).  Between 1,024 and 1,536
// columns it depends on the type: 1,500 bf16 58, a wave 48, float32 78 and 84.
template <int C, typename F>
void am_row_shape_lean(int64_t D, F go)
{
    constexpr int k = 8 / C;
    if (D > 1024 && D <= 2048) go(RowShape<256, 1 * k, C>{});
    else if (D > 6144 && D <= 8192) go(RowShape<1024, 1 * k, C>{});
    else am_row_shape<C>(D, go);
}

// And for the norm forward, whose rows with their residuals' take twice the registers:
// held up to 16,384 columns ((4000, 20000) bf16 with the residual 206 us, read again 158,
// without 100 and 80, float32 390 and 136; (2441, 32768) 148 and 161, 79 and 72).
template <int C, typename F>
void am_row_shape_norm(int64_t D, F go)
{
    if (D > 16384) go(RowShape<1024, 0, C>{});
    else am_row_shape<C>(D, go);
}

// Workgroups for M rows: at most `most`, about as many as the chip holds at
// once, each with the same number of turns.
template <typename S>
unsigned am_row_blocks(int64_t M, int64_t most)
{
    const int64_t n = (M + S::kRows - 1) / S::kRows, turns = (n + most - 1) / most;
    return static_cast<unsigned>(n ? (n + turns - 1) / turns : 0);
}

// A thread's chunks of one row, held or read when asked for.
template <typename S, typename T>
struct RowPart {
    const T *p;
    Chunk<T, S::kC> held[S::kHeld];

    __device__ __forceinline__ void hold(const T *row, int64_t cols, int t, T fill = static_cast<T>(0.0f))
    {
        p = row;
        if constexpr (S::kNv > 0)
#pragma unroll
            for (int v = 0; v < S::kNv; v++) {
                const int64_t c = (static_cast<int64_t>(v) * S::kTpr + t) * S::kC;
                held[v] = load_chunk<T, S::kC>(row + c, cols - c, fill);
            }
    }
    __device__ __forceinline__ void get(int v, int64_t c, int64_t left, float (&x)[S::kC], float fill = 0.0f) const
    {
        if constexpr (S::kNv > 0) {
#pragma unroll
            for (int e = 0; e < S::kC; e++) x[e] = static_cast<float>(held[v][e]);
        } else {
            load_floats<T, S::kC>(p + c, left, x, fill);
        }
    }
};

// LDS of the reductions.  Two sets, used in turn, so that one barrier a
// reduction is enough: a set is written again only after the other one's barrier.
struct RowScratch {
    float a[2][16], b[2][16];
};

template <typename S>
__device__ __forceinline__ float row_sum(float v, RowScratch &r, int &turn)
{
    v = wave_sum(v);
    if constexpr (S::kWaves == 1) return v;
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) r.a[turn][wave] = v;
    __syncthreads();
    float s = r.a[turn][0];
#pragma unroll
    for (int i = 1; i < S::kWaves; i++) s += r.a[turn][i];
    turn ^= 1;
    return s;
}

// two sums at once
template <typename S>
__device__ __forceinline__ void row_sums(float &u, float &v, RowScratch &r, int &turn)
{
    u = wave_sum(u), v = wave_sum(v);
    if constexpr (S::kWaves == 1) return;
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) r.a[turn][wave] = u, r.b[turn][wave] = v;
    __syncthreads();
    u = r.a[turn][0], v = r.b[turn][0];
#pragma unroll
    for (int i = 1; i < S::kWaves; i++) u += r.a[turn][i], v += r.b[turn][i];
    turn ^= 1;
}

// largest magnitude by its bits: a NaN counts as larger than an infinity
template <typename S>
__device__ __forceinline__ uint32_t row_max_u32(uint32_t v, RowScratch &r, int &turn)
{
    v = wave_max_u32(v);
    if constexpr (S::kWaves == 1) return v;
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) r.a[turn][wave] = __uint_as_float(v);
    __syncthreads();
    uint32_t m = __float_as_uint(r.a[turn][0]);
#pragma unroll
    for (int i = 1; i < S::kWaves; i++) {
        const uint32_t o = __float_as_uint(r.a[turn][i]);
        m = m > o ? m : o;
    }
    turn ^= 1;
    return m;
}

// Column sums over strips of rows: partial[strips][n] -> out[n], in order of the strips (am_norm.hip)
void am_launch_column_join(const float *partial, int64_t strips, int64_t n, float *out, hipStream_t st);

}  // namespace wfd
