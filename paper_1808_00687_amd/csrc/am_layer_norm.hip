// Layer norm of rows: forward (residual's addition, 8-bit output) and backward.
//
// Both are bound by memory: a row is read once into registers, its statistics
// are reduced there, and it is written from there.  The mean is taken first;
// the differences from it give the variance and, summed, what rounding left in
// the mean (m0 + c is the mean, to the last bits of the differences and not of
// the values).  A workgroup takes several rows in turn, so gain and bias stay in
// registers, and in the backward pass their gradients are summed there over the
// rows of a workgroup; workgroups' sums are joined by a second small kernel in a
// fixed order.
//
// (53274, 1024) bf16 with the residual to e4m3: 76 us, 382 MB, 5.0 TB/s (a large copy
// reaches 5.0); backward of (16384, 2048) bf16 with dsum: 48 us and 5 of the join, 268 MB.
#include <type_traits>

#include "am_rows.h"

namespace wfd {
namespace {

// N sums over a row's threads.  Two sets of LDS, used in turn, so one barrier is enough.
template <int N>
struct SumScratch {
    float a[2][N][16];
};

template <typename S, int N, int K>
__device__ __forceinline__ void row_sums(float (&v)[K], SumScratch<N> &r, int &turn)
{
    static_assert(K <= N, "");
#pragma unroll
    for (int k = 0; k < K; k++) v[k] = wave_sum<S::kLanes>(v[k]);
    if constexpr (S::kWaves <= 1) return;
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int k = 0; k < K; k++) r.a[turn][k][wave] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; k++) {
        v[k] = r.a[turn][k][0];
#pragma unroll
        for (int i = 1; i < S::kWaves; i++) v[k] += r.a[turn][k][i];
    }
    turn ^= 1;
}

// A thread's chunks of one row of a matrix, as RowPart's, but threads past the row's end go
// through nothing ((52429, 1280) bf16 gradients with dsum 119 us, 172 otherwise; (104858, 640)
// 131 and 170), and a chunk of 8 over it is the row's last 8 values, moved to their places: one
// load in place of seven ((23141, 2900) 168 and 227).
template <typename S, typename T>
struct Part {
    using V = Chunk<T, S::kC>;
    using Bits = std::conditional_t<sizeof(T) * S::kC == 16, unsigned __int128, uint64_t>;
    static_assert(sizeof(V) == sizeof(Bits), "");
    static constexpr bool kMoved = S::kC == 8;
    const T *p;
    V held[S::kHeld];

    __device__ __forceinline__ void hold(const T *row, int64_t cols, int t)
    {
        p = row;
        if constexpr (S::kNv > 0)
#pragma unroll
            for (int v = 0; v < S::kNv; v++) {
                const int64_t c = (static_cast<int64_t>(v) * S::kTpr + t) * S::kC, left = cols - c;
                held[v] = V{};
                if (left >= S::kC) {
                    held[v] = *(const AM_GLOBAL V *)(row + c);
                } else if (left > 0) {
                    if (kMoved && c > 0) {
                        const V u = *(const AM_GLOBAL V *)(row + (cols - S::kC));
                        held[v] = __builtin_bit_cast(V, __builtin_bit_cast(Bits, u) >> static_cast<int>((S::kC - left) * static_cast<int64_t>(sizeof(T)) * 8));
                    } else {
                        held[v] = load_chunk<T, S::kC>(row + c, left, static_cast<T>(0.0f));
                    }
                }
            }
    }
    __device__ __forceinline__ void get(int v, int64_t c, int64_t left, float (&x)[S::kC]) const
    {
        if constexpr (S::kNv > 0) {
#pragma unroll
            for (int e = 0; e < S::kC; e++) x[e] = static_cast<float>(held[v][e]);
        } else {
            load_floats<T, S::kC>(p + c, left, x);
        }
    }
};

// A row's mean is m0 + c; rho is the reciprocal of its standard deviation.
struct Moments {
    float m0, c, rho;

    __device__ __forceinline__ float unit(float s) const { return ((s - m0) - c) * rho; }
    // from the sums of the differences from m0 and of their squares over D values
    __device__ __forceinline__ void set(float sd, float sdd, float D, float eps)
    {
        c = sd / D;
        const float var = sdd / D - c * c;   // c is a rounding: nothing cancels
        rho = 1.0f / sqrtf((var < 0.0f ? 0.0f : var) + eps);
    }
};

template <typename T, typename S, bool k8Bits>
__global__ __launch_bounds__(S::kThreads) void layer_norm_kernel(wfst_am_layer_norm_args a)
{
    __shared__ SumScratch<2> sums;
    __shared__ RowScratch scratch;
    int turn = 0, turn8 = 0;
    const int64_t M = a.x.rows, D = a.x.cols, step = static_cast<int64_t>(gridDim.x) * S::kRows;
    const int t = threadIdx.x % S::kTpr;
    RowPart<S, float> gain, bias;
    if (a.gain) gain.hold(a.gain, D, t);
    if (a.bias) bias.hold(a.bias, D, t);
    Part<S, T> x, r, x_next, r_next;
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
        float total[1] = {0.0f};
        S::each(D, t, [&](int v, int64_t c, int64_t left) {
            float s[S::kC];
            sum_of(v, c, left, s);
#pragma unroll
            for (int e = 0; e < S::kC; e++) total[0] += s[e];
        });
        row_sums<S>(total, sums, turn);
        Moments mo;
        mo.m0 = total[0] / static_cast<float>(D);
        float both[2] = {0.0f, 0.0f};
        S::each(D, t, [&](int v, int64_t c, int64_t left) {
            float s[S::kC];
            sum_of(v, c, left, s);
#pragma unroll
            for (int e = 0; e < S::kC; e++) {
                const float d = e < left ? s[e] - mo.m0 : 0.0f;
                both[0] += d;
                both[1] = fmaf(d, d, both[1]);
            }
        });
        row_sums<S>(both, sums, turn);
        mo.set(both[0], both[1], static_cast<float>(D), a.eps);
        const auto value_of = [&](int v, int64_t c, int64_t left, float (&s)[S::kC]) {
#pragma unroll
            for (int e = 0; e < S::kC; e++) s[e] = mo.unit(s[e]);
            float g[S::kC];
            if (a.gain) {
                gain.get(v, c, left, g);
#pragma unroll
                for (int e = 0; e < S::kC; e++) s[e] *= g[e];
            }
            if (a.bias) {
                bias.get(v, c, left, g);
#pragma unroll
                for (int e = 0; e < S::kC; e++) s[e] += g[e];
            }
        };
        E4m3Quotient by;
        if constexpr (k8Bits) {
            uint32_t top = 0;
            S::each(D, t, [&](int v, int64_t c, int64_t left) {
                float s[S::kC];
                sum_of(v, c, left, s);
                value_of(v, c, left, s);
#pragma unroll
                for (int e = 0; e < S::kC; e++) {
                    const uint32_t b = __float_as_uint(s[e]) & 0x7FFFFFFFu;
                    top = e < left && b > top ? b : top;
                }
            });
            by.template set<(S::kWaves > 0)>(row_max_u32<S>(top, scratch, turn8));
            if (t == 0) a.y_scale[m] = by.scale;
        }
        S::each(D, t, [&](int v, int64_t c, int64_t left) {
            float s[S::kC];
            sum_of(v, c, left, s);
            if (a.sum.data) store_floats(row_out<T>(a.sum, m) + c, left, s);
            value_of(v, c, left, s);
            if constexpr (k8Bits) {
                by.divide(s);
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

// dx, and in `partial` the workgroup's sums of dy h, and behind all workgroups' of
// those the sums of dy (held rows only; else the moments of each row go to
// `moments` and a second kernel sums)
template <typename T, typename S>
__global__ __launch_bounds__(S::kThreads) void layer_norm_backward_kernel(wfst_am_layer_norm_backward_args a, float *partial, Moments *moments)
{
    __shared__ SumScratch<4> sums;
    int turn = 0;
    const int64_t M = a.s.rows, D = a.s.cols, step = static_cast<int64_t>(gridDim.x) * S::kRows;
    const int t = threadIdx.x % S::kTpr;
    RowPart<S, float> gain;
    if (a.gain) gain.hold(a.gain, D, t);
    float dg[S::kHeld][S::kC] = {}, db[S::kHeld][S::kC] = {};
    Part<S, T> s, dy, ds, s_next, dy_next;
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
        float total[1] = {0.0f};
        S::each(D, t, [&](int v, int64_t c, int64_t left) {
            float x[S::kC];
            s.get(v, c, left, x);
#pragma unroll
            for (int e = 0; e < S::kC; e++) total[0] += x[e];
        });
        row_sums<S>(total, sums, turn);
        Moments mo;
        mo.m0 = total[0] / static_cast<float>(D);
        float four[4] = {0.0f, 0.0f, 0.0f, 0.0f};   // of d, d d, u, u d
        S::each(D, t, [&](int v, int64_t c, int64_t left) {
            float x[S::kC], w[S::kC], u[S::kC];
            s.get(v, c, left, x);
            dy.get(v, c, left, w);
            u_of(v, c, left, w, u);
#pragma unroll
            for (int e = 0; e < S::kC; e++) {
                const float d = e < left ? x[e] - mo.m0 : 0.0f;
                four[0] += d;
                four[1] = fmaf(d, d, four[1]);
                four[2] += u[e];
                four[3] = fmaf(u[e], d, four[3]);
            }
        });
        row_sums<S>(four, sums, turn);
        mo.set(four[0], four[1], static_cast<float>(D), a.eps);
        if (S::kNv == 0 && moments && t == 0) moments[m] = mo;
        if (S::kNv == 0 && !a.dx.data) continue;
        const float mean_u = four[2] / static_cast<float>(D);
        const float mean_uh = (four[3] - mo.c * four[2]) / static_cast<float>(D) * mo.rho;
        S::each(D, t, [&](int v, int64_t c, int64_t left) {
            float x[S::kC], w[S::kC], u[S::kC], h[S::kC];
            s.get(v, c, left, x);
            dy.get(v, c, left, w);
            u_of(v, c, left, w, u);
#pragma unroll
            for (int e = 0; e < S::kC; e++) h[e] = mo.unit(x[e]);
            if constexpr (S::kNv > 0)
#pragma unroll
                for (int e = 0; e < S::kC; e++) {
                    dg[v][e] = fmaf(w[e], h[e], dg[v][e]);
                    db[v][e] += w[e];
                }
            if (!a.dx.data) return;
            float d[S::kC];
#pragma unroll
            for (int e = 0; e < S::kC; e++) d[e] = mo.rho * ((u[e] - mean_u) - h[e] * mean_uh);
            if (a.dsum.data) {
                ds.get(v, c, left, u);
#pragma unroll
                for (int e = 0; e < S::kC; e++) d[e] += u[e];
            }
            store_floats(row_out<T>(a.dx, m) + c, left, d);
        });
    }
    if (S::kNv == 0 || !partial) return;
    float *partial_b = partial + static_cast<int64_t>(gridDim.x) * D;
    if constexpr (S::kRows == 1) {
        S::each(D, t, [&](int v, int64_t c, int64_t left) {
            store_floats(partial + blockIdx.x * D + c, left, dg[v]);
            store_floats(partial_b + blockIdx.x * D + c, left, db[v]);
        });
    } else {
        // a wave's rows' sums, then the waves' sums one after the other
        if constexpr (S::kLanes < 64)
#pragma unroll
            for (int v = 0; v < S::kHeld; v++)
#pragma unroll
                for (int e = 0; e < S::kC; e++)
#pragma unroll
                    for (int far = S::kLanes; far < 64; far *= 2) {
                        dg[v][e] += __shfl_xor(dg[v][e], far);
                        db[v][e] += __shfl_xor(db[v][e], far);
                    }
        __shared__ float total[2][S::kHeld * S::kTpr * S::kC];
        const bool first_row = static_cast<int>(threadIdx.x & 63) < S::kTpr;
        for (int w = 0; w < S::kThreads / 64; w++) {
            __syncthreads();
            if (static_cast<int>(threadIdx.x) / 64 != w || !first_row) continue;
#pragma unroll
            for (int v = 0; v < S::kHeld; v++)
#pragma unroll
                for (int e = 0; e < S::kC; e++) {
                    const int at = (v * S::kC + e) * S::kTpr + t;
                    if (w) dg[v][e] += total[0][at], db[v][e] += total[1][at];
                    total[0][at] = dg[v][e], total[1][at] = db[v][e];
                }
        }
        if (threadIdx.x / 64 == S::kThreads / 64 - 1 && first_row)
            S::each(D, t, [&](int v, int64_t c, int64_t left) {
                store_floats(partial + blockIdx.x * D + c, left, dg[v]);
                store_floats(partial_b + blockIdx.x * D + c, left, db[v]);
            });
    }
}

// Sums of dy h and of dy over strips of rows too long to hold: a wave of a workgroup
// takes every fourth row of a strip, a lane C columns.
template <typename T, int C>
__global__ __launch_bounds__(256) void layer_norm_columns_kernel(wfst_am_layer_norm_backward_args a, const Moments *moments, float *partial)
{
    __shared__ float part[2][3][64 * C];
    const int64_t M = a.s.rows, D = a.s.cols;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = (static_cast<int64_t>(blockIdx.x) * 64 + lane) * C;
    const int64_t first = M * blockIdx.y / gridDim.y, last = M * (blockIdx.y + 1) / gridDim.y;
    float dg[C] = {}, db[C] = {};
    if (c < D)
        for (int64_t m = first + wave; m < last; m += 4) {
            const Moments mo = moments[m];
            float x[C], w[C];
            load_floats(row<T>(a.s, m) + c, D - c, x);
            load_floats(row<T>(a.dy, m) + c, D - c, w);
#pragma unroll
            for (int e = 0; e < C; e++) {
                dg[e] = fmaf(w[e], mo.unit(x[e]), dg[e]);
                db[e] += w[e];
            }
        }
    if (wave)
#pragma unroll
        for (int e = 0; e < C; e++) part[0][wave - 1][e * 64 + lane] = dg[e], part[1][wave - 1][e * 64 + lane] = db[e];
    __syncthreads();
    if (wave || c >= D) return;
#pragma unroll
    for (int e = 0; e < C; e++)
#pragma unroll
        for (int w = 0; w < 3; w++) dg[e] += part[0][w][e * 64 + lane], db[e] += part[1][w][e * 64 + lane];
    store_floats(partial + blockIdx.y * D + c, D - c, dg);
    store_floats(partial + (gridDim.y + blockIdx.y) * D + c, D - c, db);
}

// Rows of few columns share a wave: (349525, 96) bf16 to 8 bits with the residual 50 us, with a wave a row 192,
// (524288, 64) 42 and 280, (131072, 256) 42 and 73; backward of (349525, 96) with dsum 67 and 233, of (131072, 256) 55 and
// 97.  Rows of 1,025 to 1,536 16-bit columns take three chunks a lane ((52429, 1280) to 8 bits with the residual 93 us, in
// four 120; backward with dsum 112 and 118).
template <int C, typename F>
void row_shape(int64_t D, F go)
{
    constexpr int k = 8 / C;
    am_shape_of<UpTo<64, RowShape<8, 1 * k, C>>, UpTo<128, RowShape<16, 1 * k, C>>, UpTo<256, RowShape<32, 1 * k, C>>,
                UpTo<512, RowShape<64, 1 * k, C>>, UpTo<1024, RowShape<64, 2 * k, C>>, UpTo<C == 8 ? 1536 : 0, RowShape<64, 3, C>>,
                UpTo<2048, RowShape<64, 4 * k, C>>, UpTo<4096, RowShape<256, 2 * k, C>>, UpTo<6144, RowShape<256, 3 * k, C>>,
                UpTo<8192, RowShape<256, 4 * k, C>>, UpTo<16384, RowShape<1024, 2 * k, C>>, UpTo<INT64_MAX, RowShape<1024, 0, C>>>(D, go);
}

// And for the gradients: rows of 1,025 to 2,048 float32 columns take 256 threads ((11184, 1500) 53 us, a wave 59),
// 16-bit ones a wave ((22369, 1500) 68, 256 threads 130; (16384, 2048) 52 and 75).  Held up to 16,384 columns ((1024,
// 32768) bf16 132 us, held 249, float32 247 and 473).
template <int C, typename F>
void row_shape_backward(int64_t D, F go)
{
    constexpr int k = 8 / C;
    am_shape_of<UpTo<64, RowShape<8, 1 * k, C>>, UpTo<128, RowShape<16, 1 * k, C>>, UpTo<256, RowShape<32, 1 * k, C>>,
                UpTo<512, RowShape<64, 1 * k, C>>, UpTo<1024, RowShape<64, 2 * k, C>>, UpTo<C == 8 ? 1536 : 0, RowShape<64, 3, C>>,
                UpTo<2048, std::conditional_t<C == 8, RowShape<64, 4, C>, RowShape<256, 1 * k, C>>>, UpTo<4096, RowShape<256, 2 * k, C>>,
                UpTo<6144, RowShape<256, 3 * k, C>>, UpTo<8192, RowShape<256, 4 * k, C>>, UpTo<16384, RowShape<1024, 2 * k, C>>,
                UpTo<INT64_MAX, RowShape<1024, 0, C>>>(D, go);
}

// Workgroups at most.  Backward about as many as are resident, by the bytes of a matrix that a thread holds: one
// more and the last ones run alone (268 MB each, 1 to 5 a CU: 512 bf16 columns 95, 67, 62, 58, 57 us; 1,024 72, 52,
// 51, 60, 57; 2,048 64, 52, 63, 61, 61; 8,192 72, 63, 76, 79, 78; 2,048 float32 64, 49, 50, 51, 54).
//   Forward, 4, 8, 16, 24, 32 and 64 a CU: (53274, 1024) bf16 to 8 bits with the residual 80.5, 79.6, 76.7, 75.7, 74.2
// and 71.6 us, without 49.3, 46.9, 44.6, 44.2, 43.1 and 45.5; (349525, 96) 58.7, 54.1, 51.6, 49.0, 48.6 and 47.6 with it;
// (16384, 4096) 54.6 with 32 and 58.3 with 64 without.
constexpr int64_t kForwardBlocks = 256 * 32;

template <typename S>
constexpr int64_t backward_blocks(int64_t el)
{
    const int64_t held = S::kNv * S::kC * el;
    return 256 * (S::kThreads > 256 ? 1 : held <= 16 ? 5 : held <= 32 ? 3 : held <= 96 ? 2 : 1);
}

struct Sums {
    int64_t strips, moments_bytes, partial_bytes;
};

// strips of rows whose sums are joined, and what the workspace holds
Sums sums_of(int64_t M, int64_t D, int64_t el)
{
    Sums n{};
    const auto of = [&](auto shape) {
        using S = decltype(shape);
        if constexpr (S::kNv > 0) {
            n.strips = static_cast<int64_t>(am_row_blocks<S>(M, backward_blocks<S>(el)));
        } else {
            // 16 rows a wave at least, about 1,024 workgroups at most
            const int64_t wide = (D + 511) / 512, tall = M / 64, most = 1024 / wide;
            n.strips = M ? tall < most ? tall : most : 0;
            if (M && n.strips < 1) n.strips = 1;
            n.moments_bytes = (M * static_cast<int64_t>(sizeof(Moments)) + 255) & ~int64_t{255};
        }
    };
    if (el == 4) row_shape_backward<4>(D, of);
    else row_shape_backward<8>(D, of);
    n.partial_bytes = (n.strips * D * 8 + 255) & ~int64_t{255};
    return n;
}

template <typename T>
void launch_layer_norm(const wfst_am_layer_norm_args &a, hipStream_t st)
{
    const auto go = [&](auto shape) {
        using S = decltype(shape);
        const unsigned g = am_row_blocks<S>(a.x.rows, kForwardBlocks);
        if constexpr (S::kC == kChunk<T>)
            if (a.y.type == WFST_F8E4M3) return layer_norm_kernel<T, S, true><<<g, S::kThreads, 0, st>>>(a);
        layer_norm_kernel<T, S, false><<<g, S::kThreads, 0, st>>>(a);
    };
    if (kChunk<T> > 4 && a.y.type == WFST_F32) row_shape<4>(a.x.cols, go);
    else row_shape<kChunk<T>>(a.x.cols, go);
}

template <typename T>
void launch_layer_norm_backward(const wfst_am_layer_norm_backward_args &a, hipStream_t st)
{
    const int64_t M = a.s.rows, D = a.s.cols;
    const Sums n = sums_of(M, D, sizeof(T));
    const bool wanted = a.dgain || a.dbias;
    char *work = static_cast<char *>(a.workspace);
    Moments *moments = reinterpret_cast<Moments *>(work);
    float *partial = reinterpret_cast<float *>(work + n.moments_bytes);
    row_shape_backward<kChunk<T>>(D, [&](auto shape) {
        using S = decltype(shape);
        const unsigned g = M ? am_row_blocks<S>(M, S::kNv > 0 ? backward_blocks<S>(sizeof(T)) : 256 * 3) : 0;
        if constexpr (S::kNv > 0) {
            if (M) layer_norm_backward_kernel<T, S><<<g, S::kThreads, 0, st>>>(a, wanted ? partial : nullptr, nullptr);
        } else if (M) {
            if (wanted) {
                // The gradients of gain and bias before dx may overwrite dy.  In all s is gone through six times
                // and dy four: (1024, 32768) bf16 with dsum 132 us, dx alone 71.
                wfst_am_layer_norm_backward_args b = a;
                b.dx.data = nullptr;
                layer_norm_backward_kernel<T, S><<<g, S::kThreads, 0, st>>>(b, nullptr, moments);
                constexpr int C = kChunk<T>;
                const dim3 grid(static_cast<unsigned>((D + 64 * C - 1) / (64 * C)), static_cast<unsigned>(n.strips));
                layer_norm_columns_kernel<T, C><<<grid, 256, 0, st>>>(a, moments, partial);
            }
            if (a.dx.data) layer_norm_backward_kernel<T, S><<<g, S::kThreads, 0, st>>>(a, nullptr, nullptr);
        }
    });
    if (a.dgain) am_launch_column_join(partial, n.strips, D, a.dgain, a.dbias, st);
    else if (a.dbias) am_launch_column_join(partial + n.strips * D, n.strips, D, a.dbias, nullptr, st);
}

}  // namespace

hipError_t am_launch_layer_norm(const wfst_am_layer_norm_args &a, hipStream_t st)
{
    if (a.x.type == WFST_F32) launch_layer_norm<float>(a, st);
    else if (a.x.type == WFST_F16) launch_layer_norm<f16>(a, st);
    else launch_layer_norm<bf16>(a, st);
    return hipGetLastError();
}

int64_t am_layer_norm_backward_bytes(const wfst_am_layer_norm_backward_args &a)
{
    if (!a.dgain && !a.dbias) return 0;
    const Sums n = sums_of(a.s.rows, a.s.cols, am_type_bytes(a.s.type));
    return n.moments_bytes + n.partial_bytes;
}

hipError_t am_launch_layer_norm_backward(const wfst_am_layer_norm_backward_args &a, hipStream_t st)
{
    if (a.s.type == WFST_F32) launch_layer_norm_backward<float>(a, st);
    else if (a.s.type == WFST_F16) launch_layer_norm_backward<f16>(a, st);
    else launch_layer_norm_backward<bf16>(a, st);
    return hipGetLastError();
}

}  // namespace wfd
