// Tiled matrix products on the matrix cores:
//   out[i][j] = epilogue(sum_k a[i][k] b[j][k])
// with each operand stored k-contiguous (rows of k) or k-major (rows of i or
// j, one row a k).
//
// A workgroup computes a BM x BN tile, stage by stage: a stage holds 64 or 128
// bytes of k for every row of the tile.  Two to four stages lie in LDS: the later
// ones are fetched while the matrix cores work on the present one.  The fetch goes
// straight from memory to LDS (16 bytes a lane, no registers); operands that are
// not aligned to 16 bytes go through registers ((16384, 1001, 2048) forward, both
// gradients: 120, 109, 114 us; with 1024 aligned columns 70, 59, 89).
//
// 8-bit operands are widened to bf16 as they are read from LDS (each value
// exactly).  The 8-bit matrix instructions would be twice as fast, but drop the
// low bits of products far below the largest one of their 128 (errors up to
// 2^-12 of it); as bf16 the products and their sums are kept in 32 bits.
//
// LDS layout.  A stage is a row of 16-byte chunks for each row of the operand
// as stored; a chunk sits at its index XOR a function of the row, so that the
// lanes of one read meet all banks.  The memory-to-LDS fetch writes lane after
// lane, so the permutation is applied to the address that a lane reads.
//   k-contiguous: a lane's fragment is one chunk of its row
//   k-major (16 bits): a fragment is gathered by two transposing LDS reads; each
//   takes 4 rows (k) by 16 columns from a group of 16 lanes and hands every lane
//   its column's 4 values
// The order of k inside a fragment does not matter as long as both operands
// have the same.
//
// The product is issued with b as the first matrix-core operand, so a lane's
// results are 4 consecutive j of one i.  Where b is k-contiguous the rows of b
// are dealt to the fragments so that a lane holds 4 * TJ consecutive j.
//
// Gated layers have two rows of b for each result, a gate's and a value's, b.extent
// rows apart.  A tile takes half as many of either: the first half of the rows that
// make up a lane's run are gates, the second half the same results' values, so
// both meet in one lane's registers and nothing but the products' addresses and
// the epilogue differs.
//
// Measured, bf16: (16384, 4096, 1024) k-contiguous 107 us, 1,280 TFLOP/s (the
// library's product 94 us); (16384, 4096, 1024) with b k-major 120; k = 16384
// into 4096 x 1024, both k-major, 139 and 17 for joining 4 parts; with a in two parts
// 255 and 288.  The matrix cores are busy 53% of the time (403 MB of reads behind the L2s
// for two parts of both k-major; 1.3 GB when a part's tiles were dealt to all chiplets).
// Gated, (16384, 1024, 4096): 244 us, 1,127 TFLOP/s (the library's plain product of twice the
// outputs 246), with pre 310 (matrix cores busy 37 to 39%: 403 MB are stored while no products are
// formed).  No LDS bank conflicts but in
// k-contiguous stages of 64 bytes, where they take 6 to 11% of a CU's cycles (7 to 9 in 8
// bits, 11 in unaligned rows).  The rest is the waves' meeting once a stage and, for a
// short k, the start and the epilogue of a tile ((16384, 1024, 4096): 142 to 159 us).
// 256 x 256 tiles with 4 waves of twice the registers made the compiler move sums about;
// 256 x 128 ones in two workgroups a CU read half as much again from L2 (143 us instead
// of 107), but pay for 8 bits, where operands are half as large and the epilogue of one
// overlaps the other's products ((53274, 1024, 4096) e4m3 with gelu: 493 to 514 us by the
// card, 870 to 905 TFLOP/s; matrix cores busy 38%).
#pragma once

#include <type_traits>
#include <utility>

#include "am_device.h"
#include "am_plan.h"

namespace wfd {

using i16x4 = short __attribute__((ext_vector_type(4)));
using i32x4 = int __attribute__((ext_vector_type(4)));
using i32x4_any = Chunk<int, 4, 1>;   // at any address
using f32x4 = float __attribute__((ext_vector_type(4)));
using f16x8 = f16 __attribute__((ext_vector_type(8)));
using bf16x8 = bf16 __attribute__((ext_vector_type(8)));

// use(0), use(1), ... use(N - 1), each with a constant
template <int N, typename F, int... I>
__device__ __forceinline__ void am_each(F use, std::integer_sequence<int, I...>)
{
    (use(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void am_each(F use)
{
    am_each<N>(use, std::make_integer_sequence<int, N>{});
}

struct AmProduct {
    AmOperand a, b;
    const char *a_low;         // a's low parts (AmParts), laid out as a; NULL: a is all there is
    int32_t inner;             // k
    int32_t splits;            // parts of k, one workgroup each per tile; > 1: sums go to `partial`
    uint32_t first;            // tile of the launch's first workgroup
    uint32_t part_tiles;       // tiles of a part where a launch has those of several parts, else 0
    // what a workgroup reads before its first fetch lies before this
    float *partial;            // [splits][a.extent][b.extent]
    const float *a_scale, *b_scale, *bias;
    wfst_matrix residual, pre, out;
    wfst_matrix value_pre;     // gated: the values' half of pre (pre is the gates')
    int32_t activation;
};

// A float32 operand of a product as two 16-bit values: high * kHigh + low * kLow,
// within 2^-16 of it (bf16) or 2^-22 (f16, or 2^-35 if that is more).  f16's factors
// keep a layer's dz, a value times a slope (at most 1.13), below the type's largest, and
// the low part of a small one above its smallest.  A gated layer's, a product of two values
// and a slope, has no such bound: from 131,008 on its high part is an infinity.
template <typename E>
struct AmParts {
    static constexpr float kHigh = __is_same(E, f16) ? 2.0f : 1.0f;
    static constexpr float kLow = __is_same(E, f16) ? 0x1p-10f : 1.0f;
};

__device__ __forceinline__ float am_silu(float z) { return z * __builtin_amdgcn_rcpf(1.0f + am_exp(-z)); }

// The normal distribution's function at z and exp(-z^2 / 2).  For x = |z| / sqrt 2
// and t = 1 / (1 + 0.55 x), exp(x^2) erfc(x) / 2 is a polynomial of t without a
// constant, to 1.7e-8 / max(|z|, 1) after the product with exp(-x^2): the
// coefficients are a fit of that error's maximum over x (least squares, reweighted
// until the peaks are level).  The tail is not taken from 1, so gelu is as good at
// -4 as at 4.  erff costs three times as much, more than the products of a short k.
__device__ __forceinline__ float am_normal(float z, float &bell)
{
    const float x = fabsf(z) * 0.70710678f, t = __builtin_amdgcn_rcpf(fmaf(0.55f, x, 1.0f));
    bell = __builtin_amdgcn_exp2f(x * x * -1.44269504f);
    float p = fmaf(0.05319667f, t, -0.25721717f);
    p = fmaf(p, t, 0.37709814f);
    p = fmaf(p, t, -0.018625526f);
    p = fmaf(p, t, 0.19464108f);
    p = fmaf(p, t, 0.15090677f);
    const float tail = p * t * bell;
    return z < 0.0f ? tail : 1.0f - tail;
}

__device__ __forceinline__ float am_gelu(float z)
{
    float bell;
    return z * am_normal(z, bell);
}

template <int N>
__device__ __forceinline__ void am_activate(float (&v)[N], int32_t kind)
{
    if (kind == WFST_ACT_RELU)
#pragma unroll
        for (int i = 0; i < N; i++) v[i] = v[i] < 0.0f ? 0.0f : v[i];   // a NaN stays one
    else if (kind == WFST_ACT_SILU)
#pragma unroll
        for (int i = 0; i < N; i++) v[i] = am_silu(v[i]);
    else if (kind == WFST_ACT_GELU)
#pragma unroll
        for (int i = 0; i < N; i++) v[i] = am_gelu(v[i]);
}

// N consecutive values of row i from column j on; `full`: all inside.  Rows
// need no alignment (wide accesses go to any address)
template <typename T, int N>
__device__ __forceinline__ void am_store_row(const wfst_matrix &m, int64_t i, int64_t j, const float (&v)[N], bool full)
{
    T *p = static_cast<T *>(m.data) + i * m.row_stride + j;
    constexpr int kStep = N * sizeof(T) >= 16 ? 16 / sizeof(T) : N;
    using V = Chunk<T, kStep>;
    if (full) {
#pragma unroll
        for (int s = 0; s < N; s += kStep) {
            V t;
#pragma unroll
            for (int e = 0; e < kStep; e++) t[e] = static_cast<T>(v[s + e]);
            *(AM_GLOBAL V *)(p + s) = t;
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < N; e++)
        if (j + e < m.cols) ((AM_GLOBAL T *)p)[e] = static_cast<T>(v[e]);
}

template <int N>
__device__ __forceinline__ void am_store(const wfst_matrix &m, int64_t i, int64_t j, const float (&v)[N], bool full)
{
    if (m.type == WFST_BF16) am_store_row<bf16>(m, i, j, v, full);
    else if (m.type == WFST_F16) am_store_row<f16>(m, i, j, v, full);
    else am_store_row<float>(m, i, j, v, full);
}

template <typename T, int N>
__device__ __forceinline__ void am_add_row(const wfst_matrix &m, int64_t i, int64_t j, float (&v)[N], bool full)
{
    const T *p = static_cast<const T *>(m.data) + i * m.row_stride + j;
    constexpr int kStep = N * sizeof(T) >= 16 ? 16 / sizeof(T) : N;
    using V = Chunk<T, kStep>;
    if (full) {
#pragma unroll
        for (int s = 0; s < N; s += kStep) {
            const V t = *(const AM_GLOBAL V *)(p + s);
#pragma unroll
            for (int e = 0; e < kStep; e++) v[s + e] += static_cast<float>(t[e]);
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < N; e++)
        if (j + e < m.cols) v[e] += static_cast<float>(((const AM_GLOBAL T *)p)[e]);
}

template <int N>
__device__ __forceinline__ void am_add(const wfst_matrix &m, int64_t i, int64_t j, float (&v)[N], bool full)
{
    if (m.type == WFST_BF16) am_add_row<bf16>(m, i, j, v, full);
    else if (m.type == WFST_F16) am_add_row<f16>(m, i, j, v, full);
    else am_add_row<float>(m, i, j, v, full);
}

// The epilogue of N consecutive j of row i (j < cols), their scales and biases at hand.
template <int N>
__device__ __forceinline__ void am_finish(const AmProduct &p, int64_t i, int64_t j, float (&v)[N],
                                          const float (&b_scale)[N], const float (&bias)[N])
{
    const bool full = j + N <= p.b.extent;
    if (p.a_scale) {
        const float s = p.a_scale[i];
#pragma unroll
        for (int e = 0; e < N; e++) v[e] *= s * b_scale[e];
    }
    if (p.bias)
#pragma unroll
        for (int e = 0; e < N; e++) v[e] += bias[e];
    if (p.pre.data) am_store(p.pre, i, j, v, full);
    am_activate(v, p.activation);
    if (p.residual.data) am_add(p.residual, i, j, v, full);
    am_store(p.out, i, j, v, full);
}

// The epilogue of N results of a gated row i from j on (j < cols): v, scales and biases hold their gates', then their values'.
template <int N>
__device__ __forceinline__ void am_finish_gated(const AmProduct &p, int64_t i, int64_t j, float (&v)[2 * N],
                                                const float (&b_scale)[2 * N], const float (&bias)[2 * N])
{
    const bool full = j + N <= p.b.extent;
    if (p.a_scale) {
        const float s = p.a_scale[i];
#pragma unroll
        for (int e = 0; e < 2 * N; e++) v[e] *= s * b_scale[e];
    }
    if (p.bias)
#pragma unroll
        for (int e = 0; e < 2 * N; e++) v[e] += bias[e];
    float gate[N], value[N];
#pragma unroll
    for (int e = 0; e < N; e++) gate[e] = v[e], value[e] = v[N + e];
    if (p.pre.data) {
        am_store(p.pre, i, j, gate, full);
        am_store(p.value_pre, i, j, value, full);
    }
    am_activate(gate, p.activation);
#pragma unroll
    for (int e = 0; e < N; e++) gate[e] *= value[e];
    am_store(p.out, i, j, gate, full);
}

template <int N>
__device__ __forceinline__ void am_columns(const AmProduct &p, int64_t j, float (&b_scale)[N], float (&bias)[N])
{
#pragma unroll
    for (int e = 0; e < N; e++) {
        const int64_t c = j + e < p.b.extent ? j + e : p.b.extent - 1;
        b_scale[e] = p.b_scale ? p.b_scale[c] : 1.0f;
        bias[e] = p.bias ? p.bias[c] : 0.0f;
    }
}

// of gates and values of columns from j on
template <int N>
__device__ __forceinline__ void am_columns_gated(const AmProduct &p, int64_t j, float (&b_scale)[N], float (&bias)[N])
{
#pragma unroll
    for (int e = 0; e < N; e++) {
        const int64_t at = j + e % (N / 2), c = (at < p.b.extent ? at : p.b.extent - 1) + (e < N / 2 ? 0 : p.b.extent);
        b_scale[e] = p.b_scale ? p.b_scale[c] : 1.0f;
        bias[e] = p.bias ? p.bias[c] : 0.0f;
    }
}

template <typename E>
__device__ __forceinline__ f32x4 am_mfma(i32x4 x, i32x4 y, f32x4 c)
{
    if constexpr (__is_same(E, f16))
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
}

// 16 e4m3 values as bf16, which holds each exactly
__device__ __forceinline__ void am_widen(i32x4 v, i32x4 &lo, i32x4 &hi)
{
#pragma unroll
    for (int e = 0; e < 2; e++) {
        lo[2 * e] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[e], 1.0f, false));
        lo[2 * e + 1] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[e], 1.0f, true));
        hi[2 * e] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[e + 2], 1.0f, false));
        hi[2 * e + 1] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[e + 2], 1.0f, true));
    }
}

template <int e>
__device__ __forceinline__ uint32_t am_bits(const f32x4 &v)
{
    return __float_as_uint(v[e]);
}
template <int e>
__device__ __forceinline__ void am_set(f32x4 &v, uint32_t bits)
{
    v[e] = __uint_as_float(bits);
}

// Tile (ti, tj) and part of k of workgroup `block`, of parts * rows * cols in a row.
// Workgroups go to the 8 chiplets in turn; each chiplet gets a run of consecutive
// tiles of one part, and runs go through blocks of 8 rows of tiles, so a chiplet's L2
// sees few rows and columns.
__device__ __forceinline__ void am_tile_of(uint32_t block, uint32_t rows, uint32_t cols, uint32_t parts, uint32_t &ti, uint32_t &tj, uint32_t &part)
{
    const uint32_t tiles = rows * cols, count = tiles * parts, each = count / 8, more = count % 8, xcd = block % 8;
    uint32_t t = xcd * each + (xcd < more ? xcd : more) + block / 8;
    part = 0;
    if (parts > 1) part = t / tiles, t %= tiles;
    const uint32_t group = t / (8 * cols), at = t % (8 * cols);
    const uint32_t height = rows - group * 8 < 8 ? rows - group * 8 : 8;
    ti = group * 8 + at % height;
    tj = at / height;
}

constexpr int am_log2(int x) { return x <= 1 ? 0 : 1 + am_log2(x / 2); }

// One operand's part of the tile kernel: R rows (i or j) of SB bytes a stage,
// kMajor its storage, kDeal > 1: rows dealt to fragments so that a lane gets
// kDeal runs of 4 rows; kFar: rows so far apart that offsets inside a tile pass
// 31 bits; kGated: of every 4 * kDeal rows the first half are gates and the second
// half their values, which lie o.extent rows behind them.
template <typename E, int R, int SB, int kWaves, bool kMajor, int kDeal, bool kFar, bool kGated = false>
struct AmSide {
    static constexpr int kEl = sizeof(E);
    static constexpr int kWide = 16 / kEl;                       // values of a chunk
    static constexpr int kRowChunks = kMajor ? R / kWide : SB / 16;
    static constexpr int kBytes = R * SB;
    static constexpr int kPerWave = kBytes / 1024 / kWaves;      // fetches of 1 KiB a wave
    static constexpr int kHalves = SB / 64;                      // fragments along k
    static_assert(kBytes % (1024 * kWaves) == 0 && (kEl == 2 || !kMajor) && (kHalves == 1 || kHalves == 2), "");
    static_assert(!kGated || (!kMajor && kDeal > 1), "");

    // the operand's row that a tile's row is, counted from the tile's first; is it a value's?
    __device__ static __forceinline__ int source(int row)
    {
        if constexpr (kGated) return row / (4 * kDeal) * (2 * kDeal) + row % (2 * kDeal);
        else return row;
    }
    __device__ static __forceinline__ bool is_value(int row) { return kGated && row % (4 * kDeal) >= 2 * kDeal; }

    // chunk permutation of a stored row
    __device__ static __forceinline__ int permute(int row)
    {
        constexpr int kShift = 2 + am_log2(kDeal);
        if constexpr (kMajor) {
            // 16 lanes read 4 rows, 32 lanes 8: rows 0-3 and 8-11 (or 4 more), 32 bytes each
            if constexpr (kRowChunks >= 16) return ((row & 3) | ((row >> 3) & 1) << 2) << 1;
            else return (((row >> 1) & 1) | ((row >> 3) & 1) << 1) << 1;
        } else if constexpr (kHalves == 1) {
            return (row >> kShift) & 3;   // 16 lanes read 16 rows: 4 neighbours, then every 4 * kDeal
        } else {
            return ((row >> 1) & 1) | ((row >> kShift) & 3) << 1;
        }
    }

    int32_t voff[kPerWave];      // direct: byte offset of each fetch from the stage's base
    int32_t place[kMajor ? 1 : kHalves];   // of the lane's first fragment in a stage

    // the row as stored, and the chunk in it, that goes to a lane's place in LDS
    __device__ static __forceinline__ int row_of(int q, int wave, int lane) { return ((wave * kPerWave + q) * 64 + lane) / kRowChunks; }
    __device__ static __forceinline__ int chunk_of(int q, int wave, int lane)
    {
        return (lane % kRowChunks) ^ permute(row_of(q, wave, lane));
    }

    __device__ __forceinline__ void init(const AmOperand &o, int wave, int lane)
    {
#pragma unroll
        for (int q = 0; q < kPerWave; q++) {
            const int row = row_of(q, wave, lane);
            voff[q] = source(row) * static_cast<int32_t>(o.ld) + chunk_of(q, wave, lane) * 16;
            if (is_value(row)) voff[q] += o.extent * static_cast<int32_t>(o.ld);
        }
    }

    // Before the fetch of a last, partial stage with `tail` bytes of k: chunks
    // from k's end on get an offset past any range.  k-major rows past the end
    // are past the range already.
    __device__ __forceinline__ void cut(int32_t tail, int wave, int lane)
    {
        if constexpr (!kMajor)
#pragma unroll
            for (int q = 0; q < kPerWave; q++)
                voff[q] = chunk_of(q, wave, lane) * 16 < tail ? voff[q] : static_cast<int32_t>(0x80000000u);
    }

    // Straight to LDS (16-bit values): the descriptor of a stage, then its
    // fetches.  Rows past the operand's end are past the range of the descriptor
    // and read as zeros, as does a stage that is not there.
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t stage_rsrc(const AmOperand &o, int64_t first, int32_t inner, int32_t k0, bool there) const
    {
        int64_t skip, size;
        if constexpr (kMajor) {
            skip = k0 * o.ld + first * kEl;
            size = (static_cast<int64_t>(inner) - 1) * o.ld + static_cast<int64_t>(o.extent) * kEl;
        } else {
            skip = first * o.ld + static_cast<int64_t>(k0) * kEl;
            size = (static_cast<int64_t>(o.extent) * (kGated ? 2 : 1) - 1) * o.ld + static_cast<int64_t>(inner) * kEl;
        }
        const int64_t left = there ? size - skip : 0;
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(o.data) + skip, 0,
                                                 static_cast<int>(left < 0x7FFFFFFF ? left : 0x7FFFFFFF), 0x00027000);
    }
    __device__ __forceinline__ void fetch(__amdgpu_buffer_rsrc_t rsrc, int q, char *stage, int wave) const
    {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (AM_LDS void *)((AM_LDS char *)stage + (wave * kPerWave + q) * 1024),
                                                 16, voff[q], 0, 0, 0);
    }

    // Through registers, any alignment.  A chunk over its row's end is the 16
    // bytes that end there (put() moves them into place), so the loads have no
    // branch; only rows shorter than a chunk are taken value by value.  Values
    // past k's end become zeros; of a k-contiguous operand, rows past the end
    // repeat the last one, of a k-major one what follows a row's end is zeros
    // (results from neither are stored).
    __device__ __forceinline__ void load(const AmOperand &o, int64_t first, int32_t inner, int32_t k0, i32x4 (&r)[kPerWave], int wave, int lane)
    {
        using Offset = std::conditional_t<kFar, int64_t, uint32_t>;
        const AM_GLOBAL char *base = (const AM_GLOBAL char *)o.data + (kMajor ? k0 : first) * o.ld;
        const int32_t from = kMajor ? static_cast<int32_t>(first) : k0, length = kMajor ? o.extent : inner;
        const int32_t last = kMajor ? inner - k0 - 1 : o.extent - static_cast<int32_t>(first) - 1;
#pragma unroll
        for (int q = 0; q < kPerWave; q++) {
            const int32_t in_tile = row_of(q, wave, lane);
            int32_t row = source(in_tile), at = from + chunk_of(q, wave, lane) * kWide;
            row = row < last ? row : last;
            if (is_value(in_tile)) row += o.extent;
            const AM_GLOBAL char *p = base + static_cast<Offset>(row) * static_cast<Offset>(o.ld);
            if (length >= kWide) {
                at = at < length - kWide ? at : length - kWide;
                r[q] = *(const AM_GLOBAL i32x4_any *)(base + (static_cast<Offset>(row) * static_cast<Offset>(o.ld) + static_cast<Offset>(at) * kEl));
            } else {
                uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
                for (int e = 0; e < kWide; e++)
                    if (at + e < length) {
                        uint32_t t;
                        if constexpr (kEl == 2) t = ((const AM_GLOBAL uint16_t *)p)[at + e];
                        else t = ((const AM_GLOBAL uint8_t *)p)[at + e];
                        w[e * kEl / 4] |= t << (e * kEl % 4 * 8);
                    }
                r[q] = i32x4{static_cast<int>(w[0]), static_cast<int>(w[1]), static_cast<int>(w[2]), static_cast<int>(w[3])};
            }
        }
    }
    // `first`, `inner` and `k0` as for the load of r
    __device__ __forceinline__ void put(const AmOperand &o, int64_t first, int32_t inner, int32_t k0, const i32x4 (&r)[kPerWave], char *stage,
                                        int wave, int lane)
    {
        constexpr int32_t kRows = kBytes / 16 / kRowChunks;
        const int32_t from = kMajor ? static_cast<int32_t>(first) : k0, length = kMajor ? o.extent : inner;
        const int32_t k_left = inner - k0;
        const bool whole = from + kRowChunks * kWide <= length && (!kMajor || kRows <= k_left);
#pragma unroll
        for (int q = 0; q < kPerWave; q++) {
            i32x4 v = r[q];
            if (!whole) {
                // how many of the chunk's values lie before its place
                const int32_t row = row_of(q, wave, lane), at = from + chunk_of(q, wave, lane) * kWide;
                int32_t before = length >= kWide ? at - (length - kWide) : 0;
                before = before < 0 ? 0 : before;
                if (before >= kWide || (kMajor && row >= k_left)) v = i32x4{0, 0, 0, 0};
                else v = __builtin_bit_cast(i32x4, __builtin_bit_cast(unsigned __int128, v) >> (before * kEl * 8));
            }
            *reinterpret_cast<i32x4 *>(stage + ((wave * kPerWave + q) * 64 + lane) * 16) = v;
        }
    }

    // For the fragments of the wave's rows from `base` on.
    __device__ __forceinline__ void init_places(int base, int lane)
    {
        const int g = lane >> 4, s = lane & 15;
        if constexpr (kMajor) {
            const int row = g * 8 + (s >> 2);
            place[0] = row * (R * 2) + (((base >> 3) ^ permute(row)) << 4) + (s & 3) * 8;
        } else {
            const int row = base + (kDeal > 1 ? (s >> 2) * (4 * kDeal) + (s & 3) : s);
#pragma unroll
            for (int h = 0; h < kHalves; h++) place[h] = row * SB + (((h * 4 + g) ^ permute(row)) << 4);
        }
    }
    // The compiler would keep a register for each fragment's place: they are
    // taken anew in every stage instead.
    __device__ __forceinline__ void renew()
    {
        __asm__ volatile("" : "+v"(place[0]));
    }
    // Fragment f in half h of a stage's k
    template <int f, int h>
    __device__ __forceinline__ i32x4 fragment(const char *stage) const
    {
        if constexpr (kMajor) {
            i16x4 v[2];
#pragma unroll
            for (int t = 0; t < 2; t++)
                v[t] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (AM_LDS i16x4 *)((AM_LDS char *)stage + (place[0] ^ f * 32) + (h * 32 + t * 4) * (R * 2)));
            return __builtin_bit_cast(i32x4, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            return *reinterpret_cast<const i32x4 *>(stage + place[h] + f * (kDeal > 1 ? 4 : 16) * SB);
        }
    }
};

// vmcnt(n): at most n of the wave's fetches and loads under way
template <int n>
__device__ __forceinline__ void am_wait_vm()
{
    __builtin_amdgcn_s_waitcnt((n & 15) | 7 << 4 | 15 << 8 | (n >> 4) << 14);
}

// kBuffers stages of SB bytes a row in LDS
template <int BM_, int BN_, int WM_, int WN_, int SB_, int kBuffers_>
struct AmShape {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, SB = SB_, kBuffers = kBuffers_, kThreads = WM_ * WN_ * 64;
    // one workgroup a CU by its LDS may have all registers
    static constexpr int kWavesASimd = kThreads == 256 && (BM + BN) * SB * kBuffers > 80 * 1024 ? 1 : 2;
};

// kTwice: a is in two parts.  The whole of k is gone through twice into the same
// sums: the low parts, a change of scale, the high parts.
template <typename E, bool kMajorA, bool kMajorB, bool kDirect, typename S, bool kFar, bool kTwice, bool kGated>
__global__ __launch_bounds__(S::kThreads, S::kWavesASimd) void am_tile_kernel(AmProduct p)
{
#ifdef __HIP_DEVICE_COMPILE__   // the host pass needs the launch stub alone
    constexpr int BM = S::BM, BN = S::BN, WN = S::WN, SB = S::SB, kBuffers = S::kBuffers;
    constexpr int kWaves = S::WM * WN, TI = BM / S::WM / 16, TJ = BN / WN / 16, kK = SB / static_cast<int>(sizeof(E));
    constexpr int kDeal = kMajorB ? 1 : TJ;
    using SideA = AmSide<E, BM, SB, kWaves, kMajorA, 1, kFar>;
    using SideB = AmSide<E, BN, SB, kWaves, kMajorB, kDeal, kFar, kGated>;
    constexpr int kResults = kGated ? BN / 2 : BN;   // columns of a tile
    // one object a stage, so the compiler knows that a fetch into one does not touch the others
    __shared__ __attribute__((aligned(1024))) char a0[SideA::kBytes], a1[SideA::kBytes];
    __shared__ __attribute__((aligned(1024))) char a2[kBuffers > 2 ? SideA::kBytes : 1], a3[kBuffers > 3 ? SideA::kBytes : 1];
    __shared__ __attribute__((aligned(1024))) char b0[SideB::kBytes], b1[SideB::kBytes];
    __shared__ __attribute__((aligned(1024))) char b2[kBuffers > 2 ? SideB::kBytes : 1], b3[kBuffers > 3 ? SideB::kBytes : 1];
    const auto place_a = [&](auto n) -> char * {
        if constexpr (n % kBuffers == 0) return a0;
        else if constexpr (n % kBuffers == 1) return a1;
        else if constexpr (n % kBuffers == 2) return a2;
        else return a3;
    };
    const auto place_b = [&](auto n) -> char * {
        if constexpr (n % kBuffers == 0) return b0;
        else if constexpr (n % kBuffers == 1) return b1;
        else if constexpr (n % kBuffers == 2) return b2;
        else return b3;
    };

    const int lane_ = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint32_t ti, tj, k_part;
    const uint32_t rows = (p.a.extent + BM - 1) / BM, cols = (p.b.extent + kResults - 1) / kResults;
    if constexpr (kMajorB) {
        am_tile_of(p.first + blockIdx.y * p.part_tiles + blockIdx.x, rows, cols, p.part_tiles ? p.splits : 1, ti, tj, k_part);
        if (!p.part_tiles) k_part = blockIdx.y;
    } else {
        am_tile_of(p.first + blockIdx.x, rows, cols, 1, ti, tj, k_part);
    }
    const int64_t i0 = static_cast<int64_t>(ti) * BM, j0 = static_cast<int64_t>(tj) * kResults;
    const int wi = wave / WN * (BM / S::WM), wj = wave % WN * (BN / WN);

    const int32_t stages = (p.inner + kK - 1) / kK;
    const int32_t s_first = static_cast<int32_t>(static_cast<int64_t>(stages) * k_part / p.splits);
    const int32_t s_last = static_cast<int32_t>(static_cast<int64_t>(stages) * (k_part + 1) / p.splits);

    SideA sa;
    SideB sb;
    sa.init_places(wi, lane_);
    sb.init_places(wj, lane_);
    f32x4 acc[TI][TJ];
    am_each<TI>([&](auto f) { am_each<TJ>([&](auto g) { acc[f][g] = f32x4{0.0f, 0.0f, 0.0f, 0.0f}; }); });

    // A stage is kSteps steps of TJ products (8 bits: twice as many); step t has
    // half t / TI of the stage's k and rows t % TI.  Fragments are read kAhead
    // steps ahead, also over the end of a stage: its last reads are done kAhead
    // steps before its last products, and there the waves meet, a later stage is
    // fetched into this one's place and the next one's first fragments are read.
    // The scheduling fences keep that order.
    using C = std::conditional_t<sizeof(E) == 1, bf16, E>;   // what the matrix cores multiply
    constexpr int kHalves = SB / 64, kSteps = kHalves * TI, kAhead = 2, kX = 4;
    // kX divides kSteps: the next stage's first x are none of the last ones
    static_assert(kSteps % kX == 0 && 2 * kAhead <= kX && kAhead <= TI, "");
    i32x4 x[kX], y[2][TJ], y_lo[TJ], y_hi[TJ];
    // n: which stage, in turn; its half h has y in y[(n * kHalves + h) % 2]
    const auto read_y = [&](auto n, auto h) {
        am_each<TJ>([&](auto g) { y[(n * kHalves + h) % 2][g] = sb.template fragment<g, h % kHalves>(place_b(n)); });
    };
    const auto read_x = [&](auto n, auto t) { x[t % kX] = sa.template fragment<t % TI, t / TI>(place_a(n)); };
    const auto first_reads = [&](auto n) {
        sa.renew();
        sb.renew();
        read_y(n, std::integral_constant<int, 0>{});
        am_each<kAhead>([&](auto t) { read_x(n, t); });
    };
    // half(): what to do after half of a stage, next(): where the waves meet,
    // between(m): after the m-th products from there on
    const auto stage = [&](auto n, auto half, auto next, auto between) {
        am_each<kSteps>([&](auto t) {
            if constexpr (kHalves == 2 && t == TI - kAhead) read_y(n, std::integral_constant<int, 1>{});
            if constexpr (t + kAhead < kSteps) read_x(n, std::integral_constant<int, t + kAhead>{});
            if constexpr (t == kSteps / 2) half();
            if constexpr (t + kAhead == kSteps) next();
            __builtin_amdgcn_sched_barrier(0);
            constexpr int f = t % TI, in = (n * kHalves + t / TI) % 2;
            i32x4 x_lo, x_hi;
            if constexpr (sizeof(E) == 1) {
                if constexpr (f == 0) am_each<TJ>([&](auto g) { am_widen(y[in][g], y_lo[g], y_hi[g]); });
                am_widen(x[t % kX], x_lo, x_hi);
            }
            am_each<TJ>([&](auto g) {
                if constexpr (sizeof(E) == 1) {
                    acc[f][g] = am_mfma<C>(y_lo[g], x_lo, acc[f][g]);
                    acc[f][g] = am_mfma<C>(y_hi[g], x_hi, acc[f][g]);
                } else {
                    acc[f][g] = am_mfma<C>(y[in][g], x[t % kX], acc[f][g]);
                }
                if constexpr (t + kAhead >= kSteps) {
                    __builtin_amdgcn_sched_barrier(0);
                    between(std::integral_constant<int, (t + kAhead - kSteps) * TJ + g>{});
                }
            });
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    constexpr std::integral_constant<int, 0> first{};
    constexpr int kPeriod = kBuffers % 2 ? 2 * kBuffers : kBuffers;   // stages until places and y repeat
    // go(n) does a stage and says whether another one follows.  With k-major
    // operands the loop is left only after whole periods (the stages past the end
    // are zeros): every exit more costs the compiler registers, and there it
    // runs out of them.
    int32_t s;
    const auto all = [&](auto go) {
        [&]<int... n>(std::integer_sequence<int, n...>) {
            if constexpr (kMajorB) {
                do {
                    (go(std::integral_constant<int, n>{}), ...);
                } while (s < s_last);
            } else if constexpr (kGated) {
                // The stages past the end are jumped over inside the loop: with an exit at
                // each stage the sums of this epilogue are moved about and spilled ((16384, 1024,
                // 4096) bf16 1,381 us, so 238; with pre 1,646 and 313).  The copy of the count
                // keeps the compiler from making exits of the jumps.
                const auto unless_past = [&](auto m) {
                    int32_t left = s_last - s;
                    __asm__ volatile("" : "+s"(left));
                    if (m == 0 || left > 0) go(m);
                };
                do {
                    (unless_past(std::integral_constant<int, n>{}), ...);
                } while (s < s_last);
            } else {
                while ((go(std::integral_constant<int, n>{}) && ...)) {
                }
            }
        }(std::make_integer_sequence<int, kPeriod>{});
    };

    // Unrolled: as a loop the compiler kept two copies of some sums and had to fetch
    // offsets from memory inside the products' loop, each time behind the stage on its way.
#pragma clang loop unroll(full)
    for (int part = kTwice ? 0 : 1; part < 2; part++) {
    const AmOperand a{part ? p.a.data : p.a_low, p.a.ld, p.a.extent};
    s = s_first;
    int lane = lane_;   // what follows from it is computed anew for the other parts: kept, it would cost registers
    if constexpr (kTwice) __asm__ volatile("" : "+v"(lane));
    if constexpr (kDirect) {
        const int32_t tail = (p.inner % kK) * static_cast<int32_t>(sizeof(E));
        sa.init(a, wave, lane);
        sb.init(p.b, wave, lane);
        // The fetch of a stage: its descriptors, then its parts one by one.  A
        // stage that is not there is fetched from empty ranges, so that the
        // number of fetches under way is always known.
        __amdgpu_buffer_rsrc_t rsrc_a, rsrc_b;
        const auto begin = [&](int32_t s) {
            if (s + 1 == stages && tail) {
                sa.cut(tail, wave, lane);
                sb.cut(tail, wave, lane);
            }
            rsrc_a = sa.stage_rsrc(a, i0, p.inner, s * kK, s < s_last);
            rsrc_b = sb.stage_rsrc(p.b, j0, p.inner, s * kK, s < s_last);
        };
        constexpr int kParts = SideA::kPerWave + SideB::kPerWave, kEach = (kParts + kAhead * TJ - 1) / (kAhead * TJ);
        const auto part = [&](auto n, auto m) {
            if constexpr (m < SideA::kPerWave) sa.fetch(rsrc_a, m, place_a(n), wave);
            else if constexpr (m < kParts) sb.fetch(rsrc_b, m - SideA::kPerWave, place_b(n), wave);
        };
        am_each<kBuffers>([&](auto n) {
            begin(s + n);
            am_each<kParts>([&](auto m) { part(n, m); });
        });
        am_wait_vm<(kBuffers - 1) * kParts>();
        __syncthreads();
        first_reads(first);
        if (s < s_last)
            all([&](auto n) {
                stage(n, [] {}, [&] {
                    // the waves meet: the next stage has landed, later ones may be on their way
                    am_wait_vm<(kBuffers - 2) * kParts>();
                    __syncthreads();
                    first_reads(std::integral_constant<int, n + 1>{});
                    begin(s + kBuffers);
                }, [&](auto m) { am_each<kEach>([&](auto e) { part(n, std::integral_constant<int, m * kEach + e>{}); }); });
                return ++s < s_last;
            });
        am_wait_vm<0>();   // no fetch is under way when the workgroup ends
    } else {
        i32x4 ra[SideA::kPerWave], rb[SideB::kPerWave];
        const auto load = [&](int32_t s) {
            if (s >= s_last) {
                am_each<SideA::kPerWave>([&](auto q) { ra[q] = i32x4{0, 0, 0, 0}; });
                am_each<SideB::kPerWave>([&](auto q) { rb[q] = i32x4{0, 0, 0, 0}; });
                return;
            }
            sa.load(a, i0, p.inner, s * kK, ra, wave, lane);
            sb.load(p.b, j0, p.inner, s * kK, rb, wave, lane);
        };
        const auto put = [&](auto n, int32_t s) {
            sa.put(a, i0, p.inner, s * kK, ra, place_a(n), wave, lane);
            sb.put(p.b, j0, p.inner, s * kK, rb, place_b(n), wave, lane);
        };
        load(s);
        put(first, s);
        load(s + 1);
        __syncthreads();
        first_reads(first);
        if (s < s_last)
            all([&](auto n) {
                // the next stage goes to its place in the middle of this one, and the one after it on its way
                constexpr std::integral_constant<int, n + 1> next{};
                stage(n, [&] {
                    put(next, s + 1);
                    load(s + 2);
                }, [&] {
                    __syncthreads();
                    first_reads(next);
                }, [](auto) {});
                return ++s < s_last;
            });
    }
    if constexpr (kTwice) {
        // The low parts' sums in units of the high parts.  One that is not finite has
        // met an infinity or a NaN of b (low parts are finite), as the high parts will.
        const float unit = part ? AmParts<E>::kHigh : AmParts<E>::kLow / AmParts<E>::kHigh;
        am_each<TI>([&](auto f) {
            am_each<TJ>([&](auto g) {
                const f32x4 v = acc[f][g] * unit;
                const auto held = [&](float u) { return part || fabsf(u) < INFINITY ? u : 0.0f; };
                acc[f][g] = f32x4{held(v[0]), held(v[1]), held(v[2]), held(v[3])};
            });
        });
        __syncthreads();   // no wave reads a stage of these any more
    }
    }

    // A lane's run of consecutive j.  With dealt rows it has 4 * TJ already; else
    // 4 fragments' values change places between the 4 groups of 16 lanes, so that
    // group g gets fragment g: a run of 16 again.
    constexpr int kRun = 4 * TJ;
    static_assert(kDeal > 1 || TJ == 4 || TJ == 1, "");
    if constexpr (kDeal == 1 && TJ == 4)
        am_each<TI>([&](auto f) {
            am_each<4>([&](auto e) {
                const auto lo = __builtin_amdgcn_permlane32_swap(am_bits<e>(acc[f][0]), am_bits<e>(acc[f][2]), false, false);
                const auto hi = __builtin_amdgcn_permlane32_swap(am_bits<e>(acc[f][1]), am_bits<e>(acc[f][3]), false, false);
                const auto u = __builtin_amdgcn_permlane16_swap(lo[0], hi[0], false, false);
                const auto w = __builtin_amdgcn_permlane16_swap(lo[1], hi[1], false, false);
                am_set<e>(acc[f][0], u[0]);
                am_set<e>(acc[f][1], u[1]);
                am_set<e>(acc[f][2], w[0]);
                am_set<e>(acc[f][3], w[1]);
            });
        });
    if constexpr (kGated) {
        constexpr int kOwn = kRun / 2;
        const int64_t j = j0 + wj / 2 + (lane_ >> 4) * kOwn;
        if (j >= p.b.extent) return;
        float b_scale[kRun], bias[kRun];
        am_columns_gated(p, j, b_scale, bias);
        am_each<TI>([&](auto f) {
            const int64_t i = i0 + wi + f * 16 + (lane_ & 15);
            if (i >= p.a.extent) return;
            float v[kRun];
            am_each<TJ>([&](auto d) {
                const f32x4 a = acc[f][d];
                v[d * 4] = a[0], v[d * 4 + 1] = a[1], v[d * 4 + 2] = a[2], v[d * 4 + 3] = a[3];
            });
            am_finish_gated<kOwn>(p, i, j, v, b_scale, bias);
        });
        return;
    }
    const int64_t j = j0 + wj + (lane_ >> 4) * kRun;
    if (j >= p.b.extent) return;
    float b_scale[kRun], bias[kRun];
    if (p.splits == 1) am_columns(p, j, b_scale, bias);
    const wfst_matrix partial{p.partial + static_cast<int64_t>(k_part) * p.a.extent * p.b.extent, p.a.extent, p.b.extent, p.b.extent, WFST_F32, 0};
    am_each<TI>([&](auto f) {
        const int64_t i = i0 + wi + f * 16 + (lane_ & 15);
        if (i >= p.a.extent) return;
        float v[kRun];
        am_each<TJ>([&](auto d) {
            const f32x4 a = acc[f][d];
            v[d * 4] = a[0], v[d * 4 + 1] = a[1], v[d * 4 + 2] = a[2], v[d * 4 + 3] = a[3];
        });
        if (p.splits == 1) am_finish(p, i, j, v, b_scale, bias);
        else am_store_row<float>(partial, i, j, v, j + kRun <= p.b.extent);
    });
#endif
}

// --------------------------------------------------------------------------
// host side
// --------------------------------------------------------------------------

// sums the parts of a split product and finishes them (am_linear.hip)
void am_launch_join(const AmProduct &p, hipStream_t st);

template <typename E, bool kMajorA, bool kMajorB, bool kDirect, typename S, bool kTwice, bool kFar = false, bool kGated = false>
void am_launch_tiles(const AmProduct &p, hipStream_t st)
{
    const int64_t tiles = am_tiles(p.a.extent, p.b.extent, S::BM, kGated ? S::BN / 2 : S::BN);
    am_in_launches(tiles, [&](uint32_t first, uint32_t blocks) {
        AmProduct part = p;
        part.first = first;
        // The kernel does not ask for its grid's size, another read before its first fetch: (50, 512, 512) dw
        // 5.5 us, 5.9 with it; (1000, 1024, 1024) 8.9 and 9.3.
        part.part_tiles = p.splits > 1 && blocks == tiles ? blocks : 0;
        am_tile_kernel<E, kMajorA, kMajorB, kDirect, S, kFar, kTwice, kGated><<<dim3(blocks, p.splits), S::kThreads, 0, st>>>(part);
    });
    if (p.splits > 1) am_launch_join(p, st);
}

using AmLarge = AmShape<256, 256, 2, 4, 128, 2>;
using AmLarge8 = AmShape<256, 128, 2, 2, 64, 3>;   // two workgroups a CU
using AmWide = AmShape<128, 256, 2, 4, 128, 2>;
using AmMedium = AmShape<128, 128, 2, 2, 64, 3>;
using AmMediumMajor = AmShape<128, 128, 2, 2, 64, 4>;
using AmMediumDeep = AmShape<128, 128, 2, 2, 128, 4>;   // one workgroup a CU
using AmSmall = AmShape<64, 64, 2, 2, 128, 4>;
using AmSmallMajor = AmShape<64, 64, 1, 4, 128, 4>;
using AmMediumStaged = AmShape<128, 128, 2, 2, 64, 2>;
using AmSmallStaged = AmShape<64, 64, 2, 2, 128, 2>;
using AmSmallMajorStaged = AmShape<64, 64, 1, 4, 128, 2>;

template <typename E, bool kMajorA, bool kMajorB, bool kTwice = false>
void am_product(const AmProduct &p, int32_t tile, hipStream_t st)
{
    if constexpr (kMajorB && !kTwice)
        if (p.a_low) return am_product<E, kMajorA, kMajorB, true>(p, tile, st);
    if (am_direct(p.a, kMajorA, p.inner, sizeof(E)) && am_direct(p.b, kMajorB, p.inner, sizeof(E))) {
        if (tile == 256) am_launch_tiles<E, kMajorA, kMajorB, true, std::conditional_t<sizeof(E) == 1, AmLarge8, AmLarge>, kTwice>(p, st);
        else if (tile == 128 && am_tiles(p.a.extent, p.b.extent, 128, 128) * p.splits <= kComputeUnits)
            am_launch_tiles<E, kMajorA, kMajorB, true, AmMediumDeep, kTwice>(p, st);
        else if (tile == 128) am_launch_tiles<E, kMajorA, kMajorB, true, std::conditional_t<kMajorB, AmMediumMajor, AmMedium>, kTwice>(p, st);
        else am_launch_tiles<E, kMajorA, kMajorB, true, std::conditional_t<kMajorB, AmSmallMajor, AmSmall>, kTwice>(p, st);
    } else if (!am_near(p.a) || !am_near(p.b)) {
        am_launch_tiles<E, kMajorA, kMajorB, false, std::conditional_t<kMajorB, AmSmallMajorStaged, AmSmallStaged>, kTwice, true>(p, st);
    } else if (tile >= 128) {
        am_launch_tiles<E, kMajorA, kMajorB, false, AmMediumStaged, kTwice>(p, st);
    } else {
        am_launch_tiles<E, kMajorA, kMajorB, false, std::conditional_t<kMajorB, AmSmallMajorStaged, AmSmallStaged>, kTwice>(p, st);
    }
}

// y = act(a gates^T) * (a values^T), all k-contiguous: p.b the gates, the values p.b.extent rows behind them
template <typename E>
void am_gated_product(const AmProduct &p, int32_t tile, hipStream_t st)
{
    if (am_gated_direct(p.a, p.b, p.inner, sizeof(E))) {
        if (tile == 256) am_launch_tiles<E, false, false, true, std::conditional_t<sizeof(E) == 1, AmLarge8, AmLarge>, false, false, true>(p, st);
        else if (tile == kAmWide) am_launch_tiles<E, false, false, true, AmWide, false, false, true>(p, st);
        else if (tile == 128 && am_tiles(p.a.extent, 2 * int64_t{p.b.extent}, 128, 128) <= kComputeUnits)
            am_launch_tiles<E, false, false, true, AmMediumDeep, false, false, true>(p, st);
        else if (tile == 128) am_launch_tiles<E, false, false, true, AmMedium, false, false, true>(p, st);
        else am_launch_tiles<E, false, false, true, AmSmall, false, false, true>(p, st);
    } else if (!am_near(p.a) || !am_gated_near(p.b)) {
        am_launch_tiles<E, false, false, false, AmSmallStaged, false, true, true>(p, st);
    } else if (tile >= 128) {
        am_launch_tiles<E, false, false, false, AmMediumStaged, false, false, true>(p, st);
    } else {
        am_launch_tiles<E, false, false, false, AmSmallStaged, false, false, true>(p, st);
    }
}

}  // namespace wfd
