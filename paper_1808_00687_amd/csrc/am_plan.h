// Matrix products of the acoustic model: which tiles, how many workgroups.  Host
// arithmetic alone.
#pragma once

#include <cstdint>

namespace wfd {

constexpr int64_t kComputeUnits = 256;

struct AmOperand {
    const char *data;
    int64_t ld;        // bytes between rows as stored
    int32_t extent;    // i or j
};

// offsets inside a tile of 256 rows stay in 31 bits
inline bool am_near(const AmOperand &o) { return o.ld < (int64_t{1} << 22); }

// 16-byte fetches: rows aligned and ending on 16 bytes
inline bool am_direct(const AmOperand &o, bool major, int32_t inner, int el)
{
    const int64_t row = static_cast<int64_t>(major ? o.extent : inner) * el;
    return reinterpret_cast<uintptr_t>(o.data) % 16 == 0 && o.ld % 16 == 0 && row % 16 == 0 && am_near(o);
}

inline int64_t am_tiles(int64_t rows, int64_t cols, int64_t m, int64_t n) { return ((rows + m - 1) / m) * ((cols + n - 1) / n); }

// go(first, count) for consecutive runs of `blocks` workgroups, each run a launch: one
// takes fewer than 2^32 threads in a dimension (a workgroup has at most 512), and
// runs start at multiples of 8, so a block's chiplet is its index modulo 8.
template <typename F>
void am_in_launches(int64_t blocks, F go)
{
    constexpr int64_t kMost = int64_t{1} << 22;
    for (int64_t first = 0; first < blocks; first += kMost)
        go(static_cast<uint32_t>(first), static_cast<uint32_t>(blocks - first < kMost ? blocks - first : kMost));
}

// Which tiles, and into how many parts k is split.
struct AmPlan {
    int32_t tile;     // 256, 128 or 64
    int32_t splits;
};

// By an estimate of the time: rounds of workgroups over the chip times stages
// times what a stage of 64 values of k takes (measured, in microseconds, with one,
// two, ... workgroups on a CU, as many as fit).  A product that may be split (no
// epilogue, a workspace) also pays the join of its parts: 8 bytes a part and value,
// and a launch.  128 x 128 tiles that are at most one a CU have stages of twice the
// length, four of them: with the shorter ones a CU waits for memory ((4096, 1024,
// 1024) 19.4 us, so 16.2; (2048, 1024, 2048) 18.6 and 15.8; the gradient of x of
// (3000, 1024, 2048) 34.1 and 27.9).  Operands that are not `whole` (fetched straight
// to LDS) go through registers, in tiles and at times of their own: forward of (4096,
// 1024, 1024) with rows 2 bytes off 21 us in tiles of 128 and 29 of 64, gradient of x
// of (3000, 1024, 2048) 40 and 30, of w 56 and 35.
// The times are of 16-bit operands and decide for 8 bits too: of 14 products the best
// tile is missed by more than 10% in (4096, 1024, 2048) e4m3, 27 us in 256, 23 in 128,
// (3000, 1024, 2048), 25 and 22, and (53274, 512, 640), 56 and 46; of 14 in bf16 in two,
// (3000, 1024, 2048), 28.5 and 23, and (4096, 1024, 2048), 29 and 25.
inline AmPlan am_plan(int64_t rows, int64_t cols, int64_t inner, bool may_split, bool whole)
{
    struct Kind {
        int32_t tile;
        int64_t fit, most;   // workgroups on a CU, and on the chip
        double stage[4];
    };
    constexpr Kind direct[] = {{256, 1, INT64_MAX, {1.45}}, {128, 1, kComputeUnits, {0.95}}, {128, 3, INT64_MAX, {1.5, 1.9, 2.3}},
                               {64, 2, INT64_MAX, {0.5, 0.55}}};
    // forward, and with k-major operands (the gradients' products, those that may be split)
    constexpr Kind staged[2][2] = {{{128, 4, INT64_MAX, {1.2, 1.5, 2.2, 2.9}}, {64, 4, INT64_MAX, {0.58, 0.72, 1.2, 1.6}}},
                                   {{128, 4, INT64_MAX, {1.2, 1.4, 2.1, 2.85}}, {64, 4, INT64_MAX, {0.58, 0.7, 0.85, 1.15}}}};
    const int64_t stages = (inner + 63) / 64;
    AmPlan best{64, 1};
    double least = 1e30;
    for (int i = 0; i < (whole ? 4 : 2); i++) {
        const Kind &k = whole ? direct[i] : staged[may_split][i];
        for (int32_t s = 1; s <= (may_split ? 64 : 1) && (s == 1 || stages / s >= 4); s *= 2) {
            const int64_t n = am_tiles(rows, cols, k.tile, k.tile) * s, at_once = kComputeUnits * k.fit, rest = n % at_once;
            if (n > k.most) break;
            double t = static_cast<double>(n / at_once) * k.stage[k.fit - 1];
            if (rest) t += k.stage[(rest - 1) / kComputeUnits];
            t *= static_cast<double>((stages + s - 1) / s);
            if (s > 1) t += 5.0 + static_cast<double>(rows) * static_cast<double>(cols) * 8.0 * s / 4e6;
            if (t < least) least = t, best = {k.tile, s};
        }
    }
    return best;
}

inline int64_t am_partial_bytes(int64_t rows, int64_t cols, int32_t splits)
{
    return splits > 1 ? (rows * cols * splits * 4 + 255) & ~int64_t{255} : 0;
}

// The plan for operands as they lie: whole are those that are fetched straight to LDS.
inline AmPlan am_plan(const AmOperand &a, bool major_a, const AmOperand &b, bool major_b, int64_t inner, int el, int times, bool may_split)
{
    const bool whole = am_direct(a, major_a, static_cast<int32_t>(inner), el) && am_direct(b, major_b, static_cast<int32_t>(inner), el);
    return am_plan(a.extent, b.extent, inner * times, may_split, whole);
}

// Bytes that the parts of a split product take, however its operands lie.
inline int64_t am_most_partial_bytes(int64_t rows, int64_t cols, int64_t inner)
{
    const int64_t u = am_partial_bytes(rows, cols, am_plan(rows, cols, inner, true, false).splits);
    const int64_t v = am_partial_bytes(rows, cols, am_plan(rows, cols, inner, true, true).splits);
    return u > v ? u : v;
}

}  // namespace wfd
