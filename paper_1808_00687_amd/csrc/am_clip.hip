// The norm of many tensors together, and their clipping by it.
//
// Two passes: squares are summed, then values are multiplied by the factor that
// the sum gives.  Both are bound by memory.  The tensors are cut into chunks of
// 16 KB, numbered through; a workgroup takes a run of consecutive ones, so it
// looks its first tensor up once and then only steps on.  The second pass goes
// through each run backwards: what the first one read last may still be in a cache.
//
// The sum is held in 64 bits (a square of a float32 may be no float32, and a
// billion of them would lose bits): a workgroup's goes to the workspace, and every
// workgroup of the second pass adds all of them up in the same order, so there is
// no third launch and no atomic.
//
// The tensors' descriptions are arguments of the launches where they fit in
// there, and else are written to the workspace by launches of their own.
#include <algorithm>

#include "am_device.h"

namespace wfd {
namespace {

struct Tensor {
    const char *data;
    char *out;
    int64_t count;               // values
    int64_t stride, out_stride;  // elements between rows
    int64_t first;               // chunk
    int32_t cols;                // 0: rows follow one another without a gap
    int32_t type;
};

constexpr int kThreads = 256, kParts = 4;
constexpr int64_t kChunkBytes = kThreads * kParts * 16;
constexpr int64_t kMostBlocks = 256 * 8;
constexpr int kInArgs = 71;   // what fits into 4 KB of arguments with the rest

struct Table {
    Tensor t[kInArgs];
};

struct Job {
    const Tensor *table;   // in the workspace, or NULL
    double *partial;       // [blocks]
    float *norm;
    double max_norm;
    int64_t chunks;
    int32_t tensors, blocks;
};

struct FewArgs {
    Table few;
    Job job;
};
static_assert(sizeof(FewArgs) <= 4096, "");

// 16 bytes of values from value i of t on (i < count); values past the end are 0
template <typename T>
struct Piece {
    static constexpr int C = 16 / static_cast<int>(sizeof(T));
    float v[C];

    // f(index of a value here, place of it) for the values of a piece that does not lie in one run
    template <typename F>
    __device__ __forceinline__ static void each(const Tensor &t, int64_t i, int64_t stride, F f)
    {
        int64_t r = t.cols ? i / t.cols : 0, c = t.cols ? i % t.cols : i;
#pragma unroll
        for (int e = 0; e < C; e++) {
            if (i + e < t.count) f(e, r * stride + c);
            if (++c == t.cols) c = 0, r++;
        }
    }
    // where the values lie in one run: its place, else -1
    __device__ __forceinline__ static int64_t run(const Tensor &t, int64_t i, int64_t stride)
    {
        if (i + C > t.count) return -1;
        if (!t.cols) return i;
        const int64_t r = i / t.cols, c = i % t.cols;
        return c + C <= t.cols ? r * stride + c : -1;
    }
    __device__ __forceinline__ void load(const Tensor &t, int64_t i)
    {
        const T *p = reinterpret_cast<const T *>(t.data);
        const int64_t at = run(t, i, t.stride);
        if (at >= 0) {
            load_floats<T, C>(p + at, C, v);
            return;
        }
#pragma unroll
        for (int e = 0; e < C; e++) v[e] = 0.0f;
        each(t, i, t.stride, [&](int e, int64_t at) { v[e] = to_f32(((const AM_GLOBAL T *)p)[at]); });
    }
    __device__ __forceinline__ void store(const Tensor &t, int64_t i) const
    {
        T *p = reinterpret_cast<T *>(t.out);
        const int64_t at = run(t, i, t.out_stride);
        if (at >= 0) {
            store_floats<T, C>(p + at, C, v);
            return;
        }
        each(t, i, t.out_stride, [&](int e, int64_t at) { ((AM_GLOBAL T *)p)[at] = static_cast<T>(v[e]); });
    }
};

// use(the tensor as its type, first value) for the workgroup's chunks
template <bool kBackwards, typename F>
__device__ __forceinline__ void each_chunk(const Tensor *table, const Job &j, F use)
{
    const int64_t from = j.chunks * blockIdx.x / j.blocks, to = j.chunks * (blockIdx.x + 1) / j.blocks;
    if (from >= to) return;
    int lo = 0, hi = j.tensors;   // the last tensor whose first chunk is not behind the first one wanted
    const int64_t start = kBackwards ? to - 1 : from;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (table[mid].first <= start) lo = mid;
        else hi = mid;
    }
    for (int64_t n = 0; n < to - from; n++) {
        const int64_t c = kBackwards ? to - 1 - n : from + n;
        if (kBackwards) {
            if (c < table[lo].first) lo--;
        } else if (lo + 1 < j.tensors && c >= table[lo + 1].first) {
            lo++;
        }
        const Tensor &t = table[lo];
        if (t.type == WFST_F32) use(t, float{}, (c - t.first) * (kChunkBytes / 4));
        else if (t.type == WFST_F16) use(t, f16{}, (c - t.first) * (kChunkBytes / 2));
        else use(t, bf16{}, (c - t.first) * (kChunkBytes / 2));
    }
}

__device__ __forceinline__ double block_sum(double v, double (&part)[kThreads / 64])
{
#pragma unroll
    for (int s = 1; s < 64; s *= 2) v += __shfl_xor(v, s);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int w = 1; w < kThreads / 64; w++) v += part[w];
    return v;
}

__device__ __forceinline__ void square_sums(const Tensor *table, const Job &j)
{
    __shared__ double part[kThreads / 64];
    double sum = 0.0;
    each_chunk<false>(table, j, [&](const Tensor &t, auto type, int64_t first) {
        using P = Piece<decltype(type)>;
        P p[kParts];
#pragma unroll
        for (int q = 0; q < kParts; q++) {
            const int64_t i = first + (q * kThreads + static_cast<int>(threadIdx.x)) * P::C;
            if (i < t.count) p[q].load(t, i);
            else
#pragma unroll
                for (int e = 0; e < P::C; e++) p[q].v[e] = 0.0f;
        }
#pragma unroll
        for (int q = 0; q < kParts; q++)
#pragma unroll
            for (int e = 0; e < P::C; e++) {
                const double d = p[q].v[e];
                sum = fma(d, d, sum);
            }
    });
    sum = block_sum(sum, part);
    if (threadIdx.x == 0) j.partial[blockIdx.x] = sum;
}

__device__ __forceinline__ void scale_values(const Tensor *table, const Job &j)
{
    __shared__ double part[kThreads / 64];
    double sum = 0.0;
    for (int i = threadIdx.x; i < j.blocks; i += kThreads) sum += j.partial[i];
    const double norm = sqrt(block_sum(sum, part));
    if (blockIdx.x == 0 && threadIdx.x == 0) *j.norm = static_cast<float>(norm);
    const bool clipped = norm > j.max_norm;   // not with a NaN
    const double factor = clipped ? j.max_norm / norm : 1.0;
    each_chunk<true>(table, j, [&](const Tensor &t, auto type, int64_t first) {
        if (!clipped && t.out == t.data) return;
        using P = Piece<decltype(type)>;
        P p[kParts];
#pragma unroll
        for (int q = 0; q < kParts; q++) {
            const int64_t i = first + (q * kThreads + static_cast<int>(threadIdx.x)) * P::C;
            if (i < t.count) p[q].load(t, i);
        }
#pragma unroll
        for (int q = 0; q < kParts; q++) {
            const int64_t i = first + (q * kThreads + static_cast<int>(threadIdx.x)) * P::C;
            if (i >= t.count) continue;
#pragma unroll
            for (int e = 0; e < P::C; e++) p[q].v[e] = static_cast<float>(p[q].v[e] * factor);
            p[q].store(t, i);
        }
    });
}

__global__ __launch_bounds__(kThreads) void square_few_kernel(FewArgs a) { square_sums(a.few.t, a.job); }
__global__ __launch_bounds__(kThreads) void scale_few_kernel(FewArgs a) { scale_values(a.few.t, a.job); }
__global__ __launch_bounds__(kThreads) void square_kernel(Job j) { square_sums(j.table, j); }
__global__ __launch_bounds__(kThreads) void scale_kernel(Job j) { scale_values(j.table, j); }

__global__ __launch_bounds__(128) void table_kernel(Table some, Tensor *to, int32_t n)
{
    if (static_cast<int>(threadIdx.x) < n) to[threadIdx.x] = some.t[threadIdx.x];
}

// the i-th tensor's description, first chunk aside; its chunks
Tensor describe(const wfst_am_clip_args &a, int64_t i, int64_t &chunks)
{
    const wfst_matrix &g = a.grads[i], &o = a.outs ? a.outs[i] : g;
    Tensor t{};
    t.data = static_cast<const char *>(g.data);
    t.out = static_cast<char *>(o.data);
    t.count = g.rows * g.cols;
    t.stride = g.row_stride, t.out_stride = o.row_stride;
    t.type = g.type;
    const bool dense = g.rows <= 1 || (g.row_stride == g.cols && o.row_stride == g.cols);
    t.cols = dense ? 0 : static_cast<int32_t>(g.cols);
    const int64_t each = kChunkBytes / am_type_bytes(g.type);
    chunks = (t.count + each - 1) / each;
    return t;
}

int64_t table_bytes(int64_t tensors)
{
    return tensors > kInArgs ? (tensors * static_cast<int64_t>(sizeof(Tensor)) + 255) & ~int64_t{255} : 0;
}

}  // namespace

int64_t am_clip_bytes(const wfst_am_clip_args &a) { return table_bytes(a.count) + kMostBlocks * 8; }

hipError_t am_launch_clip(const wfst_am_clip_args &a, hipStream_t st)
{
    Job j{};
    j.partial = reinterpret_cast<double *>(static_cast<char *>(a.workspace) + table_bytes(a.count));
    j.norm = a.norm, j.max_norm = a.max_norm;
    const bool few = a.count <= kInArgs;
    Tensor *table = few ? nullptr : static_cast<Tensor *>(a.workspace);
    j.table = table;
    FewArgs args{};
    Table &some = args.few;
    int32_t n = 0;   // in `some`; tensors without values are left out
    for (int64_t i = 0; i < a.count; i++) {
        int64_t chunks;
        Tensor t = describe(a, i, chunks);
        if (!chunks) continue;
        t.first = j.chunks;
        j.chunks += chunks;
        some.t[n++] = t;
        if (!few && n == kInArgs) {
            table_kernel<<<1, 128, 0, st>>>(some, table + j.tensors, n);
            j.tensors += n;
            n = 0;
        }
    }
    if (!few && n) table_kernel<<<1, 128, 0, st>>>(some, table + j.tensors, n);
    j.tensors += n;
    j.blocks = static_cast<int32_t>(std::clamp<int64_t>(j.chunks, 1, kMostBlocks));
    args.job = j;
    if (few) {
        square_few_kernel<<<j.blocks, kThreads, 0, st>>>(args);
        scale_few_kernel<<<j.blocks, kThreads, 0, st>>>(args);
    } else {
        square_kernel<<<j.blocks, kThreads, 0, st>>>(j);
        scale_kernel<<<j.blocks, kThreads, 0, st>>>(j);
    }
    return hipGetLastError();
}

}  // namespace wfd
