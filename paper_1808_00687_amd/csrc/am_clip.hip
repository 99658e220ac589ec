// The norm of many tensors together, and their clipping by it.
//
// Two passes: squares are summed, then values are multiplied by the factor that
// the sum gives.  Both are bound by memory.  The tensors are cut into chunks,
// numbered through; a workgroup takes every blocks-th one and has the next one's
// loads on their way while it works on the present one.  The second pass goes
// through them backwards: what the first one read last may still be in a cache; its
// stores are not kept there.  125 tensors of 1.6 GB: 920 us, 4.9 GB in all, 5.3 TB/s (10
// more forwards, 40 more with stores that are kept); the norm alone of 1 GB: 187 us, 5.7 TB/s.
//
// Tensors whose rows have gaps are slower: each 16 bytes' row and column are a division,
// and nothing is on its way ahead.  1 GB of bf16 in rows of 8,192, 8 more apart: the
// norm 340 us, without gaps 196, with outputs 780 and 585; f32 313, 198, 719 and 580.
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

constexpr int kThreads = 256;
constexpr int64_t kMostBlocks = 256 * 8;
// Parts of 4 KB in a chunk.  The large model above takes 1,131, 1,161, 999, 920 us with 2, 4, 6, 8;
// ten tensors of 16 MB together 17 and 23 with 2 and 8, of 128 MB 69 and 73, of 256 MB 133 and 132.  So many
// from three chunks a workgroup on.
constexpr int kFewParts = 2, kManyParts = 8;
constexpr int64_t chunk_bytes(int parts) { return int64_t{kThreads} * 16 * parts; }
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
    int32_t in_place;      // all of them
};

struct FewArgs {
    Table few;
    Job job;
};
static_assert(sizeof(FewArgs) <= 4096, "");

// 16 bytes of values from value i of t on; values past the end are 0
template <typename T>
struct Piece {
    static constexpr int C = 16 / static_cast<int>(sizeof(T));
    float v[C];

    using V = T __attribute__((ext_vector_type(C)));

    __device__ __forceinline__ void take(uint32_t __attribute__((ext_vector_type(4))) raw)
    {
        const V t = __builtin_bit_cast(V, raw);
#pragma unroll
        for (int e = 0; e < C; e++) v[e] = to_f32(t[e]);
    }
    __device__ __forceinline__ uint32_t __attribute__((ext_vector_type(4))) give() const
    {
        V t;
#pragma unroll
        for (int e = 0; e < C; e++) t[e] = static_cast<T>(v[e]);
        return __builtin_bit_cast(uint32_t __attribute__((ext_vector_type(4))), t);
    }
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

using Raw = Chunk<uint32_t, 4, 1>;   // 16 bytes at any address

// A chunk of a tensor, 16 bytes a thread and part.
template <int kParts>
struct Place {
    static constexpr int64_t kBytes = chunk_bytes(kParts);
    int at;           // tensor; -1: none
    int64_t inside;   // chunk of the tensor
    int64_t run;      // bytes from this thread's first part to the end of a tensor that lies in one run, else 0

    // near: a tensor to look at first (a large one has several of a workgroup's chunks)
    __device__ __forceinline__ void find(const Tensor *table, const Job &j, int64_t c, int near)
    {
        at = -1, inside = 0, run = 0;
        if (c < 0 || c >= j.chunks) return;
        int lo = 0, hi = j.tensors;   // the last tensor whose first chunk is not behind c
        if (table[near].first > c) hi = near;
        else if (near + 1 < j.tensors && table[near + 1].first <= c) lo = near + 1;
        else lo = near, hi = near + 1;
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (table[mid].first <= c) lo = mid;
            else hi = mid;
        }
        const Tensor &t = table[lo];
        at = lo, inside = c - t.first;
        if (!t.cols) run = t.count * (t.type == WFST_F32 ? 4 : 2) - byte();
    }
    __device__ __forceinline__ int64_t byte() const { return inside * kBytes + static_cast<int64_t>(threadIdx.x) * 16; }
    // does part q lie inside the run?
    __device__ __forceinline__ bool in_run(int q) const { return run >= (q * kThreads + 1) * 16; }
    __device__ __forceinline__ void load(const Tensor *table, Raw (&r)[kParts]) const
    {
        const AM_GLOBAL char *p = (const AM_GLOBAL char *)table[at].data + byte();
#pragma unroll
        for (int q = 0; q < kParts; q++)
            if (in_run(q)) r[q] = *(const AM_GLOBAL Raw *)(p + q * kThreads * 16);
    }
};

// use(place, 16 bytes of each part that lies in a run) for the workgroup's chunks, every
// j.blocks-th one, but for tensors that are not wanted(tensor); the next one's are on
// their way meanwhile
template <int kParts, bool kBackwards, typename W, typename F>
__device__ __forceinline__ void each_chunk(const Tensor *table, const Job &j, W wanted, F use)
{
    const int64_t step = kBackwards ? -static_cast<int64_t>(j.blocks) : j.blocks;
    int64_t c = kBackwards ? j.chunks - 1 - blockIdx.x : blockIdx.x;
    Place<kParts> place, next;
    Raw r[kParts], ahead[kParts];
    place.find(table, j, c, 0);
    if (place.at >= 0 && wanted(table[place.at])) place.load(table, r);
    while (place.at >= 0) {
        c += step;
        next.find(table, j, c, place.at);
        if (next.at >= 0 && wanted(table[next.at])) next.load(table, ahead);
        if (wanted(table[place.at])) use(place, r);
        place = next;
#pragma unroll
        for (int q = 0; q < kParts; q++) r[q] = ahead[q];
    }
}

// go(type, bytes of it) with a value of the tensor's type
template <typename F>
__device__ __forceinline__ void as_type(const Tensor &t, F go)
{
    if (t.type == WFST_F32) go(float{});
    else if (t.type == WFST_F16) go(f16{});
    else go(bf16{});
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

template <int kParts>
__device__ __forceinline__ void square_sums(const Tensor *table, const Job &j)
{
    __shared__ double part[kThreads / 64];
    double sum = 0.0;
    each_chunk<kParts, false>(table, j, [](const Tensor &) { return true; }, [&](const Place<kParts> &place, const Raw (&r)[kParts]) {
        const Tensor &t = table[place.at];
        as_type(t, [&](auto type) {
            using P = Piece<decltype(type)>;
#pragma unroll
            for (int q = 0; q < kParts; q++) {
                P p;
                if (place.in_run(q)) p.take(r[q]);
                else p.load(t, place.byte() / static_cast<int64_t>(sizeof(type)) + q * kThreads * P::C);
#pragma unroll
                for (int e = 0; e < P::C; e++) {
                    const double d = p.v[e];
                    sum = fma(d, d, sum);
                }
            }
        });
    });
    sum = block_sum(sum, part);
    if (threadIdx.x == 0) j.partial[blockIdx.x] = sum;
}

template <int kParts>
__device__ __forceinline__ void scale_values(const Tensor *table, const Job &j)
{
    __shared__ double part[kThreads / 64];
    double sum = 0.0;
    for (int i = threadIdx.x; i < j.blocks; i += kThreads) sum += j.partial[i];
    const double norm = sqrt(block_sum(sum, part));
    if (blockIdx.x == 0 && threadIdx.x == 0) *j.norm = static_cast<float>(norm);
    const bool clipped = norm > j.max_norm;   // not with a NaN
    const double factor = clipped ? j.max_norm / norm : 1.0;
    if (!clipped && j.in_place) return;
    each_chunk<kParts, true>(table, j, [&](const Tensor &t) { return clipped || t.out != t.data; }, [&](const Place<kParts> &place, const Raw (&r)[kParts]) {
        const Tensor &t = table[place.at];
        as_type(t, [&](auto type) {
            using P = Piece<decltype(type)>;
#pragma unroll
            for (int q = 0; q < kParts; q++) {
                P p;
                const int64_t i = place.byte() / static_cast<int64_t>(sizeof(type)) + q * kThreads * P::C;
                if (place.in_run(q)) p.take(r[q]);
                else p.load(t, i);
#pragma unroll
                for (int e = 0; e < P::C; e++) p.v[e] = static_cast<float>(p.v[e] * factor);
                if (place.in_run(q)) __builtin_nontemporal_store(p.give(), (AM_GLOBAL Raw *)((AM_GLOBAL char *)t.out + place.byte() + q * kThreads * 16));
                else p.store(t, i);
            }
        });
    });
}

template <int kParts>
__global__ __launch_bounds__(kThreads) void square_few_kernel(FewArgs a)
{
    square_sums<kParts>(a.few.t, a.job);
}
template <int kParts>
__global__ __launch_bounds__(kThreads) void scale_few_kernel(FewArgs a)
{
    scale_values<kParts>(a.few.t, a.job);
}
template <int kParts>
__global__ __launch_bounds__(kThreads) void square_kernel(Job j)
{
    square_sums<kParts>(j.table, j);
}
template <int kParts>
__global__ __launch_bounds__(kThreads) void scale_kernel(Job j)
{
    scale_values<kParts>(j.table, j);
}

__global__ __launch_bounds__(128) void table_kernel(Table some, Tensor *to, int32_t n)
{
    if (static_cast<int>(threadIdx.x) < n) to[threadIdx.x] = some.t[threadIdx.x];
}

// the i-th tensor's description, first chunk aside
Tensor describe(const wfst_am_clip_args &a, int64_t i)
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
    return t;
}

int64_t chunks_of(const wfst_matrix &g, int parts)
{
    const int64_t each = chunk_bytes(parts) / am_type_bytes(g.type);
    return (g.rows * g.cols + each - 1) / each;
}

int64_t table_bytes(int64_t tensors)
{
    return tensors > kInArgs ? (tensors * static_cast<int64_t>(sizeof(Tensor)) + 255) & ~int64_t{255} : 0;
}

template <int kParts>
void launch(const wfst_am_clip_args &a, hipStream_t st)
{
    Job j{};
    j.partial = reinterpret_cast<double *>(static_cast<char *>(a.workspace) + table_bytes(a.count));
    j.norm = a.norm, j.max_norm = a.max_norm;
    j.in_place = !a.outs;
    const bool few = a.count <= kInArgs;
    Tensor *table = few ? nullptr : static_cast<Tensor *>(a.workspace);
    j.table = table;
    FewArgs args{};
    Table &some = args.few;
    int32_t n = 0;   // in `some`; tensors without values are left out
    for (int64_t i = 0; i < a.count; i++) {
        const int64_t chunks = chunks_of(a.grads[i], kParts);
        if (!chunks) continue;
        some.t[n] = describe(a, i);
        some.t[n++].first = j.chunks;
        j.chunks += chunks;
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
        square_few_kernel<kParts><<<j.blocks, kThreads, 0, st>>>(args);
        scale_few_kernel<kParts><<<j.blocks, kThreads, 0, st>>>(args);
    } else {
        square_kernel<kParts><<<j.blocks, kThreads, 0, st>>>(j);
        scale_kernel<kParts><<<j.blocks, kThreads, 0, st>>>(j);
    }
}

}  // namespace

int64_t am_clip_bytes(const wfst_am_clip_args &a) { return table_bytes(a.count) + kMostBlocks * 8; }

hipError_t am_launch_clip(const wfst_am_clip_args &a, hipStream_t st)
{
    int64_t chunks = 0;
    for (int64_t i = 0; i < a.count; i++) chunks += chunks_of(a.grads[i], kManyParts);
    if (chunks >= 3 * kMostBlocks) launch<kManyParts>(a, st);
    else launch<kFewParts>(a, st);
    return hipGetLastError();
}

}  // namespace wfd
