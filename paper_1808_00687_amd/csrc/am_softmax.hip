// Row operators that end in a softmax over the units: the distillation loss
// with its gradient, and log-likelihood rows.
//
// Bound by memory: a row is read once into registers; each wave takes its
// maximum and the sum of exponentials relative to it, and the waves' pairs are
// joined (a row's log sum exp in one barrier).  The teacher's entries of a row
// belong to its first wave; each is handed, by a list in LDS, to the thread that
// holds its unit, so that every gradient is written once, whole.
#include "am_rows.h"

namespace wfd {
namespace {

template <typename T>
__device__ __forceinline__ const T *row(const wfst_matrix &m, int64_t r)
{
    return static_cast<const T *>(m.data) + r * m.row_stride;
}

// log sum exp over a row; get(v, c, left, x) gives a chunk, already divided by
// the temperature, -inf beyond the row.  -inf for a row of -inf.
template <typename S, typename G>
__device__ __forceinline__ float row_lse(int64_t cols, int t, G get, RowScratch &r, int &turn)
{
    float top = -INFINITY;
    S::each(cols, t, [&](int v, int64_t c, int64_t left) {
        float x[S::kC];
        get(v, c, left, x);
#pragma unroll
        for (int e = 0; e < S::kC; e++) top = fmaxf(top, x[e]);
    });
    top = wave_max(top);
    float shift = top == -INFINITY ? 0.0f : top;
    float s = 0.0f;
    S::each(cols, t, [&](int v, int64_t c, int64_t left) {
        float x[S::kC];
        get(v, c, left, x);
#pragma unroll
        for (int e = 0; e < S::kC; e++) s += am_exp(x[e] - shift);
    });
    s = wave_sum(s);
    if constexpr (S::kWaves > 1) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) r.a[turn][wave] = top, r.b[turn][wave] = s;
        __syncthreads();
        top = r.a[turn][0];
#pragma unroll
        for (int i = 1; i < S::kWaves; i++) top = fmaxf(top, r.a[turn][i]);
        shift = top == -INFINITY ? 0.0f : top;
        s = 0.0f;
#pragma unroll
        for (int i = 0; i < S::kWaves; i++) s += r.a[turn][i] == -INFINITY ? r.b[turn][i] : r.b[turn][i] * am_exp(r.a[turn][i] - shift);
        turn ^= 1;
    }
    return shift + logf(s);
}

template <typename T, typename S>
__global__ __launch_bounds__(S::kThreads) void loglikes_kernel(wfst_am_loglikes_args a)
{
    __shared__ RowScratch scratch;
    int turn = 0;
    const int64_t M = a.logits.rows, L = a.logits.cols, step = static_cast<int64_t>(gridDim.x) * S::kRows;
    const int t = threadIdx.x % S::kTpr;
    RowPart<S, float> prior;
    if (a.log_prior) prior.hold(a.log_prior, L, t);
    RowPart<S, T> x, next;
    const T low = static_cast<T>(-INFINITY);
    int64_t m = static_cast<int64_t>(blockIdx.x) * S::kRows + threadIdx.x / S::kTpr;
    if (m < M) next.hold(row<T>(a.logits, m), L, t, low);
    for (; m < M; m += step) {
        x = next;
        if (m + step < M) next.hold(row<T>(a.logits, m + step), L, t, low);   // on its way while this row is worked on
        float *ll = static_cast<float *>(a.ll.data) + m * a.ll.row_stride;
        const float lse = row_lse<S>(L, t, [&](int v, int64_t c, int64_t left, float (&o)[S::kC]) {
            x.get(v, c, left, o, -INFINITY);
        }, scratch, turn);
        S::each(L, t, [&](int v, int64_t c, int64_t left) {
            float o[S::kC], p[S::kC] = {};
            x.get(v, c, left, o);
            if (a.log_prior) prior.get(v, c, left, p);
#pragma unroll
            for (int e = 0; e < S::kC; e++)
                o[e] = o[e] == -INFINITY || p[e] == -INFINITY ? -INFINITY : a.scale * ((o[e] - lse) - p[e]);
            store_floats(ll + c, left, o);
        });
    }
}

__device__ __forceinline__ float load_any(const wfst_matrix &m, int64_t r, int64_t c)
{
    const int64_t at = r * m.row_stride + c;
    return m.type == WFST_F32   ? static_cast<const float *>(m.data)[at]
           : m.type == WFST_F16 ? to_f32(static_cast<const f16 *>(m.data)[at])
                                : to_f32(static_cast<const bf16 *>(m.data)[at]);
}

constexpr int kEntries = WFST_AM_MAX_TOP / 64;   // a lane's

// The teacher's entries of one row, in LDS
struct Entries {
    int32_t unit[WFST_AM_MAX_TOP];   // -1: not used
    float share[WFST_AM_MAX_TOP];    // p_j
    float mass[WFST_AM_MAX_TOP];     // the unit's whole share, at its first entry
    int32_t next[WFST_AM_MAX_TOP];
};

// orders a wave's LDS accesses
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup", "local");
    __builtin_amdgcn_wave_barrier();
}

template <typename T, typename S, bool kBackward>
__global__ __launch_bounds__(S::kThreads) void distill_kernel(wfst_am_distill_args a)
{
    __shared__ RowScratch scratch;
    __shared__ Entries tables[S::kRows];
    __shared__ int32_t heads[S::kRows][S::kTpr];   // a thread's first entry
    __shared__ int32_t some[S::kRows];
    int turn = 0;
    const int64_t M = a.logits.rows, L = a.logits.cols;
    const int k = static_cast<int>(a.top_logit.cols), t = threadIdx.x % S::kTpr, sub = threadIdx.x / S::kTpr;
    const float temp = a.temperature, inv_t = 1.0f / temp;
    const int64_t step = static_cast<int64_t>(gridDim.x) * S::kRows;
    const T low = static_cast<T>(-INFINITY);
    Entries &tab = tables[sub];
    RowPart<S, T> x, next;
    int64_t m = static_cast<int64_t>(blockIdx.x) * S::kRows + sub;
    if (m < M) next.hold(row<T>(a.logits, m), L, t, low);
    for (; m < M; m += step) {
        const T *x_row = row<T>(a.logits, m);
        T *d = a.dlogits.data ? static_cast<T *>(a.dlogits.data) + m * a.dlogits.row_stride : nullptr;
        x = next;
        if (m + step < M) next.hold(row<T>(a.logits, m + step), L, t, low);   // on its way while this row is worked on
        const auto get_x = [&](int v, int64_t c, int64_t left, float (&o)[S::kC]) {
            x.get(v, c, left, o, -INFINITY);
#pragma unroll
            for (int e = 0; e < S::kC; e++) o[e] *= inv_t;
        };
        const float w = a.weight ? a.weight[m] : 1.0f;

        // the entries: shares, and for each unit one list entry with its whole mass
        int32_t unit[kEntries];
        float top[kEntries], share[kEntries], at_unit[kEntries], log_z = 0.0f;
        heads[sub][t] = -1;
        if (t < 64 && w != 0.0f) {
            float best = -INFINITY;
#pragma unroll
            for (int i = 0; i < kEntries; i++) {
                const int j = i * 64 + t;
                unit[i] = -1, top[i] = -INFINITY, share[i] = 0.0f, at_unit[i] = 0.0f;
                if (i * 64 >= k || j >= k) continue;
                const int32_t u = a.top_index[m * k + j];
                const float v = load_any(a.top_logit, m, j) * inv_t;
                if (u < 0 || u >= L || v == -INFINITY) continue;
                unit[i] = u, top[i] = v;
                at_unit[i] = to_f32(x_row[u]) * inv_t;
            }
#pragma unroll
            for (int i = 0; i < kEntries; i++) best = fmaxf(best, top[i]);
            best = wave_max(best);
            float z = 0.0f;
            bool used = false;
#pragma unroll
            for (int i = 0; i < kEntries; i++) {
                if (unit[i] < 0) continue;
                used = true;
                top[i] -= best;
                share[i] = am_exp(top[i]);
                z += share[i];
            }
            z = wave_sum(z);
            log_z = logf(z);
            if (t == 0) some[sub] = 0;
            wave_sync();
            if (used) some[sub] = 1;
#pragma unroll
            for (int i = 0; i < kEntries; i++) {
                if (i * 64 >= k) continue;
                share[i] = unit[i] < 0 ? 0.0f : share[i] / z;
                tab.unit[i * 64 + t] = unit[i];
                tab.share[i * 64 + t] = share[i];
            }
        } else if (t == 0) {
            some[sub] = 0;
        }
        if constexpr (S::kWaves > 1) __syncthreads();
        else wave_sync();
        if (t < 64 && w != 0.0f && d) {
#pragma unroll
            for (int i = 0; i < kEntries; i++) {
                if (i * 64 >= k || unit[i] < 0) continue;
                const int j = i * 64 + t;
                float mass = 0.0f;
                bool first = true;
                for (int o = 0; o < k; o++)
                    if (tab.unit[o] == unit[i]) {
                        first = first && o >= j;
                        mass += tab.share[o];
                    }
                if (!first) continue;
                tab.mass[j] = mass;
                tab.next[j] = atomicExch(&heads[sub][unit[i] / S::kC % S::kTpr], j);
            }
        }
        // every x of a unit is in registers, and the entries are in place, before dlogits may overwrite a row
        if constexpr (S::kWaves > 1) __syncthreads();
        else wave_sync();
        const bool live = w != 0.0f && some[sub] != 0;

        float lse = 0.0f;
        if constexpr (kBackward) lse = a.lse[m];
        else if (live || a.lse) lse = row_lse<S>(L, t, get_x, scratch, turn);
        if constexpr (!kBackward) {
            if (a.lse && t == 0) a.lse[m] = lse;
            if (a.loss && t < 64) {
                float sum = 0.0f;
                if (live)
#pragma unroll
                    for (int i = 0; i < kEntries; i++)   // a masked unit whose share has underflowed is worth nothing
                        if (share[i] != 0.0f) sum += share[i] * ((top[i] - log_z) - (at_unit[i] - lse));
                sum = wave_sum(sum);
                if (t == 0) a.loss[m] = live ? w * temp * temp * sum : 0.0f;
            }
        }
        if (d) {
            const float scale = w * temp;
            if (live) {
                S::each(L, t, [&](int v, int64_t c, int64_t left) {
                    float g[S::kC];
                    get_x(v, c, left, g);
#pragma unroll
                    for (int e = 0; e < S::kC; e++) g[e] = am_exp(g[e] - lse);
                    for (int j = heads[sub][t]; j >= 0; j = tab.next[j]) {
                        const int64_t at = tab.unit[j] - c;
#pragma unroll
                        for (int e = 0; e < S::kC; e++) g[e] -= at == e ? tab.mass[j] : 0.0f;
                    }
#pragma unroll
                    for (int e = 0; e < S::kC; e++) g[e] *= scale;
                    store_floats(d + c, left, g);
                });
            } else {
                const float zero[S::kC] = {};
                for (int64_t c = static_cast<int64_t>(t) * S::kC; c < L; c += S::kTpr * S::kC) store_floats(d + c, L - c, zero);
            }
        }
        // the tables are written again for the next row
        if constexpr (S::kWaves > 1) __syncthreads();
        else wave_sync();
    }
}

constexpr int64_t kBlocks = 256 * 8;

template <typename T>
void launch_loglikes(const wfst_am_loglikes_args &a, hipStream_t st)
{
    am_row_shape<4>(a.logits.cols, [&](auto shape) {
        using S = decltype(shape);
        loglikes_kernel<T, S><<<am_row_blocks<S>(a.logits.rows, kBlocks), S::kThreads, 0, st>>>(a);
    });
}

template <typename T>
void launch_distill(const wfst_am_distill_args &a, bool backward, hipStream_t st)
{
    am_row_shape<sizeof(T) == 4 ? 4 : 8>(a.logits.cols, [&](auto shape) {
        using S = decltype(shape);
        const unsigned g = am_row_blocks<S>(a.logits.rows, kBlocks);
        if (backward) distill_kernel<T, S, true><<<g, S::kThreads, 0, st>>>(a);
        else distill_kernel<T, S, false><<<g, S::kThreads, 0, st>>>(a);
    });
}

}  // namespace

hipError_t am_launch_distill(const wfst_am_distill_args &a, bool backward, hipStream_t st)
{
    if (a.logits.type == WFST_F32) launch_distill<float>(a, backward, st);
    else if (a.logits.type == WFST_F16) launch_distill<f16>(a, backward, st);
    else launch_distill<bf16>(a, backward, st);
    return hipGetLastError();
}

hipError_t am_launch_loglikes(const wfst_am_loglikes_args &a, hipStream_t st)
{
    if (a.logits.type == WFST_F32) launch_loglikes<float>(a, st);
    else if (a.logits.type == WFST_F16) launch_loglikes<f16>(a, st);
    else launch_loglikes<bf16>(a, st);
    return hipGetLastError();
}

}  // namespace wfd
