// Distillation from a teacher's top logits: loss and gradient, or the gradient
// alone.
//
// Bound by memory: a row is read once into registers and its gradient written
// from there; between them lie the row's softmax statistics (one barrier).  The
// teacher's entries of a row belong to its first wave; each is handed, by a list
// in LDS, to the thread that holds its unit, so that every gradient is written
// once, whole.
//
// (16384, 6000) bf16, 20 entries, loss and gradient: 105 us, 395 MB, 3.8 TB/s; what
// is over a copy's 77 us is the chain of a row: the entries, two reductions over a
// wave, the barrier (waves wait 64% of their time).  The exponentials are kept between the statistics and the
// gradient (recomputed, the row's arithmetic alone would take half as long again).
#include "am_softmax.h"

namespace wfd {
namespace {

__device__ __forceinline__ float load_any(const wfst_matrix &m, int64_t r, int64_t c)
{
    const int64_t at = r * m.row_stride + c;
    return m.type == WFST_F32   ? static_cast<const float *>(m.data)[at]
           : m.type == WFST_F16 ? to_f32(static_cast<const f16 *>(m.data)[at])
                                : to_f32(static_cast<const bf16 *>(m.data)[at]);
}

// The teacher's used entries of one row, in LDS: a list for each thread that
// holds one of their units.
template <int kEntries>
struct Entries {
    int32_t unit[kEntries * 64];
    float mass[kEntries * 64];       // the unit's whole share, at its first entry
    int32_t next[kEntries * 64];
    int32_t used;
};

// orders a wave's LDS accesses
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup", "local");
    __builtin_amdgcn_wave_barrier();
}

// kEntries: entries a lane of the row's first wave takes care of
template <typename T, typename S, bool kBackward, int kEntries>
__global__ __launch_bounds__(S::kThreads, kBackward && S::kTpr == 1024 && S::kNv * S::kC <= 16 ? 8 : 1) void distill_kernel(wfst_am_distill_args a)
{
    __shared__ RowScratch scratch;
    // Two sets, used in turn: the first wave fills one for its next row while
    // the others may still read the other.  A set comes round again only after
    // the barrier of the row between.
    __shared__ Entries<kEntries> tables[S::kRows][2];
    __shared__ int32_t heads[S::kRows][2][S::kTpr];   // a thread's first entry; -1 outside its row
    int turn = 0, set = 0;
    const int64_t M = a.logits.rows, L = a.logits.cols, step = static_cast<int64_t>(gridDim.x) * S::kRows;
    const int k = static_cast<int>(a.top_logit.cols), t = threadIdx.x % S::kTpr, sub = threadIdx.x / S::kTpr;
    const float temp = a.temperature, inv_t = 1.0f / temp, c2 = inv_t * kLog2e;
    const T low = static_cast<T>(-INFINITY);
    heads[sub][0][t] = heads[sub][1][t] = -1;
    if constexpr (S::kWaves > 1) __syncthreads();

    // what a row needs from memory is fetched while the row before it is worked on
    // (a forward row's logits give way to their exponentials, and the next row's
    // are fetched in their place; the other forms keep them to the end)
    constexpr bool kKeep = !kBackward && S::kNv > 0;
    RowPart<S, T> x, next;
    int32_t unit[kEntries], unit_next[kEntries];
    float top[kEntries], top_next[kEntries], at_unit[kEntries], at_next[kEntries];
    const auto hold_row = [&](int64_t r) {
        if (r < M) (kKeep ? x : next).hold(row<T>(a.logits, r), L, t, low);
    };
    const auto hold = [&](int64_t r) {
        if (r >= M || t >= 64) return;
#pragma unroll
        for (int i = 0; i < kEntries; i++) {
            const int j = i * 64 + t;
            if (i * 64 >= k) continue;
            unit_next[i] = j < k ? a.top_index[r * k + j] : -1;
            top_next[i] = j < k ? load_any(a.top_logit, r, j) : -INFINITY;
        }
    };
    const auto hold_units = [&](int64_t r) {
        if (r >= M || t >= 64 || kBackward) return;
#pragma unroll
        for (int i = 0; i < kEntries; i++)
            if (i * 64 < k && unit_next[i] >= 0 && unit_next[i] < L) at_next[i] = to_f32(row<T>(a.logits, r)[unit_next[i]]);
    };

    int64_t m = static_cast<int64_t>(blockIdx.x) * S::kRows + sub;
    hold_row(m);
    hold(m);
    hold_units(m);
    for (; m < M; m += step) {
        if constexpr (!kKeep) {
            x = next;
            hold_row(m + step);
        }
#pragma unroll
        for (int i = 0; i < kEntries; i++) unit[i] = unit_next[i], top[i] = top_next[i], at_unit[i] = at_next[i];
        hold(m + step);
        T *d = a.dlogits.data ? static_cast<T *>(a.dlogits.data) + m * a.dlogits.row_stride : nullptr;
        const auto get_x = [&](int v, int64_t c, int64_t left, float (&o)[S::kC]) { x.get(v, c, left, o, -INFINITY); };
        const float w = a.weight ? a.weight[m] : 1.0f;
        Entries<kEntries> &tab = tables[sub][set];
        int32_t &head = heads[sub][set][t];

        // the entries: shares, and for each unit one list entry with its whole mass
        float share[kEntries], log_z = 0.0f;
        if (t < 64 && w != 0.0f) {
            float best = -INFINITY, z = 0.0f;
            bool used = false;
#pragma unroll
            for (int i = 0; i < kEntries; i++) {
                if (i * 64 >= k || unit[i] < 0 || unit[i] >= L || top[i] == -INFINITY) unit[i] = -1;
                else best = fmaxf(best, top[i]);
            }
            best = wave_max(best);
#pragma unroll
            for (int i = 0; i < kEntries; i++) {
                share[i] = 0.0f;
                if (unit[i] < 0) continue;
                used = true;
                top[i] = (top[i] - best) * inv_t;
                share[i] = am_exp(top[i]);
                z += share[i];
            }
            z = wave_sum(z);
            log_z = logf(z);
            const bool any = __builtin_amdgcn_ballot_w64(used) != 0;
            if (t == 0) tab.used = any;
#pragma unroll
            for (int i = 0; i < kEntries; i++) share[i] = unit[i] < 0 ? 0.0f : share[i] / z;
            if (d) {
                // a unit's whole share, from the entries in order; they go round the wave by lane reads
                float mass[kEntries] = {};
                int32_t before[kEntries] = {};   // earlier entries of the same unit
#pragma unroll
                for (int o = 0; o < kEntries; o++) {
                    const int n = k - o * 64 < 64 ? k - o * 64 : 64;
                    for (int l = 0; l < n; l++) {
                        const int32_t u = __builtin_amdgcn_readlane(unit[o], l);
                        const float p = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(share[o]), l));
                        const int32_t j = o * 64 + l;
#pragma unroll
                        for (int i = 0; i < kEntries; i++) {
                            const bool same = unit[i] == u;
                            mass[i] += same ? p : 0.0f;
                            before[i] += same && j < i * 64 + t ? 1 : 0;
                        }
                    }
                }
                bool first[kEntries];
#pragma unroll
                for (int i = 0; i < kEntries; i++) first[i] = unit[i] >= 0 && before[i] == 0;
#pragma unroll
                for (int i = 0; i < kEntries; i++)
                    if (first[i]) {
                        const int j = i * 64 + t;
                        tab.unit[j] = unit[i];
                        tab.mass[j] = mass[i];
                        tab.next[j] = atomicExch(&heads[sub][set][unit[i] / S::kC % S::kTpr], j);
                    }
            }
        }

        // The row's statistics; their barrier also hands the entries over, and
        // comes after the last read of the row from memory.
        float kept[S::kHeld][S::kC];
        RowStat stat{0.0f, 0.0f, 1.0f};
        float lse = 0.0f, log_sum = 0.0f;
        if constexpr (kBackward) {
            lse = a.lse[m];
            if (w != 0.0f) {
                if constexpr (S::kWaves > 1) __syncthreads();
            }
        } else if (w != 0.0f || a.lse) {
            stat = row_stat<S>(L, t, c2, get_x, [&](int v, const float (&e)[S::kC]) {
                if constexpr (S::kNv > 0)
#pragma unroll
                    for (int i = 0; i < S::kC; i++) kept[v][i] = e[i];
            }, scratch, turn);
            log_sum = logf(stat.sum);
            if (a.lse && t == 0) a.lse[m] = lse_of(stat, inv_t);
        }
        if constexpr (kKeep) hold_row(m + step);
        if constexpr (S::kWaves == 1) wave_sync();
        const bool live = w != 0.0f && tab.used;
        if constexpr (!kBackward)
            if (a.loss && t < 64) {
                float sum = 0.0f;
                if (live)
#pragma unroll
                    for (int i = 0; i < kEntries; i++)   // a masked unit whose share has underflowed is worth nothing
                        if (share[i] != 0.0f) sum += w * temp * share[i] * (temp * ((top[i] - log_z) + log_sum) - (at_unit[i] - stat.top));
                sum = wave_sum(sum);
                if (t == 0) a.loss[m] = live ? sum : 0.0f;
            }
        if (d) {
            const float scale = w * temp;
            // q = e^((x - own) / temperature) * over (kept), e^((x - top) / temperature) * over, or e^(x / temperature - lse)
            const float over = scale * ((kKeep ? __builtin_amdgcn_exp2f((stat.own - stat.top) * c2) : 1.0f) / stat.sum);
            if (live) {
                const int32_t own = head;
                S::each(L, t, [&](int v, int64_t c, int64_t left) {
                    float g[S::kC];
                    if constexpr (kKeep) {
#pragma unroll
                        for (int e = 0; e < S::kC; e++) g[e] = kept[v][e] * over;
                    } else {
                        get_x(v, c, left, g);
#pragma unroll
                        for (int e = 0; e < S::kC; e++)
                            g[e] = kBackward ? scale * am_exp(tempered(g[e], inv_t) - lse) : __builtin_amdgcn_exp2f((g[e] - stat.top) * c2) * over;
                    }
                    for (int j = own; j >= 0; j = tab.next[j]) {
                        const int64_t at = tab.unit[j] - c;
                        const float mass = tab.mass[j] * scale;
#pragma unroll
                        for (int e = 0; e < S::kC; e++) g[e] -= at == e ? mass : 0.0f;
                    }
                    store_floats(d + c, left, g);
                });
                head = -1;
            } else {
                const float zero[S::kC] = {};
                for (int64_t c = static_cast<int64_t>(t) * S::kC; c < L; c += S::kTpr * S::kC) store_floats(d + c, L - c, zero);
            }
        }
        hold_units(m + step);
        if (w != 0.0f) set ^= 1;
    }
}

template <typename T>
void launch(const wfst_am_distill_args &a, bool backward, hipStream_t st)
{
    am_row_shape<sizeof(T) == 4 ? 4 : 8>(a.logits.cols, [&](auto shape) {
        using S = decltype(shape);
        constexpr int kMost = WFST_AM_MAX_TOP / 64;
        const unsigned g = am_row_blocks<S>(a.logits.rows, kSoftmaxBlocks);
        if (a.top_logit.cols <= 64) {
            if (backward) distill_kernel<T, S, true, 1><<<g, S::kThreads, 0, st>>>(a);
            else distill_kernel<T, S, false, 1><<<g, S::kThreads, 0, st>>>(a);
        } else {
            if (backward) distill_kernel<T, S, true, kMost><<<g, S::kThreads, 0, st>>>(a);
            else distill_kernel<T, S, false, kMost><<<g, S::kThreads, 0, st>>>(a);
        }
    });
}

}  // namespace

hipError_t am_launch_distill(const wfst_am_distill_args &a, bool backward, hipStream_t st)
{
    if (a.logits.type == WFST_F32) launch<float>(a, backward, st);
    else if (a.logits.type == WFST_F16) launch<f16>(a, backward, st);
    else launch<bf16>(a, backward, st);
    return hipGetLastError();
}

}  // namespace wfd
