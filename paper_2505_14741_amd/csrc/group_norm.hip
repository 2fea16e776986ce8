// Group norm over channels-last positions with an activation: a group is channels / groups neighbouring channels of one sample over all
// positions; y = (x - mean) / sqrt(var + eps) * gamma + beta, then none, tanh-GELU or SiLU.
//
// Reading x twice and writing it once is what binds.  70200 positions of 512 channels, 32 groups, SiLU, bf16 (72 MB): 14 us for the
// moments (5.2 TB/s) and 25 for the result (5.8 TB/s, beyond a device copy's rate; the second read comes from the last-level cache).  2 x 345
// positions of 320 channels, fp32, in one launch 9 us, all of it latency.  A workgroup takes a slice of whole groups (about 64 channels, so that a position is
// a whole cache line or two) over a chunk of positions.  Means and squared deviations are merged pairwise, (n, mean, M2) with
// (n', mean', M2'), from single values on: exact where the mean is far larger than the deviations, whatever the first values are.
#include "few_epilogue.h"
#include "group_norm.h"
#include "lane_sums.h"
#include "plan.h"
#include <type_traits>

namespace ps {

// over `team` neighbouring lanes (a power of two up to 64), in all of them
__device__ __forceinline__ float team_sum(float v, int team) {
    if (team == 64) return sum_of_64(v);
    for (int x = team / 2; x > 0; x /= 2) v += __shfl_xor(v, x);
    return v;
}

// Mean and M2 of the union of the items (n, (mean, M2)) that `each` gives this lane of a team: first the mean, as the mean distance from
// `pivot` (any item's), then M2 = sum of M2_i + n_i (mean_i - mean)^2.  No division but one, and the items' reads do not wait on each other.
constexpr int SINGLE_THREADS = 1024;                     // of the workgroup that does a slice alone
struct Moments { float n, mean, m2; };
template <typename Each>
__device__ __forceinline__ Moments united(const Each& each, float pivot, int team) {
    float n = 0.f, s = 0.f;
    each([&](float ni, float2 w) {
        n += ni;
        s = __builtin_fmaf(ni, w.x - pivot, s);
    });
    n = team_sum(n, team);
    const float mean = pivot + team_sum(s, team) / n;
    float m2 = 0.f;
    each([&](float ni, float2 w) {
        const float d = w.x - mean;
        m2 += __builtin_fmaf(ni * d, d, w.y);
    });
    return Moments{n, mean, team_sum(m2, team)};
}
__device__ __forceinline__ Moments merged(Moments a, Moments b) {
    const float n = a.n + b.n, d = b.mean - a.mean, w = b.n / n;
    return Moments{n, __builtin_fmaf(d, w, a.mean), a.m2 + b.m2 + d * d * (a.n * w)};
}

__device__ __forceinline__ float silu_of(float x, float) { return silu_f(x); }
__device__ __forceinline__ float silu_of(float x, bf16_t) {      // rounded to bf16 behind: two transcendentals
    return x * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * -1.4426950408889634f));
}
template <typename T, int ACT> __device__ __forceinline__ float activated(float x) {
    if constexpr (ACT == 1) return gelu_of(x, T{});
    else if constexpr (ACT == 2) return silu_of(x, T{});
    else return x;
}

// V channels, and the same in memory: at any element's address (element by element 17550 x 320 bf16 one element into rows of 321
// took 30 us, so 19; aligned 18)
template <typename T> struct ElemOf { typedef typename std::conditional<sizeof(T) == 4, float, __bf16>::type type; };
template <typename T, int V> struct ChannelsOf;
template <int V> struct ChannelsOf<float, V> {
    typedef __attribute__((ext_vector_type(V))) float type;
    typedef type mem __attribute__((aligned(4)));
};
template <int V> struct ChannelsOf<bf16_t, V> {
    typedef __attribute__((ext_vector_type(V))) __bf16 type;
    typedef type mem __attribute__((aligned(2)));
};
template <> struct ChannelsOf<float, 1> { typedef float type, mem; };
template <> struct ChannelsOf<bf16_t, 1> { typedef __bf16 type, mem; };
template <typename T, int V>
__device__ __forceinline__ void widen(const typename ChannelsOf<T, V>::type& w, float (&v)[V]) {
    if constexpr (V == 1) v[0] = (float)w;
    else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = (float)w[i];
    }
}
template <typename T, int V>
__device__ __forceinline__ void store_channels(T* p, const float (&v)[V], bool stream) {
    typename ChannelsOf<T, V>::type w;
    if constexpr (V == 1) w = (typename ElemOf<T>::type)v[0];
    else {
#pragma unroll
        for (int i = 0; i < V; ++i) w[i] = (typename ElemOf<T>::type)v[i];
    }
    store_streamed<sizeof(T)>(p, w, stream);
}

// PHASE 0: moments of the chunk's groups to a.part; 1: moments of all chunks from a.part, then the result; 2: both, one chunk.
// NT threads: `lanes` threads side by side hold the slice's channels, V each, NT / lanes positions at a time (rows); a slice of more
// than NT * V channels is walked in columns of NT * V.  A thread keeps a running mean and M2 of each of its channels; they meet in
// LDS, where `team` threads per group unite its rows x channels.  A single chunk that one batch of loads holds is read once.
template <typename T, int V, int PHASE, int ACT, int U, int NT>      // U: positions in flight per thread
__global__ void __launch_bounds__(NT)
group_norm_kernel(GroupNormArgs a, GroupNormPlan p) {
    typedef typename ChannelsOf<T, V>::type vec_t;
    typedef typename ChannelsOf<T, V>::mem mem_t;
    __shared__ float2 sums[PHASE == 1 ? 1 : NT * V + 2 * NT];     // mean, M2: rows of lanes * V channels and a fill (see p.fill)
    __shared__ float2 stats[GROUP_NORM_SLICE_GROUPS];    // mean, 1 / sqrt(var + eps)
    const int chunk = blockIdx.x, slice = blockIdx.y, b = blockIdx.z;
    const int cpg = p.cpg, g0 = slice * p.slice_groups, ng = min(p.slice_groups, a.groups - g0);
    const int c0 = g0 * cpg, nc = ng * cpg, vecs = nc / V;
    const int s0 = chunk * p.per, s1 = min(s0 + p.per, a.positions);
    const int lanes = p.lanes, rows = p.rows, team = p.team, stride = lanes * V + p.fill;
    const int myrow = (int)(threadIdx.x * p.lanes_inv >> 20), my = threadIdx.x - myrow * lanes;
    const bool active = myrow < rows;
    const int tg = threadIdx.x >> __builtin_ctz(team), tl = threadIdx.x & (team - 1);
    const T* x = (const T*)a.x + b * a.x_batch + c0;
    T* o = (T*)a.out + b * a.o_batch + c0;
    vec_t batch[U];                                      // positions past the chunk repeat the last one and do not count
    const long step = rows * a.x_position;
    // (past the chunk: repeats the last position; without these, the scheduler would move loads behind their first use to save registers)
    auto fetch = [&](const T* q, int s) {
        const T* at = q + s * a.x_position;
        if (s + (U - 1) * rows < s1) {
#pragma unroll
            for (int u = 0; u < U; ++u) batch[u] = *reinterpret_cast<const mem_t*>(at + u * step);
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) batch[u] = *reinterpret_cast<const mem_t*>(q + min(s + u * rows, s1 - 1) * a.x_position);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // what multiplies and follows a column of V channels, without the statistics
    typedef typename ChannelsOf<float, V>::type affine_t;
    typedef typename ChannelsOf<float, V>::mem affine_mem_t;
    affine_t gamma, beta;
    auto fetch_affine = [&](int col) {
        gamma = affine_t{} + 1.f;
        beta = affine_t{};
        if (a.gamma) gamma = *reinterpret_cast<const affine_mem_t*>(a.gamma + c0 + col * V);
        if (a.beta) beta = *reinterpret_cast<const affine_mem_t*>(a.beta + c0 + col * V);
    };

    Moments t{0.f, 0.f, 0.f};                            // of group tg
    if constexpr (PHASE != 0) fetch_affine(my < vecs ? my : 0);      // (now, not when the statistics are there)
    if constexpr (PHASE != 1) {
        for (int col = 0; col < vecs; col += lanes) {
            float mean[V], m2[V];
#pragma unroll
            for (int i = 0; i < V; ++i) mean[i] = m2[i] = 0.f;
            if (active && col + my < vecs) {
                const T* q = x + (col + my) * V;
                float n = 0.f;
                for (int s = s0 + myrow; s < s1; s += U * rows) {
                    fetch(q, s);
#pragma unroll
                    for (int u = 0; u < U; ++u)
                        if (s + u * rows < s1) {
                            float v[V];
                            widen<T, V>(batch[u], v);
                            n += 1.f;
                            const float r = __builtin_amdgcn_rcpf(n);
#pragma unroll
                            for (int i = 0; i < V; ++i) {
                                const float d = v[i] - mean[i];
                                mean[i] = __builtin_fmaf(d, r, mean[i]);
                                m2[i] = __builtin_fmaf(d, v[i] - mean[i], m2[i]);
                            }
                        }
                }
            }
            if (col > 0) __syncthreads();
            if (active) {
#pragma unroll
                for (int i = 0; i < V; ++i) sums[myrow * stride + my * V + i] = make_float2(mean[i], m2[i]);
            }
            __syncthreads();
            // the group's channels within this column, rows inside (rows past the chunk's end are empty)
            const int from = max(tg * cpg - col * V, 0), to = min((tg + 1) * cpg - col * V, lanes * V);
            if (tg < ng && from < to) {
                const int base = (unsigned)(s1 - s0) / (unsigned)rows, more = (s1 - s0) - base * rows, span = to - from;
                const int items = span * (base > 0 ? rows : more), dr = (unsigned)team / (unsigned)span, dc = team - dr * span;
                const int r1 = (unsigned)tl / (unsigned)span, c1 = tl - r1 * span;
                const float2* at = sums + from;
                const auto each = [&](auto f) {
                    int c = c1, r = r1;
                    for (int e = tl; e < items; e += 4 * team) {             // four reads in flight
                        float n[4];
                        float2 w[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const bool in = e + k * team < items;
                            n[k] = in ? (float)(base + (r < more)) : 0.f;
                            w[k] = at[in ? r * stride + c : 0];
                            r += dr;
                            c += dc;
                            if (c >= span) { c -= span; ++r; }
                        }
#pragma unroll
                        for (int k = 0; k < 4; ++k) f(n[k], n[k] > 0.f ? w[k] : make_float2(0.f, 0.f));
                    }
                };
                const Moments u = united(each, at[0].x, team);
                t = t.n > 0.f ? merged(t, u) : u;
            }
        }
    } else {
        if (tg < ng) {
            const float2* at = a.part + ((long)b * a.groups + g0 + tg) * p.chunks;
            const float full = (float)p.per * (float)cpg, last = (float)(a.positions - (p.chunks - 1) * p.per) * (float)cpg;
            const auto each = [&](auto f) {
                for (int k = tl; k < p.chunks; k += team) f(k + 1 < p.chunks ? full : last, at[k]);
            };
            t = united(each, at[0].x, team);
        }
    }
    if constexpr (PHASE == 0) {
        if (tg < ng && tl == 0) a.part[((long)b * a.groups + g0 + tg) * p.chunks + chunk] = make_float2(t.mean, t.m2);
        return;
    }
    if (tg < ng && tl == 0) stats[tg] = make_float2(t.mean, 1.0f / sqrtf(t.m2 / t.n + a.eps));
    __syncthreads();
    if (!active) return;
    const bool held = PHASE == 2 && vecs <= lanes && s1 - s0 <= U * rows;
    for (int col = my; col < vecs; col += lanes) {
        if (col != my) fetch_affine(col);
        float mul[V], mean[V], add[V], scale[V];
        widen<float, V>(gamma, scale);
        widen<float, V>(beta, add);
        int g = (unsigned)(col * V) / (unsigned)cpg, left = (g + 1) * cpg - col * V;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (left == 0) { ++g; left = cpg; }
            --left;
            const float2 st = stats[g];
            mean[i] = st.x;
            mul[i] = st.y * scale[i];
        }
        for (int s = s0 + myrow; s < s1; s += U * rows) {
            if (!held) fetch(x + col * V, s);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (s + u * rows < s1) {
                    float v[V];
                    widen<T, V>(batch[u], v);
#pragma unroll
                    for (int i = 0; i < V; ++i) v[i] = activated<T, ACT>(__builtin_fmaf(v[i] - mean[i], mul[i], add[i]));
                    store_channels<T, V>(o + (s + u * rows) * a.o_position + col * V, v, PHASE == 1 && a.stream);
                }
        }
    }
}

size_t group_norm_scratch_bytes(int dtype, int batch, int positions, int channels, int groups) {
    const GroupNormPlan p = group_norm_plan(positions, channels, groups, dtype == PS_BF16 ? 2 : 4);
    return p.chunks > 1 ? (size_t)batch * groups * p.chunks * sizeof(float2) : 0;
}

template <typename T, int V, int ACT>
static void launch_group_norm_act(const GroupNormArgs& a, const GroupNormPlan& p, hipStream_t st) {
    const dim3 grid(p.chunks, p.slices, a.batch);
    if (p.chunks == 1) group_norm_kernel<T, V, 2, ACT, 4, SINGLE_THREADS><<<grid, SINGLE_THREADS, 0, st>>>(a, p);
    else group_norm_kernel<T, V, 1, ACT, 4, 256><<<grid, 256, 0, st>>>(a, p);
}

template <typename T, int V>
static hipError_t launch_group_norm_as(const GroupNormArgs& a, GroupNormPlan p, hipStream_t st) {
    p.lanes = p.slice_groups * p.cpg / V;
    const int threads = p.chunks == 1 ? SINGLE_THREADS : 256;
    if (p.lanes > threads) p.lanes = threads;
    p.rows = threads / p.lanes;
    p.lanes_inv = ((1u << 20) + p.lanes - 1) / p.lanes;  // t * lanes_inv >> 20 == t / lanes for t < 1024: too large by less than lanes / 2^20
    for (p.team = 64; p.team * p.slice_groups > threads;) p.team /= 2;
    // rows of partial moments in LDS 16 entries (32 banks) apart: a team reads neighbouring channels, then rows
    p.fill = p.lanes * V % 32 == 0 && p.lanes >= 8 ? 16 : 0;      // (rows * fill <= 2 * threads)
    if (p.chunks > 1) group_norm_kernel<T, V, 0, 0, 4, 256><<<dim3(p.chunks, p.slices, a.batch), 256, 0, st>>>(a, p);
    (a.act == 2 ? launch_group_norm_act<T, V, 2> : a.act == 1 ? launch_group_norm_act<T, V, 1> : launch_group_norm_act<T, V, 0>)(a, p, st);
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_group_norm_t(const GroupNormArgs& a, hipStream_t st) {
    const GroupNormPlan p = group_norm_plan(a.positions, a.channels, a.groups, sizeof(T));
    // the widest load that divides a slice, the last one too
    const int width = p.slice_groups * p.cpg | a.channels;
    if (sizeof(T) == 2 && width % 8 == 0) return launch_group_norm_as<T, sizeof(T) == 2 ? 8 : 4>(a, p, st);
    if (width % 4 == 0) return launch_group_norm_as<T, 4>(a, p, st);
    return launch_group_norm_as<T, 1>(a, p, st);
}

hipError_t launch_group_norm(int dtype, const GroupNormArgs& args, hipStream_t st) {
    GroupNormArgs a = args;
    a.stream = (size_t)a.batch * a.positions * a.channels * (dtype == PS_BF16 ? 2 : 4) > STREAM_BYTES;
    return dtype == PS_BF16 ? launch_group_norm_t<bf16_t>(a, st) : launch_group_norm_t<float>(a, st);
}

}  // namespace ps
