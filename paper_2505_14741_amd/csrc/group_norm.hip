// Group norm over channels-last positions with an activation: a group is channels / groups neighbouring channels of one sample over all
// positions; y = (x - mean) / sqrt(var + eps) * gamma + beta, then none, tanh-GELU or SiLU.
//
// Reading x twice and writing it once is what binds.  A workgroup takes a slice of whole groups (about 64 channels, so that a position is
// a whole cache line or two) over a chunk of positions.  Means and squared deviations are merged pairwise, (n, mean, M2) with
// (n', mean', M2'), from single values on: exact where the mean is far larger than the deviations, whatever the first values are.
#include "few_epilogue.h"
#include "group_norm.h"
#include "plan.h"
#include <type_traits>

namespace ps {

struct Moments { float n, mean, m2; };
// (both may be empty; the weight of b is good for 2^-22 of itself, which is 2^-22 of the distance between the means)
__device__ __forceinline__ Moments merged(Moments a, Moments b) {
    const float n = a.n + b.n, d = b.mean - a.mean, w = n > 0.f ? b.n * __builtin_amdgcn_rcpf(n) : 0.f;
    return Moments{n, __builtin_fmaf(d, w, a.mean), a.m2 + b.m2 + d * d * (a.n * w)};
}
// over T neighbouring lanes (a power of two up to 64), in all of them
__device__ __forceinline__ Moments merged_lanes(Moments t, int T) {
    for (int x = 1; x < T; x *= 2) {
        Moments o{__shfl_xor(t.n, x), __shfl_xor(t.mean, x), __shfl_xor(t.m2, x)};
        t = (threadIdx.x & x) ? merged(o, t) : merged(t, o);     // the same order in both lanes: the same bits
    }
    return t;
}

__device__ __forceinline__ float silu_of(float x, float) { return silu_f(x); }
__device__ __forceinline__ float silu_of(float x, bf16_t) {      // rounded to bf16 behind: two transcendentals
    return x * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * -1.4426950408889634f));
}
template <typename T> __device__ __forceinline__ float activated(float x, int act) {
    if (act == 1) return gelu_of(x, T{});
    if (act == 2) return silu_of(x, T{});
    return x;
}

template <typename T, int V>
__device__ __forceinline__ void load_channels(const T* p, float (&v)[V]) {
    typedef typename std::conditional<sizeof(T) == 4, float, __bf16>::type E;
    typedef __attribute__((ext_vector_type(V))) E vec;
    if constexpr (V == 1) v[0] = (float)*reinterpret_cast<const E*>(p);
    else {
        const vec w = *reinterpret_cast<const vec*>(p);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = (float)w[i];
    }
}
template <typename T, int V>
__device__ __forceinline__ void store_channels(T* p, const float (&v)[V]) {
    typedef typename std::conditional<sizeof(T) == 4, float, __bf16>::type E;
    typedef __attribute__((ext_vector_type(V))) E vec;
    if constexpr (V == 1) *reinterpret_cast<E*>(p) = (E)v[0];
    else {
        vec w;
#pragma unroll
        for (int i = 0; i < V; ++i) w[i] = (E)v[i];
        *reinterpret_cast<vec*>(p) = w;
    }
}

// PHASE 0: moments of the chunk's groups to a.part; 1: moments of all chunks from a.part, then the result; 2: both, one chunk.
// 256 threads: `lanes` threads side by side hold the slice's channels, V each, 256 / lanes positions at a time (rows); a slice of more
// than 256 * V channels is walked in columns of 256 * V.  A thread keeps a running mean and M2 of each of its channels; they meet in
// LDS, where `team` threads per group merge its rows x channels.
template <typename T, int V, int PHASE>
__global__ void __launch_bounds__(256)
group_norm_kernel(GroupNormArgs a, GroupNormPlan p) {
    constexpr int U = 4;                                 // positions in flight per thread
    __shared__ float2 sums[PHASE == 1 ? 1 : 256 * V];    // mean, M2
    __shared__ float2 stats[GROUP_NORM_SLICE_GROUPS];    // mean, 1 / sqrt(var + eps)
    const int chunk = blockIdx.x % p.chunks, slice = blockIdx.x / p.chunks % p.slices, b = blockIdx.x / (p.chunks * p.slices);
    const int cpg = a.channels / a.groups, g0 = slice * p.slice_groups, ng = min(p.slice_groups, a.groups - g0);
    const int c0 = g0 * cpg, nc = ng * cpg, vecs = nc / V;
    const int s0 = (int)((long)a.positions * chunk / p.chunks), s1 = (int)((long)a.positions * (chunk + 1) / p.chunks);
    const int lanes = min(vecs, 256), rows = 256 / lanes;
    const int my = threadIdx.x % lanes, myrow = threadIdx.x / lanes;
    const bool active = myrow < rows;
    int team = 64;                                       // threads per group
    while (team * ng > 256) team /= 2;
    const int tg = threadIdx.x / team, tl = threadIdx.x & (team - 1);
    const T* x = (const T*)a.x + b * a.x_batch + c0;
    T* o = (T*)a.out + b * a.o_batch + c0;

    Moments t{0.f, 0.f, 0.f};                            // of group tg
    if constexpr (PHASE != 1) {
        for (int col = 0; col < vecs; col += lanes) {
            float mean[V], m2[V];
#pragma unroll
            for (int i = 0; i < V; ++i) mean[i] = m2[i] = 0.f;
            if (active && col + my < vecs) {
                const T* q = x + (col + my) * V;
                float n = 0.f;
                auto take = [&](const float (&v)[V]) {
                    n += 1.f;
                    const float r = __builtin_amdgcn_rcpf(n);
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float d = v[i] - mean[i];
                        mean[i] = __builtin_fmaf(d, r, mean[i]);
                        m2[i] = __builtin_fmaf(d, v[i] - mean[i], m2[i]);
                    }
                };
                int s = s0 + myrow;
                for (; s + (U - 1) * rows < s1; s += U * rows) {
                    float v[U][V];
#pragma unroll
                    for (int u = 0; u < U; ++u) load_channels<T, V>(q + (s + u * rows) * a.x_position, v[u]);
#pragma unroll
                    for (int u = 0; u < U; ++u) take(v[u]);
                }
                for (; s < s1; s += rows) {
                    float v[V];
                    load_channels<T, V>(q + s * a.x_position, v);
                    take(v);
                }
            }
            if (col > 0) __syncthreads();
            if (active) {
#pragma unroll
                for (int i = 0; i < V; ++i) sums[(myrow * lanes + my) * V + i] = make_float2(mean[i], m2[i]);
            }
            __syncthreads();
            // the group's channels within this column, rows inside
            if (tg < ng) {
                const int from = max(tg * cpg - col * V, 0), to = min((tg + 1) * cpg - col * V, lanes * V), items = (to - from) * rows;
                for (int e = tl; e < items; e += team) {
                    const int c = e / rows, r = e - c * rows;
                    const int n = (s1 - s0 - r + rows - 1) / rows;
                    const float2 w = sums[r * lanes * V + from + c];
                    if (n > 0) t = merged(t, Moments{(float)n, w.x, w.y});
                }
            }
        }
    } else if (tg < ng) {
        for (int k = tl; k < p.chunks; k += team) {
            const float2 w = a.part[((long)b * a.groups + g0 + tg) * p.chunks + k];
            const int n = (int)((long)a.positions * (k + 1) / p.chunks) - (int)((long)a.positions * k / p.chunks);
            t = merged(t, Moments{(float)n * (float)cpg, w.x, w.y});
        }
    }
    t = merged_lanes(t, team);
    if constexpr (PHASE == 0) {
        if (tg < ng && tl == 0) a.part[((long)b * a.groups + g0 + tg) * p.chunks + chunk] = make_float2(t.mean, t.m2);
        return;
    }
    if (tg < ng && tl == 0) stats[tg] = make_float2(t.mean, 1.0f / sqrtf(t.m2 / t.n + a.eps));
    __syncthreads();
    if (!active) return;
    for (int col = my; col < vecs; col += lanes) {
        float mul[V], mean[V], add[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = col * V + i;
            const float2 st = stats[c / cpg];
            mean[i] = st.x;
            mul[i] = st.y * (a.gamma ? a.gamma[c0 + c] : 1.f);
            add[i] = a.beta ? a.beta[c0 + c] : 0.f;
        }
        auto put = [&](float (&v)[V], int s) {
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = activated<T>(__builtin_fmaf(v[i] - mean[i], mul[i], add[i]), a.act);
            store_channels<T, V>(o + s * a.o_position + col * V, v);
        };
        int s = s0 + myrow;
        for (; s + (U - 1) * rows < s1; s += U * rows) {
            float v[U][V];
#pragma unroll
            for (int u = 0; u < U; ++u) load_channels<T, V>(x + (s + u * rows) * a.x_position + col * V, v[u]);
#pragma unroll
            for (int u = 0; u < U; ++u) put(v[u], s + u * rows);
        }
        for (; s < s1; s += rows) {
            float v[V];
            load_channels<T, V>(x + s * a.x_position + col * V, v);
            put(v, s);
        }
    }
}

size_t group_norm_scratch_bytes(int dtype, int batch, int positions, int channels, int groups) {
    const GroupNormPlan p = group_norm_plan(positions, channels, groups, dtype == PS_BF16 ? 2 : 4);
    return p.chunks > 1 ? (size_t)batch * groups * p.chunks * sizeof(float2) : 0;
}

template <typename T, int V>
static hipError_t launch_group_norm_as(const GroupNormArgs& a, const GroupNormPlan& p, hipStream_t st) {
    const unsigned grid = (unsigned)((long)a.batch * p.slices * p.chunks);
    if (p.chunks == 1) {
        group_norm_kernel<T, V, 2><<<grid, 256, 0, st>>>(a, p);
    } else {
        group_norm_kernel<T, V, 0><<<grid, 256, 0, st>>>(a, p);
        group_norm_kernel<T, V, 1><<<grid, 256, 0, st>>>(a, p);
    }
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_group_norm_t(const GroupNormArgs& a, hipStream_t st) {
    const GroupNormPlan p = group_norm_plan(a.positions, a.channels, a.groups, sizeof(T));
    // the widest load that the slices' widths, the strides and the addresses allow
    long bytes = (long)p.slice_groups * (a.channels / a.groups) * sizeof(T);
    bytes |= (long)((uintptr_t)a.x | (uintptr_t)a.out) | (long)a.channels * sizeof(T);
    if (a.positions > 1) bytes |= (a.x_position | a.o_position) * (long)sizeof(T);
    if (a.batch > 1) bytes |= (a.x_batch | a.o_batch) * (long)sizeof(T);
    if (bytes % 16 == 0) return launch_group_norm_as<T, 16 / sizeof(T)>(a, p, st);
    if (bytes % 8 == 0 && sizeof(T) == 2) return launch_group_norm_as<T, 4>(a, p, st);
    return launch_group_norm_as<T, 1>(a, p, st);
}

hipError_t launch_group_norm(int dtype, const GroupNormArgs& a, hipStream_t st) {
    return dtype == PS_BF16 ? launch_group_norm_t<bf16_t>(a, st) : launch_group_norm_t<float>(a, st);
}

}  // namespace ps
