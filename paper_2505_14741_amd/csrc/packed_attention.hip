// Attention inside the samples that are packed along one token axis: o_i = sum_j p_ij v_j / sum_j p_ij, p_ij = exp(x_ij - max), over the keys j of query
// i's own sample that it sees; x_ij = scale q_i k_j, capped by cap * tanh(x / cap), less slope * |frame(i) - frame(j)|.
//
// A sample's queries are its last tokens: query t of nq stands at nk - nq + t of the sample's nk keys.  Behind the sample's prefix, tokens lie in frames; a query
// sees the prefix and, causally, the frames up to its own: its first reach(t) keys, a number that does not fall from query to query.  So a
// tile of 64 keys is whole for a wave's rows, cut by their reach, or behind it, and only those that are cut look at single keys.
//
// Query heads that share a key head are rows of one product, row = token * share + head of the group.  Blocks of BQ rows of one (sample, key head)
// are found on the GPU, from the offsets: sample s owns the block slots from rows_before(s) / BQ + s on, which leaves room for its last, partial block
// (and at most one slot of a sample is empty), so that a slot's sample is a search in a rising sequence.
#include "packed_attention.h"
#include "lane_sums.h"
#include "plan.h"
#include "tile_ops.h"
#include <type_traits>

namespace ps {

typedef __attribute__((ext_vector_type(16))) float f32x16_t;
typedef __attribute__((ext_vector_type(4))) short s16x4_t;
typedef __attribute__((ext_vector_type(4))) int i32x4_t;

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int within(int v, int lo, int hi) { return min(max(v, lo), hi); }

// (wave-uniform)
struct PackedItem {
    int g, r0, rows, q0, k0, keys, ahead, prefix, piece, pieces, sample;
    bool any;
    // keys that a query sees, at `pos` of the sample's keys
    __device__ __forceinline__ int reach(const PackedArgs& a, int pos) const {
        if (!a.causal) return keys;
        if (pos < prefix) return prefix;
        return min((long)keys, prefix + ((long)((unsigned)(pos - prefix) / (unsigned)a.frame) + 1) * a.frame);
    }
};
template <int BQ>
__device__ __forceinline__ PackedItem packed_item(const PackedArgs& a, int lane) {
    PackedItem t;
    const int id = a.most_pieces > 1 ? (int)blockIdx.x : xcd_remap(blockIdx.x, gridDim.x);
    t.g = (int)((unsigned)id / (unsigned)a.slots);
    const int slot = a.slots - 1 - (id - t.g * a.slots);             // (a sample's last queries see most)
    t.piece = blockIdx.y;
    t.any = false;
    const auto first_slot = [&](int s) { return (int)((unsigned)within(a.q_offsets[s], 0, a.q_tokens) * (unsigned)a.share / BQ) + s; };
    int s = 0, n = a.samples, step;
    do {
        step = (n + 63) / 64;
        const int i = lane * step;
        const unsigned long long below = __ballot(i < n && first_slot(s + min(i, n - 1)) <= slot);
        if (below == 0) return t;
        const int c = (__popcll(below) - 1) * step;
        s += c;
        n = min(step, n - c);
    } while (step > 1);
    t.sample = uniform(s);
    t.q0 = uniform(within(a.q_offsets[t.sample], 0, a.q_tokens));
    const int nq = uniform(within(a.q_offsets[t.sample + 1], t.q0, a.q_tokens)) - t.q0;
    t.rows = nq * a.share;
    t.r0 = uniform((slot - first_slot(t.sample)) * BQ);
    if (t.r0 >= t.rows) return t;
    t.k0 = t.q0;
    t.keys = nq;
    if (a.kv_offsets) {
        t.k0 = uniform(within(a.kv_offsets[t.sample], 0, a.kv_tokens));
        t.keys = uniform(within(a.kv_offsets[t.sample + 1], t.k0, a.kv_tokens)) - t.k0;
    }
    t.ahead = t.keys - nq;
    t.prefix = a.prefix ? uniform(within(a.prefix[t.sample], 0, t.keys)) : 0;
    t.pieces = a.most_pieces > 1 ? packed_pieces(BQ, t.rows, t.keys, a.kv_heads) : 1;
    t.any = t.piece < t.pieces;
    return t;
}
// where the partial sums of a piece's row lie: a region of PACKED_SLOTS blocks for each sample that is divided
template <int BQ, int HD>
__device__ __forceinline__ float* packed_part(const PackedArgs& a, const PackedItem& t, int piece) {
    const int region = a.by_sample ? t.sample : t.k0 / PACKED_KEYS, block_rows = min(BQ, a.q_tokens * a.share), blocks = (t.rows + BQ - 1) / BQ;
    return a.part + (((long)region * PACKED_SLOTS + (t.g * t.pieces + piece) * blocks + t.r0 / BQ) * block_rows) * (HD + 4);
}

// offset of a row of the sample in q or o
__device__ __forceinline__ long packed_row(const PackedArgs& a, const PackedItem& t, int row, long tok, long head) {
    const int i = a.share == 1 ? row : (int)((unsigned)row / (unsigned)a.share);
    return (long)(t.q0 + i) * tok + (long)(t.g * a.share + (row - i * a.share)) * head;
}

// What a query row is to its keys: how many it sees; the distance bias' slope (0 in the prefix) and its frame.
struct PackedRow { int reach; float slope, frame; };
__device__ __forceinline__ PackedRow packed_query(const PackedArgs& a, const PackedItem& t, int row) {
    const int i = a.share == 1 ? row : (int)((unsigned)row / (unsigned)a.share), pos = t.ahead + i;
    PackedRow r;
    r.reach = t.reach(a, pos);
    r.slope = r.frame = 0.f;
    if (a.slopes && pos >= t.prefix) {
        r.slope = a.slopes[t.g * a.share + (row - i * a.share)];
        r.frame = (float)((unsigned)(pos - t.prefix) / (unsigned)a.frame);
    }
    return r;
}
// A key's frame, NaN in the prefix.
__device__ __forceinline__ float packed_frame(const PackedArgs& a, const PackedItem& t, int key) {
    return key < t.prefix ? __uint_as_float(0x7fc00000u) : (float)((unsigned)(key - t.prefix) / (unsigned)a.frame);
}
// slope * distance, 0 where the key is in the prefix
__device__ __forceinline__ float packed_bias(const PackedRow& r, float frame) {
    const float far = fabsf(r.frame - frame);
    return far == far ? r.slope * far : 0.f;
}

__device__ __forceinline__ float exp2_between(float a, float b, float c) {
    const float half = (0.5f * a - 0.5f * b) * c;
    return __builtin_amdgcn_exp2f(half + half);
}

// ------------------------------------------------------------------------------------ bf16
// Tiles are transposed: S^T = K Q^T leaves a query in lane % 32 and keys 8 (i / 4) + 4 (lane / 32) + i % 4 of every 32 in register i, which, rounded to
// bf16, are the second operand of O^T = V^T P^T as they stand (its k in the order of the registers; V fragments follow).
// The reference of a row's exponents moves only where some score of a tile exceeds it by 8 in powers of two (probabilities stay below 2^8, sums
// far from overflow).  Exponents are c s - c m in one instruction; beyond 2^10, where the rounding of c m is 2^-14, a row takes (s - m) c.
constexpr float PACKED_AHEAD = 8.0f, PACKED_FAR = 0x1p+10f;
constexpr int PACKED_BQ = 128, PACKED_BQ_F32 = 64;

__device__ __forceinline__ s16x4_t packed_read_tr16(const bf16_t* p) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(p));
}

template <int HD, bool CAP, bool BIAS>
__global__ void __launch_bounds__(256, HD > 64 ? 2 : 3)
packed_bf16_kernel(PackedArgs a) {
    constexpr int KT = 64, LDK = HD + 8, LDV = HD + 16, NB = HD < 32 ? 1 : HD / 32, QS = HD / 16, CH = HD / 8, LOADS = (KT * CH + 255) / 256;
    __shared__ __attribute__((aligned(16))) bf16_t Ks[KT * LDK], Vs[KT * LDV];
    __shared__ float Fs[KT];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), l32 = lane & 31, hi = lane >> 5;
    const PackedItem it = packed_item<PACKED_BQ>(a, lane);
    if (!it.any) return;                                 // (the whole workgroup)
    const bf16_t *kb = (const bf16_t*)a.k + (long)it.k0 * a.k_tok + it.g * a.k_head, *vb = (const bf16_t*)a.v + (long)it.k0 * a.v_tok + it.g * a.v_head;

    const int w0 = it.r0 + wave * 32, wl = min(w0 + 31, it.rows - 1), bl = min(it.r0 + PACKED_BQ, it.rows) - 1, row = min(w0 + l32, it.rows - 1);
    const bool mine = w0 < it.rows;                      // (the wave has rows)
    const int least = mine ? it.reach(a, it.ahead + w0 / a.share) : 0, most = mine ? it.reach(a, it.ahead + wl / a.share) : 0;
    const int tiles_all = (it.keys + KT - 1) / KT, tiles = (it.reach(a, it.ahead + bl / a.share) + KT - 1) / KT;
    const int j0 = (int)((long)tiles_all * it.piece / it.pieces), j1 = min(tiles, (int)((long)tiles_all * (it.piece + 1) / it.pieces));
    PackedRow me = packed_query(a, it, row);
    me.slope *= PACKED_LOG2E;

    i32x4_t kn[LOADS], vn[LOADS];
    float fn = 0.f;
    auto fetch = [&](int kv0) {                          // keys behind the sample's last one are zeros
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            const int e = threadIdx.x + 256 * u, r = e / CH, key = kv0 + r;
            kn[u] = vn[u] = i32x4_t{0, 0, 0, 0};
            if (r < KT && key < it.keys) {
                kn[u] = *reinterpret_cast<const i32x4_t*>(kb + key * a.k_tok + e % CH * 8);
                vn[u] = *reinterpret_cast<const i32x4_t*>(vb + key * a.v_tok + e % CH * 8);
            }
        }
        if constexpr (BIAS) fn = packed_frame(a, it, kv0 + (threadIdx.x & 63));
    };
    bf16x8_t qf[QS];                                     // second operand of S^T: 8 consecutive d of row l32
    {
        const bf16_t* p = (const bf16_t*)a.q + packed_row(a, it, row, a.q_tok, a.q_head) + hi * 8;
#pragma unroll
        for (int s = 0; s < QS; ++s) qf[s] = *reinterpret_cast<const bf16x8_t*>(p + s * 16);
    }
    f32x16_t acc[NB], l;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        l[i] = 0.f;
#pragma unroll
        for (int d = 0; d < NB; ++d) acc[d][i] = 0.f;
    }
    float m = -INFINITY;
    const float c0 = a.scale * PACKED_LOG2E, c = CAP || BIAS ? 1.0f : c0, ahead = fminf(PACKED_AHEAD / c, 0x1p+127f);
    const float cap2 = a.cap * PACKED_LOG2E, into = CAP ? 2.0f * c0 / a.cap : 0.f;
    const __bf16 one = (__bf16)1.0f;
    const bf16x8_t ones = {one, one, one, one, one, one, one, one};

    if (j0 < j1) fetch(j0 * KT);
    for (int j = j0; j < j1; ++j) {
        const int kv0 = j * KT;
        __syncthreads();                                 // nobody reads the last tile any more
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            const int e = threadIdx.x + 256 * u, r = e / CH, d = e % CH * 8;
            if (KT * CH % 256 && r >= KT) continue;
            *reinterpret_cast<i32x4_t*>(Ks + r * LDK + d) = kn[u];
            *reinterpret_cast<i32x4_t*>(Vs + r * LDV + d) = vn[u];
        }
        if (BIAS && threadIdx.x < KT) Fs[threadIdx.x] = fn;
        __syncthreads();
        if (j + 1 < j1) fetch(kv0 + KT);
        if (kv0 >= most) continue;                       // (the wave: nothing that its rows see)
        const bool cut = kv0 + KT > least;
        f32x16_t sc[2];
#pragma unroll
        for (int g = 0; g < 2; ++g) {
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[g][i] = 0.f;
#pragma unroll
            for (int s = 0; s < QS; ++s)
                sc[g] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8_t*>(Ks + (g * 32 + l32) * LDK + s * 16 + hi * 8), qf[s], sc[g], 0, 0, 0);
        }
        if constexpr (CAP || BIAS) {
#pragma unroll
            for (int g = 0; g < 2; ++g)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    float x = sc[g][i];
                    if constexpr (CAP) x = __builtin_fmaf(-2.0f * cap2, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * into)), cap2);
                    else x *= c0;
                    if constexpr (BIAS) x -= packed_bias(me, Fs[g * 32 + 8 * (i / 4) + 4 * hi + i % 4]);
                    sc[g][i] = x;
                }
        }
        if (cut) {
            const int left = me.reach - kv0 - 4 * hi;
#pragma unroll
            for (int g = 0; g < 2; ++g)
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[g][i] = g * 32 + 8 * (i / 4) + i % 4 < left ? sc[g][i] : -INFINITY;
        }
        float top = -INFINITY;
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[g][i]);
        if (__any(top > m + ahead)) {
            const float mn = fmaxf(m, max_xor32(top));
            const float alpha = mn == m ? 1.f : exp2_between(m, mn, c);          // 0 on the first tile
            m = mn;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                l[i] *= alpha;
#pragma unroll
                for (int d = 0; d < NB; ++d) acc[d][i] *= alpha;
            }
        }
        float mc = m == -INFINITY ? 0.f : m * c;
        if (__any(fabsf(mc) > PACKED_FAR)) {
            const bool far = fabsf(mc) > PACKED_FAR;
            const float ref = far ? m : 0.f;
            mc = far ? 0.f : mc;
#pragma unroll
            for (int g = 0; g < 2; ++g)
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[g][i] -= ref;
        }
        bf16x8_t pf[4];
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                pf[s][e] = (__bf16)__builtin_amdgcn_exp2f(__builtin_fmaf(sc[s / 2][s % 2 * 8 + e], c, -mc));
        // V^T: row d = l32 of each 32; slot (hi, e) of step s is key 16 s + 8 (e / 4) + 4 hi + e % 4
        const bf16_t* vt = Vs + (4 * hi + ((lane & 15) >> 2)) * LDV + (HD < 32 ? 0 : (lane & 16)) + (lane & 3) * 4;
        bool odd = false;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
#pragma unroll
            for (int d = 0; d < NB; ++d) {
                const bf16_t* p = vt + s * 16 * LDV + d * 32;
                s16x4_t lo = packed_read_tr16(p), up = packed_read_tr16(p + 8 * LDV);
                if (cut) {
                    // Keys that some row does not see have the weight zero there, which a value that is not finite must not meet.
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const bool ol = (lo[i] & 0x7f80) == 0x7f80, ou = (up[i] & 0x7f80) == 0x7f80;
                        odd = odd || ol || ou;
                        lo[i] = ol ? 0 : lo[i];
                        up[i] = ou ? 0 : up[i];
                    }
                }
                const bf16x8_t vf = __builtin_shufflevector(__builtin_bit_cast(bf16x4_t, lo), __builtin_bit_cast(bf16x4_t, up), 0, 1, 2, 3, 4, 5, 6, 7);
                acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[s], acc[d], 0, 0, 0);
            }
            l = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ones, pf[s], l, 0, 0, 0);
        }
        if (cut && __any(odd)) {                         // what was left out, for the rows that see it
            for (int key = 0; key < min(KT, it.keys - kv0); ++key) {
                if (kv0 + key >= me.reach) continue;
#pragma unroll
                for (int d = 0; d < NB; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int at = d * 32 + 8 * (i / 4) + 4 * hi + i % 4;
                        const float x = at < HD ? to_f32(Vs[key * LDV + at]) : 0.f;
                        if (!(fabsf(x) < INFINITY)) acc[d][i] += x;
                    }
            }
        }
    }
    const float sum = l[0];                              // (every lane has its row's whole sum)
    if (w0 + l32 >= it.rows) return;
    if (it.pieces > 1) {
        float* p = packed_part<PACKED_BQ, HD>(a, it, it.piece) + (long)(wave * 32 + l32) * (HD + 4);
#pragma unroll
        for (int d = 0; d < NB; ++d)
#pragma unroll
            for (int r = 0; r < (HD < 32 ? 2 : 4); ++r)
                *reinterpret_cast<f32x4_t*>(p + d * 32 + r * 8 + hi * 4) = f32x4_t{acc[d][4 * r], acc[d][4 * r + 1], acc[d][4 * r + 2], acc[d][4 * r + 3]};
        if (hi == 0) *reinterpret_cast<f32x2_t*>(p + HD) = f32x2_t{sum, m};
        return;
    }
    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
    bf16_t* p = (bf16_t*)a.o + packed_row(a, it, row, a.o_tok, a.o_head);
#pragma unroll
    for (int d = 0; d < NB; ++d)
#pragma unroll
        for (int r = 0; r < (HD < 32 ? 2 : 4); ++r) {
            const f32x4_t x = f32x4_t{acc[d][4 * r], acc[d][4 * r + 1], acc[d][4 * r + 2], acc[d][4 * r + 3]} * inv;
            *reinterpret_cast<bf16x4_t*>(p + d * 32 + r * 8 + hi * 4) = __builtin_convertvector(x, bf16x4_t);
        }
}

// ------------------------------------------------------------------------------------ fp32
// 16 rows per wave with full fp32 products (v_mfma_f32_16x16x4_f32): S^T = K Q^T leaves a row in lane % 16 with keys 4 (lane / 16) + i of every 16.
// Probabilities in fp32, exponentials as exact as expf.
template <int HD>
__global__ void __launch_bounds__(256, HD >= 128 ? 2 : HD == 64 ? 3 : 4)
packed_f32_kernel(PackedArgs a) {
    constexpr int KT = 64, LD = HD + 4, NB = HD / 16, CH = HD / 4, LOADS = KT * CH / 256;
    __shared__ __attribute__((aligned(16))) float Ks[KT * LD], Vs[KT * LD], Fs[KT];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), l16 = lane & 15, kgrp = lane >> 4;
    const PackedItem it = packed_item<PACKED_BQ_F32>(a, lane);
    if (!it.any) return;
    const float *kb = (const float*)a.k + (long)it.k0 * a.k_tok + it.g * a.k_head, *vb = (const float*)a.v + (long)it.k0 * a.v_tok + it.g * a.v_head;
    const int w0 = it.r0 + wave * 16, wl = min(w0 + 15, it.rows - 1), bl = min(it.r0 + PACKED_BQ_F32, it.rows) - 1, row = min(w0 + l16, it.rows - 1);
    const bool mine = w0 < it.rows;
    const int least = mine ? it.reach(a, it.ahead + w0 / a.share) : 0, most = mine ? it.reach(a, it.ahead + wl / a.share) : 0;
    const int tiles_all = (it.keys + KT - 1) / KT, tiles = (it.reach(a, it.ahead + bl / a.share) + KT - 1) / KT;
    const int j0 = (int)((long)tiles_all * it.piece / it.pieces), j1 = min(tiles, (int)((long)tiles_all * (it.piece + 1) / it.pieces));
    const PackedRow me = packed_query(a, it, row);
    f32x4_t qf[NB];
    {
        const float* p = (const float*)a.q + packed_row(a, it, row, a.q_tok, a.q_head);
#pragma unroll
        for (int d = 0; d < NB; ++d) qf[d] = *reinterpret_cast<const f32x4_t*>(p + d * 16 + kgrp * 4) * a.scale;
    }
    f32x4_t kn[LOADS], vn[LOADS];
    float fn = 0.f;
    auto fetch = [&](int kv0) {
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            const int e = threadIdx.x + 256 * u, key = kv0 + e / CH, d = e % CH * 4;
            kn[u] = vn[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            if (key < it.keys) {
                kn[u] = *reinterpret_cast<const f32x4_t*>(kb + key * a.k_tok + d);
                vn[u] = *reinterpret_cast<const f32x4_t*>(vb + key * a.v_tok + d);
            }
        }
        if (a.slopes) fn = packed_frame(a, it, kv0 + (threadIdx.x & 63));
    };
    f32x4_t acc[NB];
#pragma unroll
    for (int d = 0; d < NB; ++d) acc[d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    if (j0 < j1) fetch(j0 * KT);
    for (int j = j0; j < j1; ++j) {
        const int kv0 = j * KT;
        __syncthreads();
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            const int e = threadIdx.x + 256 * u, off = e / CH * LD + e % CH * 4;
            *reinterpret_cast<f32x4_t*>(Ks + off) = kn[u];
            *reinterpret_cast<f32x4_t*>(Vs + off) = vn[u];
        }
        if (a.slopes && threadIdx.x < KT) Fs[threadIdx.x] = fn;
        __syncthreads();
        if (j + 1 < j1) fetch(kv0 + KT);
        if (kv0 >= most) continue;
        const int blocks = min(4, (most - kv0 + 15) / 16);           // 16-key blocks that some row of the wave sees
        const bool cut = kv0 + KT > least;
        const int left = me.reach - kv0 - 4 * kgrp;
        f32x4_t sc[4];
        float top = -INFINITY, low = INFINITY;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            sc[g] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            if (g < blocks) {
#pragma unroll
                for (int d = 0; d < NB; ++d) {
                    const f32x4_t kf = *reinterpret_cast<const f32x4_t*>(Ks + (g * 16 + l16) * LD + d * 16 + kgrp * 4);
#pragma unroll
                    for (int e = 0; e < 4; ++e) sc[g] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[e], qf[d][e], sc[g], 0, 0, 0);
                }
            }
            if (a.cap > 0.f) {
#pragma unroll
                for (int i = 0; i < 4; ++i) sc[g][i] = a.cap * tanhf(sc[g][i] / a.cap);
            }
            if (a.slopes) {
                const f32x4_t f = *reinterpret_cast<const f32x4_t*>(Fs + g * 16 + kgrp * 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) sc[g][i] -= packed_bias(me, f[i]);
            }
            if (cut) {
#pragma unroll
                for (int i = 0; i < 4; ++i) sc[g][i] = g * 16 + i < left ? sc[g][i] : -INFINITY;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                top = fmaxf(top, sc[g][i]);
                low = fminf(low, sc[g][i]);
            }
        }
        const float mn = fmaxf(m, max_xor32(max_xor16(top)));
        const float alpha = mn == m ? 1.f : expf(m - mn), ref = mn == -INFINITY ? 0.f : mn;
        m = mn;
        l *= alpha;
#pragma unroll
        for (int d = 0; d < NB; ++d) acc[d] *= alpha;
        const bool near = __ballot(low - ref < EXP_NEAR) == 0;       // (of the whole wave; not with keys that a row does not see)
        bool odd = false;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            if (g >= blocks) continue;
#pragma unroll
            for (int i = 0; i < 4; ++i) sc[g][i] = near ? exp_near(sc[g][i] - ref) : expf(sc[g][i] - ref);
#pragma unroll
            for (int i = 0; i < 4; ++i) l += sc[g][i];
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int d = 0; d < NB; ++d) {
                    float x = Vs[(g * 16 + kgrp * 4 + e) * LD + d * 16 + l16];
                    if (cut) {                           // (as in the bf16 kernel)
                        const bool o = !(fabsf(x) < INFINITY);
                        odd = odd || o;
                        x = o ? 0.f : x;
                    }
                    acc[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(x, sc[g][e], acc[d], 0, 0, 0);
                }
        }
        if (cut && __any(odd)) {
            for (int key = 0; key < min(KT, it.keys - kv0); ++key) {
                if (kv0 + key >= me.reach) continue;
#pragma unroll
                for (int d = 0; d < NB; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float x = Vs[key * LD + d * 16 + 4 * kgrp + i];
                        if (!(fabsf(x) < INFINITY)) acc[d][i] += x;
                    }
            }
        }
    }
    l = sum_xor32(sum_xor16(l));
    if (w0 + l16 >= it.rows) return;
    if (it.pieces > 1) {
        float* p = packed_part<PACKED_BQ_F32, HD>(a, it, it.piece) + (long)(wave * 16 + l16) * (HD + 4);
#pragma unroll
        for (int d = 0; d < NB; ++d) *reinterpret_cast<f32x4_t*>(p + d * 16 + kgrp * 4) = acc[d];
        if (kgrp == 0) *reinterpret_cast<f32x2_t*>(p + HD) = f32x2_t{l, m};
        return;
    }
    float* p = (float*)a.o + packed_row(a, it, row, a.o_tok, a.o_head) + kgrp * 4;
#pragma unroll
    for (int d = 0; d < NB; ++d) *reinterpret_cast<f32x4_t*>(p + d * 16) = l == 0.f ? f32x4_t{0.f, 0.f, 0.f, 0.f} : acc[d] / l;
}

// Adds the pieces of a row: o = sum_i w_i acc_i / sum_i w_i l_i, w_i = exp(ref_i - max), in powers of two times c for bf16.  A workgroup
// takes a block, a wave a row at a time: HD / 4 lanes hold 4 adjacent values each, and the wave's 256 / HD teams of them take a piece each in turn.
template <typename T, int HD, int BQ>
__global__ void __launch_bounds__(256)
packed_join_kernel(PackedArgs a) {
    constexpr int W = HD / 4, TEAMS = 64 / W;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, d = lane % W * 4, team = lane / W;
    PackedItem it = packed_item<BQ>(a, lane);
    if (!it.any || it.pieces <= 1) return;
    const float c = a.cap > 0.f || a.slopes ? 1.0f : a.scale * PACKED_LOG2E;
    const long step = packed_part<BQ, HD>(a, it, 1) - packed_part<BQ, HD>(a, it, 0);
    for (int r = wave; r < min(BQ, it.rows - it.r0); r += 4) {
        const float* p = packed_part<BQ, HD>(a, it, 0) + (long)r * (HD + 4);
        float top = -INFINITY;
        for (int i = lane; i < it.pieces; i += 64) top = fmaxf(top, p[i * step + HD + 1]);
#pragma unroll
        for (int x = 1; x < 64; x *= 2) top = fmaxf(top, __shfl_xor(top, x));
        const float ref = top == -INFINITY ? 0.f : top;      // (then every weight is zero, and so are the sums)
        f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
        float l = 0.f;
#pragma unroll 4
        for (int i = team; i < it.pieces; i += TEAMS) {
            const f32x2_t s = *reinterpret_cast<const f32x2_t*>(p + i * step + HD);
            const f32x4_t v = *reinterpret_cast<const f32x4_t*>(p + i * step + d);
            const float w = sizeof(T) == 2 ? exp2_between(s[1], ref, c) : expf(s[1] - ref);
            acc += v * w;
            l = __builtin_fmaf(s[0], w, l);
        }
#pragma unroll
        for (int x = W; x < 64; x *= 2) {
            l += __shfl_xor(l, x);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i] += __shfl_xor(acc[i], x);
        }
        if (team != 0) continue;
        acc = l == 0.f ? f32x4_t{0.f, 0.f, 0.f, 0.f} : acc / l;
        T* o = (T*)a.o + packed_row(a, it, it.r0 + r, a.o_tok, a.o_head) + d;
        if constexpr (sizeof(T) == 2) *reinterpret_cast<bf16x4_t*>(o) = __builtin_convertvector(acc, bf16x4_t);
        else *reinterpret_cast<f32x4_t*>(o) = acc;
    }
}

static int packed_block(int dtype) { return dtype == PS_BF16 ? PACKED_BQ : PACKED_BQ_F32; }

size_t packed_workspace_bytes(int dtype, const PackedArgs& a) {
    if (packed_most_pieces(a.own_offsets, a.kv_tokens, a.kv_heads) <= 1) return 0;
    const long block = packed_block(dtype), rows = (long)a.q_tokens * a.share;
    return (size_t)packed_regions(a.samples, a.kv_tokens) * PACKED_SLOTS * (rows < block ? rows : block) * (a.head_dim + 4) * sizeof(float);
}

template <int HD>
static hipError_t launch_packed_hd(int dtype, PackedArgs a, hipStream_t st) {
    const int block = packed_block(dtype);
    a.slots = packed_slots(a.q_tokens, a.share, a.samples, block);
    a.most_pieces = packed_most_pieces(a.own_offsets, a.kv_tokens, a.kv_heads);
    a.by_sample = packed_regions(a.samples, a.kv_tokens) == a.samples;
    const dim3 grid((unsigned)a.slots * (unsigned)a.kv_heads, (unsigned)a.most_pieces);
    if (dtype != PS_BF16) packed_f32_kernel<HD><<<grid, 256, 0, st>>>(a);
    else if (a.cap > 0.f && a.slopes) packed_bf16_kernel<HD, true, true><<<grid, 256, 0, st>>>(a);
    else if (a.cap > 0.f) packed_bf16_kernel<HD, true, false><<<grid, 256, 0, st>>>(a);
    else if (a.slopes) packed_bf16_kernel<HD, false, true><<<grid, 256, 0, st>>>(a);
    else packed_bf16_kernel<HD, false, false><<<grid, 256, 0, st>>>(a);
    if (a.most_pieces > 1) {
        if (dtype == PS_BF16) packed_join_kernel<bf16_t, HD, PACKED_BQ><<<grid.x, 256, 0, st>>>(a);
        else packed_join_kernel<float, HD, PACKED_BQ_F32><<<grid.x, 256, 0, st>>>(a);
    }
    return hipGetLastError();
}

hipError_t launch_packed_attention(int dtype, PackedArgs a, hipStream_t st) {
    switch (a.head_dim) {
        case 16: return launch_packed_hd<16>(dtype, a, st);
        case 32: return launch_packed_hd<32>(dtype, a, st);
        case 64: return launch_packed_hd<64>(dtype, a, st);
        case 128: return launch_packed_hd<128>(dtype, a, st);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace ps
