// Attention of queries to another sequence's keys and values: o_i = sum_j p_ij v_j / sum_j p_ij, p_ij = exp(scale q_i k_j - max),
// over the keys j of the sample that count (j < kv_lens[b] and key_mask[b][j] != 0); a row without any is zero.
//
// Query heads that share a key/value head are rows of one product: row = token * share + head of the group, so that the group's keys
// are read once.  A workgroup takes a block of rows of one (sample, key/value head) and walks the keys 64 at a time through LDS, with
// the running maximum and sum of the softmax.  Tiles are transposed: S^T = K Q^T leaves a row in lane % 16 with keys 4 * (lane / 16) + i
// of every 16-key block, which is the layout the second operand of O^T = V^T P^T wants, so probabilities stay in their registers.
// Keys that do not count get a score of -infinity, and their V rows (K too in bf16) are zeros in LDS: what lies there is never multiplied.
//
// What binds: with few keys reading q and writing o (17550 x 226 keys, 30 heads of 64: 137 MB, 28 us at a device copy's rate) and the
// vector instructions per score, about as long, which do not all run beside the matrix instructions; that case takes 48 us (2.9 TB/s,
// 640 TFLOP/s).  With few rows, reading the keys: 32 tokens x 17776 keys (55 MB) 23 us and 6 to add the pieces.
#include "cross_attention.h"
#include "lane_sums.h"
#include "plan.h"
#include "tile_ops.h"
#include <type_traits>

namespace ps {

constexpr int CROSS_RESIDENT_WAVES = 8;

// the sample's keys, and which of the 64 keys from kv0 on count (wave-uniform)
__device__ __forceinline__ int cross_keys(const CrossArgs& a, int b) {
    return a.kv_lens ? min(max(a.kv_lens[b], 0), a.kv_len) : a.kv_len;
}
__device__ __forceinline__ unsigned long long cross_counts(const CrossArgs& a, int b, int kv0, int keys, int lane) {
    const int key = kv0 + lane;
    bool in = key < keys;
    if (a.key_mask && in) in = a.key_mask[b * a.mask_batch + key] != 0;
    return __ballot(in);
}

// Grid: (key/value head, piece of the keys, block of rows) in x, heads innermost, since a token's heads are neighbours in memory; samples in z.
struct CrossItem { int b, g, block, piece; };
__device__ __forceinline__ CrossItem cross_item(const CrossArgs& a) {
    CrossItem t;
    const unsigned id = blockIdx.x;
    unsigned of_head = id / (unsigned)a.kv_heads;
    t.g = (int)(id - of_head * a.kv_heads);
    t.piece = 0;
    if (a.nsplit > 1) { const unsigned q = of_head / (unsigned)a.nsplit; t.piece = (int)(of_head - q * a.nsplit); of_head = q; }
    t.block = (int)of_head;
    t.b = blockIdx.z;
    return t;
}
// offset of a row in q or o
__device__ __forceinline__ long cross_row(const CrossArgs& a, int g, int row, long tok, long head) {
    if (a.share == 1) return row * tok + g * head;
    const int t = (unsigned)row / (unsigned)a.share;
    return t * tok + (long)(g * a.share + (row - t * a.share)) * head;
}

// ------------------------------------------------------------------------------------ bf16
// The reference of a row's exponents moves only where some score of a tile exceeds it by 8 in powers of two (probabilities
// stay below 2^8, sums far from overflow): a tile then costs no rescaling and no maximum over lanes.
constexpr float CROSS_AHEAD = 8.0f;                      // (finite in units of the scores for every scale: -infinity plus it stays -infinity)
constexpr float CROSS_SUM_MAX = 0x1p+32f;
// Sums up to here are no larger than 2^8 for each of the 65 keys or more of a row with a second tile: values overflow under them only where
// they do with a reference that moves, too.
constexpr float CROSS_SUM_NEAR = 0x1p+14f;
// Exponents are c s - c m in one instruction; c m is rounded, by up to 2^-24 of itself, which all keys of a row share but two references
// do not.  Beyond 2^10, where that is 2^-14, a row takes (s - m) c instead.
constexpr float CROSS_FAR = 0x1p+10f;

typedef __attribute__((ext_vector_type(4))) short s16x4_t;
__device__ __forceinline__ s16x4_t read_tr16(const bf16_t* p) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(p));
}

typedef __attribute__((ext_vector_type(4))) int i32x4_t;

// Stores a row's outputs (16 d blocks of 4 values a lane): lanes of neighbouring kgrp swap quads of two blocks, so that each has 8
// adjacent values and the four lanes of a row write 64 bytes.
template <int NB>
__device__ __forceinline__ void cross_store(bf16_t* row, const f32x4_t (&acc)[NB], float inv, int kgrp, bool in, bool stream) {
    if constexpr (NB == 1) {
        if (in) *reinterpret_cast<bf16x4_t*>(row + kgrp * 4) = __builtin_convertvector(acc[0] * inv, bf16x4_t);
    } else {
#pragma unroll
        for (int d = 0; d < NB; d += 2) {
            typedef __attribute__((ext_vector_type(2))) unsigned u32x2_t;
            const u32x2_t x = __builtin_bit_cast(u32x2_t, __builtin_convertvector(acc[d] * inv, bf16x4_t));
            const u32x2_t y = __builtin_bit_cast(u32x2_t, __builtin_convertvector(acc[d + 1] * inv, bf16x4_t));
            const auto lo = __builtin_amdgcn_permlane16_swap(x[0], y[0], false, false), hi = __builtin_amdgcn_permlane16_swap(x[1], y[1], false, false);
            // even kgrp: block d, values 4 kgrp .. + 7; odd: block d + 1, values 4 (kgrp - 1) .. + 7
            if (in)
                store_streamed<16>(row + (d + (kgrp & 1)) * 16 + (kgrp & 2) * 4, i32x4_t{(int)lo[0], (int)hi[0], (int)lo[1], (int)hi[1]}, stream);
        }
    }
}

// The K fragments of a tile of 64 keys: first operand of S^T, 8 consecutive d (4 for heads of 16) of row l16 of each 16 keys.
// kt: the lane's place in the tile's first 16 rows.
template <int HD> struct CrossK { static constexpr int STEPS = HD < 32 ? 1 : HD / 32; bf16x8_t f[4][STEPS]; };
template <int HD, int LD>
__device__ __forceinline__ void cross_read_k(const bf16_t* kt, CrossK<HD>& k) {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        if constexpr (HD == 16) {
            const bf16x4_t w = *reinterpret_cast<const bf16x4_t*>(kt + g * 16 * LD);
            k.f[g][0] = __builtin_shufflevector(w, w, 0, 1, 2, 3, 0, 1, 2, 3);
        } else {
#pragma unroll
            for (int s = 0; s < HD / 32; ++s) k.f[g][s] = *reinterpret_cast<const bf16x8_t*>(kt + g * 16 * LD + s * 32);
        }
    }
}
template <int HD, int QT>
__device__ __forceinline__ void cross_scores(const CrossK<HD>& k, const bf16x8_t (&q)[QT][CrossK<HD>::STEPS], f32x4_t (&sc)[QT][4]) {
    constexpr f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            if constexpr (HD == 16) {
                const bf16x4_t kl = __builtin_shufflevector(k.f[g][0], k.f[g][0], 0, 1, 2, 3), ql = __builtin_shufflevector(q[t][0], q[t][0], 0, 1, 2, 3);
                sc[t][g] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4_t, kl), __builtin_bit_cast(s16x4_t, ql), zero, 0, 0, 0);
            } else {
                sc[t][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k.f[g][0], q[t][0], zero, 0, 0, 0);
            }
        }
#pragma unroll
    for (int s = 1; s < HD / 32; ++s)
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
            for (int t = 0; t < QT; ++t) sc[t][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k.f[g][s], q[t][s], sc[t][g], 0, 0, 0);
}
// The V fragments of a tile: first operand of O^T, row d = l16 of each 16 d, k slot (kgrp, e) of step s is key 32 s + 16 (e / 4) + 4 kgrp + e % 4.
// vt: the lane's place in the tile's first rows.
template <int HD> struct CrossV { bf16x8_t f[2][HD / 16]; };
template <int HD, int LD>
__device__ __forceinline__ void cross_read_v(const bf16_t* vt, CrossV<HD>& v) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int d = 0; d < HD / 16; ++d) {
            const bf16_t* p = vt + s * 32 * LD + d * 16;
            const bf16x4_t lo = __builtin_bit_cast(bf16x4_t, read_tr16(p)), hi = __builtin_bit_cast(bf16x4_t, read_tr16(p + 16 * LD));
            v.f[s][d] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        }
}

// 2^(c (a - b)) of two scores, b finite and a at most b, or -infinity (0).  Halves: the scores' difference itself may be beyond fp32 where
// c times it is not (c times a finite score is finite).
__device__ __forceinline__ float exp2_between(float a, float b, float c) {
    const float half = (0.5f * a - 0.5f * b) * c;
    return __builtin_amdgcn_exp2f(half + half);
}

// FIRST (a row's first tile, nothing has been summed): the reference is the maximum.  Else references move (in powers of two: times c)
// where a score of the tile is ahead of one, and what has been summed with them.
template <int QT, int NB, bool FIRST>
__device__ __forceinline__ void cross_softmax(const f32x4_t (&sc)[QT][4], f32x4_t (&acc)[QT][NB], float (&m)[QT], f32x4_t (&l)[QT], float c, float ahead) {
    float top[QT];
    bool over = false;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        top[t] = -INFINITY;
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
            for (int i = 0; i < 4; ++i) top[t] = fmaxf(top[t], sc[t][g][i]);
        if constexpr (FIRST) m[t] = max_xor32(max_xor16(top[t]));
        else over = over || top[t] > m[t] + ahead;
    }
    if (!FIRST && __any(over)) {
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            const float mn = fmaxf(m[t], max_xor32(max_xor16(top[t])));
            const float alpha = mn == m[t] ? 1.f : exp2_between(m[t], mn, c);        // 0 on the first tile
            m[t] = mn;
            l[t][0] *= alpha;                            // (the only one that is looked at)
#pragma unroll
            for (int d = 0; d < NB; ++d) acc[t][d] *= alpha;
        }
    }
}
// Probabilities, rounded to bf16 for the second product (the scores are used up).  NEAR: no reference is beyond CROSS_FAR, or the caller looks for it afterwards.
template <int QT, bool NEAR>
__device__ __forceinline__ void cross_weights(f32x4_t (&sc)[QT][4], const float (&m)[QT], float c, bf16x8_t (&pf)[QT][2]) {
    float mc[QT];
    bool far = false;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        mc[t] = m[t] == -INFINITY ? 0.f : m[t] * c;
        far = far || fabsf(mc[t]) > CROSS_FAR;
    }
    if (!NEAR && __any(far)) {
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            const bool mine = fabsf(mc[t]) > CROSS_FAR;
            const float ref = mine ? m[t] : 0.f;
            mc[t] = mine ? 0.f : mc[t];
#pragma unroll
            for (int g = 0; g < 4; ++g) sc[t][g] -= ref;
        }
    }
#pragma unroll
    for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                pf[t][s][e] = (__bf16)__builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][2 * s + e / 4][e % 4], c, -mc[t]));
}
// acc += V^T P^T, l += 1 P^T: the sums of the probabilities as they were rounded (one key alone has weight 1 exactly), for which the matrix
// pipes have time and the vector ones have not.  Every lane has its row's whole sum.
template <int HD, int QT, bool FIRST = false>
__device__ __forceinline__ void cross_values(const CrossV<HD>& v, const bf16x8_t (&pf)[QT][2], f32x4_t (&acc)[QT][HD / 16], f32x4_t (&l)[QT]) {
    const __bf16 one = (__bf16)1.0f;
    const bf16x8_t ones = {one, one, one, one, one, one, one, one};
    constexpr f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < 2; ++s) {
#pragma unroll
        for (int d = 0; d < HD / 16; ++d)
#pragma unroll
            for (int t = 0; t < QT; ++t)
                acc[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v.f[s][d], pf[t][s], FIRST && s == 0 ? zero : acc[t][d], 0, 0, 0);
#pragma unroll
        for (int t = 0; t < QT; ++t) l[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[t][s], FIRST && s == 0 ? zero : l[t], 0, 0, 0);
    }
}

template <int HD, int QT>
__global__ void __launch_bounds__(256, 2)
cross_bf16_kernel(CrossArgs a) {
    constexpr int KT = 64, LD = HD + 8, LDV = cross_v_pitch(HD), BQ = 4 * QT * 16, NB = HD / 16, CH = HD / 8;
    constexpr int QS = HD < 32 ? 1 : HD / 32;            // fragments of a query row
    constexpr int LOADS = (KT * CH + 255) / 256;
    __shared__ __attribute__((aligned(16))) bf16_t Ks[KT * LD], Vs[KT * LDV];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, kgrp = lane >> 4;
    const CrossItem it = cross_item(a);
    const bf16_t* kb = (const bf16_t*)a.k + it.b * a.s.k_batch + it.g * a.s.k_head;
    const bf16_t* vb = (const bf16_t*)a.v + it.b * a.s.v_batch + it.g * a.s.v_head;
    const int keys = cross_keys(a, it.b), tiles = (keys + KT - 1) / KT;
    int j0 = 0, j1 = tiles;
    if (a.nsplit > 1) { j0 = (int)((long)tiles * it.piece / a.nsplit); j1 = (int)((long)tiles * (it.piece + 1) / a.nsplit); }
    const int r0 = it.block * BQ + wave * QT * 16 + l16;
    const float c = a.scale * CROSS_LOG2E, ahead = fminf(CROSS_AHEAD / c, 0x1p+127f);

    typedef __attribute__((ext_vector_type(4))) int chunk_t;
    chunk_t kn[LOADS], vn[LOADS];                        // the next tile; rows past the end are zeros
    int at[LOADS];                                       // row of the tile
    long koff[LOADS], voff[LOADS];
#pragma unroll
    for (int u = 0; u < LOADS; ++u) {
        const int e = threadIdx.x + 256 * u;
        at[u] = e / CH;
        koff[u] = at[u] * a.s.k_tok + e % CH * 8;
        voff[u] = at[u] * a.s.v_tok + e % CH * 8;
    }
    auto fetch = [&](int kv0) {
        const bf16_t *kt = kb + kv0 * a.s.k_tok, *vt = vb + kv0 * a.s.v_tok;
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            if (kv0 + KT > keys || KT * CH % 256) {
                kn[u] = vn[u] = chunk_t{0, 0, 0, 0};
                if (at[u] >= KT || kv0 + at[u] >= keys) continue;
            }
            kn[u] = *reinterpret_cast<const chunk_t*>(kt + koff[u]);
            vn[u] = *reinterpret_cast<const chunk_t*>(vt + voff[u]);
        }
    };
    unsigned long long counts_next = j0 < j1 ? cross_counts(a, it.b, j0 * KT, keys, lane) : 0;
    if (j0 < j1) fetch(j0 * KT);

    // queries: second operand of S^T, 8 consecutive d (4 for heads of 16) of row l16; rows past the end repeat the last one
    bf16x8_t qf[QT][QS];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        const bf16_t* p = (const bf16_t*)a.q + it.b * a.s.q_batch + cross_row(a, it.g, min(r0 + t * 16, a.rows - 1), a.s.q_tok, a.s.q_head);
        if constexpr (HD == 16) {
            const bf16x4_t w = *reinterpret_cast<const bf16x4_t*>(p + kgrp * 4);
            qf[t][0] = __builtin_shufflevector(w, w, 0, 1, 2, 3, 0, 1, 2, 3);
        } else {
#pragma unroll
            for (int s = 0; s < QS; ++s) qf[t][s] = *reinterpret_cast<const bf16x8_t*>(p + s * 32 + kgrp * 8);
        }
    }
    f32x4_t acc[QT][NB];                                 // O^T: row l16, d = 16 * block + 4 * kgrp + i
    f32x4_t l[QT];                                       // [0]: the row's sum
    float m[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        m[t] = -INFINITY; l[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int d = 0; d < NB; ++d) acc[t][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    for (int j = j0; j < j1; ++j) {
        const unsigned long long counts = counts_next;
        const bool whole = counts == ~0ull;
        __syncthreads();                                 // nobody reads the last tile any more
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            if (KT * CH % 256 && at[u] >= KT) continue;
            if (!whole && !(counts >> at[u] & 1)) kn[u] = vn[u] = chunk_t{0, 0, 0, 0};
            const int d = (threadIdx.x + 256 * u) % CH * 8;
            *reinterpret_cast<chunk_t*>(Ks + at[u] * LD + d) = kn[u];
            *reinterpret_cast<chunk_t*>(Vs + at[u] * LDV + d) = vn[u];
        }
        __syncthreads();
        if (j + 1 < j1) {
            counts_next = cross_counts(a, it.b, (j + 1) * KT, keys, lane);
            fetch((j + 1) * KT);
        }
        if (counts == 0) continue;                       // (the whole workgroup)
        // reads are requested together, ahead of their use: V while the softmax runs
        CrossK<HD> kf;
        cross_read_k<HD, LD>(Ks + l16 * LD + kgrp * (HD == 16 ? 4 : 8), kf);
        if constexpr (QT * HD <= 128) __builtin_amdgcn_sched_barrier(0);     // (more would not fit the registers)
        f32x4_t sc[QT][4];
        cross_scores<HD, QT>(kf, qf, sc);
        CrossV<HD> vf;
        cross_read_v<HD, LDV>(Vs + (4 * kgrp + (l16 >> 2)) * LDV + (l16 & 3) * 4, vf);
        if constexpr (QT * HD <= 128) __builtin_amdgcn_sched_barrier(0);
        if (!whole) {
            const unsigned long long mine = counts >> (4 * kgrp);
#pragma unroll
            for (int g = 0; g < 4; ++g)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float bias = (mine >> (16 * g + i) & 1) ? 0.f : -INFINITY;     // (K rows that do not count are zeros)
#pragma unroll
                    for (int t = 0; t < QT; ++t) sc[t][g][i] += bias;
                }
        }
        cross_softmax<QT, NB, false>(sc, acc, m, l, c, ahead);
        bf16x8_t pf[QT][2];
        cross_weights<QT, false>(sc, m, c, pf);
        cross_values<HD, QT>(vf, pf, acc, l);
    }
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        const int row = r0 + t * 16;
        const float sum = l[t][0];
        if (a.nsplit > 1) {
            if (row >= a.rows) continue;
            float* p = a.part + ((((long)it.b * a.kv_heads + it.g) * a.nsplit + it.piece) * a.rows + row) * (HD + 4);
#pragma unroll
            for (int d = 0; d < NB; ++d) *reinterpret_cast<f32x4_t*>(p + d * 16 + kgrp * 4) = acc[t][d];
            if (kgrp == 0) *reinterpret_cast<f32x2_t*>(p + HD) = f32x2_t{sum, m[t]};
        } else {
            bf16_t* p = (bf16_t*)a.o + it.b * a.s.o_batch + cross_row(a, it.g, min(row, a.rows - 1), a.s.o_tok, a.s.o_head);
            cross_store<NB>(p, acc[t], sum == 0.f ? 0.f : __builtin_amdgcn_rcpf(sum), kgrp, row < a.rows, a.stream);
        }
    }
}

// Short key sequences and many rows (a prompt's states under a video's tokens; 17550 x 226 keys 70 us on cross_bf16_kernel, 48 here): all keys and
// values of a (sample, key/value head) lie in LDS, and the 8 waves of a workgroup (four per SIMD of two workgroups) take QT * 16 rows each in
// turn, without a barrier.  n workgroups share a head.  A row's values depend on the rows of its own chunk only, whatever n is.
template <int HD, int QT>
__global__ void __launch_bounds__(CROSS_RESIDENT_WAVES * 64, CROSS_RESIDENT_WAVES / 2)
cross_resident_kernel(CrossArgs a, int n) {
    constexpr int KT = 64, LDK = HD + 8, LDV = cross_v_pitch(HD), BQ = QT * 16, NB = HD / 16, CH = HD / 8, QS = HD < 32 ? 1 : HD / 32;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int slots = (a.kv_len + KT - 1) / KT * KT;     // (of the longest sample)
    bf16_t *const Ks = reinterpret_cast<bf16_t*>(lds), *const Vs = Ks + slots * LDK;
    float* const Bs = reinterpret_cast<float*>(Vs + slots * LDV);    // what the scores' sums start from: 0, or -infinity
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, kgrp = lane >> 4;
    const int part = (int)(blockIdx.x / (unsigned)a.kv_heads), g = (int)blockIdx.x - part * a.kv_heads, b = blockIdx.z;
    const bf16_t* kb = (const bf16_t*)a.k + b * a.s.k_batch + g * a.s.k_head;
    const bf16_t* vb = (const bf16_t*)a.v + b * a.s.v_batch + g * a.s.v_head;
    const bf16_t* qb = (const bf16_t*)a.q + b * a.s.q_batch;
    bf16_t* ob = (bf16_t*)a.o + b * a.s.o_batch;
    const int keys = cross_keys(a, b), tiles = (keys + KT - 1) / KT;
    const int chunks = (a.rows + BQ - 1) / BQ, stride = n * CROSS_RESIDENT_WAVES;
    const float c = a.scale * CROSS_LOG2E, ahead = fminf(CROSS_AHEAD / c, 0x1p+127f);

    // offset of row t * 16 + l16 of a chunk: the lane's share of it is the same for all chunks that are whole, if heads share no keys
    const long q_lane = l16 * a.s.q_tok + kgrp * (HD == 16 ? 4 : 8), o_lane = l16 * a.s.o_tok;
    const auto row_at = [&](int chunk, int t, long tok, long head, long of_lane, long plus) {
        const int row = chunk * BQ + t * 16;
        if (a.share == 1 && row + 16 <= a.rows) return row * tok + g * head + of_lane;
        return cross_row(a, g, min(row + l16, a.rows - 1), tok, head) + plus;
    };
    bf16x8_t qf[QT][QS];
    auto fetch = [&](int chunk) {
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            const bf16_t* p = qb + row_at(chunk, t, a.s.q_tok, a.s.q_head, q_lane, kgrp * (HD == 16 ? 4 : 8));
            if constexpr (HD == 16) {
                const bf16x4_t w = *reinterpret_cast<const bf16x4_t*>(p);
                qf[t][0] = __builtin_shufflevector(w, w, 0, 1, 2, 3, 0, 1, 2, 3);
            } else {
#pragma unroll
                for (int s = 0; s < QS; ++s) qf[t][s] = *reinterpret_cast<const bf16x8_t*>(p + s * 32);
            }
        }
    };
    int chunk = part * CROSS_RESIDENT_WAVES + wave;
    fetch(min(chunk, chunks - 1));
    constexpr int NT = CROSS_RESIDENT_WAVES * 64, U = 4; // U: keys and values in flight per thread
    const int pieces = tiles * KT * CH;
    for (int e0 = threadIdx.x; e0 < pieces; e0 += U * NT) {
        i32x4_t kv[U], vv[U];
        bool in[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int r = (e0 + u * NT) / CH, rc = min(r, keys - 1), d = (e0 + u * NT) % CH * 8;
            in[u] = r < keys && (!a.key_mask || a.key_mask[b * a.mask_batch + rc] != 0);
            kv[u] = *reinterpret_cast<const i32x4_t*>(kb + rc * a.s.k_tok + d);
            vv[u] = *reinterpret_cast<const i32x4_t*>(vb + rc * a.s.v_tok + d);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int r = (e0 + u * NT) / CH, d = (e0 + u * NT) % CH * 8;
            if (e0 + u * NT >= pieces) continue;
            *reinterpret_cast<i32x4_t*>(Ks + r * LDK + d) = in[u] ? kv[u] : i32x4_t{0, 0, 0, 0};
            *reinterpret_cast<i32x4_t*>(Vs + r * LDV + d) = in[u] ? vv[u] : i32x4_t{0, 0, 0, 0};
            if (d == 0) Bs[r] = in[u] ? 0.f : -INFINITY;
        }
    }
    __syncthreads();
    unsigned whole = 0;                                  // tiles all of whose keys count
    bool first_counts = false, any_counts = false;       // some key of the first tile does, some key at all
    for (int j = 0; j < tiles; ++j) {
        const unsigned long long in = __ballot(Bs[j * KT + lane] == 0.f);
        whole |= (in == ~0ull ? 1u : 0u) << j;
        if (j == 0) first_counts = in != 0;
        any_counts = any_counts || in != 0;
    }
    const int tracked_tiles = any_counts ? tiles : 0;    // (zeros without a product: the query need not be finite)

    const bf16_t *const k0 = Ks + l16 * LDK + kgrp * (HD == 16 ? 4 : 8), *const v0 = Vs + (4 * kgrp + (l16 >> 2)) * LDV + (l16 & 3) * 4;
    f32x4_t acc[QT][NB], l[QT];
    float m[QT];
    // One tile of the scores against the first tile's maximum (FIRST: that tile), or with a reference that moves (TRACKED).
    const auto tile = [&](int j, auto first_c, auto tracked_c) {
        constexpr bool FIRST = decltype(first_c)::value, TRACKED = decltype(tracked_c)::value;
        f32x4_t sc[QT][4];
        {
            CrossK<HD> kf;
            cross_read_k<HD, LDK>(k0 + j * (KT * LDK), kf);
            cross_scores<HD, QT>(kf, qf, sc);
        }
        if (!(whole >> j & 1)) {
#pragma unroll
            for (int g4 = 0; g4 < 4; ++g4) {
                const f32x4_t bias = *reinterpret_cast<const f32x4_t*>(Bs + j * KT + g4 * 16 + kgrp * 4);
#pragma unroll
                for (int t = 0; t < QT; ++t) sc[t][g4] += bias;
            }
        }
        if constexpr (FIRST || TRACKED) cross_softmax<QT, NB, FIRST>(sc, acc, m, l, c, ahead);
        bf16x8_t pf[QT][2];
        cross_weights<QT, !TRACKED>(sc, m, c, pf);
        CrossV<HD> vf;
        cross_read_v<HD, LDV>(v0 + j * (KT * LDV), vf);
        cross_values<HD, QT, FIRST>(vf, pf, acc, l);
    };
    const std::true_type yes;
    const std::false_type no;
    for (; chunk < chunks; chunk += stride) {
        // Relative to the first tile's maximum, which is one of the row's scores, sums are at least 1; what they are at most is looked at
        // behind the last tile, instead of every tile's maxima: rows whose later scores are so much larger (or somewhat larger, and the
        // values so large that their sums are not finite), or whose reference is beyond CROSS_FAR, are computed again.
        bool done = false;
        if (first_counts) {
            tile(0, yes, no);
            for (int j = 1; j < tiles; ++j) tile(j, no, no);
            bool fits = true;
            float sums = 0.f;                            // of the lane's rows: at least as large as each
#pragma unroll
            for (int t = 0; t < QT; ++t) {
                sums += l[t][0];
                fits = fits && !(fabsf(m[t] * c) > CROSS_FAR);
            }
            if (!__all(sums < CROSS_SUM_NEAR)) {
                float zero = 0.f;                        // (NaN if a value is not finite)
#pragma unroll
                for (int t = 0; t < QT; ++t)
#pragma unroll
                    for (int d = 0; d < NB; ++d)
#pragma unroll
                        for (int i = 0; i < 4; ++i) zero = __builtin_fmaf(acc[t][d][i], 0.f, zero);
                fits = fits && sums < CROSS_SUM_MAX && zero == 0.f;
            }
            done = __all(fits);
        }
        if (!done) {
#pragma unroll
            for (int t = 0; t < QT; ++t) {
                m[t] = -INFINITY;
                l[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int d = 0; d < NB; ++d) acc[t][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            }
            for (int j = 0; j < tracked_tiles; ++j) tile(j, no, yes);
        }
        if (chunk + stride < chunks) fetch(chunk + stride);
        // the next queries' loads are waited for here: behind the stores, whose number the compiler cannot know, it would wait for these too
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
            for (int s = 0; s < QS; ++s) asm volatile("" ::"v"(qf[t][s]));
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            const float sum = l[t][0];
            cross_store<NB>(ob + row_at(chunk, t, a.s.o_tok, a.s.o_head, o_lane, 0), acc[t], sum == 0.f ? 0.f : __builtin_amdgcn_rcpf(sum), kgrp,
                            chunk * BQ + t * 16 + l16 < a.rows, a.stream);
        }
    }
}

// Adds the pieces of a row: o = sum_i w_i acc_i / sum_i w_i l_i, w_i = exp(scale * (ref_i - max)) for bf16, whose references are scores, and
// exp(ref_i - max) for fp32, whose are scaled; a piece without a key that counts has the reference -infinity.  A wave takes a row: HD / 4 lanes
// hold 4 adjacent values each, and the wave's 256 / HD teams of them take a piece each in turn.
template <typename T, int HD>
__global__ void __launch_bounds__(256)
cross_join_kernel(CrossArgs a, long lines) {
    constexpr int W = HD / 4, TEAMS = 64 / W;
    const int lane = threadIdx.x & 63, d = lane % W * 4, team = lane / W;
    const float c = a.scale * CROSS_LOG2E;
    for (long line = (long)blockIdx.x * 4 + (threadIdx.x >> 6); line < lines; line += (long)gridDim.x * 4) {      // (whole waves)
        const long bg = line / a.rows;
        const int row = (int)(line - bg * a.rows), b = (int)(bg / a.kv_heads), g = (int)(bg - (long)b * a.kv_heads);
        const float* p = a.part + (bg * a.nsplit * a.rows + row) * (HD + 4);
        const long step = (long)a.rows * (HD + 4);
        float top = -INFINITY;
        for (int i = lane; i < a.nsplit; i += 64) top = fmaxf(top, p[i * step + HD + 1]);
#pragma unroll
        for (int x = 1; x < 64; x *= 2) top = fmaxf(top, __shfl_xor(top, x));
        const float ref = top == -INFINITY ? 0.f : top;      // (then every weight is zero, and so are the sums)
        f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
        float l = 0.f;
#pragma unroll 4
        for (int i = team; i < a.nsplit; i += TEAMS) {
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
        T* o = (T*)a.o + b * a.s.o_batch + cross_row(a, g, row, a.s.o_tok, a.s.o_head) + d;
        if constexpr (sizeof(T) == 2) *reinterpret_cast<bf16x4_t*>(o) = __builtin_convertvector(acc, bf16x4_t);
        else *reinterpret_cast<f32x4_t*>(o) = acc;
    }
}

// ------------------------------------------------------------------------------------ fp32
// The same tiles with full fp32 products (v_mfma_f32_16x16x4_f32), probabilities in fp32 and exponentials as exact as expf.
template <int HD>
__global__ void __launch_bounds__(256, HD >= 128 ? 2 : HD == 64 ? 3 : 4)
cross_f32_kernel(CrossArgs a) {
    constexpr int KT = 64, LD = HD + 4, NB = HD / 16, BQ = 64, CH = HD / 4, LOADS = KT * CH / 256;
    __shared__ __attribute__((aligned(16))) float Ks[KT * LD], Vs[KT * LD];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, kgrp = lane >> 4;
    const CrossItem it = cross_item(a);
    const float* kb = (const float*)a.k + it.b * a.s.k_batch + it.g * a.s.k_head;
    const float* vb = (const float*)a.v + it.b * a.s.v_batch + it.g * a.s.v_head;
    const int keys = cross_keys(a, it.b), tiles = (keys + KT - 1) / KT;
    const int j0 = (int)((long)tiles * it.piece / a.nsplit), j1 = (int)((long)tiles * (it.piece + 1) / a.nsplit);
    const int row = it.block * BQ + wave * 16 + l16;
    f32x4_t qf[NB];
    {
        const float* p = (const float*)a.q + it.b * a.s.q_batch + cross_row(a, it.g, min(row, a.rows - 1), a.s.q_tok, a.s.q_head);
#pragma unroll
        for (int d = 0; d < NB; ++d) qf[d] = *reinterpret_cast<const f32x4_t*>(p + d * 16 + kgrp * 4) * a.scale;
    }
    f32x4_t kn[LOADS], vn[LOADS];
    auto fetch = [&](int kv0) {
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            const int e = threadIdx.x + 256 * u, r = kv0 + e / CH, d = e % CH * 4;
            kn[u] = vn[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            if (r < keys) {
                kn[u] = *reinterpret_cast<const f32x4_t*>(kb + (long)r * a.s.k_tok + d);
                vn[u] = *reinterpret_cast<const f32x4_t*>(vb + (long)r * a.s.v_tok + d);
            }
        }
    };
    f32x4_t acc[NB];
#pragma unroll
    for (int d = 0; d < NB; ++d) acc[d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    unsigned long long counts_next = j0 < j1 ? cross_counts(a, it.b, j0 * KT, keys, lane) : 0;
    if (j0 < j1) fetch(j0 * KT);
    for (int j = j0; j < j1; ++j) {
        const unsigned long long counts = counts_next;
        __syncthreads();
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            const int e = threadIdx.x + 256 * u, r = e / CH, off = r * LD + e % CH * 4;
            *reinterpret_cast<f32x4_t*>(Ks + off) = kn[u];
            *reinterpret_cast<f32x4_t*>(Vs + off) = (counts >> r & 1) ? vn[u] : f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
        __syncthreads();
        if (j + 1 < j1) {
            counts_next = cross_counts(a, it.b, (j + 1) * KT, keys, lane);
            fetch((j + 1) * KT);
        }
        if (counts == 0) continue;
        const int blocks = min(4, (keys - j * KT + 15) / 16);        // 16-key blocks with a key in them
        const bool whole = counts == ~0ull;
        const unsigned long long mine = counts >> (4 * kgrp);
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
            if (!whole) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (!(mine >> (16 * g + i) & 1)) sc[g][i] = -INFINITY;
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
        const bool near = __ballot(low - ref < EXP_NEAR) == 0;       // (of the whole wave; not with keys that do not count)
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
                for (int d = 0; d < NB; ++d)
                    acc[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(Vs[(g * 16 + kgrp * 4 + e) * LD + d * 16 + l16], sc[g][e], acc[d], 0, 0, 0);
        }
    }
    l = sum_xor32(sum_xor16(l));
    if (row >= a.rows) return;
    if (a.nsplit > 1) {
        float* p = a.part + ((((long)it.b * a.kv_heads + it.g) * a.nsplit + it.piece) * a.rows + row) * (HD + 4);
#pragma unroll
        for (int d = 0; d < NB; ++d) *reinterpret_cast<f32x4_t*>(p + d * 16 + kgrp * 4) = acc[d];
        if (kgrp == 0) *reinterpret_cast<f32x2_t*>(p + HD) = f32x2_t{l, m};
        return;
    }
    float* p = (float*)a.o + it.b * a.s.o_batch + cross_row(a, it.g, row, a.s.o_tok, a.s.o_head) + kgrp * 4;
#pragma unroll
    for (int d = 0; d < NB; ++d) *reinterpret_cast<f32x4_t*>(p + d * 16) = l == 0.f ? f32x4_t{0.f, 0.f, 0.f, 0.f} : acc[d] / l;
}

static CrossPlan cross_plan_of(int dtype, const CrossArgs& a) {
    return cross_plan(dtype == PS_BF16, a.rows, a.kv_len, a.kv_heads, a.head_dim, compute_units());
}

size_t cross_workspace_bytes(int dtype, const CrossArgs& a) {
    const CrossPlan p = cross_plan_of(dtype, a);
    return p.nsplit > 1 ? (size_t)a.batch * a.kv_heads * p.nsplit * a.rows * (a.head_dim + 4) * sizeof(float) : 0;
}

template <int HD>
static hipError_t launch_cross_hd(int dtype, CrossArgs a, hipStream_t st) {
    const CrossPlan p = cross_plan_of(dtype, a);
    a.nsplit = p.nsplit;
    a.stream = (size_t)a.batch * a.kv_heads * a.rows * HD * (dtype == PS_BF16 ? 2 : 4) > STREAM_BYTES;
    if constexpr (HD <= 64)
    if (p.resident) {
        // workgroups per head: two for every compute unit over the whole batch, a chunk for every wave at least
        long n = 2L * compute_units() / ((long)a.kv_heads * a.batch);
        constexpr int QT = 2;
        const long most = ((a.rows + QT * 16 - 1) / (QT * 16) + CROSS_RESIDENT_WAVES - 1) / CROSS_RESIDENT_WAVES;
        n = n > most ? most : n < 1 ? 1 : n;
        const int bytes = (a.kv_len + 63) / 64 * 64 * cross_resident_key_bytes(HD);
        cross_resident_kernel<HD, QT><<<dim3((unsigned)(a.kv_heads * n), 1, a.batch), CROSS_RESIDENT_WAVES * 64, bytes, st>>>(a, (int)n);
        return hipGetLastError();
    }
    const dim3 grid((unsigned)(a.kv_heads * p.nsplit) * (unsigned)((a.rows + p.block - 1) / p.block), 1, a.batch);
    if (dtype != PS_BF16) cross_f32_kernel<HD><<<grid, 256, 0, st>>>(a);
    else if (HD > 64 || p.block == 64) cross_bf16_kernel<HD, 1><<<grid, 256, 0, st>>>(a);      // (heads of 128 always: see cross_plan)
    else if constexpr (HD <= 64) {
        if (p.block == 128) cross_bf16_kernel<HD, 2><<<grid, 256, 0, st>>>(a);
        else cross_bf16_kernel<HD, 3><<<grid, 256, 0, st>>>(a);
    }
    if (p.nsplit > 1) {
        const long lines = (long)a.batch * a.kv_heads * a.rows;
        const unsigned wgs = (unsigned)((lines + 3) / 4 < (1L << 22) ? (lines + 3) / 4 : 1L << 22);
        if (dtype == PS_BF16) cross_join_kernel<bf16_t, HD><<<wgs, 256, 0, st>>>(a, lines);
        else cross_join_kernel<float, HD><<<wgs, 256, 0, st>>>(a, lines);
    }
    return hipGetLastError();
}

hipError_t launch_cross_attention(int dtype, CrossArgs a, hipStream_t st) {
    switch (a.head_dim) {
        case 16: return launch_cross_hd<16>(dtype, a, st);
        case 32: return launch_cross_hd<32>(dtype, a, st);
        case 64: return launch_cross_hd<64>(dtype, a, st);
        case 128: return launch_cross_hd<128>(dtype, a, st);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace ps
