// Attention of queries to another sequence's keys and values: o_i = sum_j p_ij v_j / sum_j p_ij, p_ij = exp(scale q_i k_j - max),
// over the keys j of the sample that count (j < kv_lens[b] and key_mask[b][j] != 0); a row without any is zero.
//
// Query heads that share a key/value head are rows of one product: row = token * share + head of the group, so that the group's keys
// are read once.  A workgroup takes a block of rows of one (sample, key/value head) and walks the keys 64 at a time through LDS, with
// the running maximum and sum of the softmax.  Tiles are transposed: S^T = K Q^T leaves a row in lane % 16 with keys 4 * (lane / 16) + i
// of every 16-key block, which is the layout the second operand of O^T = V^T P^T wants, so probabilities stay in their registers.
// Keys that do not count get a score of -infinity, and their V rows are zeros in LDS: what lies there is never multiplied.
#include "cross_attention.h"
#include "lane_sums.h"
#include "tile_ops.h"

namespace ps {

constexpr float CROSS_LOG2E = 1.4426950408889634f;

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

// workgroup id -> sample, key/value head, block of rows and share of the keys
struct CrossItem { int b, g, block, piece; };
__device__ __forceinline__ CrossItem cross_item(const CrossArgs& a, int id) {
    CrossItem t;
    t.piece = id % a.nsplit; id /= a.nsplit;
    t.block = id % a.row_blocks; id /= a.row_blocks;
    t.g = id % a.kv_heads;
    t.b = id / a.kv_heads;
    return t;
}
// offset of a row in q (tok, head) and in o
__device__ __forceinline__ long cross_row(const CrossArgs& a, int g, int row, long tok, long head) {
    const int t = row / a.share;
    return t * tok + (long)(g * a.share + (row - t * a.share)) * head;
}

// ------------------------------------------------------------------------------------ bf16
// The reference of a row's exponents moves only where some score of a tile exceeds it by 8 in powers of two (probabilities
// stay below 2^8, sums far from overflow): a tile then costs no rescaling and no maximum over lanes.
constexpr float CROSS_AHEAD = 8.0f;

template <int HD>
__device__ __forceinline__ f32x4_t cross_scores(const bf16_t* k, const bf16x8_t* q, f32x4_t acc) {
#pragma unroll
    for (int s = 0; s < HD / 32; ++s)
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*reinterpret_cast<const bf16x8_t*>(k + s * 32), q[s], acc, 0, 0, 0);
    return acc;
}

typedef __attribute__((ext_vector_type(4))) short s16x4_t;
__device__ __forceinline__ s16x4_t read_tr16(const bf16_t* p) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(p));
}

template <int HD, int QT>
__global__ void __launch_bounds__(256, 2)
cross_bf16_kernel(CrossArgs a) {
    constexpr int KT = 64, LD = HD + 8, BQ = 4 * QT * 16, NB = HD / 16, CH = HD / 8;
    constexpr int QS = HD < 32 ? 1 : HD / 32;            // fragments of a query row
    constexpr int LOADS = (KT * CH + 255) / 256;
    __shared__ __attribute__((aligned(16))) bf16_t Ks[KT * LD], Vs[KT * LD];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, kgrp = lane >> 4;
    const CrossItem it = cross_item(a, xcd_remap(blockIdx.x, gridDim.x));
    const bf16_t* kb = (const bf16_t*)a.k + it.b * a.s.k_batch + it.g * a.s.k_head;
    const bf16_t* vb = (const bf16_t*)a.v + it.b * a.s.v_batch + it.g * a.s.v_head;
    const int keys = cross_keys(a, it.b), tiles = (keys + KT - 1) / KT;
    const int j0 = (int)((long)tiles * it.piece / a.nsplit), j1 = (int)((long)tiles * (it.piece + 1) / a.nsplit);
    const int r0 = it.block * BQ + wave * QT * 16 + l16;
    const float c = a.scale * CROSS_LOG2E, ahead = CROSS_AHEAD / c;

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

    typedef __attribute__((ext_vector_type(4))) int chunk_t;
    chunk_t kn[LOADS], vn[LOADS];                        // the next tile; rows past the end are zeros
    auto fetch = [&](int kv0) {
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            const int e = threadIdx.x + 256 * u, r = kv0 + e / CH, d = e % CH * 8;
            kn[u] = vn[u] = chunk_t{0, 0, 0, 0};
            if (e < KT * CH && r < keys) {
                kn[u] = *reinterpret_cast<const chunk_t*>(kb + (long)r * a.s.k_tok + d);
                vn[u] = *reinterpret_cast<const chunk_t*>(vb + (long)r * a.s.v_tok + d);
            }
        }
    };
    f32x4_t acc[QT][NB];                                 // O^T: row l16, d = 16 * block + 4 * kgrp + i
    float m[QT], l[QT];                                  // l: over this lane's keys only
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        m[t] = -INFINITY; l[t] = 0.f;
#pragma unroll
        for (int d = 0; d < NB; ++d) acc[t][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    unsigned long long counts_next = j0 < j1 ? cross_counts(a, it.b, j0 * KT, keys, lane) : 0;
    if (j0 < j1) fetch(j0 * KT);
    for (int j = j0; j < j1; ++j) {
        const unsigned long long counts = counts_next;
        __syncthreads();                                 // nobody reads the last tile any more
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            const int e = threadIdx.x + 256 * u, r = e / CH;
            if (e < KT * CH) {
                *reinterpret_cast<chunk_t*>(Ks + r * LD + e % CH * 8) = kn[u];
                *reinterpret_cast<chunk_t*>(Vs + r * LD + e % CH * 8) = (counts >> r & 1) ? vn[u] : chunk_t{0, 0, 0, 0};
            }
        }
        __syncthreads();
        if (j + 1 < j1) {
            counts_next = cross_counts(a, it.b, (j + 1) * KT, keys, lane);
            fetch((j + 1) * KT);
        }
        if (counts == 0) continue;                       // (the whole workgroup)
        f32x4_t sc[QT][4];
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
            for (int t = 0; t < QT; ++t) {
                const f32x4_t z = {0.f, 0.f, 0.f, 0.f};
                if constexpr (HD == 16) {
                    const s16x4_t kf = *reinterpret_cast<const s16x4_t*>(Ks + (g * 16 + l16) * LD + kgrp * 4);
                    const bf16x4_t ql = __builtin_shufflevector(qf[t][0], qf[t][0], 0, 1, 2, 3);
                    sc[t][g] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(kf, __builtin_bit_cast(s16x4_t, ql), z, 0, 0, 0);
                } else {
                    sc[t][g] = cross_scores<HD>(Ks + (g * 16 + l16) * LD + kgrp * 8, qf[t], z);
                }
            }
        if (counts != ~0ull) {
            const unsigned long long mine = counts >> (4 * kgrp);
#pragma unroll
            for (int g = 0; g < 4; ++g)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (!(mine >> (16 * g + i) & 1)) {
#pragma unroll
                        for (int t = 0; t < QT; ++t) sc[t][g][i] = -INFINITY;
                    }
        }
        float top[QT];
        bool over = false;
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            top[t] = -INFINITY;
#pragma unroll
            for (int g = 0; g < 4; ++g)
#pragma unroll
                for (int i = 0; i < 4; ++i) top[t] = fmaxf(top[t], sc[t][g][i]);
            over = over || top[t] > m[t] + ahead;
        }
        if (__any(over)) {
#pragma unroll
            for (int t = 0; t < QT; ++t) {
                const float mn = fmaxf(m[t], max_xor32(max_xor16(top[t])));
                const float alpha = mn == m[t] ? 1.f : __builtin_amdgcn_exp2f((m[t] - mn) * c);      // exp2(-inf) = 0 on the first tile
                m[t] = mn;
                l[t] *= alpha;
#pragma unroll
                for (int d = 0; d < NB; ++d) acc[t][d] *= alpha;
            }
        }
        bf16x8_t pf[QT][2];
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            const float mc = m[t] == -INFINITY ? 0.f : m[t] * c;
#pragma unroll
            for (int g = 0; g < 4; ++g)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][g][i], c, -mc));
                    l[t] += p;
                    pf[t][g >> 1][(g & 1) * 4 + i] = (__bf16)p;
                }
        }
        // k slot (kgrp, e) of step s is key 32 s + 16 (e / 4) + 4 kgrp + e % 4
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int d = 0; d < NB; ++d) {
                const bf16_t* p = Vs + (s * 32 + 4 * kgrp + (l16 >> 2)) * LD + d * 16 + (l16 & 3) * 4;
                const bf16x4_t lo = __builtin_bit_cast(bf16x4_t, read_tr16(p)), hi = __builtin_bit_cast(bf16x4_t, read_tr16(p + 16 * LD));
                const bf16x8_t vf = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
                for (int t = 0; t < QT; ++t) acc[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[t][s], acc[t][d], 0, 0, 0);
            }
    }
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        const int row = r0 + t * 16;
        const float sum = sum_xor32(sum_xor16(l[t]));
        if (row >= a.rows) continue;
        bf16_t* p = (bf16_t*)a.o + it.b * a.s.o_batch + cross_row(a, it.g, row, a.s.o_tok, a.s.o_head) + kgrp * 4;
        const float inv = sum == 0.f ? 0.f : 1.0f / sum;
#pragma unroll
        for (int d = 0; d < NB; ++d) *reinterpret_cast<bf16x4_t*>(p + d * 16) = __builtin_convertvector(acc[t][d] * inv, bf16x4_t);
    }
}

// ------------------------------------------------------------------------------------ fp32
// The same tiles with full fp32 products (v_mfma_f32_16x16x4_f32), probabilities in fp32 and exponentials as exact as expf.
template <int HD>
__global__ void __launch_bounds__(256, 2)
cross_f32_kernel(CrossArgs a) {
    constexpr int KT = 64, LD = HD + 4, NB = HD / 16, BQ = 64, CH = HD / 4, LOADS = KT * CH / 256;
    __shared__ __attribute__((aligned(16))) float Ks[KT * LD], Vs[KT * LD];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, kgrp = lane >> 4;
    const CrossItem it = cross_item(a, xcd_remap(blockIdx.x, gridDim.x));
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
        f32x4_t sc[4];
        const unsigned long long mine = counts >> (4 * kgrp);
        float top = -INFINITY;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            sc[g] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int d = 0; d < NB; ++d) {
                const f32x4_t kf = *reinterpret_cast<const f32x4_t*>(Ks + (g * 16 + l16) * LD + d * 16 + kgrp * 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) sc[g] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[e], qf[d][e], sc[g], 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (!(mine >> (16 * g + i) & 1)) sc[g][i] = -INFINITY;
                top = fmaxf(top, sc[g][i]);
            }
        }
        const float mn = fmaxf(m, max_xor32(max_xor16(top)));
        const float alpha = mn == m ? 1.f : expf(m - mn), ref = mn == -INFINITY ? 0.f : mn;
        m = mn;
        l *= alpha;
#pragma unroll
        for (int d = 0; d < NB; ++d) acc[d] *= alpha;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                sc[g][i] = expf(sc[g][i] - ref);
                l += sc[g][i];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int d = 0; d < NB; ++d)
                    acc[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(Vs[(g * 16 + kgrp * 4 + e) * LD + d * 16 + l16], sc[g][e], acc[d], 0, 0, 0);
        }
    }
    l = sum_xor32(sum_xor16(l));
    if (row >= a.rows) return;
    float* p = (float*)a.o + it.b * a.s.o_batch + cross_row(a, it.g, row, a.s.o_tok, a.s.o_head) + kgrp * 4;
#pragma unroll
    for (int d = 0; d < NB; ++d) *reinterpret_cast<f32x4_t*>(p + d * 16) = l == 0.f ? f32x4_t{0.f, 0.f, 0.f, 0.f} : acc[d] / l;
}

size_t cross_workspace_bytes(int, const CrossArgs&) { return 0; }

template <int HD>
static hipError_t launch_cross_hd(int dtype, CrossArgs a, hipStream_t st) {
    a.nsplit = 1;
    constexpr int QT = HD == 128 ? 2 : 4;
    const int bq = dtype == PS_BF16 ? 4 * QT * 16 : 64;
    a.row_blocks = (a.rows + bq - 1) / bq;
    const unsigned grid = (unsigned)((long)a.batch * a.kv_heads * a.row_blocks * a.nsplit);
    if (dtype == PS_BF16) cross_bf16_kernel<HD, QT><<<grid, 256, 0, st>>>(a);
    else cross_f32_kernel<HD><<<grid, 256, 0, st>>>(a);
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
