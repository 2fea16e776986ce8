// Rotary positions on several axes, and norms of queries and keys for each head with the rotation in the same pass.
#include "qk_norm.h"
#include "lane_sums.h"
#include "plan.h"
#include "row_eights.h"

namespace ps {

// ------------------------------------------------------------------------------------ table
// (cos, sin) of position * frequency for every token and pair.  Angles in 64 bits: at position 17776 the lowest pair's 32-bit angle would be off
// by 2^-10.  A thread per pair; the 64-bit sine and cosine bind (17776 tokens x 32 pairs).
__global__ void __launch_bounds__(256)
rope_table_kernel(const float* __restrict__ positions, long position_row, RopeAxes axes, float* __restrict__ table, unsigned n) {
    const unsigned id = blockIdx.x * 256u + threadIdx.x;
    if (id >= n) return;
    const unsigned t = id / (unsigned)axes.pairs, p = id - t * (unsigned)axes.pairs;
    double s, c;
    sincos((double)positions[t * position_row + axes.axis[p]] * axes.freq[p], &s, &c);
    reinterpret_cast<f32x2_t*>(table)[id] = f32x2_t{(float)c, (float)s};
}

hipError_t launch_rope_table(const float* positions, long position_row, const RopeAxes& axes, float* table, int tokens, hipStream_t st) {
    const unsigned n = (unsigned)tokens * (unsigned)axes.pairs;
    rope_table_kernel<<<(n + 255) / 256, 256, 0, st>>>(positions, position_row, axes, table, n);
    return hipGetLastError();
}

// ------------------------------------------------------------------------------------ norm and rotation
// y = rotate(norm(x) * gamma + beta): norm 0 none, 1 x / sqrt(mean x^2 + eps), 2 (x - mean) / sqrt(mean (x - mean)^2 + eps), over a head; pair p of the
// first 2 * pairs values turns by the table's angle p of the token: values 2p and 2p + 1, or (halves) p and p + pairs.
// Memory binds: q and k are read and written once.  A wave takes a token, L lanes a head with 8 adjacent values each; it goes over the
// token's heads 4 rounds at a time, whose loads are requested together, and has the token's angles in registers.  (17776 tokens of 60 heads of 64 in bf16, 278 MB: 65 us,
// 4.3 TB/s, where a copy reaches 4.9.)
// L: lanes of a head, a power of two (of which head_dim / 8 work).
template <int L>
__device__ __forceinline__ float sum_of_team(float v) {
    if constexpr (L >= 2) v += dpp<DPP_QUAD_XOR_1>(v);
    if constexpr (L >= 4) v += dpp<DPP_QUAD_XOR_2>(v);
    if constexpr (L >= 8) v += dpp<0x141>(v);            // lane 7 - i of 8: the other four's sum
    if constexpr (L >= 16) v += dpp<0x140>(v);           // lane 15 - i of 16
    if constexpr (L >= 32) v = sum_xor16(v);
    return v;
}

template <typename T>
__device__ __forceinline__ void qk_store(T* p, const float (&v)[8], bool stream) {
    if constexpr (sizeof(T) == 2) {
        store_streamed<2>(p, __builtin_convertvector(f32x8_t{v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]}, bf16x8_t), stream);
    } else {
        store_streamed<4>(p, f32x4_t{v[0], v[1], v[2], v[3]}, stream);
        store_streamed<4>(p + 4, f32x4_t{v[4], v[5], v[6], v[7]}, stream);
    }
}

template <typename T, int L, bool HALVES>
__global__ void __launch_bounds__(256)
qk_norm_rope_kernel(QkNormArgs a, long lines) {
    constexpr int TEAMS = 64 / L, U = 4, CS = HALVES ? 8 : 4;
    const long line = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (line >= lines) return;                           // (whole waves)
    const int b = (int)(line / a.tokens), tok = (int)(line - (long)b * a.tokens);
    const int lane = threadIdx.x & 63, l = lane & (L - 1), team = lane / L, d = l * 8;
    const bool in = d < a.head_dim, turned = d < 2 * a.pairs, high = HALVES && d >= a.pairs;
    f32x2_t cs[CS];
#pragma unroll
    for (int i = 0; i < CS; ++i) cs[i] = f32x2_t{1.f, 0.f};
    if (turned) {
        const float* t = a.table + b * a.table_batch + (long)tok * (2 * a.pairs) + (HALVES ? (high ? d - a.pairs : d) * 2 : d);
#pragma unroll
        for (int i = 0; i < CS; i += 2) {
            const f32x4_t w = *reinterpret_cast<const any_f32x4_t*>(t + 2 * i);
            cs[i] = f32x2_t{w[0], w[1]};
            cs[i + 1] = f32x2_t{w[2], w[3]};
        }
    }
    const float inv_d = 1.0f / (float)a.head_dim;
    for (int s = 0; s < 2; ++s) {
        const QkSide& q = a.side[s];
        const T* x = (const T*)q.x + b * q.x_batch + tok * q.x_tok + d;
        T* o = (T*)q.out + b * q.o_batch + tok * q.o_tok + d;
        float gamma[8], beta[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            gamma[i] = a.norm && q.gamma && in ? q.gamma[d + i] : 1.f;
            beta[i] = a.norm && q.beta && in ? q.beta[d + i] : 0.f;
        }
        for (int h0 = team; h0 - team < q.heads; h0 += U * TEAMS) {      // (every lane takes part in the sums)
            float v[U][8];
#pragma unroll
            for (int u = 0; u < U; ++u) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[u][i] = 0.f;
                if (in && h0 + u * TEAMS < q.heads) load_eight(v[u], x + (h0 + u * TEAMS) * q.x_head, 0, 8);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (h0 - team + u * TEAMS >= q.heads) continue;          // (the whole wave)
                float (&y)[8] = v[u];
                if (a.norm == 2) {
                    float sum = 0.f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum += y[i];
                    const float mean = sum_of_team<L>(sum) * inv_d;
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[i] = in ? y[i] - mean : 0.f;
                }
                if (a.norm) {
                    float sum = 0.f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(y[i], y[i], sum);
                    const float r = 1.0f / sqrtf(__builtin_fmaf(sum_of_team<L>(sum), inv_d, a.eps));
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[i] = __builtin_fmaf(y[i] * r, gamma[i], beta[i]);
                }
                if constexpr (HALVES) {
                    // the partner's value lies pairs / 8 lanes away
                    const int other = lane + (high ? -(a.pairs / 8) : a.pairs / 8);
                    float w[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[i] = __shfl(y[i], other);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float t = __builtin_fmaf(y[i], cs[i][0], (high ? w[i] : -w[i]) * cs[i][1]);
                        y[i] = turned ? t : y[i];
                    }
                } else if (turned) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float c = y[2 * i], e = y[2 * i + 1];
                        y[2 * i] = __builtin_fmaf(c, cs[i][0], -(e * cs[i][1]));
                        y[2 * i + 1] = __builtin_fmaf(e, cs[i][0], c * cs[i][1]);
                    }
                }
                if (in && h0 + u * TEAMS < q.heads) qk_store(o + (h0 + u * TEAMS) * q.o_head, y, a.stream);
            }
        }
    }
}

template <typename T, int L>
static void launch_team(const QkNormArgs& a, hipStream_t st) {
    const long lines = (long)a.batch * a.tokens;
    if constexpr (L > 1) {                               // (a head of 8 has no halves of 8)
        if (a.halves) {
            qk_norm_rope_kernel<T, L, true><<<(unsigned)((lines + 3) / 4), 256, 0, st>>>(a, lines);
            return;
        }
    }
    qk_norm_rope_kernel<T, L, false><<<(unsigned)((lines + 3) / 4), 256, 0, st>>>(a, lines);
}
template <typename T>
static hipError_t launch_typed(const QkNormArgs& a, hipStream_t st) {
    const int lanes = a.head_dim / 8;
    if (lanes <= 1) launch_team<T, 1>(a, st);
    else if (lanes <= 2) launch_team<T, 2>(a, st);
    else if (lanes <= 4) launch_team<T, 4>(a, st);
    else if (lanes <= 8) launch_team<T, 8>(a, st);
    else if (lanes <= 16) launch_team<T, 16>(a, st);
    else launch_team<T, 32>(a, st);
    return hipGetLastError();
}

hipError_t launch_qk_norm_rope(int dtype, QkNormArgs a, hipStream_t st) {
    const size_t esize = dtype == PS_BF16 ? 2 : 4;
    a.stream = (size_t)a.batch * a.tokens * (a.side[0].heads + a.side[1].heads) * a.head_dim * esize > STREAM_BYTES;
    return dtype == PS_BF16 ? launch_typed<bf16_t>(a, st) : launch_typed<float>(a, st);
}

}  // namespace ps
