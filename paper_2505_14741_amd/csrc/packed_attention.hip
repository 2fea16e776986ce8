// Attention inside the samples that are packed along one token axis: o_i = sum_j p_ij v_j / sum_j p_ij, p_ij = exp(x_ij - max), over the keys j of query
// i's own sample that it sees; x_ij = scale q_i k_j, capped by cap * tanh(x / cap), less slope * |frame(i) - frame(j)|.
//
// A sample's queries are its last tokens: query t of nq stands at nk - nq + t of the sample's nk keys.  Behind the sample's prefix, tokens lie in frames; a query
// sees the prefix and, causally, the frames up to its own: its first reach(t) keys, a number that does not fall from query to query.  So a
// tile of 64 keys is whole for a wave's rows, cut by their reach, or behind it, and only those that are cut look at single keys.
//
// Query heads that share a key head are rows of one product, row = token * share + head of the group.  Blocks of BQ rows of one (sample, key head)
// are found on the GPU, from the offsets (packed_item); the host knows how many there are at most.
#include "packed_attention.h"
#include "lane_sums.h"
#include "plan.h"
#include "tile_ops.h"
#include <algorithm>
#include <type_traits>

namespace ps {

typedef __attribute__((ext_vector_type(16))) float f32x16_t;
typedef __attribute__((ext_vector_type(4))) short s16x4_t;
typedef __attribute__((ext_vector_type(4))) int i32x4_t;

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int within(int v, int lo, int hi) { return min(max(v, lo), hi); }

// n / frame for 0 <= n < 2^24 and inv = 1 / frame: the product is off by less than one
__device__ __forceinline__ unsigned frame_of(unsigned n, unsigned frame, float inv) {
    unsigned f = (unsigned)((float)n * inv);
    f -= f * frame > n ? 1u : 0u;
    return f + (n - f * frame >= frame ? 1u : 0u);
}

// (wave-uniform)
struct PackedItem {
    int g, r0, rows, q0, k0, keys, ahead, prefix, piece, pieces, sample;
    unsigned front;                                      // rows of partial sums of a key head in front of the sample's
    float inv_frame;
    bool any;
    // keys that a query sees, at `pos` of the sample's keys
    __device__ __forceinline__ int reach(const PackedArgs& a, int pos) const {
        if (!a.causal) return keys;
        if (pos < prefix) return prefix;
        return (int)min((long)keys, prefix + ((long)frame_of((unsigned)(pos - prefix), (unsigned)a.frame, inv_frame) + 1) * a.frame);
    }
};
// Which key head and slot a workgroup takes.  Workgroup ids go to the 8 XCDs in turn, each with an L2 of its own: an XCD has kv_heads / 8 key heads to itself and
// every eighth item of the others', over 8 slots as many as all XCDs; low slots, which are long, first.
__device__ __forceinline__ void packed_place(unsigned id, int kv_heads, int& g, int& slot) {
    const unsigned x = id & 7, n = id >> 3, own = (unsigned)kv_heads / 8, rest = (unsigned)kv_heads % 8;
    const unsigned period = n / (unsigned)kv_heads, i = n - period * (unsigned)kv_heads;
    if (i < 8 * own) {
        slot = (int)(period * 8 + i / own);
        g = (int)(x * own + i % own);
    } else {
        const unsigned u = (period * rest + i - 8 * own) * 8 + x;
        slot = (int)(u / rest);
        g = (int)(8 * own + u % rest);
    }
}
// A sample's slots for a key head: its blocks, each in its pieces.
struct PackedCount { int q0, nq, k0, keys, blocks, pieces; };
template <int BQ>
__device__ __forceinline__ PackedCount packed_count(const PackedArgs& a, int s) {
    PackedCount c;
    c.q0 = within(a.q_offsets[s], 0, a.q_tokens);
    c.nq = within(a.q_offsets[s + 1], c.q0, a.q_tokens) - c.q0;
    c.k0 = c.q0;
    c.keys = c.nq;
    if (a.own_offsets) {
        c.k0 = within(a.kv_offsets[s], 0, a.kv_tokens);
        c.keys = within(a.kv_offsets[s + 1], c.k0, a.kv_tokens) - c.k0;
    }
    c.blocks = (c.nq * a.share + BQ - 1) / BQ;
    c.pieces = a.own_offsets ? packed_pieces(c.nq * a.share, c.keys, a.kv_heads) : 1;
    return c;
}
// Rows of a sample's partial sums (below 2^28; of all together below 2^30, but for offsets that fall, where sums of them may wrap around).
__device__ __forceinline__ unsigned packed_rows(const PackedArgs& a, const PackedCount& c) { return c.pieces > 1 ? (unsigned)(c.nq * a.share * c.pieces) : 0; }
// More than PACKED_SEARCH samples: a table of (sample, slot of the sample) for every slot, table[0].x of them behind it, and of the rows of partial sums in front of
// every sample; made by one workgroup.
template <int BQ>
__global__ void __launch_bounds__(1024)
packed_table_kernel(PackedArgs a) {
    __shared__ int sums[16];
    __shared__ unsigned rows[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int2* const table = a.table;
    unsigned* const fronts = reinterpret_cast<unsigned*>(table + 1 + a.slots);
    long base = 0;                                       // (offsets that fall could count far more than there are)
    unsigned front_base = 0;
    for (int s0 = 0; s0 < a.samples; s0 += 1024) {
        const int s = s0 + (int)threadIdx.x;
        int n = 0;
        unsigned own = 0;
        if (s < a.samples) {
            const PackedCount c = packed_count<BQ>(a, s);
            n = min(c.blocks * c.pieces, a.slots);
            own = packed_rows(a, c);
        }
        int upto = n;                                    // inclusive sums
        unsigned rows_upto = own;
#pragma unroll
        for (int x = 1; x < 64; x *= 2) {
            const int v = __shfl_up(upto, x);
            const unsigned u = __shfl_up(rows_upto, x);
            upto += lane >= x ? v : 0;
            rows_upto += lane >= x ? u : 0;
        }
        __syncthreads();
        if (lane == 63) {
            sums[wave] = upto;
            rows[wave] = rows_upto;
        }
        __syncthreads();
        long at = base + upto - n;
        unsigned front = front_base + rows_upto - own;
        for (int w = 0; w < 16; ++w) {
            at += w < wave ? sums[w] : 0;
            base += sums[w];
            front += w < wave ? rows[w] : 0;
            front_base += rows[w];
        }
        for (int i = 0; i < n && at + i < a.slots; ++i) table[1 + at + i] = make_int2(s, i);
        if (s < a.samples) fronts[s] = front;
    }
    if (threadIdx.x == 0) table[0] = make_int2((int)min(base, (long)a.slots), 0);
}

// The block's sample, rows and piece.  Up to 64 samples are looked through here, those with more keys first.  A sample's last blocks, whose rows see most, come
// first.
template <int BQ>
__device__ __forceinline__ PackedItem packed_item(const PackedArgs& a, int lane, unsigned id) {
    PackedItem t;
    int slot, of_sample;                                 // of_sample: which of the sample's slots
    packed_place(id, a.kv_heads, t.g, slot);
    t.any = false;
    t.front = 0;
    if (slot >= a.slots) return t;
    PackedCount c;
    if (a.samples <= PACKED_SEARCH) {
        c = packed_count<BQ>(a, min(lane, a.samples - 1));
        const int n = lane < a.samples ? c.blocks * c.pieces : 0;
        int before = 0;                                  // slots of the samples in front
        for (int i = 0; i < a.samples; ++i) {
            const int k = __builtin_amdgcn_readlane(c.keys, i), m = __builtin_amdgcn_readlane(n, i);
            before += k > c.keys || (k == c.keys && i < lane) ? m : 0;
        }
        const unsigned long long here = __ballot(slot >= before && slot < before + n);
        if (here == 0) return t;
        t.sample = __builtin_ctzll(here);
        of_sample = slot - __builtin_amdgcn_readlane(before, t.sample);
        if (__builtin_amdgcn_readlane(c.pieces, t.sample) > 1) {
            const int rows = (int)packed_rows(a, c);
            for (int i = 0; i < t.sample; ++i) t.front += (unsigned)__builtin_amdgcn_readlane(rows, i);
        }
        c.q0 = __builtin_amdgcn_readlane(c.q0, t.sample);
        c.nq = __builtin_amdgcn_readlane(c.nq, t.sample);
        c.k0 = __builtin_amdgcn_readlane(c.k0, t.sample);
        c.keys = __builtin_amdgcn_readlane(c.keys, t.sample);
        c.blocks = __builtin_amdgcn_readlane(c.blocks, t.sample);
        c.pieces = __builtin_amdgcn_readlane(c.pieces, t.sample);
    } else {
        if (slot >= uniform(a.table[0].x)) return t;
        const int2 e = a.table[1 + slot];
        t.sample = uniform(e.x);
        of_sample = uniform(e.y);
        t.front = (unsigned)uniform((int)reinterpret_cast<const unsigned*>(a.table + 1 + a.slots)[t.sample]);
        c = packed_count<BQ>(a, t.sample);
        c.q0 = uniform(c.q0); c.nq = uniform(c.nq); c.k0 = uniform(c.k0); c.keys = uniform(c.keys); c.blocks = uniform(c.blocks); c.pieces = uniform(c.pieces);
    }
    const int block = (int)((unsigned)of_sample / (unsigned)c.pieces);
    t.piece = of_sample - block * c.pieces;
    t.pieces = c.pieces;
    t.rows = c.nq * a.share;
    // (offsets that fall: the block's last pieces have no slot, or the sample's rows no place)
    if (t.pieces > 1 && (slot - t.piece + t.pieces > a.slots || t.front > a.part_rows || packed_rows(a, c) > a.part_rows - t.front)) return t;
    t.q0 = c.q0;
    t.r0 = (c.blocks - 1 - block) * BQ;
    t.k0 = c.k0;
    t.keys = c.keys;
    t.ahead = c.keys - c.nq;
    t.prefix = a.prefix ? uniform(within(a.prefix[t.sample], 0, t.keys)) : 0;
    t.inv_frame = 1.0f / (float)a.frame;
    t.any = true;
    return t;
}
// where a row's partial sums lie: [key head][row] of each of the sample's pieces
template <int HD>
__device__ __forceinline__ float* packed_part(const PackedArgs& a, const PackedItem& t, int piece, int row) {
    return a.part + ((long)t.front * a.kv_heads + ((long)piece * a.kv_heads + t.g) * t.rows + row) * (HD + 4);
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
        r.frame = (float)frame_of((unsigned)(pos - t.prefix), (unsigned)a.frame, t.inv_frame);
    }
    return r;
}
// A key's frame, NaN in the prefix.
__device__ __forceinline__ float packed_frame(const PackedArgs& a, const PackedItem& t, int key) {
    return key < t.prefix ? __uint_as_float(0x7fc00000u) : (float)frame_of((unsigned)min(key - t.prefix, (1 << 24) - 1), (unsigned)a.frame, t.inv_frame);
}
// slope * distance, 0 where the key is in the prefix
__device__ __forceinline__ float packed_bias(const PackedRow& r, float frame) {
    const float far = fabsf(r.frame - frame);
    return far == far ? r.slope * far : 0.f;
}

template <int N>
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

__device__ __forceinline__ float exp2_between(float a, float b, float c) {
    const float half = (0.5f * a - 0.5f * b) * c;
    return __builtin_amdgcn_exp2f(half + half);
}

// ------------------------------------------------------------------------------------ bf16
// Tiles are transposed: S^T = K Q^T leaves a query in lane % 32 and keys 8 (i / 4) + 4 (lane / 32) + i % 4 of every 32 in register i, which, rounded to
// bf16, are the second operand of O^T = V^T P^T as they stand (its k in the order of the registers; V fragments follow).
//
// What binds is the vector unit (an exponential, a multiply-add and half a conversion for each score) next to the matrix unit, so the loop goes
// over halves of 32 keys in three parts that do not depend on each other: the scores of the next half, the weights of this one, the values of the last one.
// K and V go straight into LDS, K a tile ahead of its use and V with it, three slots each and one hand-over per tile; rows of a tile are permuted in chunks
// of 16 bytes so that fragment reads meet different banks.
//
// A row's exponents are relative to the largest score of its first 32 keys (without the distance bias, which is not positive where slopes are not
// negative), instead of a maximum that moves: what the sums became is looked at behind the last key.  Rows whose sum is not within 2^-40 .. 2^32, or
// above 2^8 (which values may be multiplied with) with outputs that are not finite, or whose reference is beyond 2^10 (where the rounding of
// scale * score is 2^-14), are computed again by tracked(): a reference that moves where a score exceeds it by 8 in powers of two, and is
// subtracted first where it is large.  The rows next to them keep what they have, so a row's result depends neither on them nor on the block's size.
//
// Measured: five samples of 671 to 8326 tokens, 30 heads of 64 (761 GFLOP) 801 to 843 us, 0.90 to 0.95 PFLOP/s; 17776 tokens causal by frames (1305 GFLOP) 1.43 to
// 1.50 ms, 0.87 to 0.91; the simple kernel, one moving reference and a tile of 64 keys at a time, 1061 and 1810.  Vector instructions are at work 64 % of the time, the
// matrix unit 44 %, together less than half of it: what a wave's three parts leave free the other wave of the SIMD hardly takes, and at the end of the launch 1.65 of 2 waves are there.  Four slots of keys and
// a manual order of the parts: as fast; items in the order of the offsets and over all XCDs instead of as packed_place() and packed_item() have them: 931 and 1766 us
// (with them 847 and 1540, of that time's kernel).
constexpr float PACKED_AHEAD = 8.0f, PACKED_FAR = 0x1p+10f;
constexpr float PACKED_SUM_MIN = 0x1p-40f, PACKED_SUM_MAX = 0x1p+32f, PACKED_SUM_NEAR = 0x1p+8f;
constexpr int PACKED_BQ_F32 = 64;

// Largest cap that bf16 computes as cap - 2 cap / (1 + 2^(..)) alone, off by 2^-22 of the cap: 2^-14 here, where weights are rounded by 2^-8.
constexpr float PACKED_CAP_NEAR = 256.0f;
// Next to zero that form is off by more of x than its own roundings the larger the cap is; below a quarter of the cap the first terms of the series of cap * tanh(x / cap)
// take its place.  w = 2 log2(e) x / cap; x + x (-t^2 / 3 + 2 t^4 / 15 - 17 t^6 / 315 + 62 t^8 / 2835) for t = x / cap, t^2 = w^2 ln(2)^2 / 4: off by 2^-23 of x at most.
// Together with the other form: 2^-20 of x (its exponential and quotient, at a quarter of the cap).
constexpr float PACKED_CAP_SERIES = 0.5203422f;              // (log2(e) / 2)^2
__device__ __forceinline__ float packed_cap_series(float x, float w2) {
    const float p = __builtin_fmaf(__builtin_fmaf(__builtin_fmaf(4.5520010e-6f, w2, -9.3521435e-5f), w2, 1.9236258e-3f), w2, -0.040037751f);
    return __builtin_fmaf(x * w2, p, x);
}

__device__ __forceinline__ s16x4_t packed_read_tr16(const unsigned char* p) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(p));
}

enum PackedFrames { PACKED_ONE, PACKED_EACH, PACKED_ANY };
enum PackedState { ROW_REACH, ROW_SLOPE, ROW_FRAME, ROW_M, ROW_MC, ROW_STATES };     // (ROW_MC: the reference in powers of two)

// CAP: 0 none; 1 up to PACKED_CAP_NEAR; 2 above it (4276 tokens of 30 heads of 64: 220, 342 and 372 us; an exponential, a reciprocal and, of the last, the
// series for each score).
// BIAS: 0 none; 1 in frames of 64 keys and more, most tiles of which have one bias for each row; 2 in shorter ones.  Two kernels, because the loops of both
// in one leave it without registers.  (1350 rows of 30 heads against 17776 keys in frames of 1350: 316 us, with each
// key's bias looked up 381; now, with its join, 265 to 286.)
template <int HD, int QT, int CAP, int BIAS>
struct PackedBf16 {
    static constexpr int U = HD > 64 ? 32 : 64, HALVES = U / 32;     // keys of a tile
    static constexpr int SLOTS = 3;                                  // tiles of K, and of V, in LDS (four, requested a tile earlier: as fast)
    static constexpr int NB = HD < 32 ? 1 : HD / 32, QS = HD / 16, ROW = HD * 2, TILE = U * ROW;
    static constexpr int LOADS = 2 * TILE / 1024 / 4;                // 1 KB loads per wave: K's by the first waves, V's by the others
    static_assert(LOADS * 4 * 1024 == 2 * TILE, "every wave requests as many");

    const PackedArgs& a;
    const PackedItem& it;
    unsigned char *const kl, *const vl;                              // SLOTS tiles each
    float* const fl;                                                 // frames of their keys
    const bf16_t *kb, *vb;
    int lane, wave, l32, hi;
    float* const rs;                                                 // the lane's rows' state, which the steady loop has no registers for: [ROW_*][row]
    float c0, cap2, into, m[QT], ref[QT];                            // m: the reference, a score (capped or biased: in powers of two); ref: see refer()
    int koff[QS], voff[NB], now, now_end;
    bf16x8_t qf[QT][QS];
    f32x16_t acc[QT][NB];
    float l[QT];                                                     // of the lane's keys

    // chunk of a row -> its place
    __device__ __forceinline__ static int k_place(int r) { return HD == 16 ? 0 : HD == 32 ? (r >> 2) & 3 : r & 7; }
    __device__ __forceinline__ static int v_place(int r) { return HD <= 32 ? 0 : HD == 64 ? (r & 3) | (r & 2) << 1 : (r & 3) << 2; }

    __device__ __forceinline__ PackedBf16(const PackedArgs& a_, const PackedItem& it_, unsigned char* lds, float* frames, float* rows)
        : a(a_), it(it_), kl(lds), vl(lds + SLOTS * TILE), fl(frames), rs(rows) {}
    __device__ __forceinline__ float& state(int what, int q) const { return rs[what * 128 * QT + q * 32]; }
    __device__ __forceinline__ PackedRow me(int q) const { return PackedRow{__float_as_int(state(ROW_REACH, q)), state(ROW_SLOPE, q), state(ROW_FRAME, q)}; }

    __device__ __forceinline__ void start(int w0) {
        kb = (const bf16_t*)a.k + (long)it.k0 * a.k_tok + it.g * a.k_head;
        vb = (const bf16_t*)a.v + (long)it.k0 * a.v_tok + it.g * a.v_head;
        c0 = a.scale * PACKED_LOG2E;
        cap2 = a.cap * PACKED_LOG2E;
        into = CAP ? 2.0f * c0 / a.cap : 0.f;
#pragma unroll
        for (int q = 0; q < QT; ++q) {
            const int row = min(w0 + q * 32 + l32, it.rows - 1);
            const PackedRow r = packed_query(a, it, row);
            state(ROW_REACH, q) = __int_as_float(r.reach);
            state(ROW_SLOPE, q) = r.slope * PACKED_LOG2E;
            state(ROW_FRAME, q) = r.frame;
            const bf16_t* p = (const bf16_t*)a.q + packed_row(a, it, row, a.q_tok, a.q_head) + hi * 8;      // second operand of S^T: 8 consecutive d of row l32
#pragma unroll
            for (int s = 0; s < QS; ++s) qf[q][s] = *reinterpret_cast<const bf16x8_t*>(p + s * 16);
        }
#pragma unroll
        for (int s = 0; s < QS; ++s) koff[s] = l32 * ROW + ((2 * s + hi) ^ k_place(l32)) * 16;
        // V^T: row d = l32 of each 32; slot (hi, e) of a step of 16 keys is key 8 (e / 4) + 4 hi + e % 4 (heads of 16: the upper 16 rows repeat the lower)
        const int r = (lane & 15) >> 2;
#pragma unroll
        for (int d = 0; d < NB; ++d)
            voff[d] = (4 * hi + r) * ROW + ((d * 4 + (HD < 32 ? 0 : (lane & 16) >> 3) + ((lane & 3) >> 1)) ^ v_place(r)) * 16 + (lane & 1) * 8;
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int q = 0; q < QT; ++q) {
            l[q] = 0.f;
            m[q] = -INFINITY;
#pragma unroll
            for (int d = 0; d < NB; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[q][d][i] = 0.f;
        }
    }
    // requests the keys of tile tk and the values of tile tv (those that lie before `end`) into their slots; keys behind the sample's last one repeat it
    __device__ __forceinline__ void request(int tk, int kslot, int tv, int vslot, int end) {
        const bool of_k = wave < 2;                      // (uniform)
        const int tile = of_k ? tk : tv;
        if (tile < 0 || tile >= end) return;
        const bf16_t* const from = of_k ? kb : vb;
        const long tok = of_k ? a.k_tok : a.v_tok;
        unsigned char* const to = (of_k ? kl + kslot * TILE : vl + vslot * TILE) + (wave & 1) * LOADS * 1024;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int at = ((wave & 1) * LOADS + i) * 1024 + lane * 16, r = at / ROW, chunk = at % ROW / 16 ^ (of_k ? k_place(r) : v_place(r));
            lds_dma16(from + min(tile * U + r, it.keys - 1) * tok + chunk * 8, (unsigned)uniform((int)(unsigned)(size_t)PS_LDS_PTR(to + i * 1024)));
        }
    }
    __device__ __forceinline__ void frames(int tile, int slot) {     // (visible behind the next barrier)
        if (BIAS && threadIdx.x < U) fl[slot * U + threadIdx.x] = packed_frame(a, it, tile * U + (int)threadIdx.x);
    }

    __device__ __forceinline__ const unsigned char* keys_at(int slot, int half) const { return kl + slot * TILE + half * 32 * ROW; }
    __device__ __forceinline__ const unsigned char* values_at(int slot, int half) const { return vl + slot * TILE + half * 32 * ROW; }
    __device__ __forceinline__ const float* frames_at(int slot, int half) const { return fl + slot * U + half * 32; }
    // QN: query tiles that count
    template <int QN>
    __device__ __forceinline__ void scores(f32x16_t (&s)[QN], const unsigned char* kt) const {
#pragma unroll
        for (int q = 0; q < QN; ++q)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[q][i] = 0.f;
#pragma unroll
        for (int x = 0; x < QS; ++x) {
            const bf16x8_t kf = *reinterpret_cast<const bf16x8_t*>(kt + koff[x]);
#pragma unroll
            for (int q = 0; q < QN; ++q) s[q] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[q][x], s[q], 0, 0, 0);
        }
    }
    __device__ __forceinline__ float capped(float s) const {         // in powers of two
        const float w = s * into, y = __builtin_fmaf(-2.0f * cap2, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(w)), cap2);
        return CAP == 2 && w * w < PACKED_CAP_SERIES ? packed_cap_series(s * c0, w * w) : y;
    }
    // keys that the row does not see
    __device__ __forceinline__ void cut(f32x16_t& s, int q, int kv0) const {
        const int left = me(q).reach - kv0 - 4 * hi;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 8 * (i / 4) + i % 4 < left ? s[i] : -INFINITY;
    }
    // The frame of the keys at hand (-1: the prefix) and where it ends; keys come in order.  Those that lie there have one bias for each row: ref is
    // the reference and it.
    __device__ __forceinline__ void first_frame(int kv0) {
        now = kv0 < it.prefix ? -1 : uniform((int)frame_of((unsigned)(kv0 - it.prefix), (unsigned)a.frame, it.inv_frame));
        now_end = (int)min((long)it.prefix + (long)(now + 1) * a.frame, 1L << 30);
    }
    __device__ __forceinline__ void refer() {
#pragma unroll
        for (int q = 0; q < QT; ++q) {
            const float mc = state(ROW_MC, q);
            ref[q] = BIAS == 1 && now >= 0 ? __builtin_fmaf(me(q).slope, fabsf(me(q).frame - (float)now), mc) : mc;
        }
    }
    __device__ __forceinline__ void advance(int kv0) {
        while (kv0 >= now_end) {
            ++now;
            now_end = (int)min((long)now_end + a.frame, 1L << 30);
        }
        refer();
    }
    __device__ __forceinline__ static float largest(const f32x16_t& s) {
        float top = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
        return max_xor32(top);
    }
    // Weights 2^(x - reference - bias) of a half, rounded to bf16 for the second product; the same numbers whichever way their keys' frames are looked at
    // (PACKED_ONE: all in the frame at hand; PACKED_EACH: each key's, none in the prefix; PACKED_ANY) and whether some keys are not seen by some rows (CUT) or not.
    template <bool CUT, int FRAMES>
    __device__ __forceinline__ void weights(f32x16_t (&s)[QT], bf16x8_t (&pf)[QT][2], int kv0, const float* of) const {
#pragma unroll
        for (int q = 0; q < QT; ++q) {
            f32x16_t& x = s[q];
            const float c = CAP ? 1.0f : c0, mc = FRAMES == PACKED_ONE ? 0.f : state(ROW_MC, q);
            const PackedRow row = me(q);
            if constexpr (CAP) {
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = capped(x[i]);
            }
            if constexpr (CUT) cut(x, q, kv0);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float r = ref[q];
                if constexpr (FRAMES != PACKED_ONE) {
                    const float far = fabsf(row.frame - of[4 * hi + 8 * (i / 4) + i % 4]);
                    r = __builtin_fmaf(row.slope, far, mc);
                    if constexpr (FRAMES == PACKED_ANY) r = far == far ? r : mc;
                }
                pf[q][i / 8][i % 8] = (__bf16)__builtin_amdgcn_exp2f(__builtin_fmaf(x[i], c, -r));
            }
        }
    }
    // acc += V^T P^T, l += the weights as they were rounded (one key alone has weight 1 exactly).
    // CUT: some of the half's keys are not seen by some rows; they have the weight zero there, which a value that is not finite must not meet.
    template <bool CUT, int QN>
    __device__ __forceinline__ void values(const bf16x8_t (&pf)[QN][2], int kv0, const unsigned char* vt) {
        const __bf16 one = (__bf16)1.0f;
        typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
        bool odd = false;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
#pragma unroll
            for (int d = 0; d < NB; ++d) {
                s16x4_t lo = packed_read_tr16(vt + voff[d] + x * 16 * ROW), up = packed_read_tr16(vt + voff[d] + x * 16 * ROW + 8 * ROW);
                if constexpr (CUT) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const bool ol = (lo[i] & 0x7f80) == 0x7f80, ou = (up[i] & 0x7f80) == 0x7f80;
                        odd = odd || ol || ou;
                        lo[i] = ol ? 0 : lo[i];
                        up[i] = ou ? 0 : up[i];
                    }
                }
                const bf16x8_t vf = __builtin_shufflevector(__builtin_bit_cast(bf16x4_t, lo), __builtin_bit_cast(bf16x4_t, up), 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
                for (int q = 0; q < QN; ++q) acc[q][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[q][x], acc[q][d], 0, 0, 0);
            }
#pragma unroll
            for (int q = 0; q < QN; ++q)
#pragma unroll
                for (int e = 0; e < 8; e += 2)
                    l[q] = __builtin_amdgcn_fdot2_f32_bf16(bf16x2_t{pf[q][x][e], pf[q][x][e + 1]}, bf16x2_t{one, one}, l[q], false);
        }
        if (CUT && __any(odd)) {                         // what was left out, for the rows that see it
#pragma unroll 1
            for (int key = 0; key < 32; ++key) {
#pragma unroll
                for (int d = 0; d < NB; ++d)
#pragma unroll
                    for (int i = 0; i < (HD < 32 ? 8 : 16); ++i) {
                        const int at = d * 32 + 8 * (i / 4) + 4 * hi + i % 4;
                        const bf16_t* row = reinterpret_cast<const bf16_t*>(vt + key * ROW);
                        const float x = to_f32(row[(at / 8 ^ v_place(key)) * 8 + at % 8]);
#pragma unroll
                        for (int q = 0; q < QN; ++q)
                            if (kv0 + key < me(q).reach && !(fabsf(x) < INFINITY)) acc[q][d][i] += x;
                    }
            }
        }
    }
    // weights of a half with references that move
    template <int QN>
    __device__ __forceinline__ void tracked(f32x16_t (&s)[QN], bf16x8_t (&pf)[QN][2], int kv0, const float* of) {
        const float c = CAP || BIAS ? 1.0f : c0, ahead = fminf(PACKED_AHEAD / c, 0x1p+127f);
#pragma unroll
        for (int q = 0; q < QN; ++q) {
            f32x16_t& x = s[q];
            if constexpr (CAP || BIAS) {
                const float* f = of + 4 * hi;
                const PackedRow row = me(q);
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = (CAP ? capped(x[i]) : x[i] * c0) - (BIAS ? packed_bias(row, f[8 * (i / 4) + i % 4]) : 0.f);
            }
            cut(x, q, kv0);
            const float top = largest(x), mn = top > m[q] + ahead ? top : m[q], alpha = mn == m[q] ? 1.f : exp2_between(m[q], mn, c);   // 0 on the first tile
            m[q] = mn;
            l[q] *= alpha;
#pragma unroll
            for (int d = 0; d < NB; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[q][d][i] *= alpha;
            const float mm = mn == -INFINITY ? 0.f : mn * c;
            const bool far = fabsf(mm) > PACKED_FAR;
            const float first = far ? mn : 0.f, then = far ? 0.f : mm;
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int e = 0; e < 8; ++e) pf[q][y][e] = (__bf16)__builtin_amdgcn_exp2f(__builtin_fmaf(x[y * 8 + e] - first, c, -then));
        }
    }

    // Few rows (PACKED_FEW_ROWS): memory binds, and the waves take every fourth half of the keys each, through slots of their own and without a barrier; their
    // sums are united behind the last key, in the first wave's registers.  (Single tokens of eight samples against 128 MB of keys and values: 27 us,
    // 4.7 TB/s, and 7 for the join.)
    static constexpr int FEW_UNITS = HD > 64 ? 2 : 3, FEW_LOADS = 32 * ROW / 1024, FEW_HALF = 32 * ROW, FEW_BYTES = 4 * FEW_UNITS * FEW_HALF;
    static constexpr int MOST = 2 * SLOTS * TILE > FEW_BYTES ? 2 * SLOTS * TILE : FEW_BYTES, SUMS = 3 * (NB * 16 + 2) * 256, LDS_BYTES = MOST > SUMS ? MOST : SUMS;
    __device__ __forceinline__ void request_half(int h, unsigned char* to, bool of_k) {
#pragma unroll
        for (int i = 0; i < FEW_LOADS; ++i) {
            const int at = i * 1024 + lane * 16, r = at / ROW, chunk = at % ROW / 16 ^ (of_k ? k_place(r) : v_place(r)), key = min(h * 32 + r, it.keys - 1);
            const bf16_t* p = (of_k ? kb + key * a.k_tok : vb + key * a.v_tok) + chunk * 8;
            lds_dma16(p, (unsigned)uniform((int)(unsigned)(size_t)PS_LDS_PTR(to + i * 1024)));
        }
    }
    __device__ __forceinline__ void few(int first, int end) {        // halves first .. end - 1
        // Units of a wave in turn: keys, values, keys of the next half, ...; each is requested again as soon as it has been read.
        constexpr int L = FEW_LOADS, N3 = FEW_UNITS == 3;
        unsigned char* const own = kl + wave * FEW_UNITS * FEW_HALF;
        float* const of = fl + wave * 32;
        const int h0 = first + wave;
        if (h0 < end) {
            request_half(h0, own, true);
            request_half(h0, own + FEW_HALF, false);
            if (N3 && h0 + 4 < end) request_half(h0 + 4, own + 2 * FEW_HALF, true);
        }
        int u = 0;                                       // the keys' unit
        for (int h = h0; h < end; h += 4) {
            const int uv = u + 1 == FEW_UNITS ? 0 : u + 1;
            unsigned char *const ks = own + u * FEW_HALF, *const vs = own + uv * FEW_HALF;
            const bool more = h + 4 < end;
            if (N3 && more) wait_loads<2 * L>(); else wait_loads<L>();
            f32x16_t s[1];
            bf16x8_t pf[1][2];
            scores<1>(s, ks);
            if (BIAS && lane < 32) of[lane] = packed_frame(a, it, h * 32 + lane);
            wait_lds();
            if (more) request_half(h + 4, ks, !N3);      // the next values, or (of two units) the next keys
            tracked<1>(s, pf, h * 32, of);
            if (more) wait_loads<(N3 ? 2 : 1) * L>(); else wait_loads<0>();
            values<true, 1>(pf, h * 32, vs);
            wait_lds();
            if (N3 ? h + 8 < end : more) request_half(N3 ? h + 8 : h + 4, vs, N3);
            u = N3 ? (uv + 1 == FEW_UNITS ? 0 : uv + 1) : 0;
        }
        __syncthreads();                                 // (nobody reads its slots any more)
        float* const sums = reinterpret_cast<float*>(kl);            // [wave - 1][value][lane]
        constexpr int N = NB * 16 + 2;
        if (wave > 0) {
            float* to = sums + (wave - 1) * N * 64 + lane;
#pragma unroll
            for (int d = 0; d < NB; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) to[(d * 16 + i) * 64] = acc[0][d][i];
            to[(N - 2) * 64] = l[0];
            to[(N - 1) * 64] = m[0];
        }
        __syncthreads();
        if (wave > 0) return;
        const float c = CAP || BIAS ? 1.0f : c0;
        float top = m[0];
#pragma unroll
        for (int w = 0; w < 3; ++w) top = fmaxf(top, sums[(w * N + N - 1) * 64 + lane]);
        const float ref = top == -INFINITY ? 0.f : top, mine = exp2_between(m[0], ref, c);
        m[0] = top;
        l[0] *= mine;
#pragma unroll
        for (int d = 0; d < NB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[0][d][i] *= mine;
#pragma unroll
        for (int w = 0; w < 3; ++w) {
            const float* from = sums + w * N * 64 + lane;
            const float f = exp2_between(from[(N - 1) * 64], ref, c);
            l[0] = __builtin_fmaf(from[(N - 2) * 64], f, l[0]);
#pragma unroll
            for (int d = 0; d < NB; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[0][d][i] = __builtin_fmaf(from[(d * 16 + i) * 64], f, acc[0][d][i]);
        }
    }
};

template <int HD, int QT, int CAP, int BIAS>
__global__ void __launch_bounds__(256, QT == 1 && HD <= 64 ? 3 : 2)
packed_bf16_kernel(PackedArgs a) {
    typedef PackedBf16<HD, QT, CAP, BIAS> P;
    constexpr int U = P::U, NB = P::NB, HALVES = P::HALVES, BQ = 128 * QT;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[P::LDS_BYTES];
    __shared__ float fl[BIAS ? (P::SLOTS * U > 128 ? P::SLOTS * U : 128) : 1];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), l32 = lane & 31;
    const PackedItem it = packed_item<BQ>(a, lane, blockIdx.x);
    if (!it.any) return;                                 // (the whole workgroup)
    const bool few = it.rows <= PACKED_FEW_ROWS && it.keys > PACKED_FEW_MIN;         // (then all waves have the same rows)
    const int w0 = it.r0 + (few ? 0 : wave * 32 * QT), wl = min(w0 + 32 * QT - 1, it.rows - 1), bl = min(it.r0 + BQ, it.rows) - 1;
    const int most = w0 < it.rows ? it.reach(a, it.ahead + wl / a.share) : 0;        // (0: the wave has no rows)
    const int tiles_all = (it.keys + U - 1) / U, tiles = (it.reach(a, it.ahead + bl / a.share) + U - 1) / U;
    const int j0 = (int)((long)tiles_all * it.piece / it.pieces), j1 = min(tiles, (int)((long)tiles_all * (it.piece + 1) / it.pieces));
    const int end = (most + 31) / 32;                    // halves that some row of the wave sees

    __shared__ float rows[ROW_STATES * BQ];
    P t(a, it, lds, fl, rows + wave * 32 * QT + l32);
    t.lane = lane; t.wave = wave; t.l32 = l32; t.hi = lane >> 5;
    t.start(w0);
    t.clear();
    // a row's result, or its share of one
    auto store = [&](int q, bool in) {
        const int row = w0 + q * 32 + l32;
        const float sum = sum_xor32(t.l[q]);
        if (!in || row >= it.rows) return;
        if (it.pieces > 1) {
            float* p = packed_part<HD>(a, it, it.piece, row);
#pragma unroll
            for (int d = 0; d < NB; ++d)
#pragma unroll
                for (int r = 0; r < (HD < 32 ? 2 : 4); ++r)
                    *reinterpret_cast<f32x4_t*>(p + d * 32 + r * 8 + t.hi * 4) = f32x4_t{t.acc[q][d][4 * r], t.acc[q][d][4 * r + 1], t.acc[q][d][4 * r + 2], t.acc[q][d][4 * r + 3]};
            if (t.hi == 0) *reinterpret_cast<f32x2_t*>(p + HD) = f32x2_t{sum, t.m[q]};
            return;
        }
        const float inv = sum == 0.f ? 0.f : 1.0f / sum;
        bf16_t* p = (bf16_t*)a.o + packed_row(a, it, row, a.o_tok, a.o_head);
#pragma unroll
        for (int d = 0; d < NB; ++d)
#pragma unroll
            for (int r = 0; r < (HD < 32 ? 2 : 4); ++r) {
                const f32x4_t x = f32x4_t{t.acc[q][d][4 * r], t.acc[q][d][4 * r + 1], t.acc[q][d][4 * r + 2], t.acc[q][d][4 * r + 3]} * inv;
                *reinterpret_cast<bf16x4_t*>(p + d * 32 + r * 8 + t.hi * 4) = __builtin_convertvector(x, bf16x4_t);
            }
    };
    if (j0 >= j1) {                                      // (of few rows, every wave the same)
#pragma unroll
        for (int q = 0; q < QT; ++q) store(q, true);
        return;
    }
    if (few) {
        t.few(j0 * HALVES, min(j1 * HALVES, end));
        if (wave == 0) store(0, true);
        return;
    }
    f32x16_t s[2][QT];
    bf16x8_t pf[2][QT][2];
    if constexpr (BIAS) {
        t.frames(j0, 0);
        t.first_frame(j0 * U);
    }
    constexpr int SLOTS = P::SLOTS;
    t.request(j0, 0, -1, 0, j1);
    t.request(j0 + 1, 1, j0, 0, j1);
    // One tile.  Per half h (of all the sample's; parity X): the last one's values, the scores of the next one, this one's weights; the compiler mixes the three, and
    // from this order it makes the fastest code (17776 tokens 2478 us; scores, weights, values 2592, the other orders between 2533 and 2631).
    // Kinds: PACKED_ONE, all rows of the workgroup see the whole tile, which lies in one frame and is neither the first nor the last; PACKED_EACH, the same
    // behind the prefix with any frames; PACKED_ANY.
    int slot = 0;
    auto tile = [&](int j, auto x_c, auto kind_c) {
        constexpr int FRAMES = BIAS ? decltype(kind_c)::value : PACKED_ONE;
        constexpr bool STEADY = decltype(kind_c)::value != PACKED_ANY;
        wait_loads<0>();                                // K of the next tile, V of this one
        __syncthreads();                                 // ... everyone's; and nobody reads the last tile's K and the one before's V any more
        const int up = slot == 2 ? 0 : slot + 1, down = slot == 0 ? 2 : slot - 1;
        t.request(j + 2, down, j + 1, up, j1);
        if (STEADY || j + 1 < j1) t.frames(j + 1, up);
        if (!STEADY && j == j0 && j0 * HALVES < end) t.template scores<QT>(s[0], t.keys_at(slot, 0));
#pragma unroll
        for (int half = 0; half < HALVES; ++half) {
            const int X = HALVES == 2 ? half : decltype(x_c)::value, h = j * HALVES + half, kv0 = h * 32;
            const int next = half + 1 < HALVES ? slot : up, last = half > 0 ? slot : down, next_half = half + 1 < HALVES ? half + 1 : 0, last_half = half > 0 ? half - 1 : HALVES - 1;
            if constexpr (STEADY) {
                t.template values<false, QT>(pf[X ^ 1], kv0 - 32, t.values_at(last, last_half));
                t.template scores<QT>(s[X ^ 1], t.keys_at(next, next_half));
                t.template weights<false, FRAMES>(s[X], pf[X], kv0, t.frames_at(slot, half));
            } else {
                if (h + 1 < min(end, j1 * HALVES)) t.template scores<QT>(s[X ^ 1], t.keys_at(next, next_half));
                if (h < end) {
                    if (h == j0 * HALVES) {
#pragma unroll
                        for (int q = 0; q < QT; ++q) {
                            f32x16_t u = s[X][q];
                            t.cut(u, q, kv0);
                            const float top = P::largest(u);
                            const float m = top == -INFINITY ? top : CAP ? t.capped(top) : BIAS ? top * t.c0 : top;
                            t.state(ROW_M, q) = m;
                            t.state(ROW_MC, q) = top == -INFINITY ? 0.f : CAP || BIAS ? m : top * t.c0;
                        }
                        t.refer();
                    }
                    t.template weights<true, FRAMES>(s[X], pf[X], kv0, t.frames_at(slot, half));
                }
                if (h > j0 * HALVES && h - 1 < end) t.template values<true, QT>(pf[X ^ 1], kv0 - 32, t.values_at(last, last_half));
            }
        }
        slot = up;
    };
    const std::integral_constant<int, 0> c0;
    const std::integral_constant<int, 1> c1;
    const std::integral_constant<int, BIAS == 2 ? PACKED_EACH : PACKED_ONE> steady;
    const std::integral_constant<int, PACKED_ANY> general;
    const int all_see = it.reach(a, it.ahead + it.r0 / a.share);         // what the block's first row sees
    // the first tile from j on that is not as those before it: for the workgroup, or for a row's bias (counted in front of the loops: a condition that
    // changes the frame costs them their registers)
    const auto alike = [&](int j) {
        int stop = min(j1 - 1, all_see / U);
        if constexpr (BIAS == 1) {
            t.advance(j * U);
            stop = min(stop, t.now_end / U);
        }
        return BIAS == 2 && j * U < it.prefix ? j : stop;
    };
    int j = j0;
    if constexpr (HALVES == 2) {
        do {
            tile(j++, c0, general);
            for (const int stop = alike(j); j < stop; ++j) tile(j, c0, steady);
        } while (j < j1);
    } else {
        tile(j++, c0, general);
        while (j < j1) {
            for (const int stop = alike(j); j + 1 < stop; j += 2) { tile(j, c1, steady); tile(j + 1, c0, steady); }
            tile(j++, c1, general);
            if (j < j1) tile(j++, c0, general);
        }
    }
    const int h = j1 * HALVES;                           // the last half's values
    if (h - 1 < end) {
        const int last = slot == 0 ? SLOTS - 1 : slot - 1;
        if (HALVES == 2 || ((h - 1 - j0) & 1)) t.template values<true, QT>(pf[1], (h - 1) * 32, t.values_at(last, HALVES - 1));
        else t.template values<true, QT>(pf[0], (h - 1) * 32, t.values_at(last, HALVES - 1));
    }
    // rows that have to be computed again (those that see a key of the piece)
    bool redo[QT], again = false;
#pragma unroll
    for (int q = 0; q < QT; ++q) {
        redo[q] = false;
        if (end > j0 * HALVES) t.m[q] = t.state(ROW_M, q);           // (set with the wave's first half)
        if (end > j0 * HALVES && t.me(q).reach > j0 * U) {      // (a wave without rows has `end` 0)
            const float sum = sum_xor32(t.l[q]);
            redo[q] = !(sum >= PACKED_SUM_MIN && sum <= PACKED_SUM_MAX) || !(fabsf(t.state(ROW_MC, q)) <= PACKED_FAR);
            float zero = 0.f;                            // (NaN if a value is not finite)
#pragma unroll
            for (int d = 0; d < NB; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) zero = __builtin_fmaf(t.acc[q][d][i], 0.f, zero);
            zero = sum_xor32(zero);                      // (both lanes of the row alike; a maximum would lose the NaN)
            redo[q] = redo[q] || (sum > PACKED_SUM_NEAR && zero != 0.f);
        }
        store(q, !redo[q]);
        again = again || redo[q];
    }
    again = __any(again);
    if (__syncthreads_or(again)) {                       // (the whole workgroup loads)
        t.clear();
        for (int j = j0; j < j1; ++j) {
            __syncthreads();
            t.request(j, 0, j, 0, j1);
            t.frames(j, 0);
            wait_loads<0>();
            __syncthreads();
            if (again)
#pragma unroll 1
                for (int half = 0; half < HALVES; ++half)
                    if (j * HALVES + half < end) {
                        t.template scores<QT>(s[0], t.keys_at(0, half));
                        t.template tracked<QT>(s[0], pf[0], (j * HALVES + half) * 32, t.frames_at(0, half));
                        t.template values<true, QT>(pf[0], (j * HALVES + half) * 32, t.values_at(0, half));
                    }
        }
#pragma unroll
        for (int q = 0; q < QT; ++q) store(q, redo[q]);
    }
}

// ------------------------------------------------------------------------------------ fp32
// 16 rows per wave with full fp32 products (v_mfma_f32_16x16x4_f32): S^T = K Q^T leaves a row in lane % 16 with keys 4 (lane / 16) + i of every 16.
// Probabilities in fp32, exponentials as exact as expf.  What binds is the time of a step, two barriers and products and maxima that wait for each other.
// cap * tanh(x / cap), into = 2 / cap in powers of two: cap - 2 cap / (1 + 2^(into x)), the quotient refined once; the series below a quarter of the cap.
__device__ __forceinline__ float capped_of(float x, float cap, float into) {
    const float w = x * into, d = 1.0f + fminf(__builtin_amdgcn_exp2f(w), 0x1p+100f), r = __builtin_amdgcn_rcpf(d);
    const float y = __builtin_fmaf(-2.0f * cap, __builtin_fmaf(__builtin_fmaf(-d, r, 1.0f), r, r), cap);
    return w * w < PACKED_CAP_SERIES ? packed_cap_series(x, w * w) : x != x ? x : y;
}

// A workgroup takes 16 rows (of the block's 64, those of `part`), each wave a quarter of every tile's keys, and the waves' sums are united behind the last key.
// (1000, 517 and 77 tokens, 16 heads of 32, causal, capped, with a bias: 46 us, 37 since its parts lie side by side.  With rows of their own for each wave, and all
// keys, 80; 4276 tokens, 30 heads of 64, 6068 us against 1898, of 16 1825 against 560, of 128 13240 against 4360.)
template <int HD>
__device__ __forceinline__ void packed_f32_rows(const PackedArgs& a, const PackedItem& it, float* Ks, float* Vs, float* Fs, int lane, int wave, int part) {
    constexpr int KT = 64, LD = HD + 4, NB = HD / 16, CH = HD / 4, LOADS = KT * CH / 256, BQ = PACKED_BQ_F32;
    constexpr int AHEAD = HD <= 32 ? 4 : HD == 64 ? 2 : 1;           // tiles requested ahead (a step is shorter than a load)
    const int l16 = lane & 15, kgrp = lane >> 4;
    const float *kb = (const float*)a.k + (long)it.k0 * a.k_tok + it.g * a.k_head, *vb = (const float*)a.v + (long)it.k0 * a.v_tok + it.g * a.v_head;
    const int w0 = it.r0 + 16 * part, wl = min(w0 + 15, it.rows - 1), row = min(w0 + l16, it.rows - 1);
    const int least = it.reach(a, it.ahead + w0 / a.share), most = it.reach(a, it.ahead + wl / a.share);
    const int tiles_all = (it.keys + KT - 1) / KT, tiles = (most + KT - 1) / KT;
    const int j0 = (int)((long)tiles_all * it.piece / it.pieces), j1 = min(tiles, (int)((long)tiles_all * (it.piece + 1) / it.pieces));
    const PackedRow me = packed_query(a, it, row);
    const float into = a.cap > 0.f ? 2.0f * PACKED_LOG2E / a.cap : 0.f;
    f32x4_t qf[NB];
    {
        const float* p = (const float*)a.q + packed_row(a, it, row, a.q_tok, a.q_head);
#pragma unroll
        for (int d = 0; d < NB; ++d) qf[d] = *reinterpret_cast<const f32x4_t*>(p + d * 16 + kgrp * 4) * a.scale;
    }
    f32x4_t kn[AHEAD][LOADS], vn[AHEAD][LOADS];
    const int at = threadIdx.x / CH, of = threadIdx.x % CH * 4;      // the thread's first key and values of a tile
    const long k_mine = at * a.k_tok + of, v_mine = at * a.v_tok + of, k_step = 256 / CH * a.k_tok, v_step = 256 / CH * a.v_tok;
    auto fetch = [&](int n, int kv0) {                   // (keys behind the sample's last one are zeros)
        const float *kt = kb + kv0 * a.k_tok, *vt = vb + kv0 * a.v_tok;
        if (kv0 + KT <= it.keys) {
#pragma unroll
            for (int u = 0; u < LOADS; ++u) {
                kn[n][u] = *reinterpret_cast<const f32x4_t*>(kt + (k_mine + u * k_step));
                vn[n][u] = *reinterpret_cast<const f32x4_t*>(vt + (v_mine + u * v_step));
            }
            return;
        }
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            kn[n][u] = vn[n][u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            if (kv0 + at + 256 / CH * u < it.keys) {
                kn[n][u] = *reinterpret_cast<const f32x4_t*>(kt + (k_mine + u * k_step));
                vn[n][u] = *reinterpret_cast<const f32x4_t*>(vt + (v_mine + u * v_step));
            }
        }
    };
    f32x4_t acc[NB];
#pragma unroll
    for (int d = 0; d < NB; ++d) acc[d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int n = 0; n < AHEAD; ++n)
        if (j0 + n < j1) fetch(n, (j0 + n) * KT);
    auto tile = [&](int j, int n) {
        const int kv0 = j * KT;
        __syncthreads();
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            const int e = threadIdx.x + 256 * u, off = e / CH * LD + e % CH * 4;
            *reinterpret_cast<f32x4_t*>(Ks + off) = kn[n][u];
            *reinterpret_cast<f32x4_t*>(Vs + off) = vn[n][u];
        }
        if (a.slopes && threadIdx.x < KT) Fs[threadIdx.x] = packed_frame(a, it, kv0 + (int)threadIdx.x);
        __syncthreads();
        if (j + AHEAD < j1) fetch(n, kv0 + AHEAD * KT);
        const int k0 = kv0 + wave * 16;                  // the wave's keys
        if (k0 >= most) return;
        const bool cut = k0 + 16 > least;
        const int left = me.reach - k0 - 4 * kgrp;
        f32x4_t sc = {0.f, 0.f, 0.f, 0.f};
        float top = -INFINITY, low = INFINITY;
#pragma unroll
        for (int d = 0; d < NB; ++d) {
            const f32x4_t kf = *reinterpret_cast<const f32x4_t*>(Ks + (wave * 16 + l16) * LD + d * 16 + kgrp * 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) sc = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[e], qf[d][e], sc, 0, 0, 0);
        }
        if (a.cap > 0.f) {
#pragma unroll
            for (int i = 0; i < 4; ++i) sc[i] = capped_of(sc[i], a.cap, into);
        }
        if (a.slopes) {
            const f32x4_t f = *reinterpret_cast<const f32x4_t*>(Fs + wave * 16 + kgrp * 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) sc[i] -= packed_bias(me, f[i]);
        }
        if (cut) {
#pragma unroll
            for (int i = 0; i < 4; ++i) sc[i] = i < left ? sc[i] : -INFINITY;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            top = fmaxf(top, sc[i]);
            low = fminf(low, sc[i]);
        }
        const float mn = fmaxf(m, max_xor32(max_xor16(top))), ref = mn == -INFINITY ? 0.f : mn;
        if (__any(mn != m)) {
            const float alpha = mn == m ? 1.f : expf(m - mn);
            m = mn;
            l *= alpha;
#pragma unroll
            for (int d = 0; d < NB; ++d) acc[d] *= alpha;
        }
        const bool near = __ballot(low - ref < EXP_NEAR) == 0;       // (of the whole wave; not with keys that a row does not see)
        bool odd = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[i] = near ? exp_near(sc[i] - ref) : expf(sc[i] - ref);
#pragma unroll
        for (int i = 0; i < 4; ++i) l += sc[i];
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int d = 0; d < NB; ++d) {
                float x = Vs[(wave * 16 + kgrp * 4 + e) * LD + d * 16 + l16];
                if (cut) {                               // (as in the bf16 kernel)
                    const bool o = !(fabsf(x) < INFINITY);
                    odd = odd || o;
                    x = o ? 0.f : x;
                }
                acc[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(x, sc[e], acc[d], 0, 0, 0);
            }
        if (cut && __any(odd)) {
#pragma unroll 1
            for (int key = 0; key < min(16, it.keys - k0); ++key) {
                if (k0 + key >= me.reach) continue;
#pragma unroll
                for (int d = 0; d < NB; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float x = Vs[(wave * 16 + key) * LD + d * 16 + 4 * kgrp + i];
                        if (!(fabsf(x) < INFINITY)) acc[d][i] += x;
                    }
            }
        }
    };
    for (int j = j0; j < j1; j += AHEAD) {
#pragma unroll
        for (int n = 0; n < AHEAD; ++n)
            if (j + n < j1) tile(j + n, n);
    }
    l = sum_xor32(sum_xor16(l));
    constexpr int N = NB * 4 + 2;                    // [wave - 1][value][lane]
    static_assert(3 * N * 64 <= 2 * KT * LD, "scratch");
    __syncthreads();
    if (wave > 0) {
        float* to = Ks + (wave - 1) * N * 64 + lane;
#pragma unroll
        for (int d = 0; d < NB; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) to[(d * 4 + i) * 64] = acc[d][i];
        to[(N - 2) * 64] = l;
        to[(N - 1) * 64] = m;
    }
    __syncthreads();
    if (wave > 0) return;
    float top = m;
#pragma unroll
    for (int w = 0; w < 3; ++w) top = fmaxf(top, Ks[(w * N + N - 1) * 64 + lane]);
    const float ref = top == -INFINITY ? 0.f : top, f0 = expf(m - ref);
    m = top;
    l *= f0;
#pragma unroll
    for (int d = 0; d < NB; ++d) acc[d] *= f0;
#pragma unroll
    for (int w = 0; w < 3; ++w) {
        const float* from = Ks + w * N * 64 + lane;
        const float f = expf(from[(N - 1) * 64] - ref);
        l = __builtin_fmaf(from[(N - 2) * 64], f, l);
#pragma unroll
        for (int d = 0; d < NB; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[d][i] = __builtin_fmaf(from[(d * 4 + i) * 64], f, acc[d][i]);
    }
    if (w0 + l16 >= it.rows) return;
    if (it.pieces > 1) {
        float* p = packed_part<HD>(a, it, it.piece, row);
#pragma unroll
        for (int d = 0; d < NB; ++d) *reinterpret_cast<f32x4_t*>(p + d * 16 + kgrp * 4) = acc[d];
        if (kgrp == 0) *reinterpret_cast<f32x2_t*>(p + HD) = f32x2_t{l, m};
        return;
    }
    float* p = (float*)a.o + packed_row(a, it, row, a.o_tok, a.o_head) + kgrp * 4;
#pragma unroll
    for (int d = 0; d < NB; ++d) *reinterpret_cast<f32x4_t*>(p + d * 16) = l == 0.f ? f32x4_t{0.f, 0.f, 0.f, 0.f} : acc[d] / l;
}

template <int HD>
__global__ void __launch_bounds__(256, HD >= 128 ? 2 : HD == 64 ? 3 : 4)
packed_f32_kernel(PackedArgs a) {
    constexpr int KT = 64, LD = HD + 4;
    __shared__ __attribute__((aligned(16))) float lds[2 * KT * LD], Fs[KT];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    // four workgroups for each item, on one XCD and next to each other, so that what is long comes first for all of them (1000, 517 and 77 tokens, 16 heads of 32:
    // 37 us, with the four parts one behind the other 46)
    const unsigned at = blockIdx.y * gridDim.x + blockIdx.x;
    const int part = at >> 3 & 3;
    const PackedItem it = packed_item<PACKED_BQ_F32>(a, lane, at >> 5 << 3 | (at & 7));
    if (!it.any) return;                                 // (the whole workgroup)
    if (it.r0 + 16 * part < it.rows) packed_f32_rows<HD>(a, it, lds, lds + KT * LD, Fs, lane, wave, part);
}

__device__ __forceinline__ float max_of_64(float v) {    // in every lane (all lanes active)
    v = max_xor16(max_xor32(v));
    v = fmaxf(v, dpp<DPP_ROW_ROR_8>(v));
    v = fmaxf(v, dpp<DPP_ROW_ROR_4>(v));
    v = fmaxf(v, dpp<DPP_QUAD_XOR_2>(v));
    return fmaxf(v, dpp<DPP_QUAD_XOR_1>(v));
}
// Adds the pieces of a row: o = sum_i w_i acc_i / sum_i w_i l_i, w_i = exp(ref_i - max), in powers of two times c for bf16.  A workgroup
// takes a block; HD / 4 lanes, a team, hold 4 adjacent values each.  Of many pieces a wave takes a row at a time and its 256 / HD teams a piece each in turn; of up
// to four a team takes a row.
// The sums l_i come first, and weights are divided by the power of two below their sum, which is exact: then no sum of values is more than twice the largest value.
// (A bf16 piece's weights may sum to 2^32, and what each piece holds as a number the pieces together need not.)
__device__ __forceinline__ float packed_unit(float l) {  // 2^-n for 2^n <= l < 2^(n + 1)
    return l > 0.f && l < INFINITY ? __uint_as_float((254u << 23) - (__float_as_uint(l) & 0x7f800000u)) : 1.f;
}
template <typename T, int HD, int BQ>
__global__ void __launch_bounds__(256)
packed_join_kernel(PackedArgs a) {
    constexpr int W = HD / 4, TEAMS = 64 / W;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, d = lane % W * 4, team = lane / W;
    const PackedItem it = packed_item<BQ>(a, lane, blockIdx.x);
    if (!it.any || it.pieces <= 1) return;
    // (the block's rows are shared among its pieces' workgroups)
    const float c = a.cap > 0.f || a.slopes ? 1.0f : a.scale * PACKED_LOG2E;
    const long step = (long)a.kv_heads * it.rows * (HD + 4);     // from a piece to the next
    const auto weight = [c](float m, float ref) { return sizeof(T) == 2 ? exp2_between(m, ref, c) : expf(m - ref); };
    const auto result = [&](int r, f32x4_t acc, float l) {
        acc = l == 0.f ? f32x4_t{0.f, 0.f, 0.f, 0.f} : acc / l;
        T* o = (T*)a.o + packed_row(a, it, it.r0 + r, a.o_tok, a.o_head) + d;
        if constexpr (sizeof(T) == 2) *reinterpret_cast<bf16x4_t*>(o) = __builtin_convertvector(acc, bf16x4_t);
        else *reinterpret_cast<f32x4_t*>(o) = acc;
    };
    if (it.pieces <= 4) {                                // a team takes a row, all of whose pieces are loaded together
        for (int r = (it.piece * 4 + wave) * TEAMS + team; r < min(BQ, it.rows - it.r0); r += 4 * it.pieces * TEAMS) {
            const float* p = packed_part<HD>(a, it, 0, it.r0 + r);
            f32x4_t v[4], acc = {0.f, 0.f, 0.f, 0.f};
            f32x2_t s[4];
            float top = -INFINITY, l = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float* of = p + min(i, it.pieces - 1) * step;
                s[i] = *reinterpret_cast<const f32x2_t*>(of + HD);
                v[i] = *reinterpret_cast<const f32x4_t*>(of + d);
                top = fmaxf(top, s[i][1]);
            }
            const float ref = top == -INFINITY ? 0.f : top;  // (then every weight is zero, and so are the sums)
            float w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[i] = weight(s[i][1], ref);
                if (i < it.pieces) l = __builtin_fmaf(s[i][0], w[i], l);
            }
            const float f = packed_unit(l);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < it.pieces) acc += v[i] * (w[i] * f);
            result(r, acc, l * f);
        }
        return;
    }
    for (int r = wave + 4 * it.piece; r < min(BQ, it.rows - it.r0); r += 4 * it.pieces) {
        const float* p = packed_part<HD>(a, it, 0, it.r0 + r);
        const auto state = [&](int i) { return *reinterpret_cast<const f32x2_t*>(p + i * step + HD); };
        const f32x2_t mine = lane < it.pieces ? state(lane) : f32x2_t{0.f, -INFINITY};
        float top = mine[1];
        for (int i = lane + 64; i < it.pieces; i += 64) top = fmaxf(top, state(i)[1]);
        top = max_of_64(top);
        const float ref = top == -INFINITY ? 0.f : top;
        float l = mine[0] * weight(mine[1], ref);
        for (int i = lane + 64; i < it.pieces; i += 64) {
            const f32x2_t s = state(i);
            l = __builtin_fmaf(s[0], weight(s[1], ref), l);
        }
        l = sum_of_64(l);
        const float f = packed_unit(l);
        f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int i = team; i < it.pieces; i += TEAMS) {
            const f32x4_t v = *reinterpret_cast<const f32x4_t*>(p + i * step + d);
            acc += v * (weight(state(i)[1], ref) * f);
        }
#pragma unroll
        for (int x = W; x < 64; x *= 2)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i] += __shfl_xor(acc[i], x);
        if (team == 0) result(r, acc, l * f);
    }
}

static PackedPlan packed_plan_of(int dtype, const PackedArgs& a) {
    return packed_plan(dtype == PS_BF16, a.own_offsets, a.samples, a.q_tokens * a.share, a.kv_tokens, a.kv_heads, a.head_dim, compute_units(),
                       a.cap <= PACKED_CAP_NEAR ? 256 : 128);
}
// Partial sums: what they take at most, by both bounds
static size_t packed_part_bytes(const PackedPlan& p, const PackedArgs& a) {
    const long rows = packed_part_rows(a.own_offsets, a.samples, a.q_tokens * a.share, a.kv_tokens, a.kv_heads);
    return std::min(p.part_bytes, (size_t)rows * a.kv_heads * (a.head_dim + 4) * sizeof(float));
}
size_t packed_workspace_bytes(int dtype, const PackedArgs& a) {
    const PackedPlan p = packed_plan_of(dtype, a);
    return p.table_bytes + packed_part_bytes(p, a);
}

template <int HD, int QT>
static void launch_packed_bf16(const PackedArgs& a, unsigned grid, hipStream_t st) {
    if (a.samples > PACKED_SEARCH) packed_table_kernel<128 * QT><<<1, 1024, 0, st>>>(a);
    const int bias = !a.slopes ? 0 : a.frame >= 64 ? 1 : 2;
    if (a.cap > PACKED_CAP_NEAR) {                       // (hardly ever: blocks of 128 rows, one kernel for frames of every length)
        if constexpr (QT == 1) {
            if (bias == 0) packed_bf16_kernel<HD, 1, 2, 0><<<grid, 256, 0, st>>>(a);
            else packed_bf16_kernel<HD, 1, 2, 2><<<grid, 256, 0, st>>>(a);
        }
    } else if (a.cap > 0.f) {
        if (bias == 0) packed_bf16_kernel<HD, QT, 1, 0><<<grid, 256, 0, st>>>(a);
        else if (bias == 1) packed_bf16_kernel<HD, QT, 1, 1><<<grid, 256, 0, st>>>(a);
        else packed_bf16_kernel<HD, QT, 1, 2><<<grid, 256, 0, st>>>(a);
    } else {
        if (bias == 0) packed_bf16_kernel<HD, QT, 0, 0><<<grid, 256, 0, st>>>(a);
        else if (bias == 1) packed_bf16_kernel<HD, QT, 0, 1><<<grid, 256, 0, st>>>(a);
        else packed_bf16_kernel<HD, QT, 0, 2><<<grid, 256, 0, st>>>(a);
    }
    if (a.part) packed_join_kernel<bf16_t, HD, 128 * QT><<<grid, 256, 0, st>>>(a);
}

template <int HD>
static hipError_t launch_packed_hd(int dtype, PackedArgs a, hipStream_t st) {
    const PackedPlan p = packed_plan_of(dtype, a);
    a.slots = p.slots;
    a.table = p.table_bytes ? (int2*)a.scratch : nullptr;
    const size_t part_bytes = packed_part_bytes(p, a);
    a.part = part_bytes ? (float*)((char*)a.scratch + p.table_bytes) : nullptr;
    a.part_rows = (unsigned)(part_bytes / ((size_t)a.kv_heads * (HD + 4) * sizeof(float)));
    const unsigned grid = (unsigned)packed_workgroups(p.slots, a.kv_heads);
    if (dtype != PS_BF16) {
        if (a.samples > PACKED_SEARCH) packed_table_kernel<PACKED_BQ_F32><<<1, 1024, 0, st>>>(a);
        packed_f32_kernel<HD><<<dim3(grid / 2, 8), 256, 0, st>>>(a);      // (4 * grid, each dimension below 2^32 threads)
        if (a.part) packed_join_kernel<float, HD, PACKED_BQ_F32><<<grid, 256, 0, st>>>(a);
    } else if (HD > 64 || p.block == 128) {
        launch_packed_bf16<HD, 1>(a, grid, st);
    } else if constexpr (HD <= 64) {
        launch_packed_bf16<HD, 2>(a, grid, st);
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
