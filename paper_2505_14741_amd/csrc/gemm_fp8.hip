// 8-bit floating point with a power-of-two scale for each block of 128: the quantizer and the product.
//
// A matrix of R rows and K columns is held as e4m3 bytes q[R][Kp], Kp = K filled up with zeros to a multiple of 128, and one
// scale byte s (2^(s - 127)) for each row and block of 128 columns, scale[Kp / 128][pitch], pitch = R filled up to a multiple of
// 16: block after block, so that a tile's scales of one block are neighbours.
#include "fp8.h"
#include "few_epilogue.h"
#include "lane_sums.h"
#include "plan.h"
#include "tile_ops.h"
#include <type_traits>

namespace ps {

// ------------------------------------------------------------------------------------ quantizer
// A block's scale is the least power of two 2^e, e >= -127, under which its largest finite value is at most 448, the largest of
// e4m3: with amax = 1.f * 2^x, e = x - 8 where 1.f <= 1.75 and x - 7 above (448 = 1.75 * 2^8).  Multiplying by 2^-e is exact, so
// each value is rounded once, to the nearest e4m3.  What is not finite becomes NaN and does not count for the scale.
// Memory binds: 16 lanes take a block, 8 values each, a 16-byte load of bf16.  17776 x 7680 bf16 (410 MB) 73 us, 5.6 TB/s.
typedef __attribute__((ext_vector_type(8))) float f32x8_t;
// 16-byte loads from any element's address (element by element, 17776 rows of 1919 bf16 take 44 us)
typedef bf16x8_t any_bf16x8_t __attribute__((aligned(2)));
typedef f32x4_t any_f32x4_t __attribute__((aligned(4)));

__device__ __forceinline__ unsigned max_u32(unsigned a, unsigned b) { return a > b ? a : b; }
template <int CTRL>
__device__ __forceinline__ unsigned dpp_u32(unsigned v) { return __builtin_amdgcn_update_dpp(0u, v, CTRL, 0xf, 0xf, true); }

template <typename T>
__global__ void __launch_bounds__(256)
fp8_quantize_kernel(const T* __restrict__ x, unsigned char* __restrict__ q, unsigned char* __restrict__ scale, int rows, int cols,
                    long x_row, int blocks, int pitch) {
    const unsigned item = blockIdx.x * 16u + (threadIdx.x >> 4), l16 = threadIdx.x & 15;
    if (item >= (unsigned)rows * (unsigned)blocks) return;       // (whole groups of 16 lanes)
    const int row = (int)(item / (unsigned)blocks), b = (int)(item - (unsigned)row * (unsigned)blocks);
    const int col = b * 128 + (int)l16 * 8;
    const T* p = x + row * x_row + col;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
    if (col + 8 <= cols) {
        if constexpr (sizeof(T) == 2) {
            const f32x8_t w = __builtin_convertvector(*reinterpret_cast<const any_bf16x8_t*>(p), f32x8_t);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = w[i];
        } else {
            const f32x4_t a = *reinterpret_cast<const any_f32x4_t*>(p), c = *reinterpret_cast<const any_f32x4_t*>(p + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = c[i]; }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col + i < cols) v[i] = to_f32(p[i]);
    }
    unsigned amax = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const unsigned a = __float_as_uint(v[i]) & 0x7fffffffu;
        amax = max_u32(amax, a < 0x7f800000u ? a : 0u);
        if (a >= 0x7f800000u) v[i] = __uint_as_float(0x7fc00000u);
    }
    amax = max_u32(amax, dpp_u32<DPP_ROW_ROR_8>(amax));
    amax = max_u32(amax, dpp_u32<DPP_ROW_ROR_4>(amax));
    amax = max_u32(amax, dpp_u32<DPP_QUAD_XOR_2>(amax));
    amax = max_u32(amax, dpp_u32<DPP_QUAD_XOR_1>(amax));
    int s = (int)(amax >> 23) - 8 + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);
    s = s < 0 ? 0 : s;                                   // (at most 247)
    const float inv = __uint_as_float((unsigned)(254 - s) << 23);
    int lo = 0, hi = 0;
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * inv, v[1] * inv, lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[2] * inv, v[3] * inv, lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[4] * inv, v[5] * inv, hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[6] * inv, v[7] * inv, hi, true);
    *reinterpret_cast<int2*>(q + (long)row * blocks * 128 + col) = make_int2(lo, hi);
    if (l16 == 0) scale[(long)b * pitch + row] = (unsigned char)s;
    // (the fill of the scales' rows: at most 15, by the last row's lanes)
    if (row == rows - 1 && rows + (int)l16 < pitch) scale[(long)b * pitch + rows + l16] = 0;
}

template <typename T>
static hipError_t launch_quantize_as(const T* x, unsigned char* q, unsigned char* scale, int rows, int cols, long x_row, hipStream_t st) {
    const int blocks = (cols + 127) / 128, pitch = (rows + 15) / 16 * 16;
    fp8_quantize_kernel<T><<<(unsigned)quantize_workgroups(rows, cols), 256, 0, st>>>(x, q, scale, rows, cols, x_row, blocks, pitch);
    return hipGetLastError();
}

hipError_t launch_fp8_quantize(int dtype, const void* x, void* q, void* scale, int rows, int cols, long x_row, hipStream_t st) {
    if (dtype == PS_BF16) return launch_quantize_as((const bf16_t*)x, (unsigned char*)q, (unsigned char*)scale, rows, cols, x_row, st);
    return launch_quantize_as((const float*)x, (unsigned char*)q, (unsigned char*)scale, rows, cols, x_row, st);
}

// ------------------------------------------------------------------------------------ product
// out[m, n] = act(sum over blocks of 2^(sa - 127) 2^(sw - 127) sum over the block's k of qa qw + bias[n]).
// v_mfma_scale_f32_16x16x128_f8f6f4 takes the scale bytes of both operands and multiplies 128 deep: an instruction is one block,
// the sums stay in fp32 accumulators, and scaling costs no vector instruction.  (Of 8 adjacent products the instruction cuts off the
// bits below 2^-13 of the power of two of the largest, and adds exactly enough from there on: 1.3e-5 of the result's norm for
// Gaussian operands, whatever the 8-bit instruction.  The output is bf16.)  Rows of both operands are contiguous in k;
// stages of one block (128 bytes of a row) go straight into an LDS ring, with the tile's scale bytes behind them.
// 17776 x 5760, K = 1920: 194 us, 2.03 PFLOP/s; 4516 x 1920, K = 7680: 61 us, 2.18 (a library's 8-bit product of 8192^3 reaches 2.7); the tiles
// and what each measured are in plan.h.
// Slot p of LDS row r holds 16-byte chunk p ^ ((r >> 1) & 7), so that the 16 rows of a fragment read fall into different bank
// groups.  A lane's 32 bytes of a fragment are chunks l / 16 and 4 + l / 16 of its row, of both operands alike (the instruction's
// own order of k inside a block does not matter then).
// W fragments are the first operand: a lane holds 4 adjacent output columns (4 * (l / 16) ..) of row l % 16.
typedef __attribute__((ext_vector_type(8))) int i32x8_t;
typedef __attribute__((ext_vector_type(4))) int i32x4_t;

__device__ __forceinline__ void lds_dma4_base(unsigned voff, const void* sbase, unsigned lds_addr) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" ::"v"(voff), "s"(sbase), "s"(lds_addr)
                 : "memory", "m0");
}

template <int N>
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

// 4 adjacent columns of a row, behind the bias
__device__ __forceinline__ f32x4_t fp8_finish(const Fp8Product& g, f32x4_t x) {
    if (g.act) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = gelu_fast(x[i]);
    }
    return x;
}
__device__ __forceinline__ f32x4_t fp8_bias(const Fp8Product& g, int col) {
    if (g.n_out % 4 == 0) return *reinterpret_cast<const f32x4_t*>(g.bias + min(col, g.n_out - 4));
    f32x4_t b;
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = g.bias[min(col + i, g.n_out - 1)];
    return b;
}
__device__ __forceinline__ void fp8_store(const Fp8Product& g, int row, int col, f32x4_t x) {
    bf16_t* out = g.out + (long)row * g.n_out + col;
    if (g.n_out % 4 == 0) {                              // a lane's 4 columns are inside or outside together
        store_quad(out, x);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (col + i < g.n_out) out[i] = from_f32<bf16_t>(x[i]);
    }
}

// WR x WC waves of TM x TN blocks of 16 x 16 outputs (rows x columns).  A ring of NST stages of one block of k.
// A stage has two halves of TM / 2 row blocks.  The first goes row block by row block: as soon as the products of one are issued, its
// registers are read again with the one TM / 2 further down.  Then the next stage's data are waited for and the slot of this one, all of
// whose fragments are in registers, is requested anew; the second half goes column block by column block and reads the next stage's W, and
// in its last column the next stage's first A fragments.  So one set of registers per operand is enough.
template <int TM, int TN, int WR, int WC, int NST, int OCC>
__global__ void __launch_bounds__(WR * WC * 64, OCC)
gemm_fp8_kernel(Fp8Product g) {
    constexpr int NW = WR * WC, BM = WR * TM * 16, BN = WC * TN * 16, H = TM / 2;
    static_assert((BM + BN) % (8 * NW) == 0 && BM % 8 == 0 && BM <= 256 && BN <= 256 && TM % 2 == 0 && NST >= 2 && NST <= 4, "tile");
    constexpr int GPW = (BM + BN) / 8 / NW, DATA = (BM + BN) * 128, STAGE = DATA + 1024;   // scales: 256 bytes of A, 256 of W
    __shared__ __attribute__((aligned(1024))) unsigned char lds[NST * STAGE];
    int id = xcd_remap(blockIdx.x, gridDim.x), k0 = 0, nkt = g.blocks, piece = 0;
    if (g.pieces > 1) {
        const int tiles = g.tiles_m * g.tiles_n;
        piece = id / tiles;
        id -= piece * tiles;
        k0 = g.blocks * piece / g.pieces;
        nkt = g.blocks * (piece + 1) / g.pieces - k0;
    }
    const int band = id / (8 * g.tiles_n), in_band = id - band * (8 * g.tiles_n), rows_here = min(8, g.tiles_m - band * 8);
    const int tn = in_band / rows_here;
    const int m0 = (band * 8 + in_band - tn * rows_here) * BM, n0 = tn * BN;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WC, wn = wave % WC, l16 = lane & 15, kgrp = lane >> 4;

    // load group = 8 rows of the stage [A rows | W rows]; rows past the edge re-read the last one (their outputs are not stored)
    const char* base[GPW];
    unsigned off[GPW];
    const long row_bytes = (long)g.blocks * 128;
#pragma unroll
    for (int i = 0; i < GPW; ++i) {
        const int group = wave * GPW + i, row = group * 8 + (lane >> 3), chunk = (lane & 7) ^ ((row >> 1) & 7);
        const bool of_a = group * 8 < BM;
        base[i] = (of_a ? (const char*)g.a + m0 * row_bytes : (const char*)g.w + n0 * row_bytes) + (long)k0 * 128;
        off[i] = (unsigned)(of_a ? min(row, g.m - 1 - m0) : min(row - BM, g.n_out - 1 - n0)) * (unsigned)row_bytes + chunk * 16;
    }
    // every wave requests one of the two strips of scales (so that all have the same number of loads out); 4 rows a lane
    const bool scale_a = (wave & 1) == 0;
    const int pitch = scale_a ? g.a_pitch : g.w_pitch, s0 = scale_a ? m0 : n0;
    const char* const sbase = (const char*)(scale_a ? g.a_scale : g.w_scale) + s0 + (long)k0 * pitch;
    const unsigned soff = (unsigned)min(lane * 4, pitch - 4 - s0);
    const unsigned lds_base = (unsigned)(size_t)PS_LDS_PTR(lds);
    auto issue_one = [&](int kt, int slot, int i) {      // i == GPW: the scales
        if (i < GPW)
            lds_dma16_base(off[i], base[i] + (long)kt * 128, __builtin_amdgcn_readfirstlane(lds_base + slot * STAGE + (wave * GPW + i) * 1024));
        else
            lds_dma4_base(soff, sbase + (long)kt * pitch, __builtin_amdgcn_readfirstlane(lds_base + slot * STAGE + DATA + (scale_a ? 0 : 256)));
    };

    f32x4_t acc[TN][TM];
#pragma unroll
    for (int y = 0; y < TN; ++y)
#pragma unroll
        for (int x = 0; x < TM; ++x) acc[y][x] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    const int aoff = (wm * TM * 16 + l16) * 128, woff = (BM + wn * TN * 16 + l16) * 128;
    const int c0 = (kgrp ^ ((l16 >> 1) & 7)) << 4;
    auto fragment = [&](const unsigned char* row) {
        const i32x4_t lo = *reinterpret_cast<const i32x4_t*>(row + c0), hi = *reinterpret_cast<const i32x4_t*>(row + (c0 ^ 64));
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    i32x8_t fa[H], fw[TN];
    int sa[H], sw[TN];
    auto read_a = [&](const unsigned char* st, int slot, int x) {
        fa[slot] = fragment(st + aoff + x * 2048);
        sa[slot] = st[DATA + (wm * TM + x) * 16 + l16];
    };
    auto read_w = [&](const unsigned char* st, int y) {
        fw[y] = fragment(st + woff + y * 2048);
        sw[y] = st[DATA + 256 + (wn * TN + y) * 16 + l16];
    };
#pragma unroll
    for (int p = 0; p < NST; ++p)
        if (p < nkt) {
#pragma unroll
            for (int i = 0; i <= GPW; ++i) issue_one(p, p, i);
        }
    if (nkt >= NST) wait_loads<(NST - 1) * (GPW + 1)>(); else wait_loads<0>();       // stage 0
    __syncthreads();
#pragma unroll
    for (int y = 0; y < TN; ++y) read_w(lds, y);
#pragma unroll
    for (int x = 0; x < H; ++x) read_a(lds, x, x);
    int slot = 0;
    // One stage.  LEFT: stages behind it, NST or more: any number, which is the steady state; no form has a branch inside (with one the
    // compiler sinks the first half's products behind it).
    auto stage = [&](int kt, auto left_c) {
        constexpr int LEFT = decltype(left_c)::value;
        const int next = slot + 1 == NST ? 0 : slot + 1;
        const unsigned char *st = lds + slot * STAGE, *nx = lds + next * STAGE;
#pragma unroll
        for (int x = 0; x < H; ++x) {
#pragma unroll
            for (int y = 0; y < TN; ++y)
                acc[y][x] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fw[y], fa[x], acc[y][x], 0, 0, 0, sw[y], 0, sa[x]);
            read_a(st, x, x + H);
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (LEFT > 0) {
            // own share of stage kt + 1 has landed; what may be out are the stages behind it
            wait_loads<(LEFT - 1 < NST - 2 ? LEFT - 1 : NST - 2) * (GPW + 1)>();
            __syncthreads();                             // ... everyone's; and nobody reads stage kt any more
        }
        __builtin_amdgcn_sched_barrier(0);
        constexpr int LPC = (GPW + TN) / TN;             // loads per column block
#pragma unroll
        for (int y = 0; y < TN; ++y) {
            if constexpr (LEFT >= NST) {
#pragma unroll
                for (int i = y * LPC; i < (y + 1) * LPC && i <= GPW; ++i) issue_one(kt + NST, slot, i);
            }
#pragma unroll
            for (int x = 0; x < H; ++x) {
                acc[y][x + H] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fw[y], fa[x], acc[y][x + H], 0, 0, 0, sw[y], 0, sa[x]);
                if (LEFT > 0 && y == TN - 1) read_a(nx, x, x);
            }
            if constexpr (LEFT > 0) read_w(nx, y);
            __builtin_amdgcn_sched_barrier(0);
        }
        slot = next;
    };
    int kt = 0;
    for (; kt + NST < nkt; ++kt) stage(kt, std::integral_constant<int, NST>{});
    if (NST > 3 && kt + 3 < nkt) stage(kt++, std::integral_constant<int, 3>{});
    if (NST > 2 && kt + 2 < nkt) stage(kt++, std::integral_constant<int, 2>{});
    if (kt + 1 < nkt) stage(kt++, std::integral_constant<int, 1>{});
    stage(kt, std::integral_constant<int, 0>{});
    // (every load has landed: the last hand-over waited for all)
    if (g.pieces > 1) {                                  // [piece][row][column], rows of n_out rounded up to 4
        const int ldn = (g.n_out + 3) & ~3;
#pragma unroll
        for (int x = 0; x < TM; ++x) {
            const int row = m0 + (wm * TM + x) * 16 + l16;
            if (row >= g.m) continue;
#pragma unroll
            for (int y = 0; y < TN; ++y) {
                const int col = n0 + (wn * TN + y) * 16 + kgrp * 4;
                if (col < g.n_out) *reinterpret_cast<f32x4_t*>(g.ws + ((long)piece * g.m + row) * ldn + col) = acc[y][x];
            }
        }
        return;
    }
    f32x4_t bias[TN];
#pragma unroll
    for (int y = 0; y < TN; ++y) bias[y] = fp8_bias(g, n0 + (wn * TN + y) * 16 + kgrp * 4);
    const bool wide = g.n_out % 8 == 0;
#pragma unroll
    for (int x = 0; x < TM; ++x) {
        const int row = m0 + (wm * TM + x) * 16 + l16;
#pragma unroll
        for (int y = 0; y + 1 < TN; y += 2) {
            const f32x4_t u = fp8_finish(g, acc[y][x] + bias[y]), v = fp8_finish(g, acc[y + 1][x] + bias[y + 1]);
            const int col = n0 + (wn * TN + y) * 16;
            if (wide) {
                // lanes of neighbouring kgrp swap quads of two column blocks: 8 adjacent columns each, 64 bytes of a row by four lanes
                typedef __attribute__((ext_vector_type(2))) unsigned u32x2_t;
                const u32x2_t p = __builtin_bit_cast(u32x2_t, __builtin_convertvector(u, bf16x4_t));
                const u32x2_t q = __builtin_bit_cast(u32x2_t, __builtin_convertvector(v, bf16x4_t));
                const auto lo = __builtin_amdgcn_permlane16_swap(p[0], q[0], false, false), hi = __builtin_amdgcn_permlane16_swap(p[1], q[1], false, false);
                const int c = col + (kgrp & 1) * 16 + (kgrp & 2) * 4;
                const i32x4_t w = {(int)lo[0], (int)hi[0], (int)lo[1], (int)hi[1]};
                if (row < g.m && c < g.n_out) store_streamed<16>(g.out + (long)row * g.n_out + c, w, g.stream);
            } else if (row < g.m) {
                if (col + kgrp * 4 < g.n_out) fp8_store(g, row, col + kgrp * 4, u);
                if (col + 16 + kgrp * 4 < g.n_out) fp8_store(g, row, col + 16 + kgrp * 4, v);
            }
        }
        if constexpr (TN % 2) {
            const int col = n0 + (wn * TN + TN - 1) * 16 + kgrp * 4;
            if (row < g.m && col < g.n_out) fp8_store(g, row, col, fp8_finish(g, acc[TN - 1][x] + bias[TN - 1]));
        }
    }
}

// Adds the pieces of 4 adjacent columns in order.
__global__ void __launch_bounds__(256)
gemm_fp8_join_kernel(Fp8Product g, long quads) {
    const long id = (long)blockIdx.x * 256 + threadIdx.x;
    if (id >= quads) return;
    const int per_row = (g.n_out + 3) / 4;
    const long row = id / per_row;
    const int col = (int)(id - row * per_row) * 4;
    f32x4_t s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int p = 0; p < g.pieces; ++p) s += *reinterpret_cast<const f32x4_t*>(g.ws + ((long)p * g.m + row) * (per_row * 4) + col);
    fp8_store(g, (int)row, col, fp8_finish(g, s + fp8_bias(g, col)));
}

template <int TM, int TN, int WR, int WC, int NST, int OCC>
static void launch_product_tile(Fp8Product g, hipStream_t st) {
    constexpr int BM = WR * TM * 16, BN = WC * TN * 16;
    g.tiles_m = (g.m + BM - 1) / BM;
    g.tiles_n = (g.n_out + BN - 1) / BN;
    gemm_fp8_kernel<TM, TN, WR, WC, NST, OCC><<<(unsigned)((long)g.tiles_m * g.tiles_n * g.pieces), WR * WC * 64, 0, st>>>(g);
}

size_t fp8_product_workspace_bytes(int m, int n_out, int blocks) {
    const Fp8Plan p = fp8_plan(m, n_out, blocks, true, compute_units());
    return p.pieces > 1 ? (size_t)p.pieces * m * ((n_out + 3) / 4 * 4) * sizeof(float) : 0;
}

hipError_t launch_fp8_product(Fp8Product g, hipStream_t st) {
    const size_t need = fp8_product_workspace_bytes(g.m, g.n_out, g.blocks);
    const Fp8Plan p = fp8_plan(g.m, g.n_out, g.blocks, need > 0 && g.ws && g.ws_bytes >= need, compute_units());
    g.pieces = p.pieces;
    g.stream = (size_t)g.m * g.n_out * sizeof(bf16_t) > STREAM_BYTES;
    switch (p.tile) {
        case FP8_64x64: launch_product_tile<2, 2, 2, 2, 4, 2>(g, st); break;
        case FP8_128x128: launch_product_tile<2, 4, 4, 2, 3, 2>(g, st); break;
        case FP8_192x192: launch_product_tile<6, 3, 2, 4, 3, 2>(g, st); break;
        default: launch_product_tile<6, 4, 2, 4, 2, 2>(g, st); break;
    }
    if (p.pieces > 1) {
        const long quads = (long)g.m * ((g.n_out + 3) / 4);
        gemm_fp8_join_kernel<<<(unsigned)((quads + 255) / 256), 256, 0, st>>>(g, quads);
    }
    return hipGetLastError();
}

}  // namespace ps
