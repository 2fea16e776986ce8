// What the block formats share (gemm_fp8.hip, gemm_fp4.hip): the scales' loads, the epilogue of the products and the sum of
// pieces of k.
#pragma once
#include "few_epilogue.h"
#include "fp8.h"
#include "row_eights.h"

namespace ps {

typedef __attribute__((ext_vector_type(8))) int i32x8_t;
typedef __attribute__((ext_vector_type(4))) int i32x4_t;

__device__ __forceinline__ unsigned max_u32(unsigned a, unsigned b) { return a > b ? a : b; }
template <int CTRL>
__device__ __forceinline__ unsigned dpp_u32(unsigned v) { return __builtin_amdgcn_update_dpp(0u, v, CTRL, 0xf, 0xf, true); }

__device__ __forceinline__ void lds_dma4_base(unsigned voff, const void* sbase, unsigned lds_addr) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" ::"v"(voff), "s"(sbase), "s"(lds_addr)
                 : "memory", "m0");
}

template <int N>
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

// 4 adjacent columns of a row, behind the bias
__device__ __forceinline__ f32x4_t scaled_finish(const ScaledProduct& g, f32x4_t x) {
    if (g.act) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = gelu_fast(x[i]);
    }
    return x;
}
__device__ __forceinline__ f32x4_t scaled_bias(const ScaledProduct& g, int col) {
    if (g.n_out % 4 == 0) return *reinterpret_cast<const f32x4_t*>(g.bias + min(col, g.n_out - 4));
    f32x4_t b;
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = g.bias[min(col + i, g.n_out - 1)];
    return b;
}
__device__ __forceinline__ void scaled_store(const ScaledProduct& g, int row, int col, f32x4_t x) {
    bf16_t* out = g.out + (long)row * g.n_out + col;
    if (g.n_out % 4 == 0) {                              // a lane's 4 columns are inside or outside together
        store_quad(out, x);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (col + i < g.n_out) out[i] = from_f32<bf16_t>(x[i]);
    }
}

// Results of a workgroup's tile at (m0, n0): a lane of wave (wm, wn) holds 4 adjacent columns, 4 * kgrp .., of row l16 of each 16 x 16 block; or its share
// of a piece of k.
template <int TM, int TN>
__device__ __forceinline__ void scaled_results(const ScaledProduct& g, const f32x4_t (&acc)[TN][TM], int m0, int n0, int piece, int wm, int wn, int l16, int kgrp) {
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
    for (int y = 0; y < TN; ++y) bias[y] = scaled_bias(g, n0 + (wn * TN + y) * 16 + kgrp * 4);
    const bool wide = g.n_out % 8 == 0;
#pragma unroll
    for (int x = 0; x < TM; ++x) {
        const int row = m0 + (wm * TM + x) * 16 + l16;
#pragma unroll
        for (int y = 0; y + 1 < TN; y += 2) {
            const f32x4_t u = scaled_finish(g, acc[y][x] + bias[y]), v = scaled_finish(g, acc[y + 1][x] + bias[y + 1]);
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
                if (col + kgrp * 4 < g.n_out) scaled_store(g, row, col + kgrp * 4, u);
                if (col + 16 + kgrp * 4 < g.n_out) scaled_store(g, row, col + 16 + kgrp * 4, v);
            }
        }
        if constexpr (TN % 2) {
            const int col = n0 + (wn * TN + TN - 1) * 16 + kgrp * 4;
            if (row < g.m && col < g.n_out) scaled_store(g, row, col, scaled_finish(g, acc[TN - 1][x] + bias[TN - 1]));
        }
    }
}

// Adds the pieces of 4 adjacent columns in order.
static __global__ void __launch_bounds__(256)
scaled_join_kernel(ScaledProduct g, long quads) {
    const long id = (long)blockIdx.x * 256 + threadIdx.x;
    if (id >= quads) return;
    const int per_row = (g.n_out + 3) / 4;
    const long row = id / per_row;
    const int col = (int)(id - row * per_row) * 4;
    f32x4_t s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int p = 0; p < g.pieces; ++p) s += *reinterpret_cast<const f32x4_t*>(g.ws + ((long)p * g.m + row) * (per_row * 4) + col);
    scaled_store(g, (int)row, col, scaled_finish(g, s + scaled_bias(g, col)));
}

}  // namespace ps
