// 4-bit floating point with a power-of-two scale for each block of 32: the quantizer, reading back, and the product.
//
// A matrix of R rows and K columns is held as e2m1 codes q[R][Kp / 2], two to a byte, the even column in the low bits, Kp = K filled up with
// zeros to a multiple of 128, and one scale byte s (2^(s - 127); 255: NaN) for each row and block of 32 columns, scale[Kp / 32][pitch], pitch =
// R filled up to a multiple of 16: block after block, so that a tile's scales of one block are neighbours.
#include "fp4.h"
#include "lane_sums.h"
#include "plan.h"
#include "scaled_product.h"
#include <type_traits>

namespace ps {

// ------------------------------------------------------------------------------------ quantizer
// A block's scale is the least power of two 2^e, e >= -127, under which its largest value is at most 6, the largest of e2m1: with amax =
// 1.f * 2^x, e = x - 2 where 1.f <= 1.5 and x - 1 above (6 = 1.5 * 2^2).  Multiplying by 2^-e is exact, so each value is rounded once, to the
// nearest of 0 0.5 1 1.5 2 3 4 6, ties to the even code (what the conversion instruction does).  The format has no value that is not finite: a
// block with one has the scale NaN, and zeros.  (17776 x 7680 in bf16, 346 MB: 88 us at the median, 3.9 TB/s, 73 at the best.)
// Memory binds.  A workgroup takes 16 rows x 512 columns, 4 rows per wave, 8 adjacent values per lane (16 bytes of bf16, 4 lanes a
// block): the 16 scales of a block lie side by side and are stored as 16 bytes, gathered in LDS.
constexpr int FP4_ROWS = 16, FP4_COLS = 512;

template <typename T>
__global__ void __launch_bounds__(256)
fp4_quantize_kernel(const T* __restrict__ x, unsigned char* __restrict__ q, unsigned char* __restrict__ scale, int rows, int cols, long x_row,
                    int kp, int pitch, int tiles_c) {
    __shared__ __attribute__((aligned(16))) unsigned char sc[FP4_COLS / 32][FP4_ROWS];
    const int tr = (int)(blockIdx.x / (unsigned)tiles_c), tc = (int)blockIdx.x - tr * tiles_c;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = tc * FP4_COLS + lane * 8, row0 = tr * FP4_ROWS + wave * 4;
    float v[4][8];
#pragma unroll
    for (int r = 0; r < 4; ++r) load_eight(v[r], x + (long)min(row0 + r, rows - 1) * x_row + col, col, cols);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        unsigned amax = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) amax = max_u32(amax, __float_as_uint(v[r][i]) & 0x7fffffffu);
        amax = max_u32(amax, dpp_u32<DPP_QUAD_XOR_2>(amax));
        amax = max_u32(amax, dpp_u32<DPP_QUAD_XOR_1>(amax));
        const bool finite = amax < 0x7f800000u;
        int s = (int)(amax >> 23) - 2 + ((amax & 0x7fffffu) > 0x400000u ? 1 : 0);
        s = s < 0 ? 0 : s;                               // (at most 253)
        const float inv = __uint_as_float((unsigned)(254 - s) << 23);
        unsigned codes = 0;
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, v[r][0] * inv, v[r][1] * inv, 1.0f, 0);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, v[r][2] * inv, v[r][3] * inv, 1.0f, 1);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, v[r][4] * inv, v[r][5] * inv, 1.0f, 2);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, v[r][6] * inv, v[r][7] * inv, 1.0f, 3);
        if (row0 + r < rows && col < kp) *reinterpret_cast<unsigned*>(q + (long)(row0 + r) * (kp / 2) + col / 2) = finite ? codes : 0u;
        if ((lane & 3) == 0) sc[lane >> 2][wave * 4 + r] = row0 + r >= rows ? 0 : finite ? (unsigned char)s : 255;
    }
    __syncthreads();
    const int b = tc * (FP4_COLS / 32) + (int)threadIdx.x;
    if (threadIdx.x < FP4_COLS / 32 && b < kp / 32)
        *reinterpret_cast<i32x4_t*>(scale + (long)b * pitch + tr * FP4_ROWS) = *reinterpret_cast<const i32x4_t*>(sc[threadIdx.x]);
}

// Reading back: the same tiles; every value is exact in bf16 and fp32 but those beyond the largest number of the type (4 * 2^126, to which fp32's largest
// numbers are rounded), which become that.  (17776 x 7680 to bf16: 60 us, 5.8 TB/s.)
template <typename T>
__global__ void __launch_bounds__(256)
fp4_dequantize_kernel(const unsigned char* __restrict__ q, const unsigned char* __restrict__ scale, T* __restrict__ out, int rows, int cols, long out_row,
                      int kp, int pitch, int tiles_c) {
    __shared__ __attribute__((aligned(16))) unsigned char sc[FP4_COLS / 32][FP4_ROWS];
    const int tr = (int)(blockIdx.x / (unsigned)tiles_c), tc = (int)blockIdx.x - tr * tiles_c;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = tc * FP4_COLS + lane * 8, row0 = tr * FP4_ROWS + wave * 4;
    unsigned codes[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) codes[r] = *reinterpret_cast<const unsigned*>(q + (long)min(row0 + r, rows - 1) * (kp / 2) + min(col, kp - 8) / 2);
    const int b = min(tc * (FP4_COLS / 32) + (int)threadIdx.x, kp / 32 - 1);
    if (threadIdx.x < FP4_COLS / 32) *reinterpret_cast<i32x4_t*>(sc[threadIdx.x]) = *reinterpret_cast<const i32x4_t*>(scale + (long)b * pitch + tr * FP4_ROWS);
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        if (row0 + r >= rows) continue;
        const unsigned s = sc[lane >> 2][wave * 4 + r];
        const float f = s == 0 ? 0x1p-127f : s == 255 ? __uint_as_float(0x7fc00000u) : __uint_as_float(s << 23);
        const f32x2_t p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[r], 1.0f, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[r], 1.0f, 1);
        const f32x2_t p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[r], 1.0f, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[r], 1.0f, 3);
        float v[8] = {p0[0] * f, p0[1] * f, p1[0] * f, p1[1] * f, p2[0] * f, p2[1] * f, p3[0] * f, p3[1] * f};
        if (s >= 252 && s < 255) {
            const float most = sizeof(T) == 2 ? 0x1.fep+127f : 0x1.fffffep+127f;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = fminf(fmaxf(v[i], -most), most);
        }
        store_eight(out + (long)(row0 + r) * out_row + col, v, col, cols);
    }
}

template <typename T>
static hipError_t launch_quantize_as(const T* x, unsigned char* q, unsigned char* scale, int rows, int cols, long x_row, hipStream_t st) {
    const int kp = (cols + 127) / 128 * 128, pitch = (rows + 15) / 16 * 16, tiles_c = (kp + FP4_COLS - 1) / FP4_COLS;
    fp4_quantize_kernel<T><<<(unsigned)fp4_workgroups(rows, cols), 256, 0, st>>>(x, q, scale, rows, cols, x_row, kp, pitch, tiles_c);
    return hipGetLastError();
}
hipError_t launch_fp4_quantize(int dtype, const void* x, void* q, void* scale, int rows, int cols, long x_row, hipStream_t st) {
    if (dtype == PS_BF16) return launch_quantize_as((const bf16_t*)x, (unsigned char*)q, (unsigned char*)scale, rows, cols, x_row, st);
    return launch_quantize_as((const float*)x, (unsigned char*)q, (unsigned char*)scale, rows, cols, x_row, st);
}

template <typename T>
static hipError_t launch_dequantize_as(const unsigned char* q, const unsigned char* scale, T* out, int rows, int cols, long out_row, hipStream_t st) {
    const int kp = (cols + 127) / 128 * 128, pitch = (rows + 15) / 16 * 16, tiles_c = (kp + FP4_COLS - 1) / FP4_COLS;
    fp4_dequantize_kernel<T><<<(unsigned)fp4_workgroups(rows, cols), 256, 0, st>>>(q, scale, out, rows, cols, out_row, kp, pitch, tiles_c);
    return hipGetLastError();
}
hipError_t launch_fp4_dequantize(int dtype, const void* q, const void* scale, void* out, int rows, int cols, long out_row, hipStream_t st) {
    if (dtype == PS_BF16) return launch_dequantize_as((const unsigned char*)q, (const unsigned char*)scale, (bf16_t*)out, rows, cols, out_row, st);
    return launch_dequantize_as((const unsigned char*)q, (const unsigned char*)scale, (float*)out, rows, cols, out_row, st);
}

// ------------------------------------------------------------------------------------ product
// out[m, n] = act(sum over blocks of 2^(sa - 127) 2^(sw - 127) sum over the block's k of qa qw + bias[n]).
// v_mfma_scale_f32_16x16x128_f8f6f4 takes 4-bit operands and a scale byte for each 32 of k (a lane's 16 bytes are one block of its row): scaling
// costs no vector instruction.  Sums of the 128 products of an instruction are as exact as fp32 sums (measured: 5e-8 of the sum of
// magnitudes at most, whatever the blocks' scales), at twice the 8-bit rate (9.1 PFLOP/s from registers against 4.7).
// A stage is 256 k: 128 bytes of a row, which go straight into an LDS ring, with 8 strips of scale bytes of the tile's rows and
// columns behind them; where the last stage has only 128 k its other half is not multiplied.
// Slot p of LDS row r holds 16-byte chunk p ^ ((r >> 1) & 7), so that the 16 rows of a fragment read fall into different bank
// groups.  W fragments are the first operand: a lane holds 4 adjacent output columns (4 * (l / 16) ..) of row l % 16.

// Scale strips of R rows (64, 128, 192 or 256) in LDS: a load of 256 bytes holds 256 / R of them (192: one), loads lie 272 bytes apart, so that the four
// strips of a read fall into different banks.
template <int R> struct Fp4Strips {
    static constexpr int PER = R <= 128 ? 256 / R : 1, LOADS = 8 / PER, BYTES = LOADS * 272;
    __device__ __forceinline__ static int at(int strip) { return strip / PER * 272 + strip % PER * R; }
};

// Measured: 17776 x 5760, k = 1920 147 to 178 us, 2.2 to 2.67 PFLOP/s; 4516 x 1920, k = 7680 39 to 44, 3.0 to 3.4.  No unit is busy for long (the first: matrix instructions 28 % of the
// cycles, vector 32, LDS reads 18).  The loop alone reaches 4.6 PFLOP/s: a stage's 57 KB are read by 8 waves through 40 fragments and 40 scale bytes for
// every 96 products of a SIMD.  The rest is the first stage's way and the results', 7 us for each of 9 rounds of workgroups.
//
// WR x WC waves of TM x TN blocks of 16 x 16 outputs (rows x columns).  A ring of NST stages.
// A stage has two halves of TM / 2 row blocks.  The first goes row block by row block: as soon as the products of one are issued, its
// registers are read again with the one TM / 2 further down.  Then the next stage's data are waited for and the slot of this one, all of
// whose fragments are in registers, is requested anew; the second half goes column block by column block and reads the next stage's W, and
// in its last column the next stage's first A fragments.  So one set of registers per operand is enough.
template <int TM, int TN, int WR, int WC, int NST, int OCC>
__global__ void __launch_bounds__(WR * WC * 64, OCC)
gemm_fp4_kernel(ScaledProduct g) {
    constexpr int NW = WR * WC, BM = WR * TM * 16, BN = WC * TN * 16, H = TM / 2;
    typedef Fp4Strips<BM> SA;
    typedef Fp4Strips<BN> SW;
    static_assert((BM + BN) % (8 * NW) == 0 && BM % 8 == 0 && BM <= 256 && BN <= 256 && TM % 2 == 0 && NST >= 2 && NST <= 4, "tile");
    constexpr int GPW = (BM + BN) / 8 / NW, STRIPS = SA::LOADS + SW::LOADS, SPW = (STRIPS + NW - 1) / NW, LOADS = GPW + SPW;
    constexpr int DATA = (BM + BN) * 128, STAGE = (DATA + SA::BYTES + SW::BYTES + 1023) / 1024 * 1024;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[NST * STAGE];
    const int stages = (g.blocks + 1) / 2;
    int id = xcd_remap(blockIdx.x, gridDim.x), k0 = 0, nkt = stages, piece = 0;
    if (g.pieces > 1) {
        const int tiles = g.tiles_m * g.tiles_n;
        piece = id / tiles;
        id -= piece * tiles;
        k0 = stages * piece / g.pieces;
        nkt = stages * (piece + 1) / g.pieces - k0;
    }
    const bool half_last = (g.blocks & 1) && k0 + nkt == stages;
    const int band = id / (8 * g.tiles_n), in_band = id - band * (8 * g.tiles_n), rows_here = min(8, g.tiles_m - band * 8);
    const int tn = in_band / rows_here;
    const int m0 = (band * 8 + in_band - tn * rows_here) * BM, n0 = tn * BN;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WC, wn = wave % WC, l16 = lane & 15, kgrp = lane >> 4;

    // load group = 8 rows of the stage [A rows | W rows]; rows past the edge re-read the last one (their outputs are not stored)
    const char* base[GPW];
    unsigned off[GPW];
    const long row_bytes = (long)g.blocks * 64;
#pragma unroll
    for (int i = 0; i < GPW; ++i) {
        const int group = wave * GPW + i, row = group * 8 + (lane >> 3), chunk = (lane & 7) ^ ((row >> 1) & 7);
        const bool of_a = group * 8 < BM;
        base[i] = (of_a ? (const char*)g.a + m0 * row_bytes : (const char*)g.w + n0 * row_bytes) + (long)k0 * 128;
        off[i] = (unsigned)(of_a ? min(row, g.m - 1 - m0) : min(row - BM, g.n_out - 1 - n0)) * (unsigned)row_bytes + chunk * 16;
    }
    // 256 bytes of scale strips: 4 rows of a strip per lane
    const unsigned lds_base = (unsigned)(size_t)PS_LDS_PTR(lds);
    auto issue_one = [&](int kt, int slot, int i, bool half) {
        if (i < GPW) {
            // (of half a stage, the chunks that do not exist repeat those that do)
            const int group = wave * GPW + i, row = group * 8 + (lane >> 3), chunk = (lane & 7) ^ ((row >> 1) & 7);
            const unsigned o = half ? off[i] - (unsigned)(chunk & 4) * 16 : off[i];
            lds_dma16_base(o, base[i] + (long)kt * 128, __builtin_amdgcn_readfirstlane(lds_base + slot * STAGE + group * 1024));
        } else {
            const int n = (wave * SPW + i - GPW) % STRIPS;       // (every wave requests as many: some twice)
            const bool of_a = n < SA::LOADS;
            const int l = of_a ? n : n - SA::LOADS, per = of_a ? SA::PER : SW::PER, r = of_a ? BM : BN, pitch = of_a ? g.a_pitch : g.w_pitch, s0 = of_a ? m0 : n0;
            int strip = l * per + (per > 1 ? lane * 4 / r : 0);
            if (half) strip &= 3;
            const int at = per > 1 ? lane * 4 % r : lane * 4;
            const char* sb = (const char*)(of_a ? g.a_scale : g.w_scale) + s0 + (long)(k0 + kt) * 8 * pitch;
            lds_dma4_base((unsigned)strip * (unsigned)pitch + (unsigned)min(at, pitch - 4 - s0), sb,
                          __builtin_amdgcn_readfirstlane(lds_base + slot * STAGE + DATA + (of_a ? 0 : SA::BYTES) + l * 272));
        }
    };

    f32x4_t acc[TN][TM];
#pragma unroll
    for (int y = 0; y < TN; ++y)
#pragma unroll
        for (int x = 0; x < TM; ++x) acc[y][x] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    const int aoff = (wm * TM * 16 + l16) * 128, woff = (BM + wn * TN * 16 + l16) * 128;
    const int c0 = (kgrp ^ ((l16 >> 1) & 7)) << 4;
    const int as0 = DATA + SA::at(kgrp) + wm * TM * 16 + l16, as1 = DATA + SA::at(4 + kgrp) + wm * TM * 16 + l16;
    const int ws0 = DATA + SA::BYTES + SW::at(kgrp) + wn * TN * 16 + l16, ws1 = DATA + SA::BYTES + SW::at(4 + kgrp) + wn * TN * 16 + l16;
    i32x4_t fa[H][2], fw[TN][2];
    int sa[H][2], sw[TN][2];
    auto read_a = [&](const unsigned char* st, int slot, int x) {
        fa[slot][0] = *reinterpret_cast<const i32x4_t*>(st + aoff + x * 2048 + c0);
        fa[slot][1] = *reinterpret_cast<const i32x4_t*>(st + aoff + x * 2048 + (c0 ^ 64));
        sa[slot][0] = st[as0 + x * 16];
        sa[slot][1] = st[as1 + x * 16];
    };
    auto read_w = [&](const unsigned char* st, int y) {
        fw[y][0] = *reinterpret_cast<const i32x4_t*>(st + woff + y * 2048 + c0);
        fw[y][1] = *reinterpret_cast<const i32x4_t*>(st + woff + y * 2048 + (c0 ^ 64));
        sw[y][0] = st[ws0 + y * 16];
        sw[y][1] = st[ws1 + y * 16];
    };
    auto product = [&](int y, int x, int h, f32x4_t c) {
        const i32x8_t u = __builtin_shufflevector(fw[y][h], fw[y][h], 0, 1, 2, 3, -1, -1, -1, -1), v = __builtin_shufflevector(fa[x][h], fa[x][h], 0, 1, 2, 3, -1, -1, -1, -1);
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(u, v, c, 4, 4, 0, sw[y][h], 0, sa[x][h]);
    };
#pragma unroll
    for (int p = 0; p < NST; ++p)
        if (p < nkt) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) issue_one(p, p, i, half_last && p == nkt - 1);
        }
    if (nkt >= NST) wait_loads<(NST - 1) * LOADS>(); else wait_loads<0>();       // stage 0
    __syncthreads();
#pragma unroll
    for (int y = 0; y < TN; ++y) read_w(lds, y);
#pragma unroll
    for (int x = 0; x < H; ++x) read_a(lds, x, x);
    int slot = 0;
    // One stage.  LEFT: stages behind it, NST or more: any number, which is the steady state; no form has a branch inside (with one the
    // compiler sinks the first half's products behind it).  NH: halves of it that are multiplied.
    auto stage = [&](int kt, auto left_c, auto halves_c) {
        constexpr int LEFT = decltype(left_c)::value, NH = decltype(halves_c)::value;
        const int next = slot + 1 == NST ? 0 : slot + 1;
        const unsigned char *st = lds + slot * STAGE, *nx = lds + next * STAGE;
#pragma unroll
        for (int x = 0; x < H; ++x) {
#pragma unroll
            for (int h = 0; h < NH; ++h)
#pragma unroll
                for (int y = 0; y < TN; ++y) acc[y][x] = product(y, x, h, acc[y][x]);
            read_a(st, x, x + H);
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (LEFT > 0) {
            // own share of stage kt + 1 has landed; what may be out are the stages behind it
            wait_loads<(LEFT - 1 < NST - 2 ? LEFT - 1 : NST - 2) * LOADS>();
            __syncthreads();                             // ... everyone's; and nobody reads stage kt any more
        }
        __builtin_amdgcn_sched_barrier(0);
        constexpr int LPC = (LOADS + TN - 1) / TN;       // loads per column block
        const bool half = LEFT >= NST && half_last && kt + NST == nkt - 1;
#pragma unroll
        for (int y = 0; y < TN; ++y) {
            if constexpr (LEFT >= NST) {
#pragma unroll
                for (int i = y * LPC; i < (y + 1) * LPC && i < LOADS; ++i) issue_one(kt + NST, slot, i, half);
            }
#pragma unroll
            for (int h = 0; h < NH; ++h)
#pragma unroll
                for (int x = 0; x < H; ++x) {
                    acc[y][x + H] = product(y, x, h, acc[y][x + H]);
                    if (LEFT > 0 && y == TN - 1 && h == NH - 1) read_a(nx, x, x);
                }
            if constexpr (LEFT > 0) read_w(nx, y);
            __builtin_amdgcn_sched_barrier(0);
        }
        slot = next;
    };
    const std::integral_constant<int, 2> whole;
    int kt = 0;
    for (; kt + NST < nkt; ++kt) stage(kt, std::integral_constant<int, NST>{}, whole);
    if (NST > 3 && kt + 3 < nkt) stage(kt++, std::integral_constant<int, 3>{}, whole);
    if (NST > 2 && kt + 2 < nkt) stage(kt++, std::integral_constant<int, 2>{}, whole);
    if (kt + 1 < nkt) stage(kt++, std::integral_constant<int, 1>{}, whole);
    if (half_last) stage(kt, std::integral_constant<int, 0>{}, std::integral_constant<int, 1>{});
    else stage(kt, std::integral_constant<int, 0>{}, whole);
    // (every load has landed: the last hand-over waited for all)
    scaled_results<TM, TN>(g, acc, m0, n0, piece, wm, wn, l16, kgrp);
}

template <int TM, int TN, int WR, int WC, int NST, int OCC>
static void launch_product_tile(ScaledProduct g, hipStream_t st) {
    constexpr int BM = WR * TM * 16, BN = WC * TN * 16;
    g.tiles_m = (g.m + BM - 1) / BM;
    g.tiles_n = (g.n_out + BN - 1) / BN;
    gemm_fp4_kernel<TM, TN, WR, WC, NST, OCC><<<(unsigned)((long)g.tiles_m * g.tiles_n * g.pieces), WR * WC * 64, 0, st>>>(g);
}

size_t fp4_product_workspace_bytes(int m, int n_out, int blocks) {
    const Fp4Plan p = fp4_plan(m, n_out, blocks, true, compute_units());
    return p.pieces > 1 ? (size_t)p.pieces * m * ((n_out + 3) / 4 * 4) * sizeof(float) : 0;
}

hipError_t launch_fp4_product(ScaledProduct g, hipStream_t st) {
    const size_t need = fp4_product_workspace_bytes(g.m, g.n_out, g.blocks);
    const Fp4Plan p = fp4_plan(g.m, g.n_out, g.blocks, need > 0 && g.ws && g.ws_bytes >= need, compute_units());
    g.pieces = p.pieces;
    g.stream = (size_t)g.m * g.n_out * sizeof(bf16_t) > STREAM_BYTES;
    switch (p.tile) {
        case FP4_64x64: launch_product_tile<2, 2, 2, 2, 4, 2>(g, st); break;
        case FP4_128x128: launch_product_tile<2, 4, 4, 2, 3, 2>(g, st); break;
        case FP4_128x128_PAIR: launch_product_tile<4, 4, 2, 2, 2, 2>(g, st); break;
        case FP4_192x192: launch_product_tile<6, 3, 2, 4, 3, 2>(g, st); break;
        default: launch_product_tile<6, 4, 2, 4, 2, 2>(g, st); break;
    }
    if (p.pieces > 1) {
        const long quads = (long)g.m * ((g.n_out + 3) / 4);
        scaled_join_kernel<<<(unsigned)((quads + 255) / 256), 256, 0, st>>>(g, quads);
    }
    return hipGetLastError();
}

}  // namespace ps
