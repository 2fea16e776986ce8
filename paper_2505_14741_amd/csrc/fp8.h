// Interface of gemm_fp8.hip.
#pragma once
#include "common.h"

namespace ps {

hipError_t launch_fp8_quantize(int dtype, const void* x, void* q, void* scale, int rows, int cols, long x_row, hipStream_t st);

// out[m, n_out] = act(A * W^T + bias): operands of `blocks` blocks of 128 columns, scales [block][pitch]
struct ScaledProduct {
    const void *a, *w;
    const void *a_scale, *w_scale;
    const float* bias;
    bf16_t* out;
    int m, n_out, blocks, a_pitch, w_pitch, act;
    float* ws;                // fp32 sums of K pieces, or NULL
    size_t ws_bytes;
    int tiles_m, tiles_n, pieces;     // (set by the launcher)
    bool stream;              // (the same: out is larger than STREAM_BYTES)
};
size_t fp8_product_workspace_bytes(int m, int n_out, int blocks);
hipError_t launch_fp8_product(ScaledProduct g, hipStream_t st);

}  // namespace ps
