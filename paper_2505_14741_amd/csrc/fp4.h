// Interface of gemm_fp4.hip.
#pragma once
#include "fp8.h"

namespace ps {

// Columns are filled up to a multiple of 128 (one matrix instruction), scales are for blocks of 32.
hipError_t launch_fp4_quantize(int dtype, const void* x, void* q, void* scale, int rows, int cols, long x_row, hipStream_t st);
hipError_t launch_fp4_dequantize(int dtype, const void* q, const void* scale, void* out, int rows, int cols, long out_row, hipStream_t st);

// ScaledProduct of operands of `blocks` blocks of 128 columns, 64 bytes and 4 strips of scales each
size_t fp4_product_workspace_bytes(int m, int n_out, int blocks);
hipError_t launch_fp4_product(ScaledProduct g, hipStream_t st);

}  // namespace ps
