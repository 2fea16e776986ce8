// Interface of qk_norm.hip.
#pragma once
#include "common.h"

namespace ps {

constexpr int ROPE_MAX_AXES = 4, ROPE_MAX_PAIRS = 128;

// freq[pair], axis[pair]: what a position on that axis is multiplied with
struct RopeAxes { int pairs; unsigned char axis[ROPE_MAX_PAIRS]; double freq[ROPE_MAX_PAIRS]; };
hipError_t launch_rope_table(const float* positions, long position_row, const RopeAxes& axes, float* table, int tokens, hipStream_t st);

struct QkSide { const void* x; void* out; const float *gamma, *beta; int heads; long x_batch, x_tok, x_head, o_batch, o_tok, o_head; };
struct QkNormArgs {
    QkSide side[2];               // queries, keys
    const float* table;           // (cos, sin) of `pairs` pairs per token, or NULL
    long table_batch;             // floats; 0: one table for all samples
    int batch, tokens, head_dim, pairs, norm, halves;
    float eps;
    bool stream;                  // (set by the launcher)
};
hipError_t launch_qk_norm_rope(int dtype, QkNormArgs a, hipStream_t st);

}  // namespace ps
