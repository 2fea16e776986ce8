// Interface of group_norm.hip.
#pragma once
#include "common.h"

namespace ps {

struct GroupNormArgs {
    const void* x;
    void* out;
    const float *gamma, *beta;    // either may be NULL: 1 and 0
    int batch, positions, channels, groups, act;
    float eps;
    long x_batch, x_position, o_batch, o_position;
    bool stream;                  // (set by the launcher: out is larger than STREAM_BYTES)
    float2* part;                 // scratch of group_norm_scratch_bytes()
};
size_t group_norm_scratch_bytes(int dtype, int batch, int positions, int channels, int groups);
hipError_t launch_group_norm(int dtype, const GroupNormArgs& a, hipStream_t st);

}  // namespace ps
