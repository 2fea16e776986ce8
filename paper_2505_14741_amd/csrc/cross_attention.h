// Interface of cross_attention.hip.
#pragma once
#include "common.h"

namespace ps {

constexpr float CROSS_LOG2E = 1.4426950408889634f;       // scores times it and the scale are exponents of two

// A key/value head's query rows are its (token, query head of the group) pairs, row = token * share + head of the group.
struct CrossArgs {
    const void *q, *k, *v;
    void* o;
    const int32_t* kv_lens;       // keys of each sample, or NULL: kv_len
    const uint8_t* key_mask;      // 0: the key does not count; or NULL
    long mask_batch;
    int batch, rows, share, kv_len, kv_heads, head_dim;
    float scale;
    AttnStrides s;
    float* part;                  // scratch of cross_workspace_bytes()
    int nsplit;                   // (set by the launcher)
    bool stream;                  // (the same: o is larger than STREAM_BYTES)
};
size_t cross_workspace_bytes(int dtype, const CrossArgs& a);
hipError_t launch_cross_attention(int dtype, CrossArgs a, hipStream_t st);

}  // namespace ps
