// Interface of packed_attention.hip.
#pragma once
#include "common.h"

namespace ps {

constexpr float PACKED_LOG2E = 1.4426950408889634f;

// A key head's query rows of a sample are its (token, query head of the group) pairs, row = token * share + head of the group.
struct PackedArgs {
    const void *q, *k, *v;
    void* o;
    const int32_t *q_offsets, *kv_offsets, *prefix;      // kv_offsets NULL: q_offsets; prefix NULL: none
    const float* slopes;                                 // or NULL
    int samples, q_tokens, kv_tokens, kv_heads, share, head_dim, frame, causal;
    float scale, cap;                                    // cap 0: none
    long q_tok, q_head, k_tok, k_head, v_tok, v_head, o_tok, o_head;
    bool own_offsets;             // whether kv_offsets are given, for the sizes
    void* scratch;                // packed_workspace_bytes()
    int slots;                    // (set by the launcher)
    int2* table;                  // (the same: which slot is whose, and behind it the rows of partial sums in front of each sample, or NULL)
    float* part;                  // (the same: partial sums, or NULL)
    unsigned part_rows;           // (the same: of a key head)
};
size_t packed_workspace_bytes(int dtype, const PackedArgs& a);
hipError_t launch_packed_attention(int dtype, PackedArgs a, hipStream_t st);

}  // namespace ps
