// Kernel-side image of the calls that verify drafted tokens (draft_verify.hip), shared with the C ABI layer.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace difr {

struct DraftBatch {
    const void *logits;  // [D + B, ld]: the rows of sequence b are offsets[b] + b ... offsets[b + 1] + b
    int32_t dtype;
    int64_t B, D, V, ld;
    float temperature;
    const float *temperatures;  // [D + B] or null
    const int32_t *tokens;      // [D]
    const int64_t *offsets;     // [B + 1]
};
// What a chain is verified against beside the target's logits.
struct DraftChain {
    const void *draft;  // [D, ld] in the logits' type, or null: each draft has probability 1 at its token
    int64_t ld;
    float temperature;
    const float *temperatures;  // [D] or null
    const float *accept_u;      // [D]
    const float *sample_u;      // [B]
};
struct DraftTree {
    const int32_t *parents;  // [D], or null: each token's is the one before it
    const float *sample_u;   // [D + B]
};
struct DraftOutputs {
    int32_t *accepted;      // [B]
    int32_t *tokens;        // [D + B]
    int32_t *nodes;         // [D + B], trees only
    float *logp;            // [D + B] or null
    uint8_t *flags;         // [D + B]
};

// Whether the cells of D + B rows can be counted by a grid.
bool draft_shape(int64_t B, int64_t D, int64_t V);
size_t draft_workspace_bytes(int64_t B, int64_t D, int64_t V, bool draft);
int launch_draft_verify(const DraftBatch &b, const DraftChain &c, const DraftOutputs &o, void *workspace, hipStream_t stream);
int launch_tree_verify(const DraftBatch &b, const DraftTree &t, const DraftOutputs &o, void *workspace, hipStream_t stream);

}  // namespace difr
