// Launch of the streaming attention kernel (attn_stream.hip).
#pragma once
#include "rapid_internal.h"

struct StreamLaunch {
    const uint16_t* q;
    uint16_t* out;
    float* lse_out;
    const int32_t* ctx_lens;
    const int32_t* gammas;
    AttnSource own;             // codes and scales, or bf16
    float* part_o;              // [Hkv][nslots][RP][D], relative to the maximum in part_ml; slot g + b: share g's piece of sequence b
    float* part_ml;             // [Hkv][nslots][RP][2] (maximum in log2 units, sum)
    int32_t B, Qmax, Hq, Hkv, G, D, gamma, max_ctx;
    int32_t RP;                 // packed rows of a slot, a multiple of 16
    int32_t groups, nslots;     // shares of a kv head, groups + B - 1
    int32_t quantum;            // tokens that shares are cut by
    int32_t rot;                // 1: share g of slot x serves head (x + g) mod Hkv, 0: head x
    float scale_log2e;
};
// Fills the plan (RP .. rot) from the shape and the source's layout.
void plan_attn_stream(StreamLaunch& a, int n_cu);
size_t attn_stream_workspace_bytes(const StreamLaunch& a);
void bind_attn_stream(StreamLaunch& a, void* workspace);
hipError_t configure_attn_stream();
hipError_t launch_attn_stream(const StreamLaunch& a, hipStream_t stream);        // writes the partials
hipError_t launch_attn_stream_merge(const StreamLaunch& a, hipStream_t stream);
