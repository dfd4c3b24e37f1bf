// Launches of the attention kernels that divide a batch's tokens among the workgroups by themselves (attn_stream.hip, attn_prefix.hip).
#pragma once
#include "rapid_internal.h"

struct AttnSource {             // where keys and values lie; strides in elements (scales: bytes)
    const void* k;
    const void* v;
    const uint8_t* ks;          // scales, or null: bf16
    const uint8_t* vs;
    const int32_t* page_table;  // or null: contiguous
    int64_t bstride, tstride, hstride, pstride;
    int64_t sbstride, shstride, spstride;
    int32_t page_shift, page_mask, max_pages, page_hi;
};
struct StreamLaunch {
    const uint16_t* q;
    uint16_t* out;
    float* lse_out;
    const int32_t* ctx_lens;
    const int32_t* gammas;
    AttnSource own;
    float* part_o;              // [Hkv][tiles][nslots][RP][D], relative to the maximum in part_ml; slot g + b: share g's piece of sequence b
    float* part_ml;             // [Hkv][tiles][nslots][RP][2] (maximum in log2 units, sum)
    int32_t B, Qmax, Hq, Hkv, G, D, gamma, max_ctx;
    int32_t shared;             // 1: a shared prefix: one sequence (ctx_lens: its length) with the rows of the batch, which all attend all of it
    int32_t RP, tiles;          // packed rows of a slot (a multiple of 16), row tiles (1 but for a prefix)
    int32_t groups, nslots;     // shares of a kv head, groups + B - 1
    int32_t units;              // two in one launch: workgroups of a kv head, which they divide by their lengths; groups is then the most.  0: groups as they are
    int32_t quantum;            // tokens that shares are cut by
    int32_t rot;                // 1: share g of slot x serves head (x + g) mod Hkv, 0: head x
    int32_t direct;             // 1: short sequences, one workgroup for each and kv head, which writes the result; no partials
    float scale_log2e;
};
constexpr int kStreamRows = 96;      // packed rows that the streaming kernel takes
// Fill the plan (RP .. direct) from the shape and the source's layout.
void plan_attn_stream(StreamLaunch& a, int n_cu);
void plan_attn_prefix(StreamLaunch& a, int n_cu);
// Both for one launch: the tokens of a shared prefix, its rows in tiles of at most kStreamRows, and the sequences' own.  Where the two lie differently
// (one paged, the other not), for two launches in turn.
void plan_attn_stream_pair(StreamLaunch& own, StreamLaunch& prefix, int n_cu);
size_t attn_stream_workspace_bytes(const StreamLaunch& a);                       // of any plan
void bind_attn_stream(StreamLaunch& a, void* workspace);
hipError_t configure_attn_stream();
hipError_t configure_attn_prefix();
// Write the partials (direct: the result).
hipError_t launch_attn_stream(const StreamLaunch& a, hipStream_t stream);
hipError_t launch_attn_stream_pair(const StreamLaunch& own, const StreamLaunch& prefix, hipStream_t stream);
hipError_t launch_attn_prefix(const StreamLaunch& a, hipStream_t stream);
// Joins the partials of `own`, and of a shared prefix where `prefix` has any (prefix.part_o not null).
hipError_t launch_attn_stream_merge(const StreamLaunch& own, const StreamLaunch& prefix, hipStream_t stream);
