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
    int32_t window, sinks;      // window > 0: a row at position p attends tokens of (p - window, p] and the first `sinks`; 0: all up to p
    int32_t many;               // a window: 1: attn_window.hip's kernel, 0: the streaming one
    float scale_log2e;
};
constexpr int kStreamRows = 96;      // packed rows that a workgroup of the streaming kernel takes
// Fill the plan (RP .. direct) from the shape and the source's layout.
void plan_attn_stream(StreamLaunch& a, int n_cu);
// A window: row tiles of at most kStreamRows, `groups` shares of a row tile's tokens, direct where that is one.  Both return the us that they expect, the first
// infinity where its grid does not fit.
float plan_attn_stream_window(StreamLaunch& a, int n_cu);                        // q is addressed with 32 bits
void plan_attn_prefix(StreamLaunch& a, int n_cu);
float plan_attn_window(StreamLaunch& a, int n_cu);                               // attn_window.hip
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
hipError_t configure_attn_window();
size_t attn_window_workspace_bytes(const StreamLaunch& a);
void bind_attn_window(StreamLaunch& a, void* workspace);
hipError_t launch_attn_window(const StreamLaunch& a, hipStream_t stream);        // writes the result (with a second launch where groups > 1)
// Joins the partials of `own`, and of a shared prefix where `prefix` has any (prefix.part_o not null).
hipError_t launch_attn_stream_merge(const StreamLaunch& own, const StreamLaunch& prefix, hipStream_t stream);
