// Primitives of the attention kernels: loads that go from HBM straight to LDS and the waits for them, reductions over lanes.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

namespace {

// 16 bytes a lane, HBM -> LDS: lane i writes LDS bytes [lds_addr + 16 i, + 16) and fetches them from base + byte_off.
//
// The instruction is written as inline assembly on purpose: the wave keeps its own
// account of outstanding loads (wait_loads<N>() below).  Issued through the
// compiler's builtin, every later LDS read would be preceded by a compiler-inserted
// wait for ALL outstanding loads, which serialises the pipeline.  `nt` marks the
// data as streaming (read once): measured +5..10 % bandwidth over the default policy.
__device__ __forceinline__ void dma16(const char* base, uint32_t byte_off, uint32_t lds_addr)
{
    asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1 nt"
                 :
                 : "v"(byte_off), "s"(base), "s"(lds_addr)
                 : "memory", "m0");
}
// The same load without the streaming hint, for data that other workgroups read again (Q).
__device__ __forceinline__ void dma16_keep(const char* base, uint32_t byte_off, uint32_t lds_addr)
{
    asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1"
                 :
                 : "v"(byte_off), "s"(base), "s"(lds_addr)
                 : "memory", "m0");
}

// Wait until at most N of this wave's vector-memory loads are outstanding.  The
// loads complete in order, so this guarantees everything older has landed in LDS.
template <int N>
__device__ __forceinline__ void wait_loads()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// All LDS reads issued so far have returned: the slot they read may be refilled.
__device__ __forceinline__ void lds_reads_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// Reductions over the four lanes that differ in lane / 16 only, without LDS: a swap between two registers (upper half of one with the
// lower of the other, or odd rows of 16 lanes with even ones) leaves both sides of every pair in one lane.  (The copy is hidden from
// the compiler, which else takes the two for one value.)  The row max of a tile is on the way from its scores to its
// weights: with shuffles through LDS a call on 8K tokens took 12.6 us instead of 12.2, on 32K 31.4 instead of 30.9, 64 rows of 32K 35.0 instead of 34.1.
struct Pair { float x, y; };
__device__ __forceinline__ Pair lane_pair16(float v)
{
    unsigned a = __float_as_uint(v), b = a;
    asm("" : "+v"(b));
    const auto h = __builtin_amdgcn_permlane16_swap(a, b, false, false);
    return Pair{__uint_as_float(h[0]), __uint_as_float(h[1])};
}
__device__ __forceinline__ Pair lane_pair32(float v)
{
    unsigned a = __float_as_uint(v), b = a;
    asm("" : "+v"(b));
    const auto h = __builtin_amdgcn_permlane32_swap(a, b, false, false);
    return Pair{__uint_as_float(h[0]), __uint_as_float(h[1])};
}
__device__ __forceinline__ float max_over_groups(float v)
{
    Pair p = lane_pair16(v);
    p = lane_pair32(fmaxf(p.x, p.y));
    return fmaxf(p.x, p.y);
}
__device__ __forceinline__ float sum_over_groups(float v)
{
    Pair p = lane_pair16(v);
    p = lane_pair32(p.x + p.y);
    return p.x + p.y;
}

// 64 sequences at a time, one per lane: (inclusive prefix of the cost, own cost) of sequence b0 + lane.
__device__ __forceinline__ int scan_costs(int cost)
{
    cost += __builtin_amdgcn_update_dpp(0, cost, 0x111, 0xf, 0xf, false);        // row_shr 1, 2, 4, 8 inside rows of 16 lanes
    cost += __builtin_amdgcn_update_dpp(0, cost, 0x112, 0xf, 0xf, false);
    cost += __builtin_amdgcn_update_dpp(0, cost, 0x114, 0xf, 0xf, false);
    cost += __builtin_amdgcn_update_dpp(0, cost, 0x118, 0xf, 0xf, false);
    cost += __builtin_amdgcn_update_dpp(0, cost, 0x142, 0xa, 0xf, false);        // lane 15 of a row into the next: rows 1 and 3
    cost += __builtin_amdgcn_update_dpp(0, cost, 0x143, 0xc, 0xf, false);        // lane 31 into the upper half
    return cost;
}

}  // namespace
