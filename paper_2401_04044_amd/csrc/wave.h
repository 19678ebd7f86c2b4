// Internal: what the kernels with hand-counted loads share: waits, barrier, order of instructions, order of tiles.
#pragma once
#include <hip/hip_runtime.h>

namespace ffsplit {

// s_waitcnt with only the vector-memory counter constrained (gfx9 encoding: vmcnt in
// imm[3:0] and imm[15:14], expcnt imm[6:4], lgkmcnt imm[11:8])
template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x0f70);
}
template <int N>
__device__ __forceinline__ void wait_lgkmcnt() {
  __builtin_amdgcn_s_waitcnt(0xc07f | ((N < 15 ? N : 15) << 8));
}
// workgroup barrier without a memory fence (the kernels order their loads with explicit counters);
// the memory clobber keeps the compiler from moving LDS accesses across it
__device__ __forceinline__ void lds_barrier() { asm volatile("s_barrier" ::: "memory"); }
#define FFS_ORDER __builtin_amdgcn_sched_barrier(0)   // instructions keep the written order

// Workgroup i of total in an order that gives each XCD (workgroups go to them in turn) a contiguous run of tiles
__device__ __forceinline__ int xcd_remap(int i, int total) {
  const int q = total >> 3, rem = total & 7, x = i & 7;
  return x * q + (x < rem ? x : rem) + (i >> 3);
}

}  // namespace ffsplit
