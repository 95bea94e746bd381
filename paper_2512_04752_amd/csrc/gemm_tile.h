// Device pieces that the matrix-product kernels share: direct loads into LDS, their
// waits and barriers, the LDS swizzle, and the order of output tiles over the XCDs.
#pragma once

#include "common.h"

namespace spec {

typedef __attribute__((address_space(3))) char lds_char;

// Direct global -> LDS load of 16 bytes per lane from base + voff to the
// wave-uniform LDS address `lds` + 16 * lane.  In assembly, so that the
// compiler does not wait for it at the next LDS read; the kernels' own vmcnt
// waits and barriers order it.  The s_nop is the wait state that the load needs
// after a write of M0.
__device__ __forceinline__ void dma16(const void* base, uint32_t voff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(voff), "s"(base), "s"(lds)
               : "memory", "m0");
}

// Barrier that no memory access and no instruction is moved across.
__device__ __forceinline__ void phase_barrier() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_barrier" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

__device__ __forceinline__ void wait_lds() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// 16-byte chunk swizzle of tile row `row` (rows of 128 bytes): 16 consecutive
// rows reading one logical chunk hit 16 distinct 16-byte bank groups.
__device__ __forceinline__ int swz(int row) { return (row >> 1) & 7; }

// Wait until at most N vector-memory operations of this wave are in flight.
template <int N>
__device__ __forceinline__ void wait_vm() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

__device__ __forceinline__ float silu(float g) { return g / (1.0f + __expf(-g)); }

// Work-group b runs on XCD b % 8, which receives q + 1 work-groups (x < r)
// or q (x >= r) for a grid of 8q + r.  Give each XCD a contiguous range of
// logical ids, so that the M tiles sharing a weight tile (adjacent ids)
// meet in one XCD's L2.
__device__ __forceinline__ int xcd_contiguous(int b, int total) {
  const int q = total >> 3, r = total & 7, x = b & 7, j = b >> 3;
  return (x < r ? x * (q + 1) : r * (q + 1) + (x - r) * q) + j;
}

// Output tile of logical work-group id `tile`.  Up to 8 M tiles: all M tiles
// of a weight tile in a row.  More: blocks of 8 weight tiles x 4 M tiles, the
// 32 tiles an XCD runs at a time, so that its L2 is filled with 12 operand
// tiles instead of 2 + ntm (gate/up at 8192 rows 1424 -> 1274 us, at 4096 rows
// 684 -> 677 us, at 2048 rows 379 -> 387 us: hence the line).
__device__ __forceinline__ void tile_at(int tile, int ntm, int ntn, int* tm, int* tn) {
  constexpr int GN = 8, GM = 4;
  if (ntm <= 8) {
    *tm = tile % ntm;
    *tn = tile / ntm;
    return;
  }
  const int gi = tile / (GN * ntm), rem = tile % (GN * ntm);
  const int cols = min(GN, ntn - gi * GN), panel = rem / (GM * cols), in = rem - panel * GM * cols;
  const int rows = min(GM, ntm - panel * GM);
  *tm = panel * GM + in % rows;
  *tn = gi * GN + in / rows;
}

}  // namespace spec
