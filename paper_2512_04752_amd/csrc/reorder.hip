// The cache rows that follow the beams: beam j's positions [begin, end) become what its
// parent held, all beams of a group at once.
//
// A thread owns one place (8 or 16 bytes at one offset of the range) in all beams of a
// group.  It reads what every moving beam will hold, all those loads in flight together,
// and then writes: no value is overwritten before it is read, whatever the parents are
// (cycles, one parent of many), and no thread waits for another.  Bound by HBM: every
// parent is read once (a second beam's read of it hits the caches) and every moving beam
// written once; beams that stay cost nothing.
// 16 groups of 8 beams, 5 of them moving 500 tokens of the 4-bit pool (8 layers of 8 heads of
// 128): 119 us (the median; 107 at best) for 549 MB, 4.6 TB/s where a copy of 1 GiB reaches 5.15.
// 8 beams, 5 of them moving 100 tokens of the bf16 pool (16 such layers): 10.8 us for 52 MB
// (caches take part).
#include <algorithm>
#include <type_traits>

#include "kv4.h"
#include "reorder.h"

namespace spec {

namespace {

constexpr int kThreads = 256;

// Waves per SIMD that the registers shall leave room for.  Without the bound the compiler
// keeps every beam's 64-bit addresses (238 registers for 8 beams, and 2 waves per SIMD).
constexpr int min_waves(int w) { return w <= 8 ? 8 : w <= 16 ? 5 : 3; }

// The moving beams of a group into LDS, as byte places of what they read and write
// (place(beam)); their number.  One wave's work: a parent, its and the beam's descriptor.
struct Moves {
  int64_t from[64], to[64];
  int count;
};
template <class F>
__device__ __forceinline__ int moving_beams(const int32_t* parents, int width, Moves* m, F&& place) {
  if (threadIdx.x < 64) {
    const int j = threadIdx.x;
    const int p = j < width ? parents[j] : -1;
    const bool moves = p >= 0 && p < width && p != j;
    const uint64_t all = __ballot(moves);
    if (moves) {
      const int at = __popcll(all & ((1ull << j) - 1));
      m->from[at] = place(p);
      m->to[at] = place(j);
    }
    if (j == 0) m->count = __popcll(all);
  }
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(m->count);
}

// A value that all lanes have, as a scalar.
__device__ __forceinline__ int64_t scalar(int64_t x) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((int)(uint32_t)x), hi = __builtin_amdgcn_readfirstlane((int)(x >> 32));
  return (int64_t)((uint64_t)hi << 32 | lo);
}

template <int W, class Unit>
__global__ __launch_bounds__(kThreads, min_waves(W)) void reorder_kernel(ReorderBeams beams, int width, char* pool,
                                                                          int head_dim, const int32_t* parents) {
  __shared__ Moves m;
  const int g = blockIdx.z, run = blockIdx.y;
  const ReorderGroup r = (beams.groups ? beams.groups : beams.groups_here)[g];
  const ReorderBeam* b = (beams.groups ? beams.beams : beams.beams_here) + (int64_t)g * width;
  const int64_t bytes = (int64_t)(r.end - r.begin) * head_dim * 2, block = (int64_t)blockIdx.x * kThreads * sizeof(Unit);
  if (block >= bytes) return;
  const int n = moving_beams(parents + (int64_t)g * width, width, &m, [&](int j) {
    return (int64_t)b[j].block * 256 + ((int64_t)run * b[j].cap + r.begin) * head_dim * 2;
  });
  const uint32_t at = threadIdx.x * sizeof(Unit);
  if (block + at >= bytes) return;
  Unit v[W];
#pragma unroll
  for (int i = 0; i < W; ++i)
    if (i < n) v[i] = *(const Unit*)(pool + scalar(m.from[i]) + block + at);
#pragma unroll
  for (int i = 0; i < W; ++i)
    if (i < n) *(Unit*)(pool + scalar(m.to[i]) + block + at) = v[i];
}

// Which bits of word w (of a 16-byte unit `u` of a head's bytes in a page) belong to
// positions [lo, hi) of the page.
template <int HD>
__device__ __forceinline__ uint32_t bits_of(int u, int w, int lo, int hi) {
  constexpr int KEYS = kv4_value_at(HD) / 16, VALUES = kv4_kscale_at(HD) / 16, KSCALES = kv4_vscale_at(HD) / 16;
  auto inside = [&](int pos) { return pos >= lo && pos < hi; };
  if (u < KEYS) return inside(u / HD * 32 + u % 32) ? ~0u : 0u;      // a key's 32 numbers
  uint32_t m = 0;
  if (u < VALUES) {                                                  // words of eight positions' numbers
    const int p0 = (u - KEYS) / (HD / 4) * 8;
#pragma unroll
    for (int t = 0; t < 8; ++t) m |= inside(p0 + t) ? 15u << (4 * t) : 0u;
    return m;
  }
  const bool keys = u < KSCALES;
  const int per = keys ? HD / 32 : 2, b0 = (u - (keys ? VALUES : KSCALES)) * 16 + 4 * w;
#pragma unroll
  for (int t = 0; t < 4; ++t) m |= inside((b0 + t) / per) ? 255u << (8 * t) : 0u;
  return m;
}

template <int W, class Unit, int HD>
__global__ __launch_bounds__(kThreads, min_waves(W)) void kv4_reorder_kernel(ReorderPages info, int width, char* pool,
                                                                              int64_t page_bytes,
                                                                              const int32_t* parents) {
  __shared__ Moves m;
  constexpr int BYTES = sizeof(Unit), WORDS = BYTES / 4;
  const int g = blockIdx.z, page = blockIdx.y;
  const ReorderGroup r = (info.groups ? info.groups : info.groups_here)[g];
  if (page >= r.pages) return;
  const int n = moving_beams(parents + (int64_t)g * width, width, &m, [&](int j) {
    const int64_t at = r.table + (int64_t)j * r.pages + page;
    return (info.groups ? info.table[at] : (int32_t)info.table_here[at]) * page_bytes;
  });
  const int64_t block = (int64_t)blockIdx.x * kThreads * BYTES;
  const uint32_t at = threadIdx.x * BYTES;
  if (block + at >= page_bytes) return;
  const int pos0 = (r.begin / kKv4Page + page) * kKv4Page;
  const int lo = max(0, r.begin - pos0), hi = min(kKv4Page, r.end - pos0);
  uint32_t mask[WORDS], all = ~0u, some = ~0u;
  if (lo > 0 || hi < kKv4Page) {
    const int in_head = (int)((block + at) % kv4_head_bytes(HD));
    some = 0;
#pragma unroll
    for (int w = 0; w < WORDS; ++w) {
      mask[w] = bits_of<HD>(in_head / 16, in_head % 16 / 4 + w, lo, hi);
      all &= mask[w];
      some |= mask[w];
    }
    if (some == 0) return;
  }
  Unit v[W];
#pragma unroll
  for (int i = 0; i < W; ++i)
    if (i < n) v[i] = *(const Unit*)(pool + scalar(m.from[i]) + block + at);
  if (all == ~0u) {
#pragma unroll
    for (int i = 0; i < W; ++i)
      if (i < n) *(Unit*)(pool + scalar(m.to[i]) + block + at) = v[i];
  } else {
#pragma unroll
    for (int i = 0; i < W; ++i)
      if (i < n) {
        Unit* p = (Unit*)(pool + scalar(m.to[i]) + block + at);
        const Unit old = *p;
#pragma unroll
        for (int w = 0; w < WORDS; ++w) v[i][w] = (int)((uint32_t)old[w] & ~mask[w] | (uint32_t)v[i][w] & mask[w]);
        *p = v[i];
      }
  }
}

// Units of 16 bytes, of 8 where 64 beams' would not fit the registers.
template <class F>
hipError_t by_width(int width, F&& go) {
  if (width <= 8) return go(std::integral_constant<int, 8>{}, i32x4{});
  if (width <= 16) return go(std::integral_constant<int, 16>{}, i32x4{});
  if (width <= 32) return go(std::integral_constant<int, 32>{}, i32x4{});
  return go(std::integral_constant<int, 64>{}, i32x2{});
}

hipError_t grid_of(int64_t x, int64_t y, int64_t z, dim3* grid) {
  if (x > 0xffffffffll / kThreads || y > 65535 || z > 65535) return hipErrorInvalidValue;
  *grid = dim3((unsigned)x, (unsigned)y, (unsigned)z);
  return hipSuccess;
}

}  // namespace

hipError_t launch_reorder(const ReorderBeams& beams, int groups, int width, int most, bf16* pool, int n_layers,
                          int n_kv_heads, int head_dim, const int32_t* parents, hipStream_t s) {
  return by_width(width, [&](auto w, auto unit) {
    using Unit = decltype(unit);
    const int64_t units = (int64_t)most * head_dim * 2 / sizeof(Unit);
    dim3 grid;
    if (const hipError_t e = grid_of((units + kThreads - 1) / kThreads, (int64_t)n_layers * 2 * n_kv_heads, groups, &grid))
      return e;
    reorder_kernel<decltype(w)::value, Unit><<<grid, kThreads, 0, s>>>(beams, width, (char*)pool, head_dim, parents);
    return hipGetLastError();
  });
}

hipError_t launch_kv4_reorder(const ReorderPages& info, int groups, int width, int most, char* pool,
                              int64_t page_bytes, int head_dim, const int32_t* parents, hipStream_t s) {
  return by_width(width, [&](auto w, auto unit) {
    using Unit = decltype(unit);
    constexpr int W = decltype(w)::value;
    dim3 grid;
    const int64_t units = page_bytes / sizeof(Unit);
    if (const hipError_t e = grid_of((units + kThreads - 1) / kThreads, most, groups, &grid)) return e;
    if (head_dim == 128)
      kv4_reorder_kernel<W, Unit, 128><<<grid, kThreads, 0, s>>>(info, width, pool, page_bytes, parents);
    else if (head_dim == 64)
      kv4_reorder_kernel<W, Unit, 64><<<grid, kThreads, 0, s>>>(info, width, pool, page_bytes, parents);
    else
      return hipErrorInvalidValue;
    return hipGetLastError();
  });
}

}  // namespace spec
