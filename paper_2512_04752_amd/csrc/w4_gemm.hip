// Products x . W^T with W in 4 bits, on gfx950 matrix cores.
//
// The codes lie in the order in which a lane of v_mfma_f32_16x16x32_bf16 takes its
// operand: one 16-byte load gives a lane 32 consecutive columns of its row, which share
// one scale, and v_cvt_scalef32_pk_bf16_fp4 makes two of them bf16 with the scale
// applied, exactly (a code has two significant bits).  So the weights pass no LDS, and
// a product differs from one with the unpacked bf16 weights only in the order of its
// sum.  Columns meet rows of x as follows: lane group g = lane / 16 has columns 32 g ..
// 32 g + 31 of a tile, 8 at a time, and its lanes of x the same ones.
//
// The products are taken as D = W . x^T: a lane's four accumulators of a block are four
// consecutive outputs of one row of x.
#include <algorithm>

#include "e2m1.h"
#include "gemm_tile.h"
#include "w4.h"

namespace spec {

namespace {

constexpr int64_t kMaxGrid = 0xffffffffll / 512;
constexpr size_t kPartialCap = 64ull << 20;

// A group's scale; the infinity that byte 255 becomes makes every code a NaN.
__device__ __forceinline__ float scale_of(uint32_t e) { return __uint_as_float(e << 23); }

__device__ __forceinline__ bf16x8 weights_of(uint32_t word, float s) {
  return __builtin_bit_cast(bf16x8, numbers(word, s));
}

// Four outputs of one row of x, columns col .. col + 3.
__device__ __forceinline__ void store4(const W4Args& a, int row, int col, f32x4 v) {
  const int64_t at = row * a.out_stride + col;
  const bool whole = col + 4 <= a.rows;
  if (a.kind == SPEC_W4_BF16) {
    bf16* p = (bf16*)a.out + at;
    const bf16x4 b{(bf16)v[0], (bf16)v[1], (bf16)v[2], (bf16)v[3]};
    if (whole && ((uintptr_t)p & 7) == 0) *(bf16x4*)p = b;
    else
      for (int e = 0; e < 4; ++e)
        if (col + e < a.rows) p[e] = b[e];
  } else {
    float* p = (float*)a.out + at;
    if (whole && ((uintptr_t)p & 15) == 0) {
      *(f32x4*)p = a.kind == SPEC_W4_ADD ? *(const f32x4*)p + v : v;
    } else {
      for (int e = 0; e < 4; ++e)
        if (col + e < a.rows) p[e] = a.kind == SPEC_W4_ADD ? p[e] + v[e] : v[e];
    }
  }
}

__device__ __forceinline__ f32x4 gated(f32x4 g, f32x4 u) {
  return f32x4{silu(g[0]) * u[0], silu(g[1]) * u[1], silu(g[2]) * u[2], silu(g[3]) * u[3]};
}

constexpr int kWaves = 8;

// Few rows.  A work-group takes 16 MB rows of x and NB row tiles of W (of both
// matrices of a gate/up pair); its waves take column tiles in turn, and their sums meet in
// LDS, in the waves' order.
template <int MB, int NB, bool PAIR>
__global__ __launch_bounds__(64 * kWaves) void w4_rows_kernel(W4Args a) {
  constexpr int MATS = PAIR ? 2 : 1, WB = NB * MATS;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row_tiles = (a.rows + 15) / 16, T = w4_col_tiles(a.cols);
  const int groups = (row_tiles + NB - 1) / NB;
  const int group = blockIdx.x % groups, split = blockIdx.x / groups;
  const int m0 = blockIdx.y * 16 * MB;
  const int t0 = (int)((int64_t)T * split / a.plan.splits), t1 = (int)((int64_t)T * (split + 1) / a.plan.splits);
  const char* w[WB];
#pragma unroll
  for (int j = 0; j < WB; ++j)
    w[j] = (j < NB ? a.w0 : a.w1) + (int64_t)min(group * NB + j % NB, row_tiles - 1) * w4_tile_bytes(T);
  const int r = lane & 15, g = lane >> 4;
  const bf16* x[MB];
  bool live[MB];
#pragma unroll
  for (int i = 0; i < MB; ++i) {
    live[i] = m0 + 16 * i + r < a.n;
    x[i] = a.x + (live[i] ? m0 + 16 * i + r : 0) * a.x_stride + 32 * g;
  }
  f32x4 acc[MB][WB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < WB; ++j) acc[i][j] = f32x4{};
  for (int t = t0 + wave; t < t1; t += kWaves) {
    i32x4 c[WB];
    uint32_t e[WB];
    bf16x8 f[MB][4];
#pragma unroll
    for (int j = 0; j < WB; ++j) {
      c[j] = *(const i32x4*)(w[j] + (int64_t)t * 1024 + lane * 16);
      e[j] = *(const uint8_t*)(w[j] + w4_codes_bytes(T) + (t >> 2) * 256 + lane * 4 + (t & 3));
    }
    const bool inside = t * kW4Cols + 32 * g < a.cols;
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        f[i][q] = live[i] && inside ? *(const bf16x8*)(x[i] + t * kW4Cols + 8 * q) : bf16x8{};
#pragma unroll
    for (int j = 0; j < WB; ++j) {
      const float s = scale_of(e[j]);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const bf16x8 b = weights_of((uint32_t)c[j][q], s);
#pragma unroll
        for (int i = 0; i < MB; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, f[i][q], acc[i][j], 0, 0, 0);
      }
    }
  }
  // [block][wave][lane] of four sums
  f32x4* part = (f32x4*)smem;
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < WB; ++j) part[((i * WB + j) * kWaves + wave) * 64 + lane] = acc[i][j];
  __syncthreads();
  auto total = [&](int i, int j) {
    f32x4 v = part[(i * WB + j) * kWaves * 64 + lane];
#pragma unroll
    for (int k = 1; k < kWaves; ++k) v += part[((i * WB + j) * kWaves + k) * 64 + lane];
    return v;
  };
  for (int b = wave; b < MB * NB; b += kWaves) {
    const int i = b / NB, j = b % NB, tile = group * NB + j;
    const int row = m0 + 16 * i + r, col = tile * 16 + 4 * g;
    if (tile >= row_tiles || row >= a.n) continue;
    if (a.plan.splits > 1) {
#pragma unroll
      for (int k = 0; k < MATS; ++k)
        *(f32x4*)(a.partial + ((int64_t)(split * MATS + k) * a.n + row) * (row_tiles * 16) + col) = total(i, j + k * NB);
    } else if (PAIR) {
      store4(a, row, col, gated(total(i, j), total(i, j + NB)));
    } else {
      store4(a, row, col, total(i, j));
    }
  }
}

// Sum the splits, in their order, and store.
template <bool PAIR>
__global__ __launch_bounds__(256) void w4_reduce_kernel(W4Args a) {
  constexpr int MATS = PAIR ? 2 : 1;
  const int padded = (a.rows + 15) / 16 * 16;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = id / (padded / 4);
  const int col = (int)(id % (padded / 4)) * 4;
  if (row >= a.n) return;
  f32x4 v[MATS];
#pragma unroll
  for (int k = 0; k < MATS; ++k) {
    const float* p = a.partial + ((int64_t)k * a.n + row) * padded + col;
    v[k] = *(const f32x4*)p;
    for (int s = 1; s < a.plan.splits; ++s) v[k] += *(const f32x4*)(p + (int64_t)s * MATS * a.n * padded);
  }
  store4(a, (int)row, col, PAIR ? gated(v[0], v[MATS - 1]) : v[0]);
}

template <int MB, int NB, bool PAIR>
hipError_t launch_rows(const W4Args& a, hipStream_t s) {
  const int64_t groups = ((a.rows + 15) / 16 + NB - 1) / NB, blocks = (a.n + 16 * MB - 1) / (16 * MB);
  if (groups * a.plan.splits * blocks > kMaxGrid || blocks > 65535) return hipErrorInvalidValue;
  constexpr int smem = MB * NB * (PAIR ? 2 : 1) * kWaves * 1024;
  static_assert(smem <= 64 * 1024, "LDS without an attribute");
  w4_rows_kernel<MB, NB, PAIR><<<dim3((unsigned)(groups * a.plan.splits), (unsigned)blocks), 64 * kWaves, smem, s>>>(a);
  return hipGetLastError();
}

template <bool PAIR>
hipError_t launch_pair(const W4Args& a, hipStream_t s) {
  hipError_t e;
  switch (a.plan.mb) {
    case 1: e = launch_rows<1, 1, PAIR>(a, s); break;
    case 2: e = launch_rows<2, 1, PAIR>(a, s); break;
    default: e = launch_rows<4, 1, PAIR>(a, s); break;
  }
  if (e != hipSuccess || a.plan.splits == 1) return e;
  const int64_t threads = (int64_t)a.n * ((a.rows + 15) / 16 * 4);
  if ((threads + 255) / 256 > kMaxGrid) return hipErrorInvalidValue;
  w4_reduce_kernel<PAIR><<<(unsigned)((threads + 255) / 256), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

W4Plan plan_w4(int rows, int cols, int n, bool gate_up) {
  (void)rows;
  (void)cols;
  (void)gate_up;
  return W4Plan{n <= 16 ? 1 : n <= 32 ? 2 : 4, 1, 1};
}

size_t w4_partial_bytes(int rows, int cols, int n, bool gate_up) {
  const W4Plan p = plan_w4(rows, cols, n, gate_up);
  return p.splits == 1 ? 0 : (size_t)p.splits * (gate_up ? 2 : 1) * n * ((rows + 15) / 16 * 16) * 4;
}

hipError_t launch_w4(const W4Args& a, hipStream_t s) {
  if (a.n == 0) return hipSuccess;
  return a.w1 ? launch_pair<true>(a, s) : launch_pair<false>(a, s);
}

}  // namespace spec
