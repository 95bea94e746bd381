// Weights into 4 bits and back.  See specverify.h for the numbers and the layout.
//
// Both kernels are copies, bound by HBM: 2 bytes per number on one side and 17 / 32
// on the other.  A wave takes four column tiles of a row tile (16 x 512 numbers, 16 KB of
// bf16, all its loads in flight at once).  Lane l has row 4 i + l / 16 and the 8 numbers
// from column 8 (l % 16) of each tile, so that bf16 moves as 256 contiguous bytes of four
// rows; a group is four lanes, whose maximum goes by two DPP moves, and their 8 codes each
// are a word of the layout.  14336 x 4096: 37 us to pack and 23 to unpack, of 149 MB each (4.0
// and 6.4 TB/s; what the first writes was last read, what the second reads was just written);
// 61 as two calls, where a copy of as many bytes takes 58.  2048 x 2048: 5.4 and 5.0.
#include "e2m1.h"
#include "w4.h"

namespace spec {

namespace {

constexpr int64_t kMaxGrid = 0xffffffffll / 256;

// What both kernels know of their wave and lane.
struct Place {
  int rt, kt0, tiles;         // row tile, first column tile, column tiles in all
  int r4, chunk;              // row in a group of four, 8-number chunk of a tile
  bool some;                  // the wave has work
};
__device__ __forceinline__ Place place(int rows, int cols) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  Place p;
  p.tiles = w4_col_tiles(cols);
  const int quads = (p.tiles + 3) / 4;
  const int64_t id = (int64_t)blockIdx.x * 4 + wave;
  p.rt = (int)(id / quads);
  p.kt0 = (int)(id % quads) * 4;
  p.some = p.rt < (rows + 15) / 16;
  p.r4 = lane >> 4;
  p.chunk = lane & 15;
  return p;
}

// Word of the codes that lane (row r, chunk c) has in a tile, and its group's scale.
__device__ __forceinline__ int word_at(int r, int c) { return (r + 16 * (c >> 2)) * 16 + (c & 3) * 4; }
__device__ __forceinline__ int scale_at(int r, int c) { return r + 16 * (c >> 2); }

__global__ __launch_bounds__(256) void w4_pack_kernel(const bf16* w, int64_t stride, int rows, int cols,
                                                      char* data) {
  const Place p = place(rows, cols);
  if (!p.some) return;
  i32x4 v[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int row = p.rt * 16 + 4 * i + p.r4, col = (p.kt0 + j) * kW4Cols + 8 * p.chunk;
      v[i][j] = row < rows && col < cols ? *(const i32x4*)(w + row * stride + col) : i32x4{0, 0, 0, 0};
    }
  char* tile = data + p.rt * w4_tile_bytes(p.tiles);
  uint8_t* scales = (uint8_t*)tile + w4_codes_bytes(p.tiles);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = 4 * i + p.r4;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float f[8];
      uint32_t top = 0;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        f[2 * q] = __uint_as_float((uint32_t)v[i][j][q] << 16);
        f[2 * q + 1] = __uint_as_float((uint32_t)v[i][j][q] & 0xffff0000u);
      }
#pragma unroll
      for (int q = 0; q < 8; ++q) top = max(top, __float_as_uint(f[q]) & 0x7fffffffu);
      top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0xB1, 0xf, 0xf, true));   // quad_perm 1 0 3 2
      top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0x4E, 0xf, 0xf, true));   // quad_perm 2 3 0 1
      const uint32_t e = scale_byte(top, kW4Lowest);
      const uint32_t codes = pack_codes<8>(f, e);
      if (p.kt0 + j >= p.tiles) continue;
      *(uint32_t*)(tile + (int64_t)(p.kt0 + j) * 1024 + word_at(r, p.chunk)) = codes;
      if ((p.chunk & 3) == 0) scales[(p.kt0 + j) * 64 + scale_at(r, p.chunk)] = (uint8_t)e;
    }
  }
}

__global__ __launch_bounds__(256) void w4_unpack_kernel(const char* data, int rows, int cols, bf16* w,
                                                        int64_t stride) {
  const Place p = place(rows, cols);
  if (!p.some) return;
  const char* tile = data + p.rt * w4_tile_bytes(p.tiles);
  const uint8_t* scales = (const uint8_t*)tile + w4_codes_bytes(p.tiles);
  uint32_t codes[4][4], exps[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = 4 * i + p.r4;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int t = min(p.kt0 + j, p.tiles - 1);
      codes[i][j] = *(const uint32_t*)(tile + (int64_t)t * 1024 + word_at(r, p.chunk));
      exps[i][j] = scales[t * 64 + scale_at(r, p.chunk)];
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int row = p.rt * 16 + 4 * i + p.r4, col = (p.kt0 + j) * kW4Cols + 8 * p.chunk;
      // (byte 255 becomes an infinity, with which every code is a NaN)
      const i32x4 v = numbers(codes[i][j], __uint_as_float(exps[i][j] << 23));
      if (row < rows && col < cols) *(i32x4*)(w + row * stride + col) = v;
    }
}

hipError_t grid_of(int rows, int cols, unsigned* grid) {
  const int64_t waves = (int64_t)((rows + 15) / 16) * ((w4_col_tiles(cols) + 3) / 4);
  if ((waves + 3) / 4 > kMaxGrid) return hipErrorInvalidValue;
  *grid = (unsigned)((waves + 3) / 4);
  return hipSuccess;
}

}  // namespace

hipError_t launch_w4_pack(const bf16* w, int64_t stride, int rows, int cols, char* data, hipStream_t s) {
  unsigned grid;
  if (const hipError_t e = grid_of(rows, cols, &grid)) return e;
  w4_pack_kernel<<<grid, 256, 0, s>>>(w, stride, rows, cols, data);
  return hipGetLastError();
}

hipError_t launch_w4_unpack(const char* data, int rows, int cols, bf16* w, int64_t stride, hipStream_t s) {
  unsigned grid;
  if (const hipError_t e = grid_of(rows, cols, &grid)) return e;
  w4_unpack_kernel<<<grid, 256, 0, s>>>(data, rows, cols, w, stride);
  return hipGetLastError();
}

}  // namespace spec
