// Matrices in 4 bits: layout, kernel arguments and launcher prototypes.
#pragma once

#include "common.h"

namespace spec {

constexpr int kW4Rows = 16, kW4Cols = 128;      // a tile of the layout, see specverify.h
constexpr int kW4Lowest = 7;                    // lowest scale byte: 2^-120, no code of it is subnormal in bf16

// Column tiles and bytes of a row tile.
constexpr __host__ __device__ int w4_col_tiles(int cols) { return (cols + kW4Cols - 1) / kW4Cols; }
constexpr __host__ __device__ int64_t w4_codes_bytes(int col_tiles) { return (int64_t)col_tiles * 1024; }
constexpr __host__ __device__ int64_t w4_tile_bytes(int col_tiles) {
  return w4_codes_bytes(col_tiles) + (int64_t)((col_tiles + 3) / 4) * 256;      // of 64 bytes per column tile
}

// w[0, rows) x [0, cols) <-> data.
hipError_t launch_w4_pack(const bf16* w, int64_t stride, int rows, int cols, char* data, hipStream_t s);
hipError_t launch_w4_unpack(const char* data, int rows, int cols, bf16* w, int64_t stride, hipStream_t s);

// How a product runs: rows of x and row tiles of W per work-group, and K splits.
enum W4Shape { W4_STREAM, W4_TILE32, W4_TILE32W, W4_TILE64, W4_TILE64W, W4_TILE128, W4_TILE256 };
struct W4Plan {
  W4Shape shape;   // the stream kernel, or a tile's rows of x (W: with more of W)
  int wide;        // W4_STREAM: waves that share the columns
  int splits;      // of the columns, over work-groups
};

constexpr int kW4Partial = -1;    // the sums of every split stay in W4Args::partial, for who joins them

struct W4Args {
  W4Plan plan;
  const char* w0;           // W, or gate
  const char* w1;           // up; NULL: a plain product
  int rows, cols;           // of W
  const bf16* x;
  int64_t x_stride;
  int n;                    // rows of x
  void* out;
  int64_t out_stride;
  int kind;                 // SPEC_W4_*, or kW4Partial
  float* partial;           // [splits][matrices][n][16 * row tiles]
};

constexpr size_t kW4PartialCap = 64ull << 20;      // most bytes of a product's partial sums
constexpr int kMostSplitRows = 4096;     // rows of x from which on columns are not split
W4Plan plan_w4(int rows, int cols, int n, bool gate_up);
size_t w4_partial_bytes(int rows, int cols, int n, bool gate_up);
hipError_t launch_w4(const W4Args& a, hipStream_t s);

}  // namespace spec
