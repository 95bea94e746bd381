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
#include <atomic>

#include "e2m1.h"
#include "gemm_tile.h"
#include "w4.h"

namespace spec {

namespace {

constexpr int64_t kMaxGrid = 0xffffffffll / 512;

// Direct global -> LDS load of 16 bytes per lane from the lane's own address to the
// wave-uniform LDS address `lds` + 16 * lane; see dma16(base, voff, lds).
__device__ __forceinline__ void dma16_at(const void* p, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(p), "s"(lds) : "memory", "m0");
}

// A group's scale; the infinity that byte 255 becomes makes every code a NaN.
__device__ __forceinline__ float scale_of(uint32_t e) { return __uint_as_float(e << 23); }

__device__ __forceinline__ bf16x8 weights_of(uint32_t word, float s) {
  return __builtin_bit_cast(bf16x8, numbers(word, s));
}

// A row tile of a matrix as a buffer: places in it are a lane's constant offset and a scalar
// one.  (Of pointers the compiler keeps a 64-bit address per load and lane over the loops.)
struct RowTile {
  __amdgpu_buffer_rsrc_t buf;
  __device__ __forceinline__ RowTile() {}
  __device__ __forceinline__ RowTile(const char* w, int tile, int T)
      : buf(__builtin_amdgcn_make_buffer_rsrc((void*)(w + tile * w4_tile_bytes(T)), 0, (int)w4_tile_bytes(T), 0x27000)) {}
  // A lane's codes and scale of column tile t.
  __device__ __forceinline__ void load(int T, int t, int lane, i32x4* c, uint32_t* e) const {
    *c = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(buf, lane * 16, t * 1024, 0));
    *e = __builtin_amdgcn_raw_buffer_load_b8(buf, lane, (int)w4_codes_bytes(T) + t * 64, 0);
  }
};

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

// Four sums (of each matrix) of row `row`, columns col .. col + 3, of one split.
template <bool PAIR>
__device__ __forceinline__ void finish(const W4Args& a, int split, int row, int col, const f32x4 (&v)[PAIR ? 2 : 1]) {
  constexpr int MATS = PAIR ? 2 : 1;
  if (a.plan.splits > 1 || a.kind == kW4Partial) {
    const int padded = (a.rows + 15) / 16 * 16;
#pragma unroll
    for (int k = 0; k < MATS; ++k)
      *(f32x4*)(a.partial + ((int64_t)(split * MATS + k) * a.n + row) * padded + col) = v[k];
  } else {
    store4(a, row, col, PAIR ? gated(v[0], v[MATS - 1]) : v[0]);
  }
}

// Accumulators that a loop goes on with, held in registers from here on.  (Of zeros that it
// may make again where they are used, this compiler, ROCm 7.2, has left out two of the four.)
__device__ __forceinline__ f32x4 zeros() {
  f32x4 v{};
  asm volatile("" : "+v"(v));
  return v;
}

// Few rows (up to 16): bound by the weights' bytes, and so by how many of them are on their
// way at a time (some 10 MB over the chip).  The rows of x, or their columns of this split,
// lie in LDS as a whole; after that a wave only loads weights, up to 2 D column tiles of a row
// tile (of both matrices) ahead, and meets no barrier.  The sixteen waves of a work-group take
// KG ranges of the columns for 16 / KG groups of row tiles (KG > 1: their sums meet in LDS, in
// order) and go on with the next such set until there is none.  (Per wave and column tile 4 KB of x come
// out of LDS for 1 KB of weights out of HBM; read from L2 instead, x takes more of the
// load path than the weights, and its loads, waited for in order, hold theirs up.)
// Calls, three copies of the weights in turn (the last-level cache may hold them): gate/up
// 14336 x 4096, 4 rows, 12.7 us (62.5 MB, 4.9 TB/s); 4096 x 14336, 16 rows, 11.3 (31.8 MB; four
// splits, whose reduction is 3 of it); 2048 x 2048, 1 row, 5.6: the launch and one trip through
// the loads.
constexpr int kStreamWaves = 16;
template <bool PAIR>
__global__ __launch_bounds__(64 * kStreamWaves, 4) void w4_stream_kernel(W4Args a) {
  constexpr int NB = PAIR ? 2 : 1, D = 4 / NB;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row_tiles = (a.rows + 15) / 16, T = w4_col_tiles(a.cols);
  const int KG = a.plan.wide, CG = kStreamWaves / KG, kg = wave % KG, cg = wave / KG;
  const int split = blockIdx.x % a.plan.splits, first = blockIdx.x / a.plan.splits, wgs = gridDim.x / a.plan.splits;
  const int s0 = T * split / a.plan.splits, s1 = T * (split + 1) / a.plan.splits;
  const int longest = (T + a.plan.splits - 1) / a.plan.splits, pitch = (longest + 3) / 4 * 1024;
  const int r = lane & 15, g = lane >> 4;
  const int len = s1 - s0, t0 = s0 + len * kg / KG, t1 = s0 + len * (kg + 1) / KG;
  RowTile w[NB];
  auto weights_at = [&](int tile) {
#pragma unroll
    for (int j = 0; j < NB; ++j) w[j] = RowTile(j == 0 ? a.w0 : a.w1, min(tile, row_tiles - 1), T);
  };
  struct Tiles {
    i32x4 c[D][NB];
    uint32_t e[D][NB];
  };
  auto load = [&](Tiles& b, int t) {
#pragma unroll
    for (int u = 0; u < D; ++u) {
      const int tu = min(t + u, t1 - 1);         // never conditional: the compiler's waits count the loads
#pragma unroll
      for (int j = 0; j < NB; ++j) w[j].load(T, tu, lane, &b.c[u][j], &b.e[u][j]);
    }
  };
  Tiles b0, b1;
  // x into LDS: wave-load = 64 chunks of 16 bytes of one row, chunk c at place c ^ row of its 16.
  // The first weights go out behind it, and are not waited for with it.
  {
    const int per_row = pitch / 1024, loads = a.n * per_row, valid = (a.cols - s0 * kW4Cols) / 8;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_char*)smem;
    for (int l = wave; l < loads; l += kStreamWaves) {
      const int row = l / per_row, c = l % per_row * 64 + (lane ^ (row & 15));
      const bf16* p = a.x + row * a.x_stride + (int64_t)s0 * kW4Cols;
      dma16_at(p + (c < valid ? 8 * c : 0), lds0 + row * pitch + l % per_row * 1024);
    }
    weights_at(first * CG + cg);
    if (t0 < t1) {
      load(b0, t0);
      wait_vm<2 * D * NB>();
    } else {
      wait_vm<0>();
    }
    if (s1 == T && (a.cols & (kW4Cols - 1)))                   // columns that the matrix does not have
      for (int l = wave; l < loads; l += kStreamWaves) {
        const int row = l / per_row, c = l % per_row * 64 + (lane ^ (row & 15));
        if (c >= valid) *(i32x4*)(smem + row * pitch + l % per_row * 1024 + lane * 16) = i32x4{0, 0, 0, 0};
      }
    wait_lds();
    phase_barrier();
  }
  const char* xrow = smem + min(r, a.n - 1) * pitch;
  const int swz = min(r, a.n - 1) & 15;
  f32x4* sums = (f32x4*)(smem + a.n * pitch);
  for (int set = first; set * CG < row_tiles; set += wgs) {
    const int tile = set * CG + cg;
    f32x4 acc[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[j] = zeros();
    auto multiply = [&](Tiles& b, int t) {
#pragma unroll
      for (int u = 0; u < D; ++u) {
        if (t + u >= t1) break;
#pragma unroll
        for (int j = 0; j < NB; ++j) asm volatile("" : "+v"(b.c[u][j]), "+v"(b.e[u][j]));      // waited for here
        const char* p = xrow + (t + u - s0) * 256;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const bf16x8 f = *(const bf16x8*)(p + (((4 * g + q) ^ swz) << 4));
#pragma unroll
          for (int j = 0; j < NB; ++j)
            acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(weights_of((uint32_t)b.c[u][j][q], scale_of(b.e[u][j])), f,
                                                             acc[j], 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);       // not all tiles' reads of x at once: more registers than there are
      }
    };
    if (t0 < t1) {
      for (int t = t0;;) {
        if (t + D >= t1) {
          multiply(b0, t);
          break;
        }
        load(b1, t + D);
        multiply(b0, t);
        t += D;
        if (t + D >= t1) {
          multiply(b1, t);
          break;
        }
        load(b0, t + D);
        multiply(b1, t);
        t += D;
      }
      if ((set + wgs) * CG < row_tiles) {        // the next set's first weights, behind this one's sums
        weights_at((set + wgs) * CG + cg);
        load(b0, t0);
      }
    }
    if (KG > 1) {
#pragma unroll
      for (int j = 0; j < NB; ++j) sums[(wave * NB + j) * 64 + lane] = acc[j];
      wait_lds();
      phase_barrier();
      if (kg == 0) {
        for (int k = 1; k < KG; ++k)
#pragma unroll
          for (int j = 0; j < NB; ++j) acc[j] += sums[((wave + k) * NB + j) * 64 + lane];
      }
      wait_lds();
      phase_barrier();
      if (kg > 0) continue;
    }
    int row = r;
    if constexpr (PAIR) asm volatile("" : "+v"(row));      // else places of outputs are kept over the loads, in scratch
    if (tile < row_tiles && row < a.n) finish<PAIR>(a, split, row, tile * 16 + 4 * g, acc);
  }
}

// Many rows: bound by the matrix cores.  A work-group of WM x WN waves (times KG that share
// out the column tiles) takes BM = 16 MB WM rows of x and 16 NB WN rows of W (of a gate/up
// pair, half of them each one's); a wave 16 MB x 16 NB.  x moves into LDS by direct loads, a
// column tile (256 bytes of every row) at a time, the 16-byte chunk of a row XOR-ed with the row,
// so that the operand reads (16 rows, one chunk) hit all 64 banks once.  The weights go
// straight to registers.  While a column tile is multiplied, x of the next and the weights of
// the one after it are on their way; one barrier per tile.  (Weights one tile ahead: head
// 128256 x 4096, 24 rows, 58.5 us instead of 55.0; 6144 x 4096, 128 rows, 14.1 instead of 13.5; gate/up
// 14336 x 4096, 64 rows, 20.1 instead of 20.4.)  Gate/up 14336 x 4096, 1024 rows: 185 us, 1.30 PFLOP/s
// (a large bf16 product reaches 1.41), matrix cores 67 % busy, vector instructions 45 %; the
// head of 24 rows 5.3 TB/s.
template <int MB, int NB, int WM, int WN, int KG, bool PAIR>
__global__ __launch_bounds__(64 * WM * WN * KG, WM * WN * KG / 4) void w4_tile_kernel(W4Args a) {
  constexpr int BM = 16 * MB * WM, BT = NB * WN / (PAIR ? 2 : 1), STAGE = BM * 256, LOADS = BM / 4 / (WM * WN);
  static_assert(LOADS * 4 * WM * WN == BM && (!PAIR || NB % 2 == 0), "whole loads, whole pairs");
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kg = wave / (WM * WN), wm = wave % (WM * WN) / WN, wn = wave % WN;
  const int row_tiles = (a.rows + 15) / 16, T = w4_col_tiles(a.cols);
  const int ntm = (a.n + BM - 1) / BM, ntn = (row_tiles + BT - 1) / BT, tiles = ntm * ntn;
  const int bid = xcd_contiguous(blockIdx.x, gridDim.x);
  const int split = bid / tiles;
  int tm, tn;
  tile_at(bid % tiles, ntm, ntn, &tm, &tn);
  const int t0 = T * split / a.plan.splits, t1 = T * (split + 1) / a.plan.splits;
  const int r = lane & 15, g = lane >> 4;
  RowTile w[NB];
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    constexpr int HALF = PAIR ? NB / 2 : NB;
    w[j] = RowTile(j < HALF ? a.w0 : a.w1, min(tn * BT + wn * HALF + j % HALF, row_tiles - 1), T);
  }
  // Wave-load l: 4 rows, lane at row lane / 16, chunk lane % 16 of its stage; it fetches the
  // chunk that belongs there, from a scalar base (the first of the four rows) and an offset
  // of the lane's.  Rows past the last repeat it (never stored); chunks past the last column
  // repeat the row's first ones and are cleared in LDS.
  const int last = (a.cols - (T - 1) * kW4Cols) / 8;             // chunks of the last column tile
  const int lw = wave % (WM * WN);
  const char* x[LOADS];
  uint32_t off[LOADS];
#pragma unroll
  for (int l = 0; l < LOADS; ++l) {
    const int row0 = tm * BM + (lw * LOADS + l) * 4, base = min(row0, a.n - 1);
    x[l] = (const char*)(a.x + base * a.x_stride);
    off[l] = (uint32_t)((min(row0 + g, a.n - 1) - base) * a.x_stride * 2 + 16 * (r ^ ((row0 + g) & 15)));
  }
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_char*)smem + kg * 2 * STAGE + lw * LOADS * 1024;
  char* stage0 = smem + kg * 2 * STAGE;
  auto chunk_of = [&](int l) { return r ^ (((lw * LOADS + l) * 4 + g) & 15); };
  auto load_x = [&](int t, int buf) {
    if (last < 16 && t == T - 1) {
#pragma unroll
      for (int l = 0; l < LOADS; ++l) {
        const int c = chunk_of(l);
        dma16(x[l] + (int64_t)t * 256, off[l] - (c < last ? 0 : 16 * (c - c % last)), lds0 + buf * STAGE + l * 1024);
      }
    } else {
#pragma unroll
      for (int l = 0; l < LOADS; ++l) dma16(x[l] + (int64_t)t * 256, off[l], lds0 + buf * STAGE + l * 1024);
    }
  };
  auto clear_x = [&](int buf) {          // of the last column tile
#pragma unroll
    for (int l = 0; l < LOADS; ++l)
      if (chunk_of(l) >= last)
        *(i32x4*)(stage0 + buf * STAGE + (lw * LOADS + l) * 1024 + lane * 16) = i32x4{0, 0, 0, 0};
  };
  struct Weights {
    i32x4 c[NB];
    uint32_t e[NB];
  };
  auto load_w = [&](Weights& b, int t) {
#pragma unroll
    for (int j = 0; j < NB; ++j) w[j].load(T, t, lane, &b.c[j], &b.e[j]);
  };
  f32x4 acc[MB][NB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[i][j] = zeros();
  const char* arow = stage0 + (wm * 16 * MB + r) * 256;
  auto multiply = [&](const Weights& b, int buf) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      bf16x8 f[MB], v[NB];
#pragma unroll
      for (int i = 0; i < MB; ++i) f[i] = *(const bf16x8*)(arow + buf * STAGE + i * 16 * 256 + (((4 * g + q) ^ r) << 4));
#pragma unroll
      for (int j = 0; j < NB; ++j) v[j] = weights_of((uint32_t)b.c[j][q], scale_of(b.e[j]));
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[j], f[i], acc[i][j], 0, 0, 0);
    }
  };
  // Every group runs the same number of steps, one at least; past its last tile it multiplies nothing.
  const int steps = (t1 - t0 + KG - 1) / KG;
  // x a step ahead, the weights two.  Loads past the last step repeat the last tile, so that
  // waits can count them.
  Weights w0, w1, w2;
  auto step = [&](int i, Weights& now, Weights& after_next) {
    const int t = t0 + i * KG + kg, buf = i & 1;
    wait_vm<2 * NB>();                           // all but the next step's weights
    // Here and not where they are first used, behind the next loads; nor does anything of
    // theirs (the shift of the scales) move up to those.
#pragma unroll
    for (int j = 0; j < NB; ++j) asm volatile("" : "+v"(now.c[j]), "+v"(now.e[j]));
    if (last < 16 && t == T - 1) {
      clear_x(buf);
      wait_lds();
    }
    phase_barrier();
    load_x(min(t + KG, t1 - 1), buf ^ 1);
    load_w(after_next, min(t + 2 * KG, t1 - 1));
    if (t < t1) multiply(now, buf);
  };
  load_x(min(t0 + kg, t1 - 1), 0);
  load_w(w0, min(t0 + kg, t1 - 1));
  __builtin_amdgcn_sched_barrier(0);
  load_w(w1, min(t0 + KG + kg, t1 - 1));
  for (int i = 0;; i += 3) {       // left by breaks: where paths met, registers would be copied, and waited for
    step(i, w0, w2);
    if (i + 1 >= steps) break;
    step(i + 1, w1, w0);
    if (i + 2 >= steps) break;
    step(i + 2, w2, w1);
    if (i + 3 >= steps) break;
  }
  wait_vm<0>();
  if constexpr (KG > 1) {                // the groups' sums meet in LDS, in their order
    constexpr int BLOCKS = MB * NB;
    static_assert((KG - 1) * WM * WN * BLOCKS * 1024 <= KG * 2 * STAGE, "sums fit");
    __syncthreads();
    f32x4* sums = (f32x4*)smem;
    if (kg > 0)
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) sums[(((kg - 1) * WM * WN + lw) * BLOCKS + i * NB + j) * 64 + lane] = acc[i][j];
    __syncthreads();
    if (kg > 0) return;
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int k = 1; k < KG; ++k) acc[i][j] += sums[(((k - 1) * WM * WN + lw) * BLOCKS + i * NB + j) * 64 + lane];
  }
  constexpr int MATS = PAIR ? 2 : 1, HALF = NB / MATS;
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < HALF; ++j) {
      const int row = tm * BM + (wm * MB + i) * 16 + r, tile = tn * BT + wn * HALF + j;
      if (tile >= row_tiles || row >= a.n) continue;
      f32x4 v[MATS];
#pragma unroll
      for (int k = 0; k < MATS; ++k) v[k] = acc[i][j + k * HALF];
      finish<PAIR>(a, split, row, tile * 16 + 4 * g, v);
    }
}

// Sum the splits, in their order, and store.  A launch, 3 us at 16 x 4096, beside which the bytes
// (out of L2 and the last-level cache) count from about 10 MB on.
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

constexpr int kLds = 160 * 1024;         // of a CU

// Let a kernel have that much LDS, once per device (a call takes a microsecond).
hipError_t allow_lds(const void* kernel, int bytes, std::atomic<uint64_t>* ready) {
  int dev = -1;
  if (const hipError_t e = hipGetDevice(&dev)) return e;
  const uint64_t bit = dev < 64 ? 1ull << dev : 0;
  if (ready->load(std::memory_order_relaxed) & bit) return hipSuccess;
  const hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == hipSuccess) ready->fetch_or(bit, std::memory_order_relaxed);
  return e;
}

// LDS that the stream kernel needs.
int stream_lds(int cols, int n, int nb, const W4Plan& p) {
  const int T = w4_col_tiles(cols), longest = (T + p.splits - 1) / p.splits;
  return n * ((longest + 3) / 4 * 1024) + (p.wide > 1 ? kStreamWaves * nb * 1024 : 0);
}

template <bool PAIR>
hipError_t launch_stream(const W4Args& a, hipStream_t s) {
  const auto kernel = w4_stream_kernel<PAIR>;
  const int smem = stream_lds(a.cols, a.n, PAIR ? 2 : 1, a.plan);
  static std::atomic<uint64_t> ready{0};
  if (const hipError_t e = allow_lds((const void*)kernel, kLds, &ready)) return e;
  const int per = kStreamWaves / a.plan.wide, sets = ((a.rows + 15) / 16 + per - 1) / per;
  kernel<<<(unsigned)(std::min(sets, std::max(1, 256 / a.plan.splits)) * a.plan.splits), 64 * kStreamWaves, smem, s>>>(a);
  return hipGetLastError();
}

template <int MB, int NB, int WM, int WN, int KG, bool PAIR>
hipError_t launch_tile(const W4Args& a, hipStream_t s) {
  constexpr int BM = 16 * MB * WM, BT = NB * WN / (PAIR ? 2 : 1), SMEM = KG * 2 * BM * 256;
  const auto kernel = w4_tile_kernel<MB, NB, WM, WN, KG, PAIR>;
  static std::atomic<uint64_t> ready{0};
  if (const hipError_t e = allow_lds((const void*)kernel, SMEM, &ready)) return e;
  const int64_t tiles = (int64_t)((a.n + BM - 1) / BM) * (((a.rows + 15) / 16 + BT - 1) / BT);
  if (tiles * a.plan.splits > kMaxGrid) return hipErrorInvalidValue;
  kernel<<<(unsigned)(tiles * a.plan.splits), 64 * WM * WN * KG, SMEM, s>>>(a);
  return hipGetLastError();
}

template <bool PAIR>
hipError_t launch_shape(const W4Args& a, hipStream_t s) {
  switch (a.plan.shape) {
    case W4_STREAM: return launch_stream<PAIR>(a, s);
    case W4_TILE32: return launch_tile<2, 2, 1, 4, 2, PAIR>(a, s);
    case W4_TILE32W: return launch_tile<2, 4, 1, 8, 1, PAIR>(a, s);
    case W4_TILE64: return launch_tile<4, 2, 1, 4, 2, PAIR>(a, s);
    case W4_TILE64W: return launch_tile<4, 2, 1, 8, 1, PAIR>(a, s);
    case W4_TILE128: return launch_tile<4, 4, 2, 4, 1, PAIR>(a, s);
    case W4_TILE256: return launch_tile<8, 4, 2, 4, 1, PAIR>(a, s);
  }
  return hipErrorInvalidValue;
}

template <bool PAIR>
hipError_t launch_pair(const W4Args& a, hipStream_t s) {
  const hipError_t e = launch_shape<PAIR>(a, s);
  if (e != hipSuccess || a.plan.splits == 1 || a.kind == kW4Partial) return e;
  const int64_t threads = (int64_t)a.n * ((a.rows + 15) / 16 * 4);
  if ((threads + 255) / 256 > kMaxGrid) return hipErrorInvalidValue;
  w4_reduce_kernel<PAIR><<<(unsigned)((threads + 255) / 256), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

// Up to 16 rows: the stream kernel, x in LDS over as few column splits as its place there
// allows (unless these are many), and as many waves to a row tile as still leave one round of
// work-groups.  (us, the weights out of HBM: 1 row 4096 x 14336, 16 / 8 / 4 / 2 waves 9.3 / 9.9 / 12.6 / 19.5; gate/up of 4 rows,
// 14336 x 4096, 17.9 / 14.8 / 14.0 / 15.3; head of 1 row, 128256 x 4096, 73 / 54 / 52 / 50 and
// alone 49; 16 rows 4096 x 14336 in 4 splits 16.2 / 14.3 / 13.8 / 14.4, in 8 no better.)
//
// More rows: the cost model below, in us.  Work-groups run `slots` to a CU; k of them on one
// take k * each per step of a column tile (the kernel's KG at a time; the 64 x 256 tiles of one
// matrix, alone on their CU, `alone`), `fixed` more per round;
// weights stream at `tbs` TB/s; the larger of both, an eighth of the smaller (they overlap
// imperfectly), 5.9 for a launch in a graph and, where columns are split, 2.3 and the partials
// written and read at 5.8 TB/s for the reduction.  Fitted to 2550 launches (8 matrices of the 1B
// and 8B shapes, 17 to 2048 rows, all tiles, 1 to 16 splits, weights from HBM): 8 % rms, and the
// choice is on average 0.9 % slower than the best of them, at worst 8 % (128256 x 4096, 17 rows); of 1775
// others (the 8B shape's, 19 numbers of rows) 1.2 % and 8 %.  Without `alone` these are 1.0 and
// 1.9 %, at worst 12 (4096 x 14336: 900 rows 111 us instead of 99, 1024 rows 109 instead of 103).  A pair's
// tiles measure as much, but so do the others that they compete with there.
W4Plan plan_w4(int rows, int cols, int n, bool gate_up) {
  const int tiles = (rows + 15) / 16, mats = gate_up ? 2 : 1, T = w4_col_tiles(cols);
  auto partials = [&](int splits) { return 4.0 * splits * mats * n * tiles * 16; };      // bytes
  if (n <= 16) {
    W4Plan p{W4_STREAM, kStreamWaves, 1};
    while (p.splits <= 16 && stream_lds(cols, n, mats, p) > kLds) ++p.splits;
    while (p.wide > 1 && (int64_t)tiles * p.wide * p.splits > 256 * kStreamWaves) p.wide /= 2;
    if (p.splits <= 16 && (p.splits == 1 || partials(p.splits) <= kW4PartialCap)) return p;
  }
  struct Tile {
    W4Shape shape;
    int bm, bt, kg, slots;
    double alone, each, fixed, tbs;
  };
  static constexpr Tile shapes[] = {{W4_TILE32, 32, 8, 2, 3, 0, 0.538, 0.0, 4.56},
                                    {W4_TILE32W, 32, 32, 1, 1, 0, 0.880, 0.32, 5.18},
                                    {W4_TILE64, 64, 8, 2, 2, 0, 0.854, 0.33, 4.03},
                                    {W4_TILE64W, 64, 16, 1, 2, 0.88, 0.771, 0.55, 5.40},
                                    {W4_TILE128, 128, 16, 1, 1, 0, 1.614, 1.17, 2.62},
                                    {W4_TILE256, 256, 16, 1, 1, 0, 2.675, 2.28, 6.71}};
  W4Plan best{W4_TILE64, 1, 1};
  double best_us = 1e30;
  for (const Tile& s : shapes) {
    if (s.shape == W4_TILE32W && n > s.bm) continue;      // its weights would pass once per 32 rows
    const int64_t count = ((int64_t)n + s.bm - 1) / s.bm * (((int64_t)tiles * mats + s.bt - 1) / s.bt);
    for (int splits = 1; splits <= (n <= kMostSplitRows ? 16 : 1); ++splits) {
      const double part = partials(splits);
      if (splits > 1 && (T / splits < 4 || part > kW4PartialCap)) break;
      const int64_t wgs = count * splits;
      const double steps = (T + splits * s.kg - 1) / (splits * s.kg), at_once = 256.0 * s.slots;
      auto step = [&](int k) { return k == 1 && !gate_up ? std::max(s.alone, s.each) : k * s.each; };
      double work;
      if (wgs > 3 * at_once) {
        work = wgs / at_once * (steps * step(s.slots) + s.fixed);
      } else {
        const int64_t full = wgs / (256 * s.slots), rest = wgs % (256 * s.slots);
        work = steps * (full * step(s.slots) + step((int)((rest + 255) / 256))) + (full + (rest > 0)) * s.fixed;
      }
      const double stream = mats * (double)rows * cols * 17 / 32 / s.tbs / 1e6;
      double us = std::max(work, stream) + 0.13 * std::min(work, stream);
      if (splits > 1) us += 2.3 + 2 * part / 5.8e6;
      if (us < best_us) {
        best_us = us;
        best = W4Plan{s.shape, 1, splits};
      }
    }
  }
  return best;
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
