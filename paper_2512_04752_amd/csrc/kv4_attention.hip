// Tree attention over the 4-bit paged KV cache.
//
// Query row r of (sample b, kv head g) is node r / G with query head g*G + r % G
// (G query heads share a KV head).  It sees every committed key and, of the
// step's own keys, its ancestors (trees) or the ones up to itself (runs).
//
// A wave takes one or two tiles of 16 rows through 32 keys at a time, with the
// products transposed so that a row's scores and output stay in four lanes
// (l, l + 16, l + 32, l + 48, "groups" g = 0 .. 3):
//
//   S^T (keys x 16 rows)   = K . Q^T     v_mfma_scale_f32_16x16x128_f8f6f4
//   O^T (dims x 16 rows)  += V^T . P^T   v_mfma_f32_16x16x32_bf16
//
// Four bits are little enough to need no staging: the cache is stored in the
// order of the operands, a lane loads its own 16 bytes of codes, and there is no
// LDS traffic and no barrier until a wave's last key; loads run a block ahead in
// registers.
//
// K's codes and powers of two are the scaled MFMA's own format (E2M1 with a power
// of two per 32 numbers), so they are multiplied as they lie: no instruction
// decodes them.  Its other operand has 8 bits at most, so a query number is held
// as the sum of two e4m3 numbers of four significant bits each, which carries
// bf16's eight; both share a power of two per row that puts the row's largest
// magnitude in [128, 256).  Numbers more than 2^9 below the largest run into e4m3's
// smallest step and are off by up to 2^-17 of the largest, which is nothing beside the
// largest's own rounding but may be much of such a number.  Rows where that matters
// ("wide": what is lost comes, summed, to more than 2^-12 of the numbers that are more
// than 16 times below the largest, a sixteenth of what rounding them to bf16 may cost)
// get the remainders as two more e4m3 numbers, and two more products, which leaves
// 2^-34 of the largest.  Weighing the loss against the row's mean instead misses two
// equal outliers of 64 numbers, or four of 128.  Random normal rows are wide once in
// 2800 (64 numbers) or less (128).
//
// V's codes are turned into bf16 (one conversion per byte), without their power of
// two: it is the same for all dims of a key and scales the key's probability
// instead.  So K and V enter the products exactly.  Probabilities are rounded to
// bf16, as over the bf16 cache: an eight-bit significand, 2^-8 relative.
//
// Tile T of S^T takes keys 16 T + 0 .. 15 of the block, so that a load of K covers
// whole cache lines (64-byte pieces of twice as many lines stalled on the pieces
// still under way); group g then holds keys 16 T + 4 g + i.  P^T wants an octet of
// keys per group, as V's words hold them: two lane swaps per register pair.
//
// A work-group has four waves: one, two or four share a row tile (pair)'s keys, block
// by block, and merge through LDS at the end.
//
// What bounds it: up to 16 rows per KV head the cache's bytes (256 samples, 227K keys of 8
// heads, 248 MB: 45 us, 5.5 TB/s; a plain read of as many reaches 5.8); above that the vector
// instructions (4 x 64 nodes at 16K - 32K keys: 68 % of the cycles) and the matrix products (43 %),
// which two waves per SIMD do not overlap; below some 3000 keys per work-group its own latency,
// about 1000 cycles per block of a wave that has its SIMD alone, and 4 us of a merge's launch.
// Weighing what two parts lose takes four vector instructions per query number, 0.5 - 1 % of the
// time.  A first form, 32 rows by v_mfma_f32_32x32x16_bf16 with K decoded to bf16 as well, took
// (this form in brackets, us): one sample of 580 keys 12.5 (6.9); 4 x 16 nodes, 15K keys 21.6
// (16.8); 1B heads, 32 x 15 nodes 25.4 (19.6); 128 x 8 nodes, 176K keys 62.8 (55.1); 256 x 1 67
// (45.4); 4 x 64 nodes, 101K keys 151 (118); prompt pieces of 500 - 1170 rows 181 (156).  Tried and
// slower, each beside the form of its time: the next block's scores multiplied ahead of a block's
// softmax (tail 127, prompt 163 against 120, 152); three blocks of loads under way (no change);
// eight waves per work-group where each has a CU to itself (4 x 16 nodes 17.5 against 17.2); the
// merge by the last work-group of a row group (its device-wide stores: 4 x 16 nodes 37.8, tail 170).
#include <math.h>

#include <atomic>
#include <type_traits>

#include "kv4.h"

namespace spec {

namespace {

constexpr int KBLK = 32;
constexpr int kWaves = 4;

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(8))) int i32x8;

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// The running output is relative to a reference maximum that moves only when a lane's
// probabilities of a block, which are summed anyway, come to more than this: no maximum
// is taken otherwise.  The first reference is so low that any key's probability is
// infinite under it.
constexpr float kMostSum = 256.f;
constexpr float kNoKeys = -3e38f;

// IEEE maximum: one instruction, and a NaN (the score of a key that was not finite)
// stays one; fmaxf would first have to quiet the MFMA outputs.
__device__ __forceinline__ float maximum(float x, float y) { return __builtin_elementwise_maximum(x, y); }

// A value and its copy in the next group (lane ^ 16), or in lane ^ 32.
__device__ __forceinline__ uint2 with16(uint32_t x) {
  const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  return make_uint2(r[0], r[1]);
}
__device__ __forceinline__ uint2 with32(uint32_t x) {
  const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return make_uint2(r[0], r[1]);
}

// Over the four lanes of a row.
__device__ __forceinline__ float max_groups(float x) {
  uint2 r = with16(__float_as_uint(x));
  r = with32(__float_as_uint(maximum(__uint_as_float(r.x), __uint_as_float(r.y))));
  return maximum(__uint_as_float(r.x), __uint_as_float(r.y));
}
__device__ __forceinline__ float sum_groups(float x) {
  uint2 r = with16(__float_as_uint(x));
  r = with32(__float_as_uint(__uint_as_float(r.x) + __uint_as_float(r.y)));
  return __uint_as_float(r.x) + __uint_as_float(r.y);
}

// Eight codes (a word) as bf16.
__device__ __forceinline__ bf16x8 decode(uint32_t w) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 2);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.f, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Two floats as a pair of bf16, in one conversion.
__device__ __forceinline__ uint32_t pack_bf16(float x, float y) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, y}, bf16x2));
}

// A row's query as the scaled MFMA's operand.  Lane group g holds k = 16 g .. 16 g + 15
// in registers 0 .. 3 and k = 64 + 16 g .. in 4 .. 7.  HD 128: k is the dim, q[0] the
// high parts and q[1] the low ones.  HD 64: one operand, k = dim the high parts and
// k = 64 + dim the low ones (K's codes are then given twice).
template <int HD>
struct Query {
  i32x8 q[HD / 64];
  i32x8 rest[HD / 64];     // what q leaves, likewise, times 2^17; zero in a row that is not wide
  int scale, rest_scale;   // exponents + 127; 255 for a row with an infinity or NaN

  static constexpr int N = HD / 4;            // numbers of a lane
  struct Raw {
    i32x4 x[N / 8];
  };
  static __device__ __forceinline__ Raw load(const bf16* row, int g) {
    Raw raw;
#pragma unroll
    for (int c = 0; c < N / 8; ++c) raw.x[c] = *(const i32x4*)(row + 16 * g + (c & 1) * 8 + (c >> 1) * 64);
    return raw;
  }

  // Four numbers f[0 .. 3] / s as two words of e4m3, high parts and low; f keeps the remainder.
  static __device__ __forceinline__ void split(float (&f)[4], float s, int& hi, int& lo) {
    auto parts = [&]() __attribute__((always_inline)) {
      typedef __attribute__((ext_vector_type(2))) short i16x2;
      i16x2 w = {0, 0};
      w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, f[0], f[1], s, false);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, f[2], f[3], s, true);
      const int v = __builtin_bit_cast(int, w);
      const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(v, s, false);
      const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(v, s, true);
      f[0] -= a[0];
      f[1] -= a[1];
      f[2] -= b[0];
      f[3] -= b[1];
      return v;
    };
    hi = parts();
    lo = parts();
  }

  // Returns whether some row of the wave is wide.
  __device__ __forceinline__ bool convert(const Raw& raw, bool live) {
    uint32_t x[N / 2];
#pragma unroll
    for (int c = 0; c < N / 2; ++c) x[c] = live ? (uint32_t)raw.x[c >> 2][c & 3] : 0u;
    float most = 0.f;
#pragma unroll
    for (int c = 0; c < N / 2; ++c) {
      const float a = fabsf(__uint_as_float(x[c] << 16)), b = fabsf(__uint_as_float(x[c] & 0xffff0000u));
      most = maximum(maximum(most, a), b);
    }
    most = max_groups(most);
    const int e = (int)(__float_as_uint(most) >> 23 & 255);   // a NaN or infinity has 255
    scale = e == 255 ? 255 : max(e - 7, 1);
    rest_scale = e == 255 ? 255 : max(scale - 17, 1);
    const float f = __uint_as_float((uint32_t)min(scale, 247) << 23);
    const float fr = __uint_as_float((uint32_t)min(rest_scale, 247) << 23);
    auto four = [&](int c, int i, float (&v)[4]) __attribute__((always_inline)) {
      const uint32_t w0 = x[8 * c + 2 * i], w1 = x[8 * c + 2 * i + 1];
      v[0] = __uint_as_float(w0 << 16);
      v[1] = __uint_as_float(w0 & 0xffff0000u);
      v[2] = __uint_as_float(w1 << 16);
      v[3] = __uint_as_float(w1 & 0xffff0000u);
    };
    const float small = most * 0.0625f;
    float lost = 0.f, below = 0.f;             // sums: what two parts lose; the numbers below `small`
    i32x4 hi[HD / 64], lo[HD / 64];
    auto join = [&](i32x8 (&to)[HD / 64]) __attribute__((always_inline)) {
      if constexpr (HD == 128) {
        to[0] = __builtin_shufflevector(hi[0], hi[1], 0, 1, 2, 3, 4, 5, 6, 7);
        to[1] = __builtin_shufflevector(lo[0], lo[1], 0, 1, 2, 3, 4, 5, 6, 7);
      } else {
        to[0] = __builtin_shufflevector(hi[0], lo[0], 0, 1, 2, 3, 4, 5, 6, 7);
      }
    };
#pragma unroll
    for (int c = 0; c < HD / 64; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float v[4];
        int h, l;
        four(c, i, v);
#pragma unroll
        for (int j = 0; j < 4; ++j) below += fabsf(v[j]) < small ? fabsf(v[j]) : 0.f;
        split(v, f, h, l);
        lost += (fabsf(v[0]) + fabsf(v[1])) + (fabsf(v[2]) + fabsf(v[3]));
        hi[c][i] = h;
        lo[c][i] = l;
      }
    join(q);
    const bool wide = e != 255 && sum_groups(fmaf(below, -0x1p-12f, lost)) > 0.f;
#pragma unroll
    for (int c = 0; c < HD / 64; ++c) rest[c] = i32x8{0, 0, 0, 0, 0, 0, 0, 0};
    const bool any = __ballot(wide) != 0;
    if (any) {
#pragma unroll
      for (int c = 0; c < HD / 64; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float v[4];
          int h, l;
          four(c, i, v);
          split(v, f, h, l);
          split(v, fr, h, l);
          hi[c][i] = wide ? h : 0;
          lo[c][i] = wide ? l : 0;
        }
      join(rest);
    }
    return any;
  }

  // Scores of 16 keys (codes k, scale byte ks) in the lane's row; what the remainders add.
  __device__ __forceinline__ f32x4 scores(i32x4 k, int ks) const { return product(k, ks, q, scale, f32x4{0.f, 0.f, 0.f, 0.f}); }
  __device__ __forceinline__ f32x4 add_rest(i32x4 k, int ks, f32x4 s) const { return product(k, ks, rest, rest_scale, s); }

 private:
  static __device__ __forceinline__ f32x4 product(i32x4 k, int ks, const i32x8 (&x)[HD / 64], int xs, f32x4 s) {
    const i32x8 a = __builtin_shufflevector(k, k, 0, 1, 2, 3, -1, -1, -1, -1);
#pragma unroll
    for (int i = 0; i < HD / 64; ++i)
      s = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, x[i], s, 4, 0, 0, ks, 0, xs);   // E2M1 . E4M3
    return s;
  }
};

// One lane's share of a 32-key block.
template <int HD>
struct Block {
  typedef __attribute__((ext_vector_type(HD / 32))) int words;
  i32x4 k[2];              // 32 dims of key 16 T + r, r = lane % 16
  int ks[2];               // and their scale
  words v[2];              // octet g: dims 32 i + r + 16 j in v[j][i]
  i32x2 vs[2];             // value scales of keys 16 T + 4 g + 0 .. 3
};

// Codes that one wave alone reads pass the caches by: 256 samples with one row each, 45.7
// us against 50.2 (5.4 TB/s).  Where two or four waves of a work-group read the same codes
// that costs: 128 x 8 nodes out of the last-level cache 50.8 against 37.1, 1B shape 32 x 15
// nodes 23.4 against 20.4.
template <bool ONCE, class T>
__device__ __forceinline__ T load_codes(const T* p) {
  return ONCE ? __builtin_nontemporal_load(p) : *p;
}

template <int HD, int NT, bool ONCE>
__global__ __launch_bounds__(256, NT == 1 ? 3 : 2) void kv4_attention_kernel(Kv4AttnArgs a) {
  constexpr int NB = HD / 16;                 // 16-dim output tiles
  extern __shared__ __attribute__((aligned(16))) float smem[];

  const int per_xcd = gridDim.x >> 3;
  const int item = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
  if (item >= a.n_items) return;
  const Kv4Item it = a.items[item];
  if (it.waves == 0) return;                  // padding of a shorter per-XCD list
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int r = lane & 15;
  const int g = lane >> 4;
  const int KS = it.waves, part = w & (KS - 1);                     // waves per row tile (pair)
  const int pair = KS == 4 ? 0 : KS == 2 ? w >> 1 : w;
  const int G = a.group;
  auto node_of = [&](int row) { return G == 1 ? row : (int)__umulhi((uint32_t)row, a.group_inv); };
  const int row0 = it.row0 + 16 * NT * pair;

  const bool runs = a.anc == nullptr;
  // The node and query head of the lane's row in tile n.
  auto node_at = [&](int n) { return node_of(row0 + 16 * n + r); };
  auto head_at = [&](int n) { return it.kvh * G + row0 + 16 * n + r - node_at(n) * G; };
  typename Query<HD>::Raw raw[NT];
  uint64_t anc0[NT];                           // of a tree the ancestors among the first 64 nodes
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const bool ok = node_at(n) < it.ntok;
    anc0[n] = runs ? 0 : a.anc[(size_t)(it.tok0 + min(node_at(n), it.ntok - 1)) * kAncWords];
    raw[n] = Query<HD>::load(a.q + (size_t)(it.tok0 + (ok ? node_at(n) : 0)) * a.q_stride + (ok ? head_at(n) : 0) * HD, g);
  }
  Query<HD> qf[NT];
  bool wide = false;                           // wave-uniform
  auto convert = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < NT; ++n) wide |= qf[n].convert(raw[n], node_at(n) < it.ntok);
  };
  if constexpr (NT > 1) convert();             // two tiles' raw numbers would stay in registers too long

  // The wave's keys end with its last row's, and blocks past `mask_from` are masked.
  int key1 = it.key1, mask_from = it.seq_len;
  if (runs) {
    const int last = min(node_of(row0 + 16 * NT - 1), it.ntok - 1);
    key1 = min(key1, it.seq_len + last + 1);
    mask_from = it.seq_len + min(node_of(row0), it.ntok - 1) + 1;
  }
  mask_from = min(mask_from, key1);
  const int nblk = key1 > it.key0 ? (key1 - it.key0 + KBLK - 1) / KBLK : 0;
  const int mine = nblk > part ? (nblk - part + KS - 1) / KS : 0;

  const char* in_page = a.v.pool + ((int64_t)a.v.layer * a.v.n_kv_heads + it.kvh) * kv4_head_bytes(HD);
  const uint32_t* table = a.v.table + it.pages;
  const int chunk = HD == 128 ? g : g & 1;
  const uint32_t k_off = chunk * 512 + r * 16, ks_off = kv4_kscale_at(HD) + r * (HD / 32) + chunk;
  const uint32_t v_off = kv4_value_at(HD) + g * kv4_octet_bytes(HD) + r * (HD / 8);
  const uint32_t vs_off = kv4_vscale_at(HD) + 8 * g;

  auto first_key = [&](int t) { return (uint32_t)(it.key0 + (part + KS * t) * KBLK); };
  // The blocks go from the last one down, through two sets of registers.  A block's K is
  // loaded when the one two above it has been multiplied, its V likewise: a whole
  // block's work passes before it is needed.  Its page is read a block before that.
  uint32_t page = mine > 0 ? table[first_key(mine - 1) / kKv4Page] : 0;
  const char *codes, *vscales;                 // of the block whose V comes next
  auto load_k = [&](Block<HD>& b, int t) __attribute__((always_inline)) {
    const uint32_t half = first_key(t) / KBLK % 2;
    const char* base = in_page + kv4_page_offset(page);
    page = table[first_key(max(t - 1, 0)) / kKv4Page];
    codes = base + half * kv4_block_bytes(HD);
    vscales = base + half * 64;
    const char* scales = base + half * HD;     // 32 keys' scales: HD bytes of K's, 64 of V's
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      b.k[j] = load_codes<ONCE>((const i32x4*)(codes + k_off + 256 * j));
      b.ks[j] = *(const uint8_t*)(scales + ks_off + 16 * j * (HD / 32));
    }
  };
  auto load_vs = [&](Block<HD>& b) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 2; ++j) b.vs[j] = *(const i32x2*)(vscales + vs_off + 32 * j);
  };
  auto load_v = [&](Block<HD>& b) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 2; ++j) b.v[j] = load_codes<ONCE>((const typename Block<HD>::words*)(codes + v_off + j * 2 * HD));
  };

  const float sl2 = 1.4426950408889634f / sqrtf((float)HD);   // log2(e) / sqrt(d)
  float m_run[NT], l_run[NT];                 // the row's reference maximum; this lane's share of its sum
  f32x4 o[NT][NB];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    m_run[n] = kNoKeys;
    l_run[n] = 0.f;
#pragma unroll
    for (int i = 0; i < NB; ++i) o[n][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // Block `t`, whose loads are in b; then b takes the loads of block t - 2 (of block 0
  // again when there is none: the waits below count on them).
  auto step = [&](Block<HD>& b, int t) __attribute__((always_inline)) {
    const int kb = (int)first_key(t);
    f32x4 x[NT][2];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int n = 0; n < NT; ++n) x[n][j] = qf[n].scores(b.k[j], b.ks[j]);
    if (wide)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int n = 0; n < NT; ++n) x[n][j] = qf[n].add_rest(b.k[j], b.ks[j], x[n][j]);
    float s[NT][8];                            // s[n][e]: key kb + 16 (e / 4) + 4 g + e % 4
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 8; ++e) s[n][e] = x[n][e >> 2][e & 3];
    load_k(b, max(t - 2, 0));
    float vscale[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t pair = (uint32_t)b.vs[e >> 2][(e >> 1) & 1];
      vscale[e] = __uint_as_float(e & 1 ? pair & 0xffff0000u : pair << 16);
    }
    // Keys that a row does not see score -inf and weigh 0.  Blocks that reach past
    // `mask_from` only; there a value scale that is not a number (or was never written) is
    // taken as 0, and the rows that see the key score NaN instead.
    if (kb + KBLK > mask_from) {
      int at_lane = lane;                      // nothing of this is worth a register between blocks
      asm("" : "+v"(at_lane) : "s"(kb));
      const int r = at_lane & 15, g = at_lane >> 4;
      auto below = [](int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1; };   // bits 0 .. n - 1
      uint32_t seen[NT];                       // bit e, of keys e = 4 .. 7 bit 12 + e
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const int node = min(node_of(row0 + 16 * n + r), it.ntok - 1), x0 = kb - it.seq_len;
        uint32_t see;                          // bit k: key kb + k
        if (runs) {
          see = below(node + 1 - x0);
        } else if (x0 < 0) {                   // committed keys, all seen, then the first nodes
          see = x0 <= -32 ? ~0u : (uint32_t)(anc0[n] << -x0) | below(-x0);
        } else {
          const uint64_t* anc = a.anc + (size_t)(it.tok0 + node) * kAncWords;
          const int i = x0 >> 6, shift = x0 & 63;
          const uint64_t lo = i == 0 ? anc0[n] : i < kAncWords ? anc[i] : 0;
          see = (uint32_t)(lo >> shift);
          if (shift > 32 && i + 1 < kAncWords) see |= (uint32_t)(anc[i + 1] << (64 - shift));
        }
        see &= below(key1 - kb);
        seen[n] = see >> (4 * g);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool bad = (__float_as_uint(vscale[e]) & 0x7f800000u) == 0x7f800000u;
#pragma unroll
        for (int n = 0; n < NT; ++n)
          s[n][e] = !(seen[n] >> (e < 4 ? e : 12 + e) & 1u) ? -INFINITY : bad ? __uint_as_float(0x7fc00000u) : s[n][e];
        vscale[e] = bad ? 0.f : vscale[e];
      }
    }
    float p[NT][8], psum[NT];
    auto weigh = [&](int n) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < 8; ++e) p[n][e] = fast_exp2(fmaf(s[n][e], sl2, -m_run[n]));
      psum[n] = ((p[n][0] + p[n][1]) + (p[n][2] + p[n][3])) + ((p[n][4] + p[n][5]) + (p[n][6] + p[n][7]));
    };
    bool grows = false;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      weigh(n);
      grows |= psum[n] > kMostSum;
    }
    if (__ballot(grows)) {
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float most = maximum(maximum(maximum(s[n][0], s[n][1]), s[n][2]), maximum(maximum(s[n][3], s[n][4]), s[n][5]));
        most = maximum(maximum(most, s[n][6]), s[n][7]);
        const float m_new = maximum(m_run[n], max_groups(most) * sl2);
        const float alpha = fast_exp2(m_run[n] - m_new);
        l_run[n] *= alpha;
#pragma unroll
        for (int i = 0; i < NB; ++i) o[n][i] *= alpha;
        m_run[n] = m_new;
        weigh(n);
      }
    }
    i32x4 pb[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      l_run[n] += psum[n];
#pragma unroll
      for (int e = 0; e < 8; e += 2)
        pb[n][e >> 1] = (int)pack_bf16(p[n][e] * vscale[e], p[n][e + 1] * vscale[e + 1]);
      // [tile 0: groups' keys 0-3, 4-7, 8-11, 12-15; tile 1: 16-19, ..] -> group g: keys 8 g .. 8 g + 7
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const auto x = __builtin_amdgcn_permlane32_swap(pb[n][i], pb[n][2 + i], false, false);
        const auto y = __builtin_amdgcn_permlane16_swap(x[0], x[1], false, false);
        pb[n][i] = (int)y[0];
        pb[n][2 + i] = (int)y[1];
      }
    }
    load_vs(b);
#pragma unroll
    for (int i = 0; i < HD / 32; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const bf16x8 vt = decode((uint32_t)b.v[j][i]);
#pragma unroll
        for (int n = 0; n < NT; ++n)
          o[n][2 * i + j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, __builtin_bit_cast(bf16x8, pb[n]),
                                                                   o[n][2 * i + j], 0, 0, 0);
      }
    load_v(b);
  };

  if (mine > 0) {
    Block<HD> b0, b1;
    int t = mine - 1;
    // In the order in which step() issues them, which is what its waits count on.
    auto fill = [&](Block<HD>& b, int at) __attribute__((always_inline)) {
      load_k(b, at);
      __builtin_amdgcn_sched_barrier(0);
      load_vs(b);
      __builtin_amdgcn_sched_barrier(0);
      load_v(b);
      __builtin_amdgcn_sched_barrier(0);
    };
    fill(b0, t);
    fill(b1, max(t - 1, 0));
    if constexpr (NT == 1) convert();          // while the first keys are on their way
    __builtin_amdgcn_sched_barrier(0);
    for (; t > 0; t -= 2) {
      step(b0, t);
      __builtin_amdgcn_sched_barrier(0);       // the registers of two blocks' steps at once are too many
      step(b1, t - 1);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (t == 0) step(b0, 0);
  }

  asm("" : "+v"(r) : "v"(l_run[0]));            // nor of this
  // o[n][i][j]: dim 16 i + 4 g + j of row row0 + 16 n + r.  Row r of tile n, normalised by
  // its sum l: to the output, or to its key range's partial state.
  const bool split = it.nsplit > 1;
  auto put = [&](int n, int i, f32x4 x) __attribute__((always_inline)) {
    if (split) {
      const size_t row = (size_t)(it.part + (NT * pair + n) * it.nsplit) * 16 + r;
      *(f32x4*)(a.part_o + row * HD + 16 * i + 4 * g) = x;
    } else {
      bf16* dst = a.out + ((size_t)(it.tok0 + node_at(n)) * a.n_heads + head_at(n)) * HD + 16 * i + 4 * g;
      *(i32x2*)dst = i32x2{(int)pack_bf16(x[0], x[1]), (int)pack_bf16(x[2], x[3])};
    }
  };
  auto put_ml = [&](int n, float m, float l) __attribute__((always_inline)) {
    const size_t row = (size_t)(it.part + (NT * pair + n) * it.nsplit) * 16 + r;
    if (split && g == 0) *(float2*)(a.part_ml + row * 2) = make_float2(m, l);
  };
  if (KS == 1) {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const float l = sum_groups(l_run[n]), inv = l == 0.f ? 0.f : 1.f / l;
      if (node_at(n) >= it.ntok) continue;
      put_ml(n, m_run[n], l);
#pragma unroll
      for (int i = 0; i < NB; ++i) put(n, i, o[n][i] * inv);
    }
    return;
  }
  // Waves that share a row tile leave their states in LDS, lane by lane; each then merges
  // its share of the dims.
  constexpr int STATE = (NB * 4 + 2) * 64;     // floats of a wave and tile
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    float* p = smem + (w * NT + n) * STATE;
#pragma unroll
    for (int i = 0; i < NB; ++i) *(f32x4*)(p + i * 256 + lane * 4) = o[n][i];
    *(float2*)(p + NB * 256 + lane * 2) = make_float2(m_run[n], l_run[n]);
  }
  __syncthreads();
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    if (row0 + 16 * n >= it.ntok * G) break;   // wave-uniform: no row in the tile
    const float* p = smem + (w - part) * NT * STATE + n * STATE;
    float2 ml[kWaves];
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int k = 0; k < kWaves; ++k)
      if (k < KS) {
        ml[k] = *(const float2*)(p + k * NT * STATE + NB * 256 + lane * 2);
        m = maximum(m, ml[k].x);
      }
#pragma unroll
    for (int k = 0; k < kWaves; ++k)
      if (k < KS) {
        ml[k].x = fast_exp2(ml[k].x - m);
        l += ml[k].x * ml[k].y;
      }
    l = sum_groups(l);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    if (node_at(n) >= it.ntok) continue;
    if (part == 0) put_ml(n, m, l);
    for (int i = part * NB / KS; i < (part + 1) * NB / KS; ++i) {
      f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < kWaves; ++k)
        if (k < KS) x += ml[k].x * *(const f32x4*)(p + k * NT * STATE + i * 256 + lane * 4);
      put(n, i, x * inv);
    }
  }
}

// Merge the partial states of a row tile's key ranges: a 256-thread block takes
// 256 / (HD / 4) rows, HD / 4 lanes each with four dims.  Range s weighs
// l_s 2^(m_s - M); ranges are added in order, four loads in flight.
template <int HD>
__global__ __launch_bounds__(256) void kv4_combine_kernel(Kv4AttnArgs a) {
  constexpr int LPR = HD / 4, RPB = 256 / LPR, MAXS = 64;
  __shared__ float wgt[RPB][MAXS];
  const Kv4Merge ci = a.comb[blockIdx.x];        // a tile of 16 rows
  const int lane = threadIdx.x % LPR, rr = threadIdx.x / LPR;
  const int row = blockIdx.y * RPB + rr;
  const int G = a.group;
  const int gr = ci.row0 + row, nd = gr / G;
  if (nd >= ci.ntok) return;                   // a row's lanes lie in one wave: nobody waits for them
  const int ns = ci.nsplit;
  float M = -INFINITY;
  for (int sp = lane; sp < ns; sp += LPR) M = maximum(M, a.part_ml[((size_t)(ci.part0 + sp) * 16 + row) * 2]);
#pragma unroll
  for (int m = LPR / 2; m >= 1; m >>= 1) M = maximum(M, __shfl_xor(M, m));
  float L = 0.f;
  for (int sp = lane; sp < ns; sp += LPR) {
    const size_t slot = (size_t)(ci.part0 + sp) * 16 + row;
    const float ms = a.part_ml[slot * 2];
    const float f = fast_exp2(ms - M) * a.part_ml[slot * 2 + 1];
    wgt[rr][sp] = f;
    L += f;
  }
#pragma unroll
  for (int m = LPR / 2; m >= 1; m >>= 1) L += __shfl_xor(L, m);
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  const float* src = a.part_o + ((size_t)ci.part0 * 16 + row) * HD + 4 * lane;
  constexpr size_t STRIDE = (size_t)16 * HD;   // elements between consecutive ranges
  f32x4 O = {0.f, 0.f, 0.f, 0.f};
  int sp = 0;
  for (; sp + 4 <= ns; sp += 4) {
    f32x4 p[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) p[u] = *(const f32x4*)(src + (sp + u) * STRIDE);
#pragma unroll
    for (int u = 0; u < 4; ++u) O += wgt[rr][sp + u] * p[u];
  }
  for (; sp < ns; ++sp) O += wgt[rr][sp] * *(const f32x4*)(src + sp * STRIDE);
  const float inv = 1.f / L;
  bf16x4 v;
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = (bf16)(O[j] * inv);
  *(bf16x4*)(a.out + ((size_t)(ci.tok0 + nd) * a.n_heads + ci.kvh * G + gr % G) * HD + 4 * lane) = v;
}

template <int HD, int NT, bool ONCE>
hipError_t launch_tiles(const Kv4AttnArgs& a, hipStream_t s) {
  constexpr int SMEM = kWaves * NT * (HD / 4 + 2) * 64 * 4;
  const auto kernel = kv4_attention_kernel<HD, NT, ONCE>;
  if constexpr (SMEM > 64 * 1024) {
    static std::atomic<uint64_t> configured{0};               // a bit per device
    int dev = 0;
    if (const hipError_t e = hipGetDevice(&dev)) return e;
    const uint64_t bit = 1ull << (dev & 63);
    if (!(configured.load() & bit)) {
      if (const hipError_t e = hipFuncSetAttribute((const void*)kernel,
                                                   hipFuncAttributeMaxDynamicSharedMemorySize, SMEM))
        return e;
      configured.fetch_or(bit);
    }
  }
  kernel<<<(a.n_items + 7) / 8 * 8, 64 * kWaves, SMEM, s>>>(a);
  return hipGetLastError();
}

template <int HD>
hipError_t launch_hd(const Kv4AttnArgs& a, hipStream_t s) {
  const hipError_t e = a.wave_tiles == 2 ? launch_tiles<HD, 2, false>(a, s)
                       : a.once          ? launch_tiles<HD, 1, true>(a, s)
                                         : launch_tiles<HD, 1, false>(a, s);
  if (e != hipSuccess) return e;
  if (a.n_comb) kv4_combine_kernel<HD><<<dim3(a.n_comb, 16 / (256 / (HD / 4))), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv4_attention(const Kv4AttnArgs& a, hipStream_t s) {
  if (a.v.head_dim == 128) return launch_hd<128>(a, s);
  if (a.v.head_dim == 64) return launch_hd<64>(a, s);
  return hipErrorInvalidValue;
}

}  // namespace spec
