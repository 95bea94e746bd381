// The 4-bit paged KV cache: rows quantised into it, read back, and moved when a
// branch is committed.
//
// A number is an E2M1 code times its group's power of two s = 2^e: 32
// consecutive dims of a key make a group, so do all dims of a value.  e is the
// smallest exponent in [-126, 125] with max |x| <= 6 s, or 125; the code is the one
// nearest to x / s, the even one of two equally near.
#include <algorithm>
#include <math.h>

#include "kv4.h"

namespace spec {

namespace {

constexpr int kWaves = 4;                        // waves per work-group
constexpr int64_t kMaxGrid = 0xffffffffll / 256;

// x as fp32 so that rounding it to a code (two significant bits, in steps of 2^-127 at
// least) gives what one rounding of x would: 21 significant bits, the last one set when
// something was cut off.  What is finite stays finite.
__device__ __forceinline__ float round_to_odd(double x) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t hi = (uint32_t)(b >> 32) | ((uint32_t)b != 0 ? 1u : 0u);
  const float f = (float)__builtin_bit_cast(double, (uint64_t)hi << 32);
  return isinf(f) && !isinf(x) ? copysignf(3.4028234663852886e38f, f) : f;
}

// The larger magnitude; a NaN when there is one.
__device__ __forceinline__ float largest(float x, float y) {
  return __builtin_elementwise_maximum(fabsf(x), fabsf(y));
}

// x of the lane with its index's bit 0, 1 or 2 flipped, given (for 2 and 4) that lanes
// that differ in a lower bit hold the same; over 16 lanes likewise.
__device__ __forceinline__ uint32_t lane_xor1(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xf, 0xf, true);      // quad_perm 1 0 3 2
}
template <int LANES>
__device__ __forceinline__ uint32_t max_over(uint32_t x) {
  x = max(x, lane_xor1(x));
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xf, 0xf, true));   // quad_perm 2 3 0 1
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x141, 0xf, 0xf, true));  // row_half_mirror
  if constexpr (LANES == 16) x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x140, 0xf, 0xf, true));
  return x;
}

// cos and sin of an angle, to about an ulp of double.  Below 2^31 (every position, with a
// rotary base of 1 or more): x = n pi/2 + r, |r| <= pi/4, with pi/2 in two doubles, of
// which the first product leaves no rounding error (n pi_hi and an x that has an n are
// multiples of 2^-53, and their difference is below 1); then the series, cut where the
// next term is below 2^-53 of the result.  About 40 instructions.
__device__ __forceinline__ double2 cos_sin(double x) {
  if (!(fabs(x) < 0x1p31)) {
    double s, c;
    sincos(x, &s, &c);
    return make_double2(c, s);
  }
  const double n = rint(x * 0.63661977236758134308);
  const double r = fma(-n, 6.123233995736766e-17, fma(-n, 1.5707963267948966, x)), z = r * r;
  auto series = [z](const double (&c)[8]) __attribute__((always_inline)) {
    double y = c[7];
#pragma unroll
    for (int i = 6; i >= 0; --i) y = fma(y, z, c[i]);
    return y;
  };
  // 1 / (2 i + 3)! and 1 / (2 i + 4)!, with their signs
  constexpr double S[8] = {-1.0 / 6, 1.0 / 120, -1.0 / 5040, 1.0 / 362880, -1.0 / 39916800, 1.0 / 6227020800.0,
                           -1.0 / 1307674368000.0, 1.0 / 355687428096000.0};
  constexpr double C[8] = {1.0 / 24, -1.0 / 720, 1.0 / 40320, -1.0 / 3628800, 1.0 / 479001600.0, -1.0 / 87178291200.0,
                           1.0 / 20922789888000.0, -1.0 / 6402373705728000.0};
  const double sn = fma(r * z, series(S), r);
  const double half = 0.5 * z, one = 1.0 - half;                   // 1 - z / 2 loses what is added back
  const double cn = one + fma(z * z, series(C), (1.0 - one) - half);
  const int q = (int)n;
  const double c = q & 1 ? sn : cn, t = q & 1 ? cn : sn;
  return make_double2((q + 1) & 2 ? -c : c, q & 2 ? -t : t);
}

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// e + 127 for a group whose largest magnitude has the fp32 bits `top`; 255 when
// the group holds an infinity or NaN.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
  if (top >= 0x7f800000u) return 255u;
  // top = 1.m 2^(E - 127) <= 6 2^e = 1.5 2^(e + 2)
  return (uint32_t)min(max(((int)top + 0x3fffff - (2 << 23)) >> 23, 1), 252);
}

// N (4 or 8) E2M1 codes of f / 2^(byte - 127), dim n in bits 4n .. 4n + 3; 0 for a
// group without a scale, and 0 rather than -0.
template <int N>
__device__ __forceinline__ uint32_t pack_codes(const float* f, uint32_t byte) {
  const float s = __uint_as_float(byte << 23);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[0], f[1], s, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[2], f[3], s, 1);
  if constexpr (N == 8) {
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[4], f[5], s, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[6], f[7], s, 3);
  }
  const uint32_t some = ((w & 0x77777777u) + 0x77777777u) & 0x88888888u;   // magnitude bits set
  w &= some | 0x77777777u;
  return byte == 255u ? 0u : w;
}

// The number of a code: its exponent and mantissa bits read as fp32's are 2^-126
// times the E2M1 number, subnormals included.
__device__ __forceinline__ float code_value(uint32_t code, float s) {
  const float m = __uint_as_float((code & 7u) << 22) * 0x1p126f;
  return (code & 8u ? -m : m) * s;
}

// Eight numbers of a word of codes, s a power of two, as bf16.
__device__ __forceinline__ i32x4 numbers(uint32_t w, float s) {
  return i32x4{__builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0)),
               __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1)),
               __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2)),
               __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3))};
}

// A row's lanes: HD / 8 lanes, so a wave holds 64 / (HD / 8) rows at a time and takes an
// octet's 8 keys in KPL steps.  Lane l has 8 consecutive dims from 8 l; of a key that is
// appended the two halves of its rotated pairs, 4 dims from 4 l and 4 from HD / 2 + 4 l.
template <int HD>
struct Rows {
  static constexpr int LPR = HD / 8;
  static constexpr int RPW = 64 / LPR;
  static constexpr int KPL = 8 / RPW;
  static constexpr int WORDS = HD / 64;       // value-code words of an octet per lane
};

// Work-groups go to the eight XCDs in turn; consecutive octets to one of them, so that
// lines that the octets of a page share (the scales) are put together in its L2.
__device__ __forceinline__ int octet_of_block() {
  return (int)((blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3));
}

// Quantise one octet's rows of a sample, a wave per head at a time.
//
// The rotation is computed in doubles and rounded once, to the code: every
// angle's sine and cosine is taken once per work-group (position and pair) and
// shared by its heads through LDS.  A head's rows are loaded while the angles, or the
// head before it, are computed.
// A value's codes are held with the octet's 8 keys in one word per dim, so the
// wave transposes them through LDS; positions of the octet that are not written
// keep their codes.
//
// Bound by bytes and vector instructions about alike: 29.7K rows of 8 heads of 128 (122
// MB in, 32 MB out, 31 us at a copy's rate) take 36 us, 38 before the clock has risen, with
// some 500 instructions per octet and head.  With the library's sincos, a conversion of
// both numbers of a pair in both of their lanes, and no load under way it was 44 us (before
// the clock had risen, as the next) and 665; a wave per head and no second one to load for,
// 48 us.  One row: 3.6 us (5.1).
template <int HD>
__global__ __launch_bounds__(256) void kv4_append_kernel(Kv4RowArgs a, int heads_per_wg) {
  using R = Rows<HD>;
  constexpr int HALF = HD / 2;
  __shared__ double2 turn[8][HALF + HALF / 8];        // one pad every 8: lanes of a row 144 bytes apart
  __shared__ uint32_t vcode[kWaves][8][HD / 8];
  const int at_octet = octet_of_block();
  if (at_octet >= a.n_octets) return;
  const Kv4Octet oc = a.octets[at_octet];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int q = lane / R::LPR, l = lane % R::LPR;
  const int at = oc.slot0 % kKv4Page;                 // in the page
  char* page = a.v.pool + kv4_page_offset(oc.page);
  const int h0 = blockIdx.y * heads_per_wg, h1 = min(h0 + heads_per_wg, a.v.n_kv_heads);
  const int64_t ks = a.blocks ? HD : a.k_stride, vs = a.blocks ? HD : a.v_stride;
  const int64_t hs = a.blocks ? (int64_t)oc.ntok * HD : HD;             // between heads
  const bf16* k0 = a.k + oc.row0 * ks;
  const bf16* v0 = a.val + oc.row0 * vs;
  if (a.blocks) {
    k0 = a.k + (int64_t)oc.tok0 * 2 * a.v.n_kv_heads * HD + (int64_t)(oc.row0 - oc.tok0) * HD;
    v0 = k0 + a.v.n_kv_heads * hs;
  }
  // Lanes of a position that the step does not write do the work of one that it does.
  int row[R::KPL];
  const bf16 *kp[R::KPL], *vp[R::KPL];
#pragma unroll
  for (int kk = 0; kk < R::KPL; ++kk) {
    row[kk] = min(max(q + R::RPW * kk, oc.lo), oc.hi - 1);
    kp[kk] = k0 + row[kk] * ks + 4 * l;
    vp[kk] = v0 + row[kk] * vs + 8 * l;
  }
  struct Values {
    i32x2 k[R::KPL][2];
    i32x4 v[R::KPL];
  } next;
  auto load = [&](int head) __attribute__((always_inline)) {
#pragma unroll
    for (int kk = 0; kk < R::KPL; ++kk) {
      next.k[kk][0] = *(const i32x2*)(kp[kk] + head * hs);
      next.k[kk][1] = *(const i32x2*)(kp[kk] + head * hs + HALF);
      next.v[kk] = *(const i32x4*)(vp[kk] + head * hs);
    }
  };
  if (h0 + w < h1) load(h0 + w);                       // under way while the angles are computed
  if (a.rotate) {
    for (int x = threadIdx.x; x < 8 * HALF; x += 256) {
      const int t = x / HALF, j = x % HALF;
      if (t >= oc.lo && t < oc.hi) {
        const int pos = a.toks ? a.toks[oc.row0 + t].pos : oc.slot0 + t;
        turn[t][j + j / 8] = cos_sin((double)pos * a.freq[j]);
      }
    }
    __syncthreads();
  }
  for (int head = h0 + w; head < h1; head += kWaves) {
    char* base = page + ((int64_t)a.v.layer * a.v.n_kv_heads + head) * kv4_head_bytes(HD);
    const Values x = next;
    if (head + kWaves < h1) load(head + kWaves);
#pragma unroll
    for (int kk = 0; kk < R::KPL; ++kk) {
      const int t = q + R::RPW * kk;
      const bool live = t >= oc.lo && t < oc.hi;
      float f[8];                              // of a key: 4 of the low half, 4 of the high one
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f[2 * i] = bf16_lo((uint32_t)x.k[kk][i >> 1][i & 1]);
        f[2 * i + 1] = bf16_hi((uint32_t)x.k[kk][i >> 1][i & 1]);
      }
      uint32_t low, high;                      // largest magnitudes (or NaN) of f[0 .. 3], f[4 .. 7]
      auto tops = [&]() __attribute__((always_inline)) {
        low = __float_as_uint(largest(largest(f[0], f[1]), largest(f[2], f[3])));
        high = __float_as_uint(largest(largest(f[4], f[5]), largest(f[6], f[7])));
      };
      if (a.rotate) {
        const double2* cs = &turn[row[kk]][4 * l + l / 2];
        // Where the nearest fp32 number has two significant bits or three it may be midway
        // between two codes, and the number itself not: those, and what fp32 does not
        // reach, are rounded by round_to_odd().
        uint32_t least = 0xffffffffu;          // 0: low 21 bits are 0
        auto rotated = [&](auto round) __attribute__((always_inline)) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t lw = (uint32_t)x.k[kk][0][i >> 1], hw = (uint32_t)x.k[kk][1][i >> 1];
            const double lo = (double)(i & 1 ? bf16_hi(lw) : bf16_lo(lw));
            const double hi = (double)(i & 1 ? bf16_hi(hw) : bf16_lo(hw));
            f[i] = round(fma(-hi, cs[i].y, lo * cs[i].x));
            f[4 + i] = round(fma(lo, cs[i].y, hi * cs[i].x));
            least = min(least, min(__float_as_uint(f[i]) << 11, __float_as_uint(f[4 + i]) << 11));
          }
          tops();
        };
        rotated([](double x) { return (float)x; });
        if (__ballot(least == 0 || max(low, high) >= 0x7f800000u)) {
          asm volatile("");                    // keeps this out of the usual path
          rotated(round_to_odd);
        }
      } else {
        tops();
      }
      low = scale_byte(max_over<8>(low));
      high = scale_byte(max_over<8>(high));
      // 4 dims make two bytes.  Even lanes store four of the low half, odd ones of the high.
      const uint32_t cl = pack_codes<4>(f, low), ch = pack_codes<4>(f + 4, high);
      const uint32_t other = lane_xor1(l & 1 ? cl : ch);
      if (live) {
        const uint32_t s = at + t, d = (l & 1 ? HALF : 0) + 4 * (l & ~1);  // first of 8 dims
        *(uint32_t*)(base + (s / 32 * kv4_block_bytes(HD) + d / 32 * 512 + s % 32 * 16 + d % 32 / 2)) =
            l & 1 ? other | ch << 16 : cl | other << 16;
        if (l % 8 == 0) {
          uint8_t* scales = (uint8_t*)(base + (kv4_kscale_at(HD) + s * (HD / 32) + l / 8));
          scales[0] = (uint8_t)low;
          scales[HALF / 32] = (uint8_t)high;
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f[2 * i] = bf16_lo((uint32_t)x.v[kk][i]);
        f[2 * i + 1] = bf16_hi((uint32_t)x.v[kk][i]);
      }
      tops();
      const uint32_t vb = scale_byte(max_over<R::LPR>(max(low, high)));
      vcode[w][t][l] = pack_codes<8>(f, vb);
      if (live && l == 0)
        *(uint16_t*)(base + (uint32_t)(kv4_vscale_at(HD) + 2 * (at + t))) = vb == 255u ? 0x7fc0 : (uint16_t)(vb << 7);
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    // Word (m, i) of the octet: dim 32 i + m of keys 0 .. 7.
    uint32_t* vw = (uint32_t*)(base + (uint32_t)(kv4_value_at(HD) + (at / 8) * kv4_octet_bytes(HD) +
                                                 lane * R::WORDS * 4));
    const uint32_t hi_mask = oc.hi == 8 ? 0xffffffffu : (1u << (4 * oc.hi)) - 1;
    const uint32_t mask = hi_mask & ~((1u << (4 * oc.lo)) - 1);
#pragma unroll
    for (int x = 0; x < R::WORDS; ++x) {
      const int wi = lane * R::WORDS + x, m = wi / (HD / 32), d = 32 * (wi % (HD / 32)) + m;
      uint32_t word = 0;
#pragma unroll
      for (int t = 0; t < 8; ++t) word |= (vcode[w][t][d / 8] >> (4 * (d % 8)) & 15u) << (4 * t);
      if (mask != 0xffffffffu) word = (vw[x] & ~mask) | (word & mask);
      vw[x] = word;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

// What the cache holds for one octet's rows, as bf16 (exact: two significant bits).  Bound
// by its writes: 29.7K rows of 8 heads of 128 (122 MB) 25 us; with every number built from
// its bits 26.5, the vector units 99 % busy.
template <int HD>
__global__ __launch_bounds__(256) void kv4_read_kernel(Kv4RowArgs a, int heads_per_wg) {
  using R = Rows<HD>;
  __shared__ uint32_t vword[kWaves][HD];
  const int at_octet = octet_of_block();
  if (at_octet >= a.n_octets) return;
  const Kv4Octet oc = a.octets[at_octet];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int q = lane / R::LPR, l = lane % R::LPR;
  const int at = oc.slot0 % kKv4Page;
  const char* page = a.v.pool + kv4_page_offset(oc.page);
  const int h0 = blockIdx.y * heads_per_wg, h1 = min(h0 + heads_per_wg, a.v.n_kv_heads);
  for (int head = h0 + w; head < h1; head += kWaves) {
    const char* base = page + ((int64_t)a.v.layer * a.v.n_kv_heads + head) * kv4_head_bytes(HD);
    const uint32_t* vw = (const uint32_t*)(base + kv4_value_at(HD) + (at / 8) * kv4_octet_bytes(HD));
#pragma unroll
    for (int x = 0; x < R::WORDS; ++x) vword[w][lane * R::WORDS + x] = vw[lane * R::WORDS + x];
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int kk = 0; kk < R::KPL; ++kk) {
      const int t = q + R::RPW * kk;
      if (t < oc.lo || t >= oc.hi) continue;
      const int s = at + t;
      const uint32_t kw = *(const uint32_t*)(base + (s / 32) * kv4_block_bytes(HD) + (l / 4) * 512 +
                                             (s % 32) * 16 + (l % 4) * 4);
      const uint32_t sb = *(const uint8_t*)(base + kv4_kscale_at(HD) + s * (HD / 32) + l / 4);
      const uint32_t vs = *(const uint16_t*)(base + kv4_vscale_at(HD) + 2 * s);
      uint32_t vcodes = 0;                     // the row's eight dims, as kw
#pragma unroll
      for (int n = 0; n < 8; ++n) {
        const int d = 8 * l + n;
        vcodes |= (vword[w][(d % 32) * (HD / 32) + d / 32] >> (4 * t) & 15u) << (4 * n);
      }
      i32x4 ko, vo;
      // Scales that leave no number subnormal: two numbers at once.
      const bool normal = sb - 2u <= 250u && (vs & 0x807fu) == 0 && (vs >> 7) - 2u <= 250u;
      if (__ballot(!normal) == 0) {
        ko = numbers(kw, __uint_as_float(sb << 23));
        vo = numbers(vcodes, __uint_as_float(vs << 16));
      } else {
        const float ks = sb == 255u ? __uint_as_float(0x7fc00000u) : __uint_as_float(sb << 23);
        const float fs = __uint_as_float(vs << 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t kb[2], vb[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            kb[j] = __float_as_uint(code_value(kw >> (8 * i + 4 * j) & 15u, ks)) >> 16;
            vb[j] = __float_as_uint(code_value(vcodes >> (8 * i + 4 * j) & 15u, fs)) >> 16;
          }
          ko[i] = (int)(kb[0] | kb[1] << 16);
          vo[i] = (int)(vb[0] | vb[1] << 16);
        }
      }
      *(i32x4*)(a.k + (oc.row0 + t) * a.k_stride + head * HD + 8 * l) = ko;
      *(i32x4*)(a.val + (oc.row0 + t) * a.v_stride + head * HD + 8 * l) = vo;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

// Move the accepted branch of one sample, one layer and head: position seq_len + d
// takes the codes and scales of node path[d] > d, d = 1 .. accepted_len.  A thread
// owns one word column of the keys and one dim of the values, and within those it
// goes up in d.  What it overwrites lies at d, what it still has to read at
// path[d'] > d' > d, so nothing is lost and no thread waits for another.
// Bound by that thread's chain of loads, PER of the keys and 8 of the values under way:
// 127 rows moved in 128 samples, 32 layers of 8 heads of 128 (8.7 MB in and out) take 80 us.
template <int HD>
__global__ __launch_bounds__(128) void kv4_compact_kernel(const Kv4CommitInfo* info, char* pool,
                                                          int64_t page_bytes, int n_kv_heads,
                                                          const int32_t* accepted_len,
                                                          const int32_t* accepted_nodes,
                                                          int32_t* new_seq_lens) {
  constexpr int PER = 8;
  const int b = blockIdx.x, layer = blockIdx.y, head = blockIdx.z, x = threadIdx.x;
  const Kv4CommitInfo& c = info[b];
  const int S = c.seq_len;
  int acc = accepted_len[b];
  acc = min(max(acc, 0), min(kMaxTree - 1, c.cap - 1 - S));
  if (layer == 0 && head == 0 && x == 0) new_seq_lens[b] = S + acc + 1;
  if (acc == 0) return;
  const int32_t* path = accepted_nodes + (size_t)b * kMaxTree;
  const int first = S / kKv4Page * kKv4Page;
  const int64_t in_page = ((int64_t)layer * n_kv_heads + head) * kv4_head_bytes(HD);
  auto base = [&](int slot) { return pool + (int64_t)c.pages[(slot - first) / kKv4Page] * page_bytes + in_page; };
  // The node that position S + d takes, or -1 when it keeps what it has.
  auto source = [&](int d) {
    const int nd = path[d];
    return nd > d && nd < kMaxTree && S + nd < c.cap ? nd : -1;
  };
  // One column of the keys: codes (a word of every row), then scales.
  constexpr int KW = HD / 8;
  if (x < KW) {
    auto word = [&](int slot) {
      const int s = slot % kKv4Page;
      return (uint32_t*)(base(slot) + (s / 32) * kv4_block_bytes(HD) + (x / 4) * 512 + (s % 32) * 16 + (x % 4) * 4);
    };
    for (int d0 = 1; d0 <= acc; d0 += PER) {
      uint32_t v[PER];
      int nd[PER];
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        nd[i] = d0 + i <= acc ? source(d0 + i) : -1;
        if (nd[i] >= 0) v[i] = *word(S + nd[i]);
      }
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (nd[i] >= 0) *word(S + d0 + i) = v[i];
    }
  } else if (x >= 64 && x < 64 + HD / 32 + 2) {       // a byte column of the key or value scales
    const int y = x - 64;
    auto byte = [&](int slot) {
      const int s = slot % kKv4Page;
      return (uint8_t*)(base(slot) + (y < HD / 32 ? kv4_kscale_at(HD) + s * (HD / 32) + y
                                                  : kv4_vscale_at(HD) + 2 * s + y - HD / 32));
    };
    for (int d0 = 1; d0 <= acc; d0 += PER) {
      uint8_t v[PER];
      int nd[PER];
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        nd[i] = d0 + i <= acc ? source(d0 + i) : -1;
        if (nd[i] >= 0) v[i] = *byte(S + nd[i]);
      }
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (nd[i] >= 0) *byte(S + d0 + i) = v[i];
    }
  }
  // One dim of the values: a word of every octet.
  if (x < HD) {
    const int m = x % 32, i = x / 32;
    auto word = [&](int slot) {
      return (uint32_t*)(base(slot) + kv4_value_at(HD) + (slot % kKv4Page) / 8 * kv4_octet_bytes(HD)) +
             m * (HD / 32) + i;
    };
    for (int o = (S + 1) / 8 * 8; o <= S + acc; o += 8) {
      uint32_t got[8];
      uint32_t mask = 0;
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        const int d = o + t - S;
        const int nd = d >= 1 && d <= acc ? source(d) : -1;
        got[t] = 0;
        if (nd >= 0) {
          got[t] = (*word(S + nd) >> (4 * ((S + nd) % 8)) & 15u) << (4 * t);
          mask |= 15u << (4 * t);
        }
      }
      if (mask == 0) continue;
      uint32_t v = *word(o) & ~mask;
#pragma unroll
      for (int t = 0; t < 8; ++t) v |= got[t];
      *word(o) = v;
    }
  }
}

// Heads per work-group of the row kernels: all of them when there are octets
// enough to fill the chip (an angle is then taken once), else one per wave.
int heads_per_wg(int n_octets, int n_kv_heads) {
  return n_octets >= 1024 ? n_kv_heads : std::min(n_kv_heads, kWaves);
}

template <class K64, class K128>
hipError_t launch_rows(const Kv4RowArgs& a, hipStream_t s, K64 k64, K128 k128) {
  if (a.n_octets == 0) return hipSuccess;
  if (a.n_octets > kMaxGrid) return hipErrorInvalidValue;
  const int hpw = heads_per_wg(a.n_octets, a.v.n_kv_heads);
  const dim3 grid((a.n_octets + 7) / 8 * 8, (a.v.n_kv_heads + hpw - 1) / hpw);
  if ((int64_t)grid.x * grid.y > kMaxGrid) return hipErrorInvalidValue;
  if (a.v.head_dim == 128) k128<<<grid, 256, 0, s>>>(a, hpw);
  else if (a.v.head_dim == 64) k64<<<grid, 256, 0, s>>>(a, hpw);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv4_append(const Kv4RowArgs& a, hipStream_t s) {
  return launch_rows(a, s, kv4_append_kernel<64>, kv4_append_kernel<128>);
}

hipError_t launch_kv4_read(const Kv4RowArgs& a, hipStream_t s) {
  return launch_rows(a, s, kv4_read_kernel<64>, kv4_read_kernel<128>);
}

hipError_t launch_kv4_compact(const Kv4CommitInfo* info, int batch, char* pool, int64_t page_bytes,
                              int n_layers, int n_kv_heads, int head_dim, const int32_t* accepted_len,
                              const int32_t* accepted_nodes, int32_t* new_seq_lens, hipStream_t s) {
  const dim3 grid(batch, n_layers, n_kv_heads);
  if (head_dim == 128)
    kv4_compact_kernel<128><<<grid, 128, 0, s>>>(info, pool, page_bytes, n_kv_heads, accepted_len,
                                                 accepted_nodes, new_seq_lens);
  else if (head_dim == 64)
    kv4_compact_kernel<64><<<grid, 128, 0, s>>>(info, pool, page_bytes, n_kv_heads, accepted_len,
                                                accepted_nodes, new_seq_lens);
  else
    return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace spec
