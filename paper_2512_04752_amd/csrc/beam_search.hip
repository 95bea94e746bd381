// The k best continuations of a sample's beams.
//
// Candidate (w, y) scores s_w + z_wy - lse_w with lse_w = log sum_y exp z_wy.  Within a beam
// the order is that of its logits, so one pass over them finds both what the normaliser
// needs and the k best logits of every piece of a row, exactly; the scores are only formed
// for those few, in doubles, where beams are compared.
//
//   beam_scan_kernel   a wave per segment of a row: sum of exponentials and its k best logits
//   beam_pick_kernel   a work-group per sample: normalisers, and the k best of all candidates
//
// The sums are doubles, terms included: two beams' candidates can lie next to each other,
// and an fp32 exponential (relative error 6e-8 and more) would decide between them.
#include <algorithm>

#include "beam.h"
#include "gemm_tile.h"

namespace spec {

namespace {

// e^d for -708 <= d <= 690 (the result's exponent is a normal one), relative error below 5e-11:
// d log2 e = n + f, |f| <= 1/2, and 2^n times the polynomial of degree 7 that is 1 at 0 with the
// smallest largest relative error of 2^f (4.67e-11 by Remez's exchange; the series needs degree 9
// for that).  e^0 is 1 exactly (without that 4.0e-11), so that beams that are sure of a token, and
// beams with equally many equally likely ones, have equal normalisers.  n comes out of an
// addition that leaves it in the low bits, and goes into the exponent by an integer one: all of
// it at the rate of fp64 additions.  The constants are held in scalar registers (of constants
// that the compiler knows, it copies each into the result first and then accumulates, twice the
// instructions), but the 1, which an instruction has itself.
struct Exp {
  double log2e, big, c[8];
  __device__ __forceinline__ Exp()
      : c{1.0, 0.693147180704532, 0.24022651066560827, 0.055504103659919514, 0.009618038132083197,
          0.0013333935054941355, 0.00015466756313134368, 1.5196156729123239e-05} {
    log2e = 1.44269504088896340736;
    // 1.5 * 2^52, and 2^12 that the shift drops: without it the low word is 0, and then this
    // compiler (ROCm 7.2) loads it by s_mov_b64 with a 64-bit literal, which there is none of.
    big = 6755399441055744.0 + 4096.0;
    asm volatile("" : "+s"(log2e), "+s"(big), "+v"(c[7]));         // an instruction reads one scalar pair
#pragma unroll
    for (int i = 1; i < 7; ++i) asm volatile("" : "+s"(c[i]));
  }
  __device__ __forceinline__ double operator()(double d) const {
    const double m = fma(d, log2e, big), f = fma(d, log2e, big - m);
    double y = fma(f, c[7], c[6]);
#pragma unroll
    for (int i = 5; i >= 0; --i) y = fma(y, f, c[i]);
    i32x2 b = __builtin_bit_cast(i32x2, y);
    b[1] += __builtin_bit_cast(i32x2, m)[0] << 20;
    return __builtin_bit_cast(double, b);
  }
  // x e^d, d <= 690; a NaN for a NaN in either; 0 where that is below e^-690 of x.
  __device__ __forceinline__ double scaled(double x, double d) const {
    return d != d ? d : x * (d < -690.0 ? 0.0 : (*this)(d));
  }
};

constexpr float kLowest = -3.4028234663852886e38f;

// A logit and its token as one number, larger for a higher logit, then for a lower token; 0:
// none.
__device__ __forceinline__ uint64_t key_of(float z, int y) {
  const uint32_t b = __float_as_uint(z + 0.0f);              // -0 as 0
  return (uint64_t)(b ^ ((uint32_t)((int)b >> 31) | 0x80000000u)) << 32 | (uint32_t)~y;
}
__device__ __forceinline__ float logit_of(uint64_t key) {
  const uint32_t u = (uint32_t)(key >> 32);
  return key == 0 ? -INFINITY : __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u);
}
__device__ __forceinline__ int token_of(uint64_t key) { return (int)~(uint32_t)key; }

// Lane i gets lane i - 1's x.
__device__ __forceinline__ int from_below(int x) {
  return __builtin_amdgcn_update_dpp(x, x, 0x138, 0xf, 0xf, false);      // wave_shr:1
}

__device__ __forceinline__ float lane_value(float x, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane));
}

template <class X>
__device__ __forceinline__ X lane_value64(X x, int lane) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)b, lane), hi = __builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), lane);
  return __builtin_bit_cast(X, (uint64_t)hi << 32 | lo);
}
template <class X>
__device__ __forceinline__ X from_below64(X x) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = from_below((int)(uint32_t)b), hi = from_below((int)(uint32_t)(b >> 32));
  return __builtin_bit_cast(X, (uint64_t)hi << 32 | lo);
}

// Both halves of 2 S lanes, whose S lanes each have the same of their own: x and its partner's,
// the same pair in all.  Moves inside and between rows of 16 lanes; through LDS (a shuffle)
// each takes some 100 cycles, which at a wave's end nothing hides.
template <int S>
__device__ __forceinline__ void halves_of(uint32_t x, uint32_t* a, uint32_t* b) {
  if constexpr (S < 16) {
    constexpr int MOVE = S == 1 ? 0xb1 : S == 2 ? 0x4e : S == 4 ? 0x141 : 0x140;    // quads' lanes, mirrors of 8 and 16
    *a = x;
    *b = (uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, MOVE, 0xf, 0xf, false);
  } else {
    const auto r = S == 16 ? __builtin_amdgcn_permlane16_swap(x, x, false, false)
                           : __builtin_amdgcn_permlane32_swap(x, x, false, false);
    *a = r[0];
    *b = r[1];
  }
}
template <int S>
__device__ __forceinline__ float max_of_halves(float x) {
  uint32_t a, b;
  halves_of<S>(__float_as_uint(x), &a, &b);
  return __builtin_elementwise_maximum(__uint_as_float(a), __uint_as_float(b));
}
template <int S>
__device__ __forceinline__ double sum_of_halves(double x) {
  const i32x2 v = __builtin_bit_cast(i32x2, x);
  uint32_t a[2], b[2];
  halves_of<S>((uint32_t)v[0], &a[0], &b[0]);
  halves_of<S>((uint32_t)v[1], &a[1], &b[1]);
  return __builtin_bit_cast(double, i32x2{(int)a[0], (int)a[1]}) + __builtin_bit_cast(double, i32x2{(int)b[0], (int)b[1]});
}
// Over groups of `lanes` neighbours (a power of two), every lane of a group the same.
__device__ __forceinline__ float max_over(float x, int lanes) {
  if (lanes > 1) x = max_of_halves<1>(x);
  if (lanes > 2) x = max_of_halves<2>(x);
  if (lanes > 4) x = max_of_halves<4>(x);
  if (lanes > 8) x = max_of_halves<8>(x);
  if (lanes > 16) x = max_of_halves<16>(x);
  if (lanes > 32) x = max_of_halves<32>(x);
  return x;
}
__device__ __forceinline__ double sum_over(double x, int lanes) {
  if (lanes > 1) x = sum_of_halves<1>(x);
  if (lanes > 2) x = sum_of_halves<2>(x);
  if (lanes > 4) x = sum_of_halves<4>(x);
  if (lanes > 8) x = sum_of_halves<8>(x);
  if (lanes > 16) x = sum_of_halves<16>(x);
  if (lanes > 32) x = sum_of_halves<32>(x);
  return x;
}

// The largest float below x; -infinity and NaN stay.
__device__ __forceinline__ float float_below(float x) {
  const int b = __float_as_int(x);
  return !(x > -INFINITY) ? x : b == 0 ? -1e-45f : __int_as_float(b > 0 ? b - 1 : b + 1);
}

// A bound that at least k of the wave's N x 64 numbers are not below, within 2^-7 of the
// k-th largest (k <= 64 N): the leading 16 bits of its place in the order of floats, found
// from the top by counting, BITS at a time (a step waits for its counts, some 100 cycles).
// -infinity where it is that.
template <int BITS, int N>
__device__ __forceinline__ float kth_bound(const float (&x)[N], int k) {
  uint32_t u[N], t = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t b = __float_as_uint(x[i]);
    u[i] = b ^ ((uint32_t)((int)b >> 31) | 0x80000000u);
  }
#pragma unroll
  for (int bit = 32 - BITS; bit >= 16; bit -= BITS) {
    uint32_t up = 0;
#pragma unroll
    for (uint32_t c = 1; c < 1u << BITS; ++c) {
      int n = 0;
#pragma unroll
      for (int i = 0; i < N; ++i) n += __popcll(__ballot(u[i] >= (t | c << bit)));
      up += n >= k;
    }
    t |= up << bit;
  }
  return t <= 0x007fffffu ? -INFINITY : __uint_as_float(t & 0x80000000u ? t ^ 0x80000000u : ~t);
}

// LDS written by lanes of a wave is there for its other lanes.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// A wave's list of the k best is one key per lane, best first, 0 past the last.
// Put one more into it.
__device__ __forceinline__ void insert(uint64_t& l, uint64_t key, int lane) {
  const int pos = __popcll(__ballot(l > key));
  const uint64_t b = from_below64(l);
  l = lane < pos ? l : lane == pos ? key : b;
}

// Put n <= 64 more into it, by counting for each what is better: about 5 instructions per new
// entry and 3 per old one, where insert() takes 20 for each.
constexpr int kFew = 5, kEnough = 32;
__device__ __forceinline__ void merge(uint64_t& l, const uint64_t* found, uint64_t* merged, int n, int k, int lane) {
  const uint64_t x = lane < n ? found[lane] : 0;
  int rank = 0, old = lane;
  merged[lane] = l;
  wave_sync();
#pragma unroll 4
  for (int q = 0; q < n; ++q) {
    const uint64_t f = found[q];
    rank += f > x;
    old += f > l;
  }
  if (lane_value64(l, 0) != 0) {
#pragma unroll 4
    for (int q = 0; q < k; ++q) rank += merged[q] > x;
  }
  wave_sync();
  merged[lane] = 0;
  wave_sync();
  if (lane < k && l != 0 && old < k) merged[old] = l;
  if (lane < n && rank < k) merged[rank] = x;
  wave_sync();
  l = merged[lane];
}

// Whether a beam is read at all: its score is finite and it has not ended.
__device__ __forceinline__ bool beam_live(const BeamArgs& a, int row) {
  const float s = a.scores[row];
  return fabsf(s) < INFINITY && !(a.eos >= 0 && a.last[row] == a.eos);
}

// 16 bytes of a row, wherever it starts: which elements a lane takes, and so the order of
// a row's sum, goes by their index alone, and equal rows have equal normalisers.
template <class T>
struct Vectors {
  static constexpr int PER = 16 / sizeof(T);
  typedef i32x4 __attribute__((aligned(2))) Loose;
  const T* row;
  int vocab;
  // Elements v * PER ..; what is past the row, or vector v1, reads as -infinity.
  __device__ __forceinline__ i32x4 load(int v, int v1) const {
    constexpr int NONE = PER == 4 ? (int)0xff800000 : (int)0xff80ff80;
    const int e0 = v * PER;
    i32x4 x{NONE, NONE, NONE, NONE};
    if (v < v1) {
      if (e0 + PER <= vocab) {
        x = *(const Loose*)(row + e0);
      } else {
#pragma unroll
        for (int i = 0; i < PER - 1; ++i)
          if (e0 + i < vocab) {
            const T t = row[e0 + i];
            if constexpr (PER == 4) x[i] = __builtin_bit_cast(int, t);
            else {
              const uint32_t b = (uint32_t)__builtin_bit_cast(uint16_t, t), at = 16 * (i & 1);
              x[i / 2] = (int)(((uint32_t)x[i / 2] & ~(0xffffu << at)) | b << at);
            }
          }
      }
    }
    return x;
  }
  static __device__ __forceinline__ void numbers(const i32x4& x, float* z) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (PER == 4) {
        z[i] = __uint_as_float((uint32_t)x[i]);
      } else {
        z[2 * i] = __uint_as_float((uint32_t)x[i] << 16);
        z[2 * i + 1] = __uint_as_float((uint32_t)x[i] & 0xffff0000u);
      }
    }
  }
};

// A wave goes through its segment in batches of kVecs vectors per lane, the next batch on
// its way while one is worked on.  Per number: 15 instructions of fp64 rate for its term,
// one comparison with the k-th best so far, and the few that pass (k ln(n / k) of n in random
// order) go side by side and into the list when there are enough of them.  The first batch
// gives a bound to start with.  128 x 8 x 128256 fp32: 102 us for 525 MB (5.1 TB/s), vector
// instructions 80 % busy; 17 x 12 x 50001 bf16, k 24: 18 us for 20 MB, 61 % busy, half of whose
// 1270 instructions per wave are the terms; 4 x 32000 fp32: 5.2, launch and one trip.
//
// TEAM: the four waves of a work-group have four segments of one row, of which the k best
// matter.  Each tells the others its k / 4-th best so far: k numbers are not below the
// smallest of these four, and what is stays out of every list (which need not fill up).  They
// are read as they are, however old: a bound only rises.
constexpr int kTeam = 4;
constexpr int64_t kMaxGrid = 0xffffffffll / (64 * kTeam);      // a grid has less than 2^32 threads
template <class T, bool TEAM>
__global__ __launch_bounds__(64 * kTeam, 4) void beam_scan_kernel(BeamArgs a) {
  constexpr int PER = Vectors<T>::PER, kVecs = 16 / PER;
  __shared__ uint64_t found[kTeam][64], merged[kTeam][64];
  __shared__ __attribute__((aligned(16))) float told[kTeam];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int teams = (a.segs + kTeam - 1) / kTeam;
  const int64_t id = (int64_t)blockIdx.x * kTeam + wave;
  const int row = TEAM ? (int)(blockIdx.x / teams) : (int)(id / a.segs);
  const int seg = TEAM ? (int)(blockIdx.x % teams) * kTeam + wave : (int)(id % a.segs);
  if (row >= a.groups * a.width || !beam_live(a, row)) return;
  const int members = TEAM ? min(kTeam, a.segs - (seg - wave)) : 1, share = (a.k + members - 1) / members;
  if (TEAM && wave >= members) {
    if (lane == 0) told[wave] = INFINITY;
    wait_lds();
    phase_barrier();
    return;
  }
  auto told_by_all = [&]() {
    const f32x4 t = *(const volatile f32x4*)told;
    return float_below(fminf(fminf(t[0], t[1]), fminf(t[2], t[3])));
  };
  const Vectors<T> vec{(const T*)a.logits + row * a.row_stride, a.vocab};
  const int v0 = seg * a.seg, v1 = min((a.vocab + PER - 1) / PER, v0 + a.seg);
  float top = kLowest;          // the lane's reference: its largest logit so far, less 32 at most
  const Exp exp;
  double sum = 0.0;
  uint64_t best = 0;
  float least = -INFINITY;      // only what is above can be one of the k best: tokens come in ascending order
  int n = 0;                    // found since
  bool first = true;
  constexpr int kStep = 64 * kVecs;
  const T* at_lane = vec.row + (int64_t)(v0 + lane) * PER;
  i32x4 next[kVecs];
  for (int v = v0 - kStep; v < v1; v += kStep) {       // batch v, and loads of the one after it
    float z[kVecs][PER], m[kVecs];
#pragma unroll
    for (int j = 0; j < kVecs; ++j) Vectors<T>::numbers(next[j], z[j]);
    const int after = v + kStep;
    if (after + kStep <= v1 && (int64_t)(after + kStep) * PER <= a.vocab) {
#pragma unroll
      for (int j = 0; j < kVecs; ++j) next[j] = *(const typename Vectors<T>::Loose*)(at_lane + j * 64 * PER);
    } else if (after < v1) {
      int l = lane;
      asm volatile("" : "+v"(l));              // its addresses are not kept in registers over the loop
      for (int j = 0; j < kVecs; ++j) next[j] = vec.load(after + 64 * j + l, v1);
    }
    at_lane += kStep * PER;
    if (v < v0) continue;
#pragma unroll
    for (int j = 0; j < kVecs; ++j) {
      m[j] = z[j][0];
#pragma unroll
      for (int i = 1; i < PER; ++i) m[j] = __builtin_elementwise_maximum(m[j], z[j][i]);   // a NaN when there is one
    }
    float most = m[0], lowest = z[0][0];
#pragma unroll
    for (int j = 1; j < kVecs; ++j) most = __builtin_elementwise_maximum(most, m[j]);
#pragma unroll
    for (int j = 0; j < kVecs; ++j)
#pragma unroll
      for (int i = 0; i < PER; ++i) lowest = __builtin_elementwise_minimum(lowest, z[j][i]);
    // Terms relative to `top`; what is below e^-690 of it counts as that.  A NaN makes the sum
    // one, an infinity `top`.  Lanes rescale their sums by themselves, by e^-32 or less: a second
    // time leaves nothing of what met a first one, so a term meets four exponentials at most (its
    // own, this one, those at the wave's and at the row's end), and errors do not add up along a
    // row.  A logit that has all the probability is its lane's reference, and its term 1.
    // (Differences are compared: of numbers so large that neighbours are further apart, top + 32
    // would be another float than it is.)
    const bool far = !(most - top <= 32.f);
    if (__ballot(far)) {
      if (far) {
        sum = exp.scaled(sum, (double)top - (double)most);
        top = most;
      }
    }
    // (Vectors past the segment add nothing, and most rows have nothing to clamp.)
    const int vecs = min(kVecs, (v1 - v + 63) / 64);
    const double base = (double)top;
    auto add = [&](auto clamp) {
#pragma unroll
      for (int j = 0; j < kVecs; ++j) {
        if (j >= vecs) break;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          const double d = (double)z[j][i] - base;
          sum += exp(clamp ? fmax(d, -690.0) : d);
        }
        __builtin_amdgcn_sched_barrier(0);     // else all terms at once, in more registers than there are
      }
    };
    if (__ballot(!(lowest - top >= -680.f))) add(std::true_type{});
    else add(std::false_type{});
    if (first) {
      first = false;
      // k of the maxima of halves of the lanes' numbers are not below it.  What equals it has to pass.
      float half[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int j = 0; j < kVecs; ++j)
#pragma unroll
        for (int i = 0; i < PER; ++i) half[i & 1] = fmaxf(half[i & 1], z[j][i]);
      const float bound = kth_bound<1>(half, share);
      if constexpr (TEAM) {
        if (lane == 0) told[wave] = bound;
        wait_lds();
        phase_barrier();
      }
      least = TEAM ? told_by_all() : float_below(bound);
    }
    if constexpr (TEAM) least = fmaxf(least, told_by_all());
    const bool none = __ballot(most > least) == 0;
    if (none && (n == 0 || v + kStep < v1)) continue;
    // What can be among the k best, side by side.  Within a batch the order is another: once
    // the bound has risen in it, what equals the bound passes too.
    float kth = least;
    auto flush = [&]() {
      wave_sync();
      if (lane < n) {
        const uint64_t x = found[wave][lane];
        found[wave][lane] = key_of(__uint_as_float((uint32_t)(x >> 32)), (int)(uint32_t)x);
      }
      wave_sync();
      if (n > kFew) {
        merge(best, found[wave], merged[wave], n, a.k, lane);
      } else {
        for (int q = 0; q < n; ++q) insert(best, found[wave][q], lane);
      }
      n = 0;
      kth = fmaxf(least, logit_of(lane_value64(best, a.k - 1)));
      if (TEAM && lane == 0) told[wave] = fmaxf(told[wave], logit_of(lane_value64(best, share - 1)));
    };
#pragma unroll
    for (int j = 0; j < kVecs; ++j) {
      if (__ballot(m[j] > least) == 0) continue;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        uint64_t pass = __ballot(z[j][i] > least);
        if (pass == 0) continue;
        if (n + __popcll(pass) > 64) {
          flush();
          least = float_below(kth);
          pass = __ballot(z[j][i] > least);
        }
        const int at = __builtin_amdgcn_mbcnt_hi((uint32_t)(pass >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)pass, n));
        if (pass >> lane & 1)
          found[wave][at] = (uint64_t)__float_as_uint(z[j][i]) << 32 | (uint32_t)((v + 64 * j + lane) * PER + i);
        n += __popcll(pass);
      }
    }
    if (n >= kEnough || v + kStep >= v1) flush();
    least = kth;
  }
  // over the wave
  const float all = max_over(top, 64);
  sum = sum_over(exp.scaled(sum, (double)top - (double)all), 64);
  const int64_t at = (int64_t)row * a.segs + seg;
  if (lane == 0) {
    a.tops[at] = all;
    a.sums[at] = sum;
  }
  if (lane < a.k) {
    a.cand_z[at * a.k + lane] = logit_of(best);
    a.cand_y[at * a.k + lane] = best ? token_of(best) : -1;
  }
}

// A candidate of the last stage: a higher score is better, then a lower id, which is the
// beam above the token above a bit; score -infinity: none.  The bit: the next lower float as a
// logit would have the same score.
struct Cand {
  double s;
  uint64_t id;
};
__device__ __forceinline__ bool better(const Cand& p, const Cand& q) {
  return (p.s > q.s) | ((p.s == q.s) & (p.id < q.id));
}
__device__ __forceinline__ uint64_t id_of(int w, int y) { return (uint64_t)(uint32_t)w << 32 | (uint32_t)y << 1; }
constexpr int kPick = 512;         // threads
constexpr int kListed = 1024;      // candidates that can be ranked side by side
constexpr int kMaxLists = 1024;    // lists of a group: plan_beam()
static_assert(kPick / 64 * kMaxBeams <= kListed && kMaxBeams <= 128, "the waves' lists, and the bound's rank");

// -infinity by way of vector registers: as a scalar one this compiler (ROCm 7.2) makes it
// s_mov_b64 with a 64-bit literal, which the instruction does not have, and it arrives as 0.
__device__ __forceinline__ double no_score() {
  double x = -INFINITY;
  asm volatile("" : "+v"(x));
  return x;
}

// The normalisers, then the k best of the rows' lists.  Bound by latency, a few loads one
// after the other, so candidates are only looked at where they can be chosen: every thread
// takes the best of some lists' first entries; the k-th best of these bounds the group's
// k-th best from below, and only lists that begin at or above it are read.  All that these
// hold bounds it again (one beam far ahead of the others has k better ones than the second
// beam's best), and what is not below (about k, unless many are equal) is ranked by counting.
// Where that is more than fits, each wave keeps a sorted list instead, and these are ranked.
// Lists go by logits, and scores may be equal where logits are not (of 1e30, or of logits near
// 1e-20): then the beams that have the k-th best score are gone through once more for it.
// 6.7 us for 128 groups of 8 x 4 lists of 8, 7.8 for 17 of 12 x 20 of 24, 5.6 for one of 4 x 125 of
// 4; launch and end are 3.4 of each.
__global__ __launch_bounds__(kPick) void beam_pick_kernel(BeamArgs a) {
  constexpr int kWaves = kPick / 64;
  __shared__ double lse[kMaxBeams];              // NaN: the beam offers nothing
  __shared__ float score[kMaxBeams];
  __shared__ Cand listed[kListed];
  __shared__ float heads[kPick];
  __shared__ uint16_t open[kMaxLists];
  __shared__ int count, opened, merges, above, passing[kPick / 64];
  __shared__ uint32_t over[2], tied[2];          // beams, a bit each
  __shared__ double kth;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = blockIdx.x, k = a.k;
  const int per_row = a.segs * k, lists = a.width * a.segs, total = a.width * per_row;
  const int64_t first = (int64_t)g * a.width * per_row;
  // Candidate e of list l.
  auto entry = [&](int l, int e) { return first + l * k + e; };
  auto candidate = [&](int w, float z, int y) {
    Cand c{no_score(), id_of(w, y)};
    const double norm = lse[w];
    if (norm == norm && y >= 0) c.s = (double)score[w] + ((double)z - norm);
    return c;
  };
  auto with_bit = [&](Cand c, float z) {
    const int w = (int)(c.id >> 32);
    c.id |= candidate(w, float_below(z), 0).s == c.s;
    return c;
  };
  auto ended = [&](int w) {                      // a beam that has ended, as a candidate
    Cand c{no_score(), id_of(w, a.eos)};
    if (a.eos >= 0 && w < a.width) {
      const float s = a.scores[g * a.width + w];
      if (fabsf(s) < INFINITY && a.last[g * a.width + w] == a.eos) c.s = s;
    }
    return c;
  };
  // Normalisers: as many lanes (a power of two) per row as there are for all rows at once.
  const Exp exp;
  int lg = 6;
  while (lg > 0 && ((1 << (lg - 1)) >= a.segs || a.width << lg > kPick)) --lg;
  const int lanes = 1 << lg, rows_at_once = 64 >> lg, sub = lane & (lanes - 1);
  // Threads' own entries, in the order of all lists' first entries, then all second ones ..
  const int mine = min((int)threadIdx.x, total - 1);
  int l0 = mine, e0 = 0;
  float z0;
  int y0;
  if (threadIdx.x == 0) count = opened = merges = above = tied[0] = tied[1] = 0;
  for (int w0 = wave * rows_at_once, trip = 0; trip == 0 || w0 < a.width; w0 += kWaves * rows_at_once, ++trip) {
    const int w = w0 + (lane >> lg), row = g * a.width + min(w, a.width - 1);
    // Every lane's first two segments before anything waits, then the others.  (What is read
    // of a beam that is not live is not used.)
    const float* tops = a.tops + (int64_t)row * a.segs;
    const double* sums = a.sums + (int64_t)row * a.segs;
    const int i0 = min(sub, a.segs - 1), i1 = min(sub + lanes, a.segs - 1);
    const float s = a.scores[row], t0 = tops[i0], t1 = tops[i1];
    const double x0 = sums[i0], x1 = sums[i1];
    const bool live = beam_live(a, row);
    if (trip == 0) {
      if (lists < kPick) {
        e0 = mine / lists;
        l0 = mine - e0 * lists;
      }
      z0 = a.cand_z[entry(l0, e0)];
      y0 = a.cand_y[entry(l0, e0)];
    }
    float top = __builtin_elementwise_maximum(t0, t1);
#pragma unroll 4
    for (int i = sub + 2 * lanes; i < a.segs; i += lanes) top = __builtin_elementwise_maximum(top, tops[i]);
    top = max_over(top, lanes);
    double sum = sub < a.segs ? exp.scaled(x0, (double)t0 - (double)top) : 0.0;
    if (sub + lanes < a.segs) sum += exp.scaled(x1, (double)t1 - (double)top);
#pragma unroll 4
    for (int i = sub + 2 * lanes; i < a.segs; i += lanes) sum += exp.scaled(sums[i], (double)tops[i] - (double)top);
    sum = sum_over(sum, lanes);
    if (sub == 0 && w < a.width) {
      lse[w] = live && top < INFINITY ? (double)top + log(sum) : NAN;
      score[w] = s;
    }
  }
  __syncthreads();
  double head = no_score();
  if ((int)threadIdx.x < total) head = candidate(l0 / a.segs, z0, y0).s;
  const double own = head;
  for (int l = threadIdx.x + kPick; l < lists; l += kPick)
    head = fmax(head, candidate(l / a.segs, a.cand_z[entry(l, 0)], a.cand_y[entry(l, 0)]).s);
  // A bound that k of the threads' candidates are not below, from the maxima of 64 groups (of
  // threads 64 apart: neighbours often have the same beam) while k is far below that, of 128
  // otherwise.  A step of the search takes three counts of 64, or six.
  auto kth_of = [&](double x) {
    float h = (float)x;                          // not above the double
    if ((double)h > x) h = float_below(h);
    __syncthreads();
    heads[threadIdx.x] = h;
    __syncthreads();
    float most[2] = {heads[lane], heads[64 + lane]};
#pragma unroll
    for (int i = 2; i < kWaves; ++i) most[i & 1] = fmaxf(most[i & 1], heads[64 * i + lane]);
    if (k > 24) return (double)kth_bound<2>(most, k);
    const float one[1] = {fmaxf(most[0], most[1])};
    return (double)kth_bound<2>(one, k);
  };
  double least_score = kth_of(head);
  for (int l = threadIdx.x; l < lists; l += kPick) {
    const double s = l < kPick && e0 == 0 ? own : candidate(l / a.segs, a.cand_z[entry(l, 0)], a.cand_y[entry(l, 0)]).s;
    if (s >= least_score && s > -INFINITY) open[atomicAdd(&opened, 1)] = (uint16_t)l;
  }
  if (wave == 0 && a.eos >= 0) {
    const Cand c = ended(lane);
    if (fabs(c.s) < INFINITY) listed[atomicAdd(&count, 1)] = c;
    const uint64_t all = __ballot(fabs(c.s) < INFINITY);
    if (lane < 2) over[lane] = (uint32_t)(all >> 32 * lane);
  }
  __syncthreads();
  // The open lists in blocks of `deep` entries of each, as many as there are threads for.
  const int lists_open = opened, deep = max(1, kPick / max(1, lists_open)), block = lists_open * deep;
  auto opened_entry = [&](int i, int at, float* z) {
    const int l = open[i % lists_open], e = at + i / lists_open;
    if (e >= k) return Cand{no_score(), 0};
    *z = a.cand_z[entry(l, e)];
    return candidate(l / a.segs, *z, a.cand_y[entry(l, e)]);
  };
  Cand first_one{no_score(), 0};                 // of the first block
  float first_z = 0.f, z;
  if ((int)threadIdx.x < block) first_one = opened_entry(threadIdx.x, 0, &first_z);
  if (lists_open * k > 2 * kMaxBeams) {          // a closer bound
    head = first_one.s;
    for (int i = threadIdx.x + kPick; i < block; i += kPick) head = fmax(head, opened_entry(i, 0, &z).s);
    least_score = fmax(least_score, kth_of(head));
  }
  for (int at = 0; at < k && lists_open > 0; at += deep) {
    bool more = false;                           // a list's last entry here passes
    for (int i = threadIdx.x; i < block; i += kPick) {
      z = first_z;
      Cand c = at == 0 && i < kPick ? first_one : opened_entry(i, at, &z);
      if (c.s >= least_score && c.s > -INFINITY) {
        more |= i >= block - lists_open;
        c = with_bit(c, z);
        if (c.id & 1) merges = 1;
        const int to = atomicAdd(&count, 1);
        if (to < kListed) listed[to] = c;
      }
    }
    if (!__syncthreads_or(more)) break;          // the lists are sorted
  }
  __syncthreads();
  int n = count;
  if (n > kListed) {
    __syncthreads();
    if (threadIdx.x == 0) count = 0;
    Cand best{no_score(), ~0ull}, least = best;
    auto offer = [&](const Cand& c, bool some) {
      uint64_t pass = __ballot(some && better(c, least));
      while (pass) {
        const int l = __ffsll((unsigned long long)pass) - 1;
        pass &= pass - 1;
        const Cand x{lane_value64(c.s, l), lane_value64(c.id, l)};
        if (!better(x, least)) continue;
        const int pos = __popcll(__ballot(better(best, x)));
        const Cand b{from_below64(best.s), from_below64(best.id)};
        if (lane >= pos) best = lane == pos ? x : b;
        least = Cand{lane_value64(best.s, k - 1), lane_value64(best.id, k - 1)};
      }
    };
    for (int i = wave * 64; i < total; i += kPick) {
      const int at = min(i + lane, total - 1);
      const float z = a.cand_z[first + at];
      const Cand c = with_bit(candidate(at / per_row, z, a.cand_y[first + at]), z);
      offer(c, i + lane < total && c.s > -INFINITY);
    }
    if (a.eos >= 0 && wave == 0) {
      const Cand c = ended(lane);
      offer(c, fabs(c.s) < INFINITY);
    }
    __syncthreads();
    if (lane < k && fabs(best.s) < INFINITY) listed[atomicAdd(&count, 1)] = best;
    __syncthreads();
    n = count;
  }
  // Eight threads to a candidate count what is better.
  for (int i0 = 0; i0 < n; i0 += kPick / 8) {
    const int i = i0 + (threadIdx.x >> 3);
    const Cand c = listed[min(i, n - 1)];
    uint32_t rank = 0, other;
#pragma unroll 4
    for (int j = threadIdx.x & 7; j < n; j += 8) rank += better(listed[j], c);
    halves_of<1>(rank, &rank, &other);
    rank += other;
    halves_of<2>(rank, &rank, &other);
    rank += other;
    halves_of<4>(rank, &rank, &other);
    rank += other;
    if (i < n && (threadIdx.x & 7) == 0 && (int)rank < k) {
      const int64_t at = (int64_t)g * k + rank;
      a.parents[at] = (int32_t)(c.id >> 32);
      a.tokens[at] = (int32_t)((uint32_t)c.id >> 1);
      a.new_scores[at] = (float)c.s;
      if ((int)rank == k - 1) kth = c.s;
    }
  }
  // What is better than the k-th best score is listed, and where that score is (a beam that has
  // it has it listed too): of the tokens that have it the lowest, beam after beam.  A row of
  // 128256 takes 60 us if its last token is the one; most often there are some among the first.
  if (merges && n >= k) {
    __syncthreads();
    if (threadIdx.x == 0) merges = 0;
    __syncthreads();
    const double score_k = kth;
    for (int i = threadIdx.x; i < n; i += kPick) {
      const Cand c = listed[i];
      if (c.s > score_k) atomicAdd(&above, 1);
      if (c.s == score_k) atomicOr(&tied[c.id >> 37], 1u << (c.id >> 32 & 31));
      if (c.s == score_k && (c.id & 1)) merges = 1;
    }
    __syncthreads();
    int at = merges ? above : k;                 // not where only better ones' neighbours merge
    auto put = [&](int w, int y, int to) {
      a.parents[(int64_t)g * k + to] = w;
      a.tokens[(int64_t)g * k + to] = y;
      a.new_scores[(int64_t)g * k + to] = (float)score_k;
    };
    for (int w = 0; w < a.width && at < k; ++w) {
      if (!(tied[w >> 5] >> (w & 31) & 1)) continue;
      if (a.eos >= 0 && (over[w >> 5] >> (w & 31) & 1)) {
        if (threadIdx.x == 0) put(w, a.eos, at);
        ++at;
        continue;
      }
      const int64_t row = (int64_t)(g * a.width + w) * a.row_stride;
      constexpr int kAhead = 8;
      for (int y0 = threadIdx.x; y0 - (int)threadIdx.x < a.vocab && at < k; y0 += kAhead * kPick) {
        float x[kAhead];
        uint32_t has = 0;
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
          const int64_t from = row + min(y0 + j * kPick, a.vocab - 1);
          x[j] = a.is_bf16 ? (float)((const bf16*)a.logits)[from] : ((const float*)a.logits)[from];
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
          const int y = y0 + j * kPick;
          has |= (uint32_t)(y < a.vocab && x[j] > -INFINITY && candidate(w, x[j], y).s == score_k) << j;
        }
        if (!__syncthreads_or(has)) continue;
        for (int j = 0; j < kAhead && at < k; ++j) {
          const uint64_t all = __ballot(has >> j & 1);
          if (lane == 0) passing[wave] = __popcll(all);
          __syncthreads();
          int to = at + __popcll(all & ((1ull << lane) - 1));
          for (int i = 0; i < kWaves; ++i) {
            if (i < wave) to += passing[i];
            at += passing[i];
          }
          if ((has >> j & 1) && to < k) put(w, y0 + j * kPick, to);
          __syncthreads();
        }
      }
    }
  }
  for (int i = n + threadIdx.x; i < k; i += kPick) {
    const int64_t at = (int64_t)g * k + i;
    a.parents[at] = a.tokens[at] = -1;
    a.new_scores[at] = -INFINITY;
  }
}

}  // namespace

// Segments: about 4096 waves' worth of rows' pieces fill the chip (4 to a SIMD), none below 64
// vectors (one load of each lane), at most kMaxLists in a group, each a list that one
// work-group picks from, and 128 in a row, whose normaliser takes two loads of 64 lanes.  us,
// with 2048 / 4096 / 6144 / 8192 waves: 17 x 12 x 50001 bf16, k 24, 28.3 / 24.6 / 25.1 / 25.4; 3 x 64 x
// 32000, k 64, 32.5 / 27.2 / 27.1 / 27.2; 128 x 8 x 128256 112 / 109 / 111 / 113.  With 512 / 1024 /
// 2048 lists: 1 x 32 x 128256 bf16, k 64, 34.0 / 27.6 / 28.0; 1 x 64 x 128000, k 64, 46.8 / 36.9 / 35.6;
// 1 x 16 x 128256, k 16, 19.6 / 17.4 / 20.0.  With 64 / 128 / 256 segments: 8 x 128256, k 8, 14.1 /
// 13.4 / 17.2; 4 x 128256, k 4, - / 11.6 / 13.5.
// Many rows have few segments: four, for a team, where 16 or more are chosen from 1000 vectors or
// more (with less than four / four: 90 x 24 x 32000, k 24, 91.6 / 75.6; 128 x 64 x 8000 bf16, k 64,
// 107 / 99; but 150 x 10 x 50001, k 10, 70.2 / 73.0; 128 x 64 x 2000, k 32, 39.7 / 52.5).
void plan_beam(BeamArgs* a) {
  const int per = a->is_bf16 ? 8 : 4;
  const int64_t rows = (int64_t)a->groups * a->width;
  const int64_t vectors = (a->vocab + per - 1) / per;
  const int64_t want = std::max<int64_t>(a->k >= 16 && vectors >= 1000 ? kTeam : 1, 4096 / rows);
  const int64_t most = (vectors + 63) / 64;
  const int64_t segs = std::min<int64_t>({want, most, 128, kMaxLists / a->width});
  a->seg = (int)((vectors + 64 * segs - 1) / (64 * segs) * 64);
  a->segs = (int)((vectors + a->seg - 1) / a->seg);
}

size_t beam_scratch(BeamArgs* a, char* base) {
  const size_t n = (size_t)a->groups * a->width * a->segs;
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  size_t off = 0;
  a->sums = (double*)(base + off);
  off += up(n * 8);
  a->tops = (float*)(base + off);
  off += up(n * 4);
  a->cand_z = (float*)(base + off);
  off += up(n * a->k * 4);
  a->cand_y = (int32_t*)(base + off);
  off += up(n * a->k * 4);
  return off;
}

hipError_t launch_beam(const BeamArgs& a, hipStream_t s) {
  const int64_t rows = (int64_t)a.groups * a.width;
  auto scan = [&](auto kernel, int64_t blocks) {
    if (blocks > kMaxGrid) return hipErrorInvalidValue;
    kernel<<<(unsigned)blocks, 64 * kTeam, 0, s>>>(a);
    return hipGetLastError();
  };
  const int64_t teams = rows * ((a.segs + kTeam - 1) / kTeam), pieces = (rows * a.segs + kTeam - 1) / kTeam;
  // Up to 8 best the team's words cost more than they save (us: 4 x 32000, k 4, 13.2 alone and 13.5
  // as teams; 8 x 128256, k 8, 15.6 and 15.9; 16 x 128256, k 16, 20.9 and 20.6; 17 x 12 x 50001, k 24,
  // 29.2 and 27.6; 3 x 64 x 32000, k 64, 36.7 and 30.8; 4 x 64 x 128256 bf16, k 64, 69.5 and 57.6).
  const bool team = a.segs >= kTeam && a.k > 8;
  const hipError_t e = a.is_bf16 ? team ? scan(beam_scan_kernel<bf16, true>, teams)
                                        : scan(beam_scan_kernel<bf16, false>, pieces)
                                 : team ? scan(beam_scan_kernel<float, true>, teams)
                                        : scan(beam_scan_kernel<float, false>, pieces);
  if (e != hipSuccess) return e;
  beam_pick_kernel<<<a.groups, kPick, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace spec
