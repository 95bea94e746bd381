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

namespace spec {

namespace {

constexpr int64_t kMaxGrid = 0xffffffffll / 1024;

// 2^t for -1100 <= t <= 1000, relative error below 1e-14: 2^n times the series of
// exp(f ln 2), |f| <= 1/2, cut where the next term, (ln 2 / 2)^12 / 12!, is 6e-15.
__device__ __forceinline__ double exp2_double(double t) {
  constexpr double L = 0.69314718055994530942;
  constexpr double C[12] = {1.0,
                            L,
                            L * L / 2,
                            L * L * L / 6,
                            L * L * L * L / 24,
                            L * L * L * L * L / 120,
                            L * L * L * L * L * L / 720,
                            L * L * L * L * L * L * L / 5040,
                            L * L * L * L * L * L * L * L / 40320,
                            L * L * L * L * L * L * L * L * L / 362880,
                            L * L * L * L * L * L * L * L * L * L / 3628800,
                            L * L * L * L * L * L * L * L * L * L * L / 39916800};
  const double n = rint(t), f = t - n;
  double y = C[11];
#pragma unroll
  for (int i = 10; i >= 0; --i) y = fma(y, f, C[i]);
  return ldexp(y, (int)n);
}

constexpr double kLog2e = 1.44269504088896340736;
constexpr float kLowest = -3.4028234663852886e38f;

// A wave's running list of the k best, one entry per lane, best first; entries past the
// filled ones hold -infinity.
struct List {
  float z;
  int y;
};

// Lane i gets lane i - 1's x.
__device__ __forceinline__ int from_below(int x) {
  return __builtin_amdgcn_update_dpp(x, x, 0x138, 0xf, 0xf, false);      // wave_shr:1
}

__device__ __forceinline__ float lane_value(float x, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane));
}

// Put (z, y) into the list, behind entries that are as good: a caller that comes to tokens in
// ascending order so keeps the lower one of equal logits first.
__device__ __forceinline__ void insert(List& l, float z, int y, int lane) {
  const int pos = __popcll(__ballot(l.z >= z));
  const float zb = __int_as_float(from_below(__float_as_int(l.z)));
  const int yb = from_below(l.y);
  l.z = lane < pos ? l.z : lane == pos ? z : zb;
  l.y = lane < pos ? l.y : lane == pos ? y : yb;
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
  // Elements v * PER ..; what is past the row reads as -infinity.
  __device__ __forceinline__ void load(int v, float* z) const {
    const int e0 = v * PER;
    if (e0 + PER <= vocab) {
      const i32x4 x = *(const Loose*)(row + e0);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (PER == 4) {
          z[i] = __uint_as_float((uint32_t)x[i]);
        } else {
          z[2 * i] = __uint_as_float((uint32_t)x[i] << 16);
          z[2 * i + 1] = __uint_as_float((uint32_t)x[i] & 0xffff0000u);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < PER; ++i) z[i] = e0 + i < vocab ? (float)row[e0 + i] : -INFINITY;
    }
  }
};

template <class T>
__global__ __launch_bounds__(256) void beam_scan_kernel(BeamArgs a) {
  constexpr int PER = Vectors<T>::PER;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t id = (int64_t)blockIdx.x * 4 + wave;
  const int row = (int)(id / a.segs), seg = (int)(id % a.segs);
  if (row >= a.groups * a.width || !beam_live(a, row)) return;
  const T* p = (const T*)a.logits + row * a.row_stride;
  const Vectors<T> vec{p, a.vocab};
  const int vectors = (a.vocab + PER - 1) / PER;
  const int v0 = seg * a.seg, v1 = min(vectors, v0 + a.seg);
  float top = kLowest;          // the lane's reference: at least a logit of its own less 600
  double sum = 0.0;
  List best{-INFINITY, -1};
  float least = -INFINITY;      // of the k best
  for (int v = v0; v < v1; v += 64) {
    float z[PER];
    if (v + lane < v1) {
      vec.load(v + lane, z);
    } else {
#pragma unroll
      for (int i = 0; i < PER; ++i) z[i] = -INFINITY;
    }
    float m = z[0];
#pragma unroll
    for (int i = 1; i < PER; ++i) m = __builtin_elementwise_maximum(m, z[i]);   // a NaN when there is one
    // Terms relative to `top`: doubles hold e^600, and what is e^-690 of `top` counts as that.
    if (__ballot(!(m <= top + 600.f) || top < -1e37f)) {
      if (!(m <= top)) {
        sum = m - top > 690.f ? 0.0 : sum * exp2_double(((double)top - (double)m) * kLog2e);
        top = m;
      }
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const double d = (double)z[i] - (double)top;
        sum += d != d ? d : d < -690.0 ? 0.0 : exp2_double(d * kLog2e);
      }
    } else {
#pragma unroll
      for (int i = 0; i < PER; ++i)
        sum += exp2_double(((double)fmaxf(z[i], top - 690.f) - (double)top) * kLog2e);
    }
    uint64_t pass = __ballot(m > least || m != m);
    while (pass) {
      const int l = __ffsll((unsigned long long)pass) - 1;
      pass &= pass - 1;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const float x = lane_value(z[i], l);
        if (x > least) {
          insert(best, x, (v + l) * PER + i, lane);
          least = lane_value(best.z, a.k - 1);
        }
      }
    }
  }
  // over the wave
#pragma unroll
  for (int x = 32; x >= 1; x >>= 1) {
    const float t = __shfl_xor(top, x);
    const double s = __shfl_xor(sum, x);
    const float m = __builtin_elementwise_maximum(top, t);
    auto scaled = [&](double q, float from) {
      const double d = (double)from - (double)m;
      return d != d ? d : d < -690.0 ? 0.0 : q * exp2_double(d * kLog2e);
    };
    sum = scaled(sum, top) + scaled(s, t);
    top = m;
  }
  const int64_t at = (int64_t)row * a.segs + seg;
  if (lane == 0) {
    a.tops[at] = top;
    a.sums[at] = sum;
  }
  if (lane < a.k) {
    a.cand_z[at * a.k + lane] = best.z;
    a.cand_y[at * a.k + lane] = best.y;
  }
}

// A candidate of the last stage: better is a higher score, then a lower beam, then a lower token.
struct Cand {
  double s;
  int w, y;
};
__device__ __forceinline__ bool better(const Cand& p, const Cand& q) {
  return p.s > q.s || (p.s == q.s && (p.w < q.w || (p.w == q.w && p.y < q.y)));
}
__device__ __forceinline__ double readlane_double(double x, int lane) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)b, lane), hi = __builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), lane);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double double_from_below(double x) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = from_below((int)(uint32_t)b), hi = from_below((int)(uint32_t)(b >> 32));
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

constexpr int kPickWaves = 8;

__global__ __launch_bounds__(64 * kPickWaves) void beam_pick_kernel(BeamArgs a) {
  __shared__ double lse[kMaxBeams];              // NaN: the beam offers nothing
  __shared__ Cand lists[kPickWaves * kMaxBeams];
  __shared__ int count;
  __shared__ Cand kth[kPickWaves];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = blockIdx.x, k = a.k;
  if (threadIdx.x == 0) count = 0;
  // normalisers
  for (int w = wave; w < a.width; w += kPickWaves) {
    const int row = g * a.width + w;
    double v = NAN;
    if (beam_live(a, row)) {
      const float* tops = a.tops + (int64_t)row * a.segs;
      const double* sums = a.sums + (int64_t)row * a.segs;
      float top = -INFINITY;
      for (int i = lane; i < a.segs; i += 64) top = __builtin_elementwise_maximum(top, tops[i]);
#pragma unroll
      for (int x = 32; x >= 1; x >>= 1) top = __builtin_elementwise_maximum(top, __shfl_xor(top, x));
      double sum = 0.0;
      for (int i = lane; i < a.segs; i += 64) {
        const double d = (double)tops[i] - (double)top;
        sum += d != d ? d : d < -690.0 ? 0.0 : sums[i] * exp2_double(d * kLog2e);
      }
#pragma unroll
      for (int x = 32; x >= 1; x >>= 1) sum += __shfl_xor(sum, x);
      v = top < INFINITY ? (double)top + log(sum) : NAN;
    }
    if (lane == 0) lse[w] = v;
  }
  __syncthreads();
  // each wave's k best
  // -infinity by way of vector registers: as a scalar one this compiler (ROCm 7.2) makes it
  // s_mov_b64 with a 64-bit literal, which the instruction does not have, and it arrives as 0.
  double none = -INFINITY;
  asm volatile("" : "+v"(none));
  Cand best{none, 0x7fffffff, 0x7fffffff}, least = best;
  auto offer = [&](const Cand& c, bool some) {
    uint64_t pass = __ballot(some && better(c, least));
    while (pass) {
      const int l = __ffsll((unsigned long long)pass) - 1;
      pass &= pass - 1;
      const Cand n{readlane_double(c.s, l), __builtin_amdgcn_readlane(c.w, l), __builtin_amdgcn_readlane(c.y, l)};
      if (!better(n, least)) continue;
      const int pos = __popcll(__ballot(better(best, n)));
      const Cand b{double_from_below(best.s), from_below(best.w), from_below(best.y)};
      if (lane >= pos) best = lane == pos ? n : b;
      least = Cand{readlane_double(best.s, k - 1), __builtin_amdgcn_readlane(best.w, k - 1),
                   __builtin_amdgcn_readlane(best.y, k - 1)};
    }
  };
  const int per_row = a.segs * k, total = a.width * per_row;
  for (int i = wave * 64; i < total; i += 64 * kPickWaves) {
    const int at = i + lane, w = min(at, total - 1) / per_row, row = g * a.width + w;
    Cand c{};
    bool some = false;
    if (at < total && lse[w] == lse[w]) {
      const int64_t from = (int64_t)row * per_row + at - w * per_row;
      const float z = a.cand_z[from];
      c = Cand{(double)a.scores[row] + ((double)z - lse[w]), w, a.cand_y[from]};
      some = z > -INFINITY;
    }
    offer(c, some);
  }
  if (a.eos >= 0 && wave == 0) {                 // beams that have ended
    const int row = g * a.width + min(lane, a.width - 1);
    const float s = a.scores[row];
    offer(Cand{(double)s, lane, a.eos}, lane < a.width && fabsf(s) < INFINITY && a.last[row] == a.eos);
  }
  // The best k-th of any wave bounds the group's from below; what passes is ranked.
  if (lane == 0) kth[wave] = least;
  __syncthreads();
  Cand floor = kth[0];
#pragma unroll
  for (int i = 1; i < kPickWaves; ++i)
    if (better(kth[i], floor)) floor = kth[i];
  if (lane < k && best.s > -INFINITY && !better(floor, best)) lists[atomicAdd(&count, 1)] = best;
  __syncthreads();
  const int n = count;
  for (int i = threadIdx.x; i < n; i += 64 * kPickWaves) {
    const Cand c = lists[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += better(lists[j], c);
    if (rank < k) {
      const int64_t at = (int64_t)g * k + rank;
      a.parents[at] = c.w;
      a.tokens[at] = c.y;
      a.new_scores[at] = (float)c.s;
    }
  }
  for (int i = n + threadIdx.x; i < k; i += 64 * kPickWaves) {
    const int64_t at = (int64_t)g * k + i;
    a.parents[at] = a.tokens[at] = -1;
    a.new_scores[at] = -INFINITY;
  }
}

}  // namespace

// Segments: about 4096 waves' worth of rows' pieces fill the chip, none below 64 vectors
// (one load of each lane), at most 256 of a row.
void plan_beam(BeamArgs* a) {
  const int per = a->is_bf16 ? 8 : 4;
  const int64_t rows = (int64_t)a->groups * a->width;
  const int64_t vectors = (a->vocab + per - 1) / per;
  const int64_t want = std::max<int64_t>(1, 4096 / rows), most = (vectors + 63) / 64;
  const int64_t segs = std::min<int64_t>({want, most, 256});
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
  const int64_t waves = (int64_t)a.groups * a.width * a.segs;
  if ((waves + 3) / 4 > kMaxGrid) return hipErrorInvalidValue;
  const unsigned grid = (unsigned)((waves + 3) / 4);
  if (a.is_bf16) beam_scan_kernel<bf16><<<grid, 256, 0, s>>>(a);
  else beam_scan_kernel<float><<<grid, 256, 0, s>>>(a);
  if (const hipError_t e = hipGetLastError()) return e;
  beam_pick_kernel<<<a.groups, 64 * kPickWaves, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace spec
