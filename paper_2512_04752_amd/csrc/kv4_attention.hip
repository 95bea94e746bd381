// Tree attention over the 4-bit paged KV cache.
//
// Query row r of (sample b, kv head g) is node r / G with query head g*G + r % G
// (G query heads share a KV head).  It sees every committed key and, of the
// step's own keys, its ancestors (trees) or the ones up to itself (runs).
//
// A wave takes a tile of 32 rows through 32 keys at a time, with the products
// transposed so that a lane owns one query row (its softmax state and output
// column never leave the lane and its partner, lane ^ 32):
//
//   S^T (32 keys x 32 rows)  = K . Q^T     v_mfma_f32_32x32x16_bf16
//   O^T (dims x 32 rows)    += V^T . P^T   the same, P straight from S^T's registers
//
// The cache is stored in the order of those operands.  Four bits are little
// enough to need no staging: a lane loads its own 16 bytes of codes (K: 32 dims
// of one key; V: its dims of 8 keys, one word each), 1 KB contiguous per wave
// and load, and turns a byte into two bf16 numbers with one conversion.  K's
// power of two goes into that conversion (a lane's 32 dims share one); V's is
// the same for all dims of a key, so it scales the key's probability instead.
// So K and V enter the products exactly; probabilities are rounded to bf16, as
// in the bf16 cache's kernels.  There is no LDS traffic and no barrier until a
// wave's last key; loads run a few blocks ahead in registers.
//
// Row r of K's operand takes key kappa(r) of the block, bits 2 and 3 of r
// swapped: S^T's accumulators of lane half h are then 8 consecutive keys each
// (16 k + 8 h ..), which is an octet of V's layout.
//
// A work-group has four waves: RT row tiles, and 4 / RT waves per tile that deal
// its keys in blocks and merge through LDS at the end.
#include <math.h>

#include <atomic>

#include "kv4.h"

namespace spec {

namespace {

constexpr int KBLK = 32;
constexpr int kWaves = 4;

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// The running output is relative to a reference maximum that moves only when a
// row's maximum outgrows it by this many binary orders (a wave-uniform test).
constexpr float kRescaleSlack = 8.f;

// max / sum of a value and its copy in lane ^ 32.
__device__ __forceinline__ float max_xor32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_xor32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Eight codes (a word) as bf16, times the power of two s.
__device__ __forceinline__ bf16x8 decode(uint32_t w, float s) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// One lane's share of a 32-key block.
template <int HD>
struct Block;
template <>
struct Block<128> {
  i32x4 k[2], v[2];        // k[j]: dims 32 (2j + h) .. of key kappa(r); v[k][i]: dim 32 i + r of octet 2k + h
  uint32_t ks;             // the key's four scale bytes
  i32x4 vs[2];             // value scales of the two octets
};
template <>
struct Block<64> {
  i32x4 k[1];
  i32x2 v[2];
  uint32_t ks;
  i32x4 vs[2];
};

template <int HD, int RT>
__global__ __launch_bounds__(256, 2) void kv4_attention_kernel(Kv4AttnArgs a, const AttnItem* items,
                                                               int n_items) {
  constexpr int KS = kWaves / RT;             // waves per row tile
  constexpr int NB = HD / 32;                 // 32-dim output blocks
  constexpr int NJ = HD / 64;                 // 16-byte key loads per lane
  constexpr int AHEAD = 2;                    // blocks in registers
  constexpr int PITCH = HD + 4;               // floats per merged row
  extern __shared__ __attribute__((aligned(16))) float smem[];

  const int per_xcd = gridDim.x >> 3;
  const int item = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
  if (item >= n_items) return;
  const AttnItem it = items[item];
  if (it.sample < 0) return;                  // padding of a shorter per-XCD list
  const SampleInfo si = a.v.samples[it.sample];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 31, h = lane >> 5;
  const int tile = w / KS, part = w % KS;
  const int G = a.n_heads / a.v.n_kv_heads;
  const int row0 = it.row0 + 32 * tile;

  const int grow = row0 + r;
  const int node = grow / G, head = it.kvh * G + grow % G;
  const bool row_ok = node < si.ntok;
  bf16x8 qf[HD / 16];
  {
    const bf16* qrow = a.q + (size_t)(si.tok0 + (row_ok ? node : 0)) * a.q_stride + (row_ok ? head : 0) * HD;
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        qf[4 * j + u] = *(const bf16x8*)(qrow + 32 * (2 * j + h) + 8 * u);
        if (!row_ok) qf[4 * j + u] = bf16x8{};
      }
  }
  // What the row sees: of a tree its ancestors, of a run the keys before `limit`.
  const bool runs = a.anc == nullptr;
  NodeSet anc;
  anc.clear();
  anc.w0 = 1ull;
  if (!runs && row_ok) anc.load(a.anc + (size_t)(si.tok0 + node) * kAncWords);
  const int limit = si.seq_len + min(node, si.ntok - 1) + 1;

  // The tile's keys end with its last row's, and blocks past `mask_from` are masked.
  int key1 = it.key1, mask_from = si.seq_len;
  if (runs) {
    const int last = min((row0 + 31) / G, si.ntok - 1);
    key1 = min(key1, si.seq_len + last + 1);
    mask_from = si.seq_len + min(row0 / G, si.ntok - 1) + 1;
  }
  mask_from = min(mask_from, key1);
  const int nblk = key1 > it.key0 ? (key1 - it.key0 + KBLK - 1) / KBLK : 0;
  const int mine = nblk > part ? (nblk - part + KS - 1) / KS : 0;

  const char* in_page = a.v.pool + ((int64_t)a.v.layer * a.v.n_kv_heads + it.kvh) * kv4_head_bytes(HD);
  const int32_t* table = a.v.table + si.kv_base;
  const int kappa = (r & 0x13) | ((r & 4) << 1) | ((r & 8) >> 1);
  const int k_off = h * 512 + kappa * 16, ks_off = kv4_kscale_at(HD) + kappa * (HD / 32);
  const int v_off = kv4_value_at(HD) + h * kv4_octet_bytes(HD) + r * (HD / 8);
  const int vs_off = kv4_vscale_at(HD) + 16 * h;

  auto first_key = [&](int t) { return it.key0 + (part + KS * t) * KBLK; };
  auto load = [&](Block<HD>& b, int t) {
    const int kb = first_key(t);
    const char* base = in_page + (int64_t)table[kb / kKv4Page] * a.v.page_bytes;
    const int half = kb / KBLK % 2;
    const char* codes = base + half * kv4_block_bytes(HD);
#pragma unroll
    for (int j = 0; j < NJ; ++j) b.k[j] = *(const i32x4*)(codes + k_off + j * 1024);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      b.v[k] = *(const decltype(b.v[0] + b.v[0])*)(codes + v_off + 2 * k * kv4_octet_bytes(HD));
      b.vs[k] = *(const i32x4*)(base + half * 64 + vs_off + 32 * k);
    }
    if constexpr (HD == 128) b.ks = *(const uint32_t*)(base + half * 128 + ks_off);
    else b.ks = *(const uint16_t*)(base + half * 64 + ks_off);
  };

  const float sl2 = 1.4426950408889634f / sqrtf((float)HD);   // log2(e) / sqrt(d)
  float m_run = -INFINITY, l_run = 0.f;
  f32x16 o[NB];
#pragma unroll
  for (int i = 0; i < NB; ++i) o[i] = f32x16{};

  auto compute = [&](const Block<HD>& b, int kb) {
    f32x16 s0 = f32x16{}, s1 = f32x16{};
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const float ks = __uint_as_float((b.ks >> (16 * j + 8 * h) & 255u) << 23);
#pragma unroll
      for (int u = 0; u < 4; u += 2) {
        s0 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(decode((uint32_t)b.k[j][u], ks), qf[4 * j + u], s0, 0, 0, 0);
        s1 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(decode((uint32_t)b.k[j][u + 1], ks), qf[4 * j + u + 1], s1, 0,
                                                     0, 0);
      }
    }
    f32x16 s = s0 + s1;                        // s[e]: key kb + 16 (e / 8) + 8 h + e % 8
    const bool mask = kb + KBLK > mask_from;
    if (mask) {
      const int t0 = kb - si.seq_len;
      const uint64_t lo = anc.word(t0), hi = anc.word(t0 + 31);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int key = kb + 16 * (e >> 3) + 8 * h + (e & 7);
        const int tt = key - si.seq_len;
        const uint64_t word = (tt >> 6) == (t0 >> 6) ? lo : hi;
        const bool in_tree = (tt < 0) | (bool)((word >> (tt & 63)) & 1ull);
        const bool seen = (key < key1) & (runs ? key < limit : in_tree);
        s[e] = seen ? s[e] : -INFINITY;
      }
    }
    float smax = s[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) smax = fmaxf(smax, s[e]);
    smax = max_xor32(smax);
    const float m_new = fmaxf(m_run, smax * sl2);
    if (__ballot(m_new > m_run + kRescaleSlack)) {
      const float alpha = m_new == -INFINITY ? 1.f : fast_exp2(m_run - m_new);
      l_run *= alpha;
#pragma unroll
      for (int i = 0; i < NB; ++i) o[i] *= alpha;
      m_run = m_new;
    }
    const float mb = m_run == -INFINITY ? 0.f : m_run;
    float psum = 0.f;
    bf16x8 pb[2];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float pe = fast_exp2(fmaf(s[e], sl2, -mb));
      psum += pe;
      const uint32_t sw = (uint32_t)b.vs[e >> 3][(e & 7) >> 1];
      float ps = pe * __uint_as_float(e & 1 ? sw & 0xffff0000u : sw << 16);
      if (mask) ps = s[e] == -INFINITY ? 0.f : ps;     // an unseen key's scale may be anything
      pb[e >> 3][e & 7] = (bf16)ps;
    }
    l_run += psum;
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < NB; ++i)
        o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(decode((uint32_t)b.v[k][i], 1.f), pb[k], o[i], 0, 0, 0);
  };

  Block<HD> blk[AHEAD];
#pragma unroll
  for (int u = 0; u < AHEAD; ++u)
    if (u < mine) load(blk[u], u);
  for (int t0 = 0; t0 < mine; t0 += AHEAD) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int t = t0 + u;
      if (t >= mine) break;
      compute(blk[u], first_key(t));
      if (t + AHEAD < mine) load(blk[u], t + AHEAD);
    }
  }
  l_run = sum_xor32(l_run);

  // Every wave leaves its 32 rows in LDS; a tile's waves then share its rows.
  float* own = smem + w * 32 * PITCH;
  float* ml = smem + kWaves * 32 * PITCH;      // [wave][32][2]
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int c = 0; c < 4; ++c)
      *(f32x4*)(own + r * PITCH + 32 * i + 8 * c + 4 * h) =
          f32x4{o[i][4 * c], o[i][4 * c + 1], o[i][4 * c + 2], o[i][4 * c + 3]};
  if (h == 0) {
    ml[(w * 32 + r) * 2] = m_run;
    ml[(w * 32 + r) * 2 + 1] = l_run;
  }
  __syncthreads();
  constexpr int LPR = HD / 8, RPP = 64 / LPR;  // lanes per row, rows per pass
  const bool split = it.nsplit > 1;
  const int slot = it.part + tile * it.nsplit;
#pragma unroll
  for (int p = 0; p < 32 / KS; p += RPP) {
    const int rr = part * (32 / KS) + p + lane / LPR, d = lane % LPR * 8;
    const int gr = row0 + rr, nd = gr / G;
    if (nd >= si.ntok) continue;
    float m = -INFINITY;
#pragma unroll
    for (int k = 0; k < KS; ++k) m = fmaxf(m, ml[((tile * KS + k) * 32 + rr) * 2]);
    float l = 0.f;
    f32x4 x0 = {0.f, 0.f, 0.f, 0.f}, x1 = x0;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      const float mk = ml[((tile * KS + k) * 32 + rr) * 2];
      const float f = mk == -INFINITY ? 0.f : fast_exp2(mk - m);
      const float* src = smem + ((tile * KS + k) * 32 + rr) * PITCH + d;
      l += f * ml[((tile * KS + k) * 32 + rr) * 2 + 1];
      x0 += f * *(const f32x4*)src;
      x1 += f * *(const f32x4*)(src + 4);
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    x0 *= inv;
    x1 *= inv;
    if (split) {
      float* dst = a.part_o + ((size_t)slot * 32 + rr) * HD + d;
      *(f32x4*)dst = x0;
      *(f32x4*)(dst + 4) = x1;
      if (d == 0) {
        a.part_ml[((size_t)slot * 32 + rr) * 2] = m;
        a.part_ml[((size_t)slot * 32 + rr) * 2 + 1] = l;
      }
    } else {
      bf16x8 y;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        y[j] = (bf16)x0[j];
        y[4 + j] = (bf16)x1[j];
      }
      *(bf16x8*)(a.out + ((size_t)(si.tok0 + nd) * a.n_heads + it.kvh * G + gr % G) * HD + d) = y;
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
  const CombineItem ci = a.comb[blockIdx.x];
  const int lane = threadIdx.x % LPR, rr = threadIdx.x / LPR;
  const int row = blockIdx.y * RPB + rr;
  const SampleInfo si = a.v.samples[ci.sample];
  const int G = a.n_heads / a.v.n_kv_heads;
  const int gr = ci.row0 + row, nd = gr / G;
  if (nd >= si.ntok) return;                   // a row's lanes lie in one wave: nobody waits for them
  const int ns = ci.nsplit;
  float M = -INFINITY;
  for (int sp = lane; sp < ns; sp += LPR) M = fmaxf(M, a.part_ml[((size_t)(ci.part0 + sp) * 32 + row) * 2]);
#pragma unroll
  for (int m = LPR / 2; m >= 1; m >>= 1) M = fmaxf(M, __shfl_xor(M, m));
  float L = 0.f;
  for (int sp = lane; sp < ns; sp += LPR) {
    const size_t slot = (size_t)(ci.part0 + sp) * 32 + row;
    const float ms = a.part_ml[slot * 2];
    const float f = ms == -INFINITY ? 0.f : fast_exp2(ms - M) * a.part_ml[slot * 2 + 1];
    wgt[rr][sp] = f;
    L += f;
  }
#pragma unroll
  for (int m = LPR / 2; m >= 1; m >>= 1) L += __shfl_xor(L, m);
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  const float* src = a.part_o + ((size_t)ci.part0 * 32 + row) * HD + 4 * lane;
  constexpr size_t STRIDE = (size_t)32 * HD;   // elements between consecutive ranges
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
  *(bf16x4*)(a.out + ((size_t)(si.tok0 + nd) * a.n_heads + ci.kvh * G + gr % G) * HD + 4 * lane) = v;
}

template <int HD, int RT>
hipError_t launch_tiles(const Kv4AttnArgs& a, const AttnItem* items, int n, hipStream_t s) {
  if (n == 0) return hipSuccess;
  constexpr int SMEM = kWaves * 32 * (HD + 4 + 2) * 4;
  const auto kernel = kv4_attention_kernel<HD, RT>;
  static std::atomic<uint64_t> configured{0};  // a bit per device
  int dev = 0;
  if (const hipError_t e = hipGetDevice(&dev)) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (!(configured.load() & bit)) {
    if (const hipError_t e = hipFuncSetAttribute((const void*)kernel,
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, SMEM))
      return e;
    configured.fetch_or(bit);
  }
  kernel<<<(n + 7) / 8 * 8, 64 * kWaves, SMEM, s>>>(a, items, n);
  return hipGetLastError();
}

template <int HD>
hipError_t launch_hd(const Kv4AttnArgs& a, hipStream_t s) {
  hipError_t e = launch_tiles<HD, 1>(a, a.items[0], a.n_items[0], s);
  if (e == hipSuccess) e = launch_tiles<HD, 2>(a, a.items[1], a.n_items[1], s);
  if (e == hipSuccess) e = launch_tiles<HD, 4>(a, a.items[2], a.n_items[2], s);
  if (e == hipSuccess && a.n_comb) {
    kv4_combine_kernel<HD><<<dim3(a.n_comb, 32 / (256 / (HD / 4))), 256, 0, s>>>(a);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

hipError_t launch_kv4_attention(const Kv4AttnArgs& a, hipStream_t s) {
  if (a.v.head_dim == 128) return launch_hd<128>(a, s);
  if (a.v.head_dim == 64) return launch_hd<64>(a, s);
  return hipErrorInvalidValue;
}

}  // namespace spec
