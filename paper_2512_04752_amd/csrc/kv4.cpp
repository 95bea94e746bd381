// Host side of the 4-bit paged KV cache: page tables, a step's plan (row octets,
// attention work items) and its one upload, and the launches of append, read,
// attend and commit.
#include <algorithm>
#include <cmath>
#include <new>
#include <string>
#include <vector>

#include "kv4_host.h"

using namespace spec;

namespace {

constexpr int kPartCap = 8192;          // partial tiles of 16 rows per step, at most
constexpr int kResident1 = 768;         // attention work-groups that fit the chip, a wave on one row tile
constexpr int kResident2 = 512;         // and on two
constexpr double kUneven1 = 2.25;       // largest work of one over the average of that many
constexpr double kUneven2 = 1.5;
constexpr int kPairRows = 128;          // rows per KV head from which on a wave takes two tiles
constexpr int kMinWork = 2048;          // keys x (row tile share) of a work-group, lower bound
constexpr int kUnsplit = 2816;          // nothing is split when no range is above this
constexpr int kMaxSplits = 64;          // key ranges per row tile (combine kernel's table)

int64_t page_bytes_of(const spec_model_config* c) {
  return (int64_t)c->n_layers * c->n_kv_heads * kv4_head_bytes(c->head_dim);
}

// Positions that the sample's mapped pages hold.
int64_t mapped(const spec_kv4* kv, int sample) { return (int64_t)kv->pages[sample].size() * kKv4Page; }

// No page of positions [begin, end) of a sample may be another sample's too.
int check_unshared(const spec_kv4* kv, int sample, int64_t begin, int64_t end) {
  for (int64_t p = begin / kKv4Page; p * kKv4Page < end; ++p) {
    const int page = kv->pages[sample][p];
    if (kv->uses[page] > 1)
      return fail(SPEC_ERR_INVALID, "sample %d: page %d of positions to be written is mapped to %d samples", sample,
                  page, kv->uses[page]);
  }
  return SPEC_OK;
}

// Partial tiles that the plan of such a step may have: every row tile in as many key ranges
// as the shortest range, kMinWork shared by a work-group's four tiles, leaves of its keys.
int64_t part_cap(const spec_model_config* c, int64_t batch, int64_t rows, int64_t pages) {
  const int64_t tiles = rows * (c->n_heads / c->n_kv_heads) / 16 + batch;
  const int64_t ranges = std::min<int64_t>(kMaxSplits, (pages * kKv4Page + kMinWork / 4 - 1) / (kMinWork / 4));
  return std::min<int64_t>(kPartCap, c->n_kv_heads * tiles * ranges);
}

struct StepLayout {
  size_t blob, toks, anc, part_o, part_ml, total;
};

StepLayout step_layout(const spec_model_config* c, int64_t batch, int64_t rows, int64_t pages) {
  const int64_t G = c->n_heads / c->n_kv_heads;
  const int64_t groups = (int64_t)c->n_kv_heads * (rows * G / 64 + batch);   // of four row tiles at least, or a sample's last
  const int64_t parts = part_cap(c, batch, rows, pages);
  const int64_t items = 8 * (groups + parts);                                // padded per XCD
  const int64_t octets = rows / 8 + 2 * batch;
  const size_t blob = align_up(batch * sizeof(SampleInfo)) + align_up(rows * 4) + align_up(pages * 4) +
                      align_up(c->head_dim / 2 * sizeof(double)) + align_up(octets * sizeof(Kv4Octet)) +
                      align_up(items * sizeof(Kv4Item)) +
                      align_up(parts * sizeof(Kv4Merge));
  StepLayout L{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off += align_up(bytes);
    return at;
  };
  L.blob = take(blob);
  L.toks = take(rows * sizeof(TokInfo));
  L.anc = take(rows * 8 * kAncWords);
  L.part_o = take((size_t)parts * 16 * c->head_dim * 4);
  L.part_ml = take((size_t)parts * 16 * 2 * 4);
  L.total = off;
  return L;
}

// The attention work of a step: work-groups, as they go to the XCDs, and the merges of
// split key ranges.
struct AttnPlan {
  std::vector<Kv4Item> items;
  std::vector<Kv4Merge> comb;
  int wave_tiles = 1;
  bool once = false;
};

// A (sample, kv head) has ceil(T G / 16) row tiles.  A wave takes one (three waves per
// SIMD) or, when some sample has more than kPairRows rows, two (two per SIMD, and V is
// decoded once for both).  A work-group's four waves share the keys of the first tile
// (pair) by four, of two by two, or have one each; more tiles go to more work-groups.
// A group's key range is cut evenly, so that the step's work-groups (work: keys x waves'
// share) fit the chip at once, kResident, unless one would then have kUneven times the
// average; but none below kMinWork is made, and with no range above kUnsplit nothing is
// cut, which saves the merge's launch.  Measured side by side when the rules were set, us, 8B heads:
//                                   one tile per wave   two tiles
//   128 samples, 176K keys, 32 rows        55.7            62.1
//   4 samples, 15K keys, 64 rows           17.0            20.5
//   4 samples, 101K keys, 256 rows         139             120
//   prompt pieces of 500 - 1170 rows       173             153
// kUneven 1 / 1.5 / 2 / 2.25 / 4: first row 60.0 / 58.5 / 57.7 / 55.6 / 55.7, third 143 /
// 121 / 121 / 120 / 119, fourth 158 / 155 / 153 / 153 / 153; but with one sample of 30000
// keys among 100 of 64 rows and 1000 keys 66.9 / 90 for the last two, and among 8 of 1024
// rows 211 / 306 (192 at 1.5; a work-group that is left alone runs faster where three share a CU than
// where two do).  Chunks of one length for all, 1.5 rounds of them: 58.8, 124, 157, 70, 179.
// At least 1024 / 2048 per work-group: the second row 19.8 / 17.4.  A range of 2100 (of
// 4064) in one piece 11.4 (17.7), in two 14.2 (14.3).
void plan_attention(const spec_model_config* c, const std::vector<SampleInfo>& si, bool runs, int64_t parts,
                    AttnPlan* plan) {
  const int G = c->n_heads / c->n_kv_heads, nkv = c->n_kv_heads;
  struct Group {
    int b, tile0, tiles, keys;
  };
  std::vector<Group> groups;
  int64_t most_rows = 0;
  for (const SampleInfo& x : si) most_rows = std::max(most_rows, (int64_t)x.ntok * G);
  plan->wave_tiles = most_rows <= kPairRows ? 1 : 2;
  plan->once = most_rows <= 16;               // one row tile
  const int wt = plan->wave_tiles;
  auto waves_of = [&](int tiles) { return tiles <= wt ? 4 : tiles <= 2 * wt ? 2 : 1; };
  auto weight = [&](int tiles) { return 4 / waves_of(tiles); };
  double work = 0.0;
  int64_t longest = 0;
  for (int b = 0; b < (int)si.size(); ++b) {
    const int64_t rows = (int64_t)si[b].ntok * G;
    const int tiles = (int)((rows + 15) / 16);
    for (int t = 0; t < tiles; t += 4 * wt) {
      const int n = std::min(4 * wt, tiles - t);
      const int64_t last = std::min<int64_t>(rows, 16ll * (t + n)) - 1;      // last row of the group
      const int keys = si[b].seq_len + (runs ? (int)(last / G) + 1 : si[b].ntok);
      groups.push_back(Group{b, t, n, keys});
      work += (double)nkv * keys * weight(n);
      longest = std::max(longest, (int64_t)keys * weight(n));
    }
  }
  auto splits_of = [&](const Group& g, double unit) {
    const double per = std::max(128.0, unit / weight(g.tiles));
    return (int)std::min<int64_t>(kMaxSplits, std::max<int64_t>(1, (int64_t)std::ceil(g.keys / per)));
  };
  auto chunk_of = [&](const Group& g, int ns) { return ((int64_t)g.keys + 128 * ns - 1) / (128 * ns) * 128; };
  const int slots_at_once = wt == 1 ? kResident1 : kResident2;
  const double least = longest <= kUnsplit ? kUnsplit : kMinWork, even = work / slots_at_once;
  const double uneven = wt == 1 ? kUneven1 : kUneven2;
  double unit = std::max(least, even);
  for (;;) {      // ends: with units beyond the longest range times four nothing is split
    int64_t slots = 0, wgs = 0;
    for (const Group& g : groups) {
      const int ns = splits_of(g, unit);
      wgs += (int64_t)ns * nkv;
      if (ns > 1) slots += (int64_t)ns * nkv * g.tiles;
    }
    if (slots <= parts && (wgs <= slots_at_once || slots == 0 || unit > uneven * even)) break;
    unit *= 1.03;
  }
  std::vector<Kv4Item> list;
  std::vector<AttnItem> order;     // with ranges as long as the work; `pad` is an index into `list`
  int slot = 0;
  for (const Group& g : groups) {
    const int64_t ch = chunk_of(g, splits_of(g, unit));
    const int ns = (int)((g.keys + ch - 1) / ch);
    const SampleInfo& b = si[g.b];
    for (int kvh = 0; kvh < nkv; ++kvh) {
      for (int k = 0; k < ns; ++k) {
        const int key0 = (int)(k * ch), key1 = (int)std::min<int64_t>(g.keys, (k + 1) * ch);
        const int64_t end = key0 + (int64_t)(key1 - key0) * weight(g.tiles);
        order.push_back(AttnItem{g.b, kvh, 0, key0, (int)std::min<int64_t>(end, 0x7fffffff), 0, 0, (int)list.size()});
        list.push_back(Kv4Item{kvh, g.tile0 * 16, key0, key1, ns, ns > 1 ? slot + k : 0, waves_of(g.tiles), b.seq_len,
                               b.tok0, b.ntok, (uint32_t)b.kv_base, {}});
      }
      if (ns > 1) {
        for (int t = 0; t < g.tiles; ++t)
          plan->comb.push_back(Kv4Merge{kvh, (g.tile0 + t) * 16, ns, slot + t * ns, b.tok0, b.ntok, {}});
        slot += ns * g.tiles;
      }
    }
  }
  deal_items(order);
  plan->items.reserve(order.size());
  for (const AttnItem& x : order)  // sample -1: padding of a shorter per-XCD list
    plan->items.push_back(x.sample < 0 ? Kv4Item{} : list[x.pad]);
}

}  // namespace

namespace spec {

int refuse_capture(void* stream) {
  hipStreamCaptureStatus st = hipStreamCaptureStatusNone;
  HIP_TRY(hipStreamIsCapturing((hipStream_t)stream, &st), "stream capture status");
  if (st != hipStreamCaptureStatusNone)
    return fail(SPEC_ERR_INVALID, "the call uploads its plan and cannot be captured into a graph");
  return SPEC_OK;
}

int kv4_check_rows(const spec_kv4* kv, int32_t batch, const int32_t* sample_ids, const int32_t* offsets,
                   const int32_t* parents, const int32_t* seq_lens) {
  if (batch < 1) return fail(SPEC_ERR_INVALID, "batch must be >= 1");
  if (int rc = check_sample_ids(kv->n, batch, sample_ids)) return rc;
  if (offsets[0] != 0) return fail(SPEC_ERR_TREE, "row_offsets[0] must be 0");
  for (int b = 0; b < batch; ++b) {
    const int64_t T = (int64_t)offsets[b + 1] - offsets[b];
    if (T < 1) return fail(SPEC_ERR_TREE, "sample %d has %lld rows", b, (long long)T);
    const int64_t G = kv->cfg.n_heads / kv->cfg.n_kv_heads;
    if (T * G * G > 0xffffffffll)
      return fail(SPEC_ERR_UNSUPPORTED, "sample %d: %lld rows of %lld query heads each are more than one step takes", b,
                  (long long)T, (long long)G);
    if (parents && T > SPEC_MAX_TREE) return fail(SPEC_ERR_UNSUPPORTED, "sample %d has %lld tree nodes", b, (long long)T);
    const int S = seq_lens[b];
    if (S < 0) return fail(SPEC_ERR_INVALID, "seq_lens[%d] = %d", b, S);
    if (S + T > mapped(kv, sample_ids[b]))
      return fail(SPEC_ERR_CAPACITY, "sample %d: %d committed + %lld rows exceed the %lld positions of its pages", b, S,
                  (long long)T, (long long)mapped(kv, sample_ids[b]));
    if (int rc = check_unshared(kv, sample_ids[b], S, S + T)) return rc;
    if (!parents) continue;
    const int32_t* p = parents + offsets[b];
    if (p[0] != -1) return fail(SPEC_ERR_TREE, "sample %d: root parent must be -1", b);
    for (int i = 1; i < T; ++i)
      if (p[i] < 0 || p[i] >= i)
        return fail(SPEC_ERR_TREE, "sample %d node %d: parent %d not before the node", b, i, p[i]);
  }
  return SPEC_OK;
}

size_t kv4_step_bytes(const spec_model_config* cfg, int64_t batch, int64_t rows, int64_t pages) {
  return step_layout(cfg, batch, rows, pages).total;
}

int64_t kv4_step_pages(const spec_kv4*, int32_t batch, const int32_t* offsets, const int32_t* seq_lens) {
  int64_t pages = 0;
  for (int b = 0; b < batch; ++b)
    pages += ((int64_t)seq_lens[b] + offsets[b + 1] - offsets[b] + kKv4Page - 1) / kKv4Page;
  return pages;
}

int kv4_plan_step(spec_kv4* kv, int32_t batch, const int32_t* sample_ids, const int32_t* offsets,
                  const int32_t* parents, const int32_t* seq_lens, void* workspace, hipStream_t s,
                  const spec_debug& dbg, spec_kv4_step* st) {
  const spec_model_config& c = kv->cfg;
  const int64_t N = offsets[batch];
  const int64_t pages = kv4_step_pages(kv, batch, offsets, seq_lens);
  const bool runs = parents == nullptr;
  std::vector<SampleInfo> si(batch);
  std::vector<uint32_t> table;
  table.reserve(pages);
  const uint32_t page_units = (uint32_t)(page_bytes_of(&c) / kKv4Unit);
  std::vector<Kv4Octet> octets;
  octets.reserve(N / 8 + 2 * batch);
  for (int b = 0; b < batch; ++b) {
    const int id = sample_ids[b], S = seq_lens[b], T = offsets[b + 1] - offsets[b];
    const int np = (int)(((int64_t)S + T + kKv4Page - 1) / kKv4Page);
    si[b] = SampleInfo{(int64_t)table.size(), np * kKv4Page, S, offsets[b], T, 0, 0};
    for (int p = 0; p < np; ++p) table.push_back((uint32_t)kv->pages[id][p] * page_units);
    for (int o = S / 8 * 8; o < S + T; o += 8)
      octets.push_back(Kv4Octet{table[si[b].kv_base + o / kKv4Page], o, std::max(0, S - o), std::min(8, S + T - o),
                                offsets[b] + (o - S), offsets[b], T, 0});
  }
  AttnPlan plan;
  plan_attention(&c, si, runs, part_cap(&c, batch, N, pages), &plan);
  std::vector<double> freq(c.head_dim / 2);
  for (int j = 0; j < c.head_dim / 2; ++j)
    freq[j] = std::pow((double)c.rope_theta, -2.0 * j / c.head_dim);

  // ---- one upload ----
  const StepLayout L = step_layout(&c, batch, N, pages);
  std::vector<char> blob;
  auto put = [&](const void* src, size_t bytes) {
    const size_t at = align_up(blob.size());
    blob.resize(at + bytes);
    if (bytes) memcpy(blob.data() + at, src, bytes);
    return at;
  };
  const size_t o_si = put(si.data(), si.size() * sizeof(SampleInfo));
  const size_t o_par = put(parents, runs ? 0 : N * 4);
  const size_t o_table = put(table.data(), table.size() * 4);
  const size_t o_freq = put(freq.data(), freq.size() * sizeof(double));
  const size_t o_oct = put(octets.data(), octets.size() * sizeof(Kv4Octet));
  const size_t o_items = put(plan.items.data(), plan.items.size() * sizeof(Kv4Item));
  const size_t o_comb = put(plan.comb.data(), plan.comb.size() * sizeof(Kv4Merge));
  char* ws = (char*)workspace;
  char* d = ws + L.blob;
  if (int rc = kv->ring.upload(blob.data(), blob.size(), d, s)) return rc;
  const SampleInfo* d_si = (const SampleInfo*)(d + o_si);
  TokInfo* toks = (TokInfo*)(ws + L.toks);
  uint64_t* anc = (uint64_t*)(ws + L.anc);
  if (!runs)
    HIP_TRY(launch_tree_meta(d_si, batch, (const int32_t*)(d + o_par), toks, anc, dbg.depth, dbg.pos, dbg.anc, s),
            "tree meta");

  st->kv = kv;
  st->n_rows = (int)N;
  Kv4View view{kv->pool, (const uint32_t*)(d + o_table), d_si, 0, c.n_kv_heads, c.head_dim};
  st->rows = Kv4RowArgs{view, (const Kv4Octet*)(d + o_oct), (int)octets.size(), runs ? nullptr : toks,
                        (const double*)(d + o_freq), nullptr, nullptr, 0, 0, 0, 0};
  Kv4AttnArgs& a = st->attn;
  a = Kv4AttnArgs{};
  a.v = view;
  a.anc = runs ? nullptr : anc;
  a.items = (const Kv4Item*)(d + o_items);
  a.n_items = (int)plan.items.size();
  a.wave_tiles = plan.wave_tiles;
  a.once = plan.once;
  a.part_o = (float*)(ws + L.part_o);
  a.part_ml = (float*)(ws + L.part_ml);
  a.n_heads = c.n_heads;
  a.group = c.n_heads / c.n_kv_heads;
  a.group_inv = (uint32_t)(((1ull << 32) + a.group - 1) / a.group);
  a.comb = (const Kv4Merge*)(d + o_comb);
  a.n_comb = (int)plan.comb.size();
  return SPEC_OK;
}

int kv4_append(const spec_kv4_step* st, int layer, const bf16* k, int64_t k_stride, const bf16* v, int64_t v_stride,
               int rotate, hipStream_t s) {
  Kv4RowArgs a = st->rows;
  a.v.layer = layer;
  a.k = const_cast<bf16*>(k);
  a.val = const_cast<bf16*>(v);
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.rotate = rotate;
  HIP_TRY(timed(SPEC_K_KV4_APPEND, s, [&] { return launch_kv4_append(a, s); }), "kv4 append");
  return SPEC_OK;
}

int kv4_append_blocks(const spec_kv4_step* st, int layer, const bf16* kv, hipStream_t s) {
  Kv4RowArgs a = st->rows;
  a.v.layer = layer;
  a.k = a.val = const_cast<bf16*>(kv);
  a.blocks = 1;
  HIP_TRY(timed(SPEC_K_KV4_APPEND, s, [&] { return launch_kv4_append(a, s); }), "kv4 append");
  return SPEC_OK;
}

int kv4_attend(const spec_kv4_step* st, int layer, const bf16* q, int64_t q_stride, bf16* out, hipStream_t s) {
  Kv4AttnArgs a = st->attn;
  a.v.layer = layer;
  a.q = q;
  a.q_stride = q_stride;
  a.out = out;
  HIP_TRY(timed(SPEC_K_ATTENTION, s, [&] { return launch_kv4_attention(a, s); }), "kv4 attention");
  return SPEC_OK;
}

}  // namespace spec

SPEC_API size_t spec_kv4_page_bytes(const spec_model_config* cfg) {
  std::string why;
  if (!cfg || !config_ok(cfg, &why)) return 0;
  return (size_t)page_bytes_of(cfg);
}

SPEC_API size_t spec_kv4_bytes(const spec_model_config* cfg, int32_t n_samples, int32_t n_pages) {
  const size_t page = spec_kv4_page_bytes(cfg);
  if (page == 0 || n_samples < 1 || n_pages < 1) return 0;
  return align_up(page * n_pages) + align_up((size_t)n_samples * sizeof(Kv4CommitInfo));
}

SPEC_API int spec_kv4_alloc(const spec_model_config* cfg, int32_t n_samples, int32_t n_pages, void* device_buf,
                            size_t buf_bytes, spec_kv4** out) {
  return guarded([&]() -> int {
    if (!cfg || !device_buf || !out) return fail(SPEC_ERR_INVALID, "null argument");
    if (n_samples < 1 || n_pages < 1) return fail(SPEC_ERR_INVALID, "n_samples and n_pages must be >= 1");
    std::string why;
    if (!config_ok(cfg, &why)) return fail(SPEC_ERR_UNSUPPORTED, "%s", why.c_str());
    if ((uintptr_t)device_buf % kAlign) return fail(SPEC_ERR_INVALID, "device_buf not 256-byte aligned");
    if ((int64_t)n_pages > (int64_t)0xffffffff / (page_bytes_of(cfg) / kKv4Unit))
      return fail(SPEC_ERR_UNSUPPORTED, "%d pages are more than the 512 GB a pool can have", n_pages);
    const size_t need = spec_kv4_bytes(cfg, n_samples, n_pages);
    if (buf_bytes < need)
      return fail(SPEC_ERR_CAPACITY, "KV buffer holds %zu bytes, needs %zu", buf_bytes, need);
    spec_kv4* kv = new spec_kv4;
    kv->cfg = *cfg;
    kv->n = n_samples;
    kv->pages.resize(n_samples);
    kv->uses.assign(n_pages, 0);
    kv->pool = (char*)device_buf;
    kv->ctl_off = align_up((size_t)page_bytes_of(cfg) * n_pages);
    *out = kv;
    return SPEC_OK;
  });
}

SPEC_API int spec_kv4_free(spec_kv4* kv) {
  if (!kv) return fail(SPEC_ERR_INVALID, "null handle");
  const int rc = kv->ring.release();
  delete kv;
  return rc;
}

SPEC_API int spec_kv4_map(spec_kv4* kv, int32_t sample, int32_t n_pages, const int32_t* pages) {
  return guarded([&]() -> int {
    if (!kv || (n_pages > 0 && !pages)) return fail(SPEC_ERR_INVALID, "null argument");
    if (sample < 0 || sample >= kv->n) return fail(SPEC_ERR_INVALID, "sample %d out of range", sample);
    const int total = (int)kv->uses.size();
    if (n_pages < 0 || n_pages > total || n_pages > 0x7fffffff / kKv4Page)
      return fail(SPEC_ERR_INVALID, "%d pages of %d", n_pages, total);
    std::vector<char> seen(total, 0);
    for (int i = 0; i < n_pages; ++i) {
      if (pages[i] < 0 || pages[i] >= total)
        return fail(SPEC_ERR_INVALID, "pages[%d] = %d outside the pool's %d", i, pages[i], total);
      if (seen[pages[i]]) return fail(SPEC_ERR_INVALID, "page %d appears twice", pages[i]);
      seen[pages[i]] = 1;
    }
    std::vector<int32_t> next(pages, pages + n_pages);
    for (const int32_t p : kv->pages[sample]) --kv->uses[p];
    for (const int32_t p : next) ++kv->uses[p];
    kv->pages[sample].swap(next);
    return SPEC_OK;
  });
}

SPEC_API size_t spec_kv4_step_bytes(const spec_model_config* cfg, int32_t max_batch, int32_t max_rows,
                                    int32_t max_pages) {
  std::string why;
  if (!cfg || max_batch < 1 || max_rows < max_batch || max_pages < 1 || !config_ok(cfg, &why)) return 0;
  return step_layout(cfg, max_batch, max_rows, max_pages).total;
}

SPEC_API int spec_kv4_step_begin(spec_kv4* kv, int32_t batch, const int32_t* sample_ids, const int32_t* row_offsets,
                                 const int32_t* parents, const int32_t* seq_lens, void* workspace, size_t ws_bytes,
                                 void* stream, spec_kv4_step** out) {
  return guarded([&]() -> int {
    if (!kv || !sample_ids || !row_offsets || !seq_lens || !workspace || !out)
      return fail(SPEC_ERR_INVALID, "null argument");
    if (int rc = kv4_check_rows(kv, batch, sample_ids, row_offsets, parents, seq_lens)) return rc;
    if ((uintptr_t)workspace % kAlign) return fail(SPEC_ERR_INVALID, "workspace not 256-byte aligned");
    const size_t need = kv4_step_bytes(&kv->cfg, batch, row_offsets[batch],
                                       kv4_step_pages(kv, batch, row_offsets, seq_lens));
    if (ws_bytes < need) return fail(SPEC_ERR_WORKSPACE, "workspace %zu bytes, needs %zu", ws_bytes, need);
    if (int rc = refuse_capture(stream)) return rc;
    spec_kv4_step* st = new spec_kv4_step;
    int rc;
    try {
      rc = kv4_plan_step(kv, batch, sample_ids, row_offsets, parents, seq_lens, workspace, (hipStream_t)stream,
                         spec_debug{}, st);
    } catch (...) {
      delete st;
      throw;
    }
    if (rc != SPEC_OK) {
      delete st;
      return rc;
    }
    *out = st;
    return SPEC_OK;
  });
}

SPEC_API int spec_kv4_step_free(spec_kv4_step* step) {
  if (!step) return fail(SPEC_ERR_INVALID, "null handle");
  delete step;
  return SPEC_OK;
}

namespace {

int check_layer(const spec_kv4_step* step, int32_t layer) {
  if (layer < 0 || layer >= step->kv->cfg.n_layers) return fail(SPEC_ERR_INVALID, "layer %d out of range", layer);
  return SPEC_OK;
}

// Rows of `width` values `stride` apart, accessed 16 bytes at a time.
int check_strided(const char* what, const void* p, int64_t stride, int64_t width) {
  if (!p) return fail(SPEC_ERR_INVALID, "null argument");
  if ((uintptr_t)p % 16) return fail(SPEC_ERR_INVALID, "%s not 16-byte aligned", what);
  if (stride < width || stride % 8)
    return fail(SPEC_ERR_INVALID, "%s: row stride %lld must be a multiple of 8 and at least %lld", what,
                (long long)stride, (long long)width);
  return SPEC_OK;
}

int check_kv_rows(const spec_kv4_step* step, int32_t layer, const void* k, int64_t k_stride, const void* v,
                  int64_t v_stride) {
  if (!step) return fail(SPEC_ERR_INVALID, "null argument");
  if (int rc = check_layer(step, layer)) return rc;
  const spec_model_config& c = step->kv->cfg;
  if (int rc = check_strided("k", k, k_stride, (int64_t)c.n_kv_heads * c.head_dim)) return rc;
  return check_strided("v", v, v_stride, (int64_t)c.n_kv_heads * c.head_dim);
}

}  // namespace

SPEC_API int spec_kv4_append(const spec_kv4_step* step, int32_t layer, const void* k, int64_t k_stride, const void* v,
                             int64_t v_stride, int32_t rotate, void* stream) {
  return guarded([&]() -> int {
    if (int rc = check_kv_rows(step, layer, k, k_stride, v, v_stride)) return rc;
    return kv4_append(step, layer, (const bf16*)k, k_stride, (const bf16*)v, v_stride, rotate != 0,
                      (hipStream_t)stream);
  });
}

SPEC_API int spec_kv4_read(const spec_kv4_step* step, int32_t layer, void* k, int64_t k_stride, void* v,
                           int64_t v_stride, void* stream) {
  return guarded([&]() -> int {
    if (int rc = check_kv_rows(step, layer, k, k_stride, v, v_stride)) return rc;
    Kv4RowArgs a = step->rows;
    a.v.layer = layer;
    a.k = (bf16*)k;
    a.val = (bf16*)v;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    HIP_TRY(launch_kv4_read(a, (hipStream_t)stream), "kv4 read");
    return SPEC_OK;
  });
}

SPEC_API int spec_kv4_attend(const spec_kv4_step* step, int32_t layer, const void* q, int64_t q_stride, void* out,
                             void* stream) {
  return guarded([&]() -> int {
    if (!step || !out) return fail(SPEC_ERR_INVALID, "null argument");
    if (int rc = check_layer(step, layer)) return rc;
    const spec_model_config& c = step->kv->cfg;
    if (int rc = check_strided("q", q, q_stride, (int64_t)c.n_heads * c.head_dim)) return rc;
    if ((uintptr_t)out % 16) return fail(SPEC_ERR_INVALID, "out not 16-byte aligned");
    return kv4_attend(step, layer, (const bf16*)q, q_stride, (bf16*)out, (hipStream_t)stream);
  });
}

SPEC_API int spec_kv4_commit(spec_kv4* kv, int32_t batch, const int32_t* sample_ids, const int32_t* seq_lens,
                             const int32_t* accepted_len, const int32_t* accepted_nodes, int32_t* new_seq_lens,
                             void* stream) {
  return guarded([&]() -> int {
    if (!kv || !sample_ids || !seq_lens || !accepted_len || !accepted_nodes || !new_seq_lens)
      return fail(SPEC_ERR_INVALID, "null argument");
    if (batch < 1 || batch > kv->n) return fail(SPEC_ERR_INVALID, "batch %d out of range", batch);
    if (int rc = check_sample_ids(kv->n, batch, sample_ids)) return rc;
    std::vector<Kv4CommitInfo> info(batch);
    for (int b = 0; b < batch; ++b) {
      const int id = sample_ids[b], S = seq_lens[b];
      const int64_t cap = mapped(kv, id);
      if (S < 0 || S >= cap)
        return fail(SPEC_ERR_CAPACITY, "seq_lens[%d] = %d outside the %lld positions of its pages", b, S,
                    (long long)cap);
      if (int rc = check_unshared(kv, id, S, std::min<int64_t>(cap, (int64_t)S + SPEC_MAX_TREE))) return rc;
      info[b] = Kv4CommitInfo{S, (int32_t)cap, {-1, -1, -1, -1, -1, -1}};
      for (int i = 0; i < 6 && S / kKv4Page + i < (int)kv->pages[id].size(); ++i)
        info[b].pages[i] = kv->pages[id][S / kKv4Page + i];
    }
    if (int rc = refuse_capture(stream)) return rc;
    hipStream_t s = (hipStream_t)stream;
    void* ctl = kv->pool + kv->ctl_off;
    if (int rc = kv->ring.upload(info.data(), batch * sizeof(Kv4CommitInfo), ctl, s)) return rc;
    const spec_model_config& c = kv->cfg;
    HIP_TRY(timed(SPEC_K_COMMIT, s, [&] {
              return launch_kv4_compact((const Kv4CommitInfo*)ctl, batch, kv->pool, page_bytes_of(&c), c.n_layers,
                                        c.n_kv_heads, c.head_dim, accepted_len, accepted_nodes, new_seq_lens, s);
            }),
            "kv4 compact");
    return SPEC_OK;
  });
}
