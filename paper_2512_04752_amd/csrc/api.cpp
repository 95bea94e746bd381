// Host side of the specverify C ABI: argument validation, per-call planning
// (per-sample descriptors, split-KV attention work list), workspace carving,
// one staged host-to-device upload per call and the launch sequence of the
// verify step.  Every step of the computation itself runs in the HIP kernels.
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include <algorithm>
#include <cmath>
#include <string>
#include <vector>

#include "common.h"
#include "kv4_host.h"
#include "reorder.h"
#include "specverify.h"
#include "w4.h"

using namespace spec;

namespace {

thread_local std::string g_err;

}  // namespace

namespace spec {

Profiler g_prof;

int fail(int code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  g_err = buf;
  return code;
}

int hip_fail(hipError_t e, const char* what) {
  return fail(SPEC_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

void clear_error() { g_err.clear(); }

bool config_ok(const spec_model_config* c, std::string* why) {
  char buf[256];
  auto bad = [&](const char* m) {
    snprintf(buf, sizeof buf, "unsupported model shape: %s", m);
    *why = buf;
    return false;
  };
  if (c->n_layers < 1 || c->hidden < 1 || c->n_heads < 1 || c->n_kv_heads < 1 || c->ffn < 1 ||
      c->vocab < 1 || c->head_dim < 1)
    return bad("non-positive dimension");
  if (c->head_dim != 64 && c->head_dim != 128) return bad("head_dim must be 64 or 128");
  if (c->n_heads % c->n_kv_heads) return bad("n_heads must be a multiple of n_kv_heads");
  if (c->hidden % 128) return bad("hidden must be a multiple of 128");
  if ((c->n_heads * c->head_dim) % 128) return bad("n_heads*head_dim must be a multiple of 128");
  if ((c->n_kv_heads * c->head_dim) % 128)
    return bad("n_kv_heads*head_dim must be a multiple of 128");
  if (c->ffn % 128) return bad("ffn must be a multiple of 128");
  if (c->vocab % 128) return bad("vocab must be a multiple of 128");
  if (!(c->rope_theta > 0.f) || !(c->rms_eps >= 0.f)) return bad("rope_theta/rms_eps");
  return true;
}

bool same_config(const spec_model_config* a, const spec_model_config* b) {
  return a->n_layers == b->n_layers && a->hidden == b->hidden && a->n_heads == b->n_heads &&
         a->n_kv_heads == b->n_kv_heads && a->head_dim == b->head_dim && a->ffn == b->ffn &&
         a->vocab == b->vocab;
}

}  // namespace spec

namespace {

constexpr int kPartCap = 8192;          // split-KV partial tiles per call
constexpr int kTargetSlots = 512;       // attention CU slots aimed for (two rounds of 256 CUs)
constexpr int kMinChunk = 64;           // keys per split, lower bound
constexpr int kSmallChunk = 256;        // small calls: chunks of 64-key multiples up to this
constexpr int kMaxSplits = 64;          // key ranges per row tile (combine kernel's table)

size_t sample_bytes(const spec_model_config* c, int32_t cap) {
  return align_up((size_t)c->n_layers * 2 * c->n_kv_heads * (size_t)cap * c->head_dim * 2);
}

// Workspace carving; every region 256-byte aligned.
struct WsLayout {
  size_t blob, toks, anc, rope, x, h, q, o, act, part_o, part_ml, lm_val, lm_idx, argmax, splitk,
      logits, resid, kv4_step, kv4_rows, total;
  size_t blob_bytes;
};

int64_t max_row_tiles(const spec_model_config* c, int64_t max_batch, int64_t max_tokens) {
  const int64_t G = c->n_heads / c->n_kv_heads;
  return (int64_t)c->n_kv_heads * ((max_tokens * G + 31) / 32 + max_batch);
}

// kv4_pages > 0: over the 4-bit pool, the attention's plan and partials are the step's.
// w4: with weights in 4 bits, whose products leave q, k, v and the logits in fp32.
WsLayout ws_layout(const spec_model_config* c, int64_t max_batch, int64_t max_tokens,
                   bool sampling = false, int64_t kv4_pages = 0, bool w4 = false) {
  WsLayout L{};
  const bool kv4 = kv4_pages > 0;
  const int64_t part_cap = kv4 ? 0 : kPartCap;
  // attention items: one per row tile and split, then padded per XCD (at most 8x)
  const int64_t items = kv4 ? 0 : 8 * (max_row_tiles(c, max_batch, max_tokens) + kPartCap);
  L.blob_bytes = align_up(max_batch * sizeof(SampleInfo)) + 2 * align_up(max_tokens * 4) +
                 align_up(items * sizeof(AttnItem)) + 2 * kAlign +  // narrow + two wide lists
                 align_up(part_cap * sizeof(CombineItem));
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off += align_up(bytes);
    return at;
  };
  const size_t nq_hd = (size_t)c->n_heads * c->head_dim;
  L.blob = take(L.blob_bytes);
  L.toks = take(kv4 ? 0 : max_tokens * sizeof(TokInfo));
  L.anc = take(kv4 ? 0 : max_tokens * 8 * kAncWords);
  L.rope = take(max_tokens * (size_t)(c->head_dim / 2) * 8);
  L.x = take(max_tokens * (size_t)c->hidden * 4);
  L.h = take(max_tokens * (size_t)c->hidden * 2);
  L.q = take(max_tokens * nq_hd * 2);
  L.o = take(max_tokens * nq_hd * 2);
  L.act = take(max_tokens * (size_t)c->ffn * 2);
  L.part_o = take((size_t)part_cap * 32 * c->head_dim * 2);
  L.part_ml = take((size_t)part_cap * 32 * 2 * 4);
  L.lm_val = take(max_tokens * (size_t)(c->vocab / 64) * 4);
  L.lm_idx = take(max_tokens * (size_t)(c->vocab / 64) * 4);
  L.argmax = take(max_tokens * 4);
  const size_t qkv = nq_hd + 2 * (size_t)c->n_kv_heads * c->head_dim;
  L.splitk = take(w4 ? std::max(kW4PartialCap, max_tokens * std::max(qkv, (size_t)c->hidden) * 4) : gemm_partial_bytes());
  if (sampling || w4) L.logits = take(max_tokens * (size_t)c->vocab * 4);
  if (sampling)     // speculative sampling: node decisions, fp64 residual rows
    L.resid = take(sample_accept_scratch((int)max_batch, (int)max_tokens, c->vocab));
  if (kv4) {   // the step's plan, and one layer's rotated K/V on their way into the cache
    L.kv4_step = take(kv4_step_bytes(c, max_batch, max_tokens, kv4_pages));
    L.kv4_rows = take(max_tokens * 2 * (size_t)c->n_kv_heads * c->head_dim * 2);
  }
  L.total = off;
  return L;
}

// The plan of one product (SPEC_K_*) of a verify step of n rows.
GemmPlan product_plan(const spec_model_config* c, int kind, int n) {
  const int q = c->n_heads * c->head_dim, kv = c->n_kv_heads * c->head_dim;
  switch (kind) {
    case SPEC_K_GEMM_QKV: return plan_gemm(EPI_QKV, n, q + 2 * kv, c->hidden, q, kv, false);
    case SPEC_K_GEMM_O: return plan_gemm(EPI_RESID, n, c->hidden, q, c->hidden, 0, true);
    case SPEC_K_GEMM_GATE_UP:
      return plan_gemm(EPI_GATE_UP, n, 2 * c->ffn, c->hidden, c->ffn, c->ffn, false);
    case SPEC_K_GEMM_DOWN: return plan_gemm(EPI_RESID, n, c->hidden, c->ffn, c->hidden, 0, true);
    default: return plan_gemm(EPI_ARGMAX, n, c->vocab, c->hidden, c->vocab, 0, false);
  }
}

}  // namespace

// Library-owned part of a KV pool: capacities, block offsets and a two-slot
// pinned staging ring for the per-call host->device uploads.
struct spec_kv {
  spec_model_config cfg;
  int32_t n = 0;
  std::vector<int32_t> cap;
  std::vector<int64_t> base;     // element offsets of the sample blocks
  bf16* pool = nullptr;
  size_t bytes = 0;
  size_t ctl_off = 0;            // byte offset of the control area (commit descriptors)
  StagingRing<2> ring;
};

namespace {

int check_samples(const spec_kv* kv, int32_t batch, const int32_t* ids) {
  return check_sample_ids(kv->n, batch, ids);
}

}  // namespace

namespace spec {

int check_reorder(int n, int32_t groups, int32_t width, const int32_t* ids, const int32_t* begin,
                  const int32_t* end, const int32_t* parents) {
  if (!ids || !begin || !end || !parents) return fail(SPEC_ERR_INVALID, "null argument");
  if (width < 1 || width > kMaxReorder) return fail(SPEC_ERR_INVALID, "width %d outside 1 .. %d", width, kMaxReorder);
  if (groups < 1 || (int64_t)groups * width > n)
    return fail(SPEC_ERR_INVALID, "%d groups of %d beams over %d samples", groups, width, n);
  if (groups > 65535) return fail(SPEC_ERR_UNSUPPORTED, "%d groups, at most 65535", groups);
  if ((uintptr_t)parents % 4) return fail(SPEC_ERR_INVALID, "parents not 4-byte aligned");
  for (int g = 0; g < groups; ++g)
    if (begin[g] < 0 || end[g] < begin[g])
      return fail(SPEC_ERR_INVALID, "group %d: positions [%d, %d)", g, begin[g], end[g]);
  return check_sample_ids(n, groups * width, ids);
}

int check_sample_ids(int n, int32_t batch, const int32_t* ids) {
  std::vector<char> seen(n, 0);
  for (int b = 0; b < batch; ++b) {
    const int id = ids[b];
    if (id < 0 || id >= n) return fail(SPEC_ERR_INVALID, "sample_ids[%d] = %d out of range", b, id);
    if (seen[id]) return fail(SPEC_ERR_INVALID, "sample id %d appears twice", id);
    seen[id] = 1;
  }
  return SPEC_OK;
}

void deal_items(std::vector<AttnItem>& list) {
  struct Group { size_t first, count; int64_t work; };
  std::vector<Group> groups;
  for (size_t i = 0; i < list.size();) {
    size_t j = i;
    while (j < list.size() && list[j].sample == list[i].sample && list[j].kvh == list[i].kvh &&
           list[j].key0 == list[i].key0)
      ++j;
    groups.push_back(Group{i, j - i, (int64_t)(list[i].key1 - list[i].key0) * (int64_t)(j - i)});
    i = j;
  }
  std::stable_sort(groups.begin(), groups.end(),
                   [](const Group& x, const Group& y) { return x.work > y.work; });
  std::vector<AttnItem> xcd[8];
  int64_t load[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  for (const Group& gp : groups) {
    const int x = (int)(std::min_element(load, load + 8) - load);
    load[x] += gp.work;
    xcd[x].insert(xcd[x].end(), list.begin() + gp.first, list.begin() + gp.first + gp.count);
  }
  size_t per = 0;
  for (auto& v : xcd) per = std::max(per, v.size());
  std::vector<AttnItem> dealt;
  dealt.reserve(per * 8);
  for (auto& v : xcd) {
    dealt.insert(dealt.end(), v.begin(), v.end());
    dealt.resize(dealt.size() + (per - v.size()), AttnItem{-1, 0, 0, 0, 0, 1, 0, 0});
  }
  list.swap(dealt);
}

}  // namespace spec

SPEC_API const char* spec_last_error(void) { return g_err.c_str(); }

namespace spec {
int set_error(int code, const char* msg) {
  g_err = msg;
  return code;
}
}  // namespace spec

SPEC_API size_t spec_kv_bytes(const spec_model_config* cfg, int32_t n_samples,
                              const int32_t* capacity) {
  std::string why;
  if (!cfg || !capacity || n_samples < 1 || !config_ok(cfg, &why)) return 0;
  size_t total = 0;
  for (int i = 0; i < n_samples; ++i) {
    if (capacity[i] < 1) return 0;
    total += sample_bytes(cfg, capacity[i]);
  }
  return total + align_up((size_t)n_samples * sizeof(SampleInfo));
}

SPEC_API int spec_kv_alloc(const spec_model_config* cfg, int32_t n_samples,
                           const int32_t* capacity, void* device_buf, size_t buf_bytes,
                           spec_kv** out) {
  g_err.clear();
  if (!cfg || !capacity || !device_buf || !out) return fail(SPEC_ERR_INVALID, "null argument");
  if (n_samples < 1) return fail(SPEC_ERR_INVALID, "n_samples must be >= 1");
  std::string why;
  if (!config_ok(cfg, &why)) return fail(SPEC_ERR_UNSUPPORTED, "%s", why.c_str());
  if ((uintptr_t)device_buf % kAlign) return fail(SPEC_ERR_INVALID, "device_buf not 256-byte aligned");
  for (int i = 0; i < n_samples; ++i)
    if (capacity[i] < 1) return fail(SPEC_ERR_INVALID, "capacity[%d] = %d", i, capacity[i]);
  const size_t need = spec_kv_bytes(cfg, n_samples, capacity);
  if (buf_bytes < need)
    return fail(SPEC_ERR_CAPACITY, "KV buffer holds %zu bytes, needs %zu", buf_bytes, need);
  spec_kv* kv = new spec_kv;
  kv->cfg = *cfg;
  kv->n = n_samples;
  kv->cap.assign(capacity, capacity + n_samples);
  kv->base.resize(n_samples);
  size_t off = 0;
  for (int i = 0; i < n_samples; ++i) {
    kv->base[i] = (int64_t)(off / 2);
    off += sample_bytes(cfg, capacity[i]);
  }
  kv->ctl_off = off;
  kv->pool = (bf16*)device_buf;
  kv->bytes = buf_bytes;
  *out = kv;
  return SPEC_OK;
}

SPEC_API int spec_kv_free(spec_kv* kv) {
  if (!kv) return fail(SPEC_ERR_INVALID, "null handle");
  const int rc = kv->ring.release();
  delete kv;
  return rc;
}

SPEC_API int spec_kv_sample_layout(const spec_kv* kv, int32_t sample, int64_t* byte_offset,
                                   int32_t* capacity) {
  if (!kv || !byte_offset || !capacity) return fail(SPEC_ERR_INVALID, "null argument");
  if (sample < 0 || sample >= kv->n) return fail(SPEC_ERR_INVALID, "sample %d out of range", sample);
  *byte_offset = kv->base[sample] * 2;
  *capacity = kv->cap[sample];
  return SPEC_OK;
}

SPEC_API size_t spec_workspace_bytes(const spec_model_config* cfg, int32_t max_batch,
                                     int32_t max_tokens) {
  std::string why;
  if (!cfg || max_batch < 1 || max_tokens < max_batch || !config_ok(cfg, &why)) return 0;
  return ws_layout(cfg, max_batch, max_tokens).total;
}

namespace {

// Attention work items of a step over the bf16 pool, by kernel, and the combine jobs.
struct AttnWork {
  std::vector<AttnItem> items, wide4, wide8;
  std::vector<CombineItem> comb;
};

void plan_split_kv(const spec_model_config* cfg, const std::vector<SampleInfo>& si, AttnWork* out) {
  const int batch = (int)si.size(), nkv = cfg->n_kv_heads, G = cfg->n_heads / nkv;
  // Split-KV plan.  A row tile is 32 query rows of one (sample, kv head).  A
  // (sample, kv head) with one tile gets narrow items (2 waves dealing the
  // keys among themselves, two work-groups per CU); 2-4 tiles get one 4-wave
  // wide group (two per CU); more get 8-wave groups of 8 tiles (one per CU).
  // Every (sample, kv head) key range is cut into chunks of `chunk` keys,
  // sized so that the whole call is about kTargetSlots chunk-sized CU
  // occupancies (a few per CU, for balance), with at most kMaxSplits chunks
  // per range and at most kPartCap partial states.
  auto tiles_of = [&](int b) { return (si[b].ntok * G + 31) / 32; };
  auto keys_of = [&](int b) { return (int64_t)si[b].seq_len + si[b].ntok; };
  // Cost weight of one chunk's work-groups: their CU occupancy, except that a
  // narrow item counts as a whole CU (measured: sizing its chunks as half a
  // CU's worth, i.e. twice as many splits, is slower).
  auto cu_weight = [&](int tiles) {
    return tiles == 1 ? 1.0 : tiles <= 4 ? 0.5 : (double)((tiles + 7) / 8);
  };
  int64_t max_keys = 0;
  double work = 0.0;
  for (int b = 0; b < batch; ++b) {
    max_keys = std::max(max_keys, keys_of(b));
    work += (double)nkv * keys_of(b) * cu_weight(tiles_of(b));
  }
  auto part_slots = [&](int64_t c) {
    int64_t slots = 0;
    for (int b = 0; b < batch; ++b) {
      const int64_t ns = (keys_of(b) + c - 1) / c;
      if (ns > 1) slots += ns * nkv * tiles_of(b);
    }
    return slots;
  };
  // Chunk length: a multiple of 128 keys.  A small call (under kSmallChunk
  // keys of work per slot at that target) instead aims at one round of the
  // 256 CUs, in multiples of 64 keys between kMinChunk and kSmallChunk: a
  // single short sample gets more, shorter chunks (each work-group's block
  // chain is serial), and a few samples with multi-tile trees do not spill
  // into a second round.  Measured per 32-layer step against a 256-key floor:
  // batch 1, 1.1K keys, attention 0.50 -> 0.44 ms; against the two-round
  // target at 64-key granularity: batch 4 x 16 nodes 5.75 -> 5.48 ms.
  auto round128 = [](int64_t x) { return (x + 127) / 128 * 128; };
  auto round64 = [](int64_t x) { return (x + 63) / 64 * 64; };
  const int64_t min_split = (max_keys + kMaxSplits - 1) / kMaxSplits;
  const int64_t want = std::max<int64_t>(min_split, (int64_t)(work / kTargetSlots));
  int64_t chunk = round128(want);
  if (want < kSmallChunk)
    chunk = std::min<int64_t>(kSmallChunk, round64(std::max<int64_t>({kMinChunk, min_split, (int64_t)(work / 256)})));
  while (part_slots(chunk) > kPartCap) chunk += 128;    // terminates: one chunk per range has none
  // Work items.  Split key ranges write their partial states to per-tile
  // slots part + tile * ns + split.
  std::vector<AttnItem>&items = out->items, &wide4 = out->wide4, &wide8 = out->wide8;
  std::vector<CombineItem>& comb = out->comb;
  int part = 0;
  for (int b = 0; b < batch; ++b) {
    const int keys = (int)keys_of(b);
    const int ns = (int)((keys + chunk - 1) / chunk);
    const int tiles = tiles_of(b);
    for (int g = 0; g < nkv; ++g) {
      for (int t = 0; t < tiles && ns > 1; ++t)
        comb.push_back(CombineItem{b, g, t * 32, ns, part + t * ns, 0, 0, 0});
      for (int k = 0; k < ns; ++k) {
        const int k0 = (int)(k * chunk), k1 = (int)std::min<int64_t>(keys, (k + 1) * chunk);
        const int p = ns > 1 ? part + k : 0;
        if (tiles == 1)
          items.push_back(AttnItem{b, g, 0, k0, k1, ns, p, 0});
        else if (tiles <= 4)
          wide4.push_back(AttnItem{b, g, 0, k0, k1, ns, p, 0});
        else
          for (int rg = 0; rg < (tiles + 7) / 8; ++rg)
            wide8.push_back(AttnItem{b, g, rg * 256, k0, k1, ns, ns > 1 ? p + rg * 8 * ns : 0, 0});
      }
      if (ns > 1) part += ns * tiles;
    }
  }
  deal_items(items);
  deal_items(wide4);
  deal_items(wide8);
}

int check_w4_matrix(const spec_w4& m, int rows, int cols, const char* what) {
  if (!m.data) return fail(SPEC_ERR_INVALID, "null weight pointer: %s", what);
  if ((uintptr_t)m.data % kAlign) return fail(SPEC_ERR_INVALID, "%s: matrix data not 256-byte aligned", what);
  if (m.rows != rows || m.cols != cols)
    return fail(SPEC_ERR_INVALID, "%s is %d x %d, the model's %d x %d", what, m.rows, m.cols, rows, cols);
  return SPEC_OK;
}

int check_w4_weights(const spec_model_config* c, const spec_weights_w4* w) {
  if (!w->tok_embed || !w->final_norm || !w->attn_norm || !w->wqkv || !w->wo || !w->ffn_norm || !w->w_gate ||
      !w->w_up || !w->w_down)
    return fail(SPEC_ERR_INVALID, "null weight pointer");
  const int q = c->n_heads * c->head_dim, kv = c->n_kv_heads * c->head_dim;
  if (int rc = check_w4_matrix(w->lm_head, c->vocab, c->hidden, "lm_head")) return rc;
  for (int l = 0; l < c->n_layers; ++l) {
    if (!w->attn_norm[l] || !w->ffn_norm[l]) return fail(SPEC_ERR_INVALID, "null weight pointer in layer %d", l);
    if (int rc = check_w4_matrix(w->wqkv[l], q + 2 * kv, c->hidden, "wqkv")) return rc;
    if (int rc = check_w4_matrix(w->wo[l], c->hidden, q, "wo")) return rc;
    if (int rc = check_w4_matrix(w->w_gate[l], c->ffn, c->hidden, "w_gate")) return rc;
    if (int rc = check_w4_matrix(w->w_up[l], c->ffn, c->hidden, "w_up")) return rc;
    if (int rc = check_w4_matrix(w->w_down[l], c->hidden, c->ffn, "w_down")) return rc;
  }
  return SPEC_OK;
}

// Over the bf16 pool `kv`, or over the 4-bit one `kv4`; with weights w, or w4.
int verify_impl(const spec_model_config* cfg, const spec_weights* w, spec_kv* kv, spec_kv4* kv4,
                int32_t batch, const int32_t* sample_ids, const int32_t* tree_offsets, const int32_t* tree_tokens,
                const int32_t* tree_parents, const int32_t* seq_lens, void* workspace,
                size_t ws_bytes, void* stream, const spec_sampling* samp, int32_t* accepted_len,
                int32_t* next_token, int32_t* accepted_nodes, const spec_debug* dbg,
                bool noalloc = false, const spec_weights_w4* w4 = nullptr) {
  // ---- validation (no side effects) ----
  if (!cfg || (!w && !w4) || (!kv && !kv4) || !sample_ids || !tree_offsets || !tree_tokens || !tree_parents ||
      !seq_lens || (!workspace && !noalloc) || !accepted_len || !next_token || !accepted_nodes)
    return fail(SPEC_ERR_INVALID, "null argument");
  std::string why;
  if (!config_ok(cfg, &why)) return fail(SPEC_ERR_UNSUPPORTED, "%s", why.c_str());
  if (!same_config(cfg, kv4 ? &kv4->cfg : &kv->cfg)) return fail(SPEC_ERR_INVALID, "config differs from the KV pool's");
  if (batch < 1) return fail(SPEC_ERR_INVALID, "batch must be >= 1");
  if (w4) {
    if (int rc = check_w4_weights(cfg, w4)) return rc;
  } else if (!w->tok_embed || !w->final_norm || !w->lm_head || !w->attn_norm || !w->wq || !w->wk ||
             !w->wv || !w->wo || !w->ffn_norm || !w->w_gate || !w->w_up || !w->w_down) {
    return fail(SPEC_ERR_INVALID, "null weight pointer");
  }
  for (int l = 0; !w4 && l < cfg->n_layers; ++l)
    if (!w->attn_norm[l] || !w->wq[l] || !w->wk[l] || !w->wv[l] || !w->wo[l] || !w->ffn_norm[l] ||
        !w->w_gate[l] || !w->w_up[l] || !w->w_down[l])
      return fail(SPEC_ERR_INVALID, "null weight pointer in layer %d", l);
  if (kv4) {
    if (int rc = kv4_check_rows(kv4, batch, sample_ids, tree_offsets, tree_parents, seq_lens)) return rc;
    for (int i = 0; i < tree_offsets[batch]; ++i)
      if (tree_tokens[i] < 0 || tree_tokens[i] >= cfg->vocab)
        return fail(SPEC_ERR_TREE, "row %d: token %d out of range", i, tree_tokens[i]);
  } else {
    if (int rc = check_samples(kv, batch, sample_ids)) return rc;
    if (tree_offsets[0] != 0) return fail(SPEC_ERR_TREE, "tree_offsets[0] must be 0");
    for (int b = 0; b < batch; ++b) {
      const int T = tree_offsets[b + 1] - tree_offsets[b];
      if (T < 1 || T > SPEC_MAX_TREE)
        return fail(T < 1 ? SPEC_ERR_TREE : SPEC_ERR_UNSUPPORTED, "sample %d has %d tree nodes", b, T);
      const int S = seq_lens[b];
      if (S < 0) return fail(SPEC_ERR_INVALID, "seq_lens[%d] = %d", b, S);
      if ((int64_t)S + T > kv->cap[sample_ids[b]])
        return fail(SPEC_ERR_CAPACITY, "sample %d: %d committed + %d nodes exceed capacity %d", b, S,
                    T, kv->cap[sample_ids[b]]);
      const int t0 = tree_offsets[b];
      if (tree_parents[t0] != -1) return fail(SPEC_ERR_TREE, "sample %d: root parent must be -1", b);
      for (int i = 0; i < T; ++i) {
        const int tok = tree_tokens[t0 + i];
        if (tok < 0 || tok >= cfg->vocab)
          return fail(SPEC_ERR_TREE, "sample %d node %d: token %d out of range", b, i, tok);
        if (i > 0) {
          const int p = tree_parents[t0 + i];
          if (p < 0 || p >= i)
            return fail(SPEC_ERR_TREE, "sample %d node %d: parent %d not before the node", b, i, p);
        }
      }
    }
  }
  const bool sampled = samp && samp->temperature > 0.f;
  if (samp) {
    if (!(samp->temperature >= 0.f) || !std::isfinite(samp->temperature))
      return fail(SPEC_ERR_INVALID, "temperature must be finite and >= 0");
    if (samp->eos_token < -1 || samp->eos_token >= cfg->vocab)
      return fail(SPEC_ERR_INVALID, "eos_token %d out of range", samp->eos_token);
    if (sampled && (!samp->draft_probs || !samp->uniforms))
      return fail(SPEC_ERR_INVALID, "sampling needs draft_probs and uniforms");
  }
  const int N = tree_offsets[batch];
  const int64_t pages = kv4 ? kv4_step_pages(kv4, batch, tree_offsets, seq_lens) : 0;
  if (w4 && N > 65535) return fail(SPEC_ERR_UNSUPPORTED, "%d tree nodes in one call, at most 65535", N);
  const WsLayout ly = ws_layout(cfg, batch, N, sampled, pages, w4 != nullptr);
  const size_t need = ly.total;
  if (noalloc && need > SPEC_NOALLOC_SCRATCH_BYTES)
    return fail(SPEC_ERR_WORKSPACE,
                "%d samples with %d tree nodes need %zu bytes of workspace, more than the %zu "
                "bytes of spec_verify_noalloc's static scratch",
                batch, N, need, (size_t)SPEC_NOALLOC_SCRATCH_BYTES);
  if (noalloc) {
    HIP_TRY(noalloc_scratch(&workspace), "static scratch lookup");
    ws_bytes = SPEC_NOALLOC_SCRATCH_BYTES;
  }
  if (ws_bytes < need) return fail(SPEC_ERR_WORKSPACE, "workspace %zu bytes, needs %zu", ws_bytes, need);
  if (kv4 || w4) {
    if ((uintptr_t)workspace % kAlign) return fail(SPEC_ERR_INVALID, "workspace not 256-byte aligned");
    if (int rc = refuse_capture(stream)) return rc;
  }

  // ---- planning ----
  const int L = cfg->n_layers, H = cfg->hidden, nq = cfg->n_heads, nkv = cfg->n_kv_heads;
  const int hd = cfg->head_dim, F = cfg->ffn, V = cfg->vocab;
  char* ws = (char*)workspace;
  hipStream_t s = (hipStream_t)stream;

  std::vector<SampleInfo> si(batch);
  for (int b = 0; b < batch; ++b) {
    const int id = sample_ids[b], T = tree_offsets[b + 1] - tree_offsets[b];
    // The q/k/v product writes K/V to the bf16 pool, or, on their way to the 4-bit one, to
    // this layer's rows: a block [K, V][kv head][node][head_dim] per sample.
    si[b] = kv4 ? SampleInfo{(int64_t)tree_offsets[b] * 2 * nkv * hd, T, 0, tree_offsets[b], T, 0, 0}
                : SampleInfo{kv->base[id], kv->cap[id], seq_lens[b], tree_offsets[b], T, 0, 0};
  }
  AttnWork aw;
  if (!kv4) plan_split_kv(cfg, si, &aw);
  const std::vector<AttnItem>&items = aw.items, &wide4 = aw.wide4, &wide8 = aw.wide8;
  const std::vector<CombineItem>& comb = aw.comb;

  // ---- one upload of the per-call descriptors ----
  const size_t o_si = 0;
  const size_t o_tok = align_up(batch * sizeof(SampleInfo));
  const size_t o_par = o_tok + align_up((size_t)N * 4);
  const size_t o_items = o_par + align_up((size_t)N * 4);
  const size_t o_wide4 = o_items + align_up(items.size() * sizeof(AttnItem));
  const size_t o_wide8 = o_wide4 + align_up(wide4.size() * sizeof(AttnItem));
  const size_t o_comb = o_wide8 + align_up(wide8.size() * sizeof(AttnItem));
  const size_t blob_bytes = o_comb + comb.size() * sizeof(CombineItem);
  std::vector<char> blob(blob_bytes, 0);
  memcpy(blob.data() + o_si, si.data(), batch * sizeof(SampleInfo));
  memcpy(blob.data() + o_tok, tree_tokens, (size_t)N * 4);
  memcpy(blob.data() + o_par, tree_parents, (size_t)N * 4);
  memcpy(blob.data() + o_items, items.data(), items.size() * sizeof(AttnItem));
  if (!wide4.empty()) memcpy(blob.data() + o_wide4, wide4.data(), wide4.size() * sizeof(AttnItem));
  if (!wide8.empty()) memcpy(blob.data() + o_wide8, wide8.data(), wide8.size() * sizeof(AttnItem));
  if (!comb.empty()) memcpy(blob.data() + o_comb, comb.data(), comb.size() * sizeof(CombineItem));
  if (noalloc)   // no pinned staging: a copy from pageable memory, done before the call returns
    HIP_TRY(hipMemcpyAsync(ws + ly.blob, blob.data(), blob_bytes, hipMemcpyHostToDevice, s),
            "upload");
  else if (int rc = kv4 ? kv4->ring.upload(blob.data(), blob_bytes, ws + ly.blob, s)
                        : kv->ring.upload(blob.data(), blob_bytes, ws + ly.blob, s))
    return rc;

  const SampleInfo* d_si = (const SampleInfo*)(ws + ly.blob + o_si);
  const int32_t* d_tok = (const int32_t*)(ws + ly.blob + o_tok);
  const int32_t* d_par = (const int32_t*)(ws + ly.blob + o_par);
  const AttnItem* d_items = (const AttnItem*)(ws + ly.blob + o_items);
  const AttnItem* d_wide4 = (const AttnItem*)(ws + ly.blob + o_wide4);
  const AttnItem* d_wide8 = (const AttnItem*)(ws + ly.blob + o_wide8);
  const CombineItem* d_comb = (const CombineItem*)(ws + ly.blob + o_comb);
  const TokInfo* d_toks = (const TokInfo*)(ws + ly.toks);
  const uint64_t* d_anc = (const uint64_t*)(ws + ly.anc);
  float2* d_rope = (float2*)(ws + ly.rope);
  float* d_x = (float*)(ws + ly.x);
  bf16* d_h = (bf16*)(ws + ly.h);
  bf16* d_q = (bf16*)(ws + ly.q);
  bf16* d_o = (bf16*)(ws + ly.o);
  bf16* d_act = (bf16*)(ws + ly.act);
  float* d_lmv = (float*)(ws + ly.lm_val);
  int32_t* d_lmi = (int32_t*)(ws + ly.lm_idx);
  int32_t* d_arg = (int32_t*)(ws + ly.argmax);

  const spec_debug nodbg{};
  const spec_debug& D = dbg ? *dbg : nodbg;

  // ---- the step ----
  spec_kv4_step step;
  bf16* d_kv4 = (bf16*)(ws + ly.kv4_rows);
  if (kv4) {
    if (int rc = kv4_plan_step(kv4, batch, sample_ids, tree_offsets, tree_parents, seq_lens, ws + ly.kv4_step, s, D,
                               &step))
      return rc;
    d_toks = step.rows.toks;
    d_anc = step.attn.anc;
  } else {
    HIP_TRY(launch_tree_meta(d_si, batch, d_par, (TokInfo*)(ws + ly.toks), (uint64_t*)(ws + ly.anc), D.depth, D.pos,
                             D.anc, s),
            "tree meta");
  }
  const void* const* attn_norm = w4 ? w4->attn_norm : w->attn_norm;
  const void* const* ffn_norm = w4 ? w4->ffn_norm : w->ffn_norm;
  const void* final_norm = w4 ? w4->final_norm : w->final_norm;
  const void* tok_embed = w4 ? w4->tok_embed : w->tok_embed;
  HIP_TRY(launch_row_front(d_toks, d_tok, (const bf16*)tok_embed, (const bf16*)attn_norm[0], d_x, d_h,
                           N, H, cfg->rms_eps, hd, cfg->rope_theta, d_rope, s),
          "row front");

  GemmArgs ga{};
  ga.M = N;
  ga.samples = d_si;
  ga.toks = d_toks;
  ga.kv_pool = kv4 ? d_kv4 : kv->pool;
  ga.n_kv_heads = nkv;
  ga.head_dim = hd;
  ga.rope_cs = d_rope;
  ga.partial = (float*)(ws + ly.splitk);
  AttnArgs aa{};
  aa.q = d_q;
  aa.kv_pool = ga.kv_pool;
  aa.samples = d_si;
  aa.toks = d_toks;
  aa.anc = d_anc;
  aa.items = d_items;
  aa.n_items = (int)items.size();
  aa.wide = d_wide4;
  aa.n_wide = (int)wide4.size();
  aa.wide8 = d_wide8;
  aa.n_wide8 = (int)wide8.size();
  aa.part_o = (f16*)(ws + ly.part_o);
  aa.part_ml = (float*)(ws + ly.part_ml);
  aa.out = d_o;
  aa.n_heads = nq;
  aa.n_kv_heads = nkv;
  aa.head_dim = hd;
  aa.comb = d_comb;
  aa.n_comb = (int)comb.size();

  // Every RMSNorm after the first follows a residual product (O or down
  // projection); when that product is split over K the norm runs inside its
  // split-K reduction, otherwise on its own.
  bool fused;
  auto resid_then_norm = [&](int kind, GemmArgs g, const void* gain, const char* what) -> int {
    fused = false;
    g.norm_gain = (const bf16*)gain;
    g.norm_out = d_h;
    g.norm_eps = cfg->rms_eps;
    g.norm_done = &fused;
    HIP_TRY(timed(kind, s, [&] { return launch_gemm(EPI_RESID, g, s); }), what);
    if (!fused) HIP_TRY(launch_rmsnorm(d_x, (const bf16*)gain, d_h, N, H, cfg->rms_eps, s), "rmsnorm");
    return SPEC_OK;
  };
  // One product with weights in 4 bits, of the plan that its kind of product has in all layers.
  auto w4_product = [&](int kind, const W4Plan& plan, const spec_w4& m, const spec_w4* up, const bf16* x, void* out,
                        int out_kind, const char* what) -> int {
    const W4Args a{plan, (const char*)m.data, up ? (const char*)up->data : nullptr, m.rows, m.cols, x, m.cols, N,
                   out, m.rows, out_kind, (float*)(ws + ly.splitk)};
    HIP_TRY(timed(kind, s, [&] { return launch_w4(a, s); }), what);
    return SPEC_OK;
  };
  auto attend = [&](int l) -> int {
    if (kv4) {
      if (int rc = kv4_append_blocks(&step, l, d_kv4, s)) return rc;
      return kv4_attend(&step, l, d_q, (int64_t)nq * hd, d_o, s);
    }
    aa.layer = l;
    HIP_TRY(timed(SPEC_K_ATTENTION, s, [&] { return launch_attention(aa, s); }), "attention");
    return SPEC_OK;
  };
  if (w4) {
    float* partial = (float*)(ws + ly.splitk);
    float* logits = D.logits ? D.logits : (float*)(ws + ly.logits);
    const int wide = (nq + 2 * nkv) * hd;
    const W4Plan p_qkv = plan_w4(wide, H, N, false), p_o = plan_w4(H, nq * hd, N, false),
                 p_gate_up = plan_w4(F, H, N, true), p_down = plan_w4(H, F, N, false),
                 p_head = plan_w4(V, H, N, false);
    // x += a product, and the norm that follows in the kernel that joins its splits.
    auto resid_norm = [&](int kind, const W4Plan& plan, const spec_w4& m, const bf16* x, const void* gain,
                          const char* what) -> int {
      if (int rc = w4_product(kind, plan, m, nullptr, x, nullptr, kW4Partial, what)) return rc;
      GemmArgs g = ga;
      g.plan.splits = plan.splits;
      g.N = H;
      g.x = d_x;
      g.norm_gain = (const bf16*)gain;
      g.norm_out = d_h;
      g.norm_eps = cfg->rms_eps;
      g.norm_done = &fused;
      fused = false;
      HIP_TRY(launch_resid_reduce(g, s), what);
      if (!fused) HIP_TRY(launch_rmsnorm(d_x, (const bf16*)gain, d_h, N, H, cfg->rms_eps, s), "rmsnorm");
      return SPEC_OK;
    };
    for (int l = 0; l < L; ++l) {
      const void* next_norm = l + 1 < L ? attn_norm[l + 1] : final_norm;
      if (int rc = w4_product(SPEC_K_GEMM_QKV, p_qkv, w4->wqkv[l], nullptr, d_h, nullptr, kW4Partial, "qkv product"))
        return rc;
      HIP_TRY(launch_place_qkv(partial, p_qkv.splits, N, d_si, d_toks, d_rope, d_q, kv4 ? d_kv4 : kv->pool, kv4 ? 0 : l, nq, nkv, hd,
                               s),
              "place q, k, v");
      if (int rc = attend(l)) return rc;
      if (int rc = resid_norm(SPEC_K_GEMM_O, p_o, w4->wo[l], d_o, ffn_norm[l], "o product")) return rc;
      if (int rc = w4_product(SPEC_K_GEMM_GATE_UP, p_gate_up, w4->w_gate[l], &w4->w_up[l], d_h, d_act, SPEC_W4_BF16,
                              "gate/up product"))
        return rc;
      if (int rc = resid_norm(SPEC_K_GEMM_DOWN, p_down, w4->w_down[l], d_act, next_norm, "down product")) return rc;
    }
    if (int rc = w4_product(SPEC_K_LM_HEAD, p_head, w4->lm_head, nullptr, d_h, logits, SPEC_W4_F32, "lm head"))
      return rc;
    HIP_TRY(launch_logit_max(logits, N, V, d_lmv, d_lmi, s), "logits' maxima");
  } else {
    const GemmPlan p_qkv = product_plan(cfg, SPEC_K_GEMM_QKV, N), p_o = product_plan(cfg, SPEC_K_GEMM_O, N),
                   p_gate_up = product_plan(cfg, SPEC_K_GEMM_GATE_UP, N),
                   p_down = product_plan(cfg, SPEC_K_GEMM_DOWN, N), p_head = product_plan(cfg, SPEC_K_LM_HEAD, N);
    for (int l = 0; l < L; ++l) {
      GemmArgs g = ga;
      g.plan = p_qkv;
      g.A = d_h;
      g.K = H;
      g.B0 = (const bf16*)w->wq[l];
      g.B1 = (const bf16*)w->wk[l];
      g.B2 = (const bf16*)w->wv[l];
      g.n0 = nq * hd;
      g.n1 = g.n2 = nkv * hd;
      g.N = g.n0 + g.n1 + g.n2;
      g.q_out = d_q;
      g.layer = kv4 ? 0 : l;
      HIP_TRY(timed(SPEC_K_GEMM_QKV, s, [&] { return launch_gemm(EPI_QKV, g, s); }), "qkv gemm");
      if (int rc = attend(l)) return rc;
      g = ga;
      g.plan = p_o;
      g.A = d_o;
      g.K = nq * hd;
      g.B0 = (const bf16*)w->wo[l];
      g.n0 = g.N = H;
      g.x = d_x;
      if (int rc = resid_then_norm(SPEC_K_GEMM_O, g, ffn_norm[l], "o gemm")) return rc;
      g = ga;
      g.plan = p_gate_up;
      g.A = d_h;
      g.K = H;
      g.B0 = (const bf16*)w->w_gate[l];
      g.B1 = (const bf16*)w->w_up[l];
      g.n0 = g.n1 = F;
      g.N = 2 * F;
      g.act_out = d_act;
      HIP_TRY(timed(SPEC_K_GEMM_GATE_UP, s, [&] { return launch_gemm(EPI_GATE_UP, g, s); }), "gate/up gemm");
      g = ga;
      g.plan = p_down;
      g.A = d_act;
      g.K = F;
      g.B0 = (const bf16*)w->w_down[l];
      g.n0 = g.N = H;
      g.x = d_x;
      const void* next_norm = l + 1 < L ? attn_norm[l + 1] : final_norm;
      if (int rc = resid_then_norm(SPEC_K_GEMM_DOWN, g, next_norm, "down gemm")) return rc;
    }
    GemmArgs g = ga;
    g.plan = p_head;
    g.A = d_h;
    g.K = H;
    g.B0 = (const bf16*)w->lm_head;
    g.n0 = g.N = V;
    g.part_val = d_lmv;
    g.part_idx = d_lmi;
    g.logits = D.logits ? D.logits : sampled ? (float*)(ws + ly.logits) : nullptr;
    HIP_TRY(timed(SPEC_K_LM_HEAD, s, [&] { return launch_gemm(EPI_ARGMAX, g, s); }), "lm head");
  }
  HIP_TRY(launch_argmax_reduce(d_lmv, d_lmi, N, w4 ? logit_parts(V) : V / 64, d_arg, D.argmax, s), "argmax");
  if (sampled) {
    const float* logits = D.logits ? D.logits : (const float*)(ws + ly.logits);
    HIP_TRY(timed(SPEC_K_ACCEPT, s, [&] {
              return launch_sample_accept(d_si, batch, N, d_toks, d_tok, d_par, logits, d_arg,
                                          samp->draft_probs, samp->uniforms, V, samp->temperature,
                                          samp->eos_token, ws + ly.resid, accepted_len, next_token,
                                          accepted_nodes, s);
            }),
            "sampled accept");
  } else {
    HIP_TRY(timed(SPEC_K_ACCEPT, s, [&] {
              return launch_accept(d_si, batch, d_tok, d_par, d_toks, d_anc, d_arg,
                                   samp ? samp->eos_token : -1, accepted_len, next_token, accepted_nodes,
                                   s);
            }),
            "accept");
  }
  return SPEC_OK;
}

}  // namespace

SPEC_API int spec_verify(const spec_model_config* cfg, const spec_weights* w, spec_kv* kv,
                         int32_t batch, const int32_t* sample_ids, const int32_t* tree_offsets,
                         const int32_t* tree_tokens, const int32_t* tree_parents,
                         const int32_t* seq_lens, void* workspace, size_t ws_bytes, void* stream,
                         int32_t* accepted_len, int32_t* next_token, int32_t* accepted_nodes,
                         const spec_debug* dbg) {
  g_err.clear();
  return verify_impl(cfg, w, kv, nullptr, batch, sample_ids, tree_offsets, tree_tokens, tree_parents,
                     seq_lens, workspace, ws_bytes, stream, nullptr, accepted_len, next_token,
                     accepted_nodes, dbg);
}

SPEC_API size_t spec_workspace_bytes_sampled(const spec_model_config* cfg, int32_t max_batch,
                                             int32_t max_tokens) {
  std::string why;
  if (!cfg || max_batch < 1 || max_tokens < max_batch || !config_ok(cfg, &why)) return 0;
  return ws_layout(cfg, max_batch, max_tokens, true).total;
}

SPEC_API int spec_verify_sampled(const spec_model_config* cfg, const spec_weights* w,
                                 spec_kv* kv, int32_t batch, const int32_t* sample_ids,
                                 const int32_t* tree_offsets, const int32_t* tree_tokens,
                                 const int32_t* tree_parents, const int32_t* seq_lens,
                                 void* workspace, size_t ws_bytes, void* stream,
                                 const spec_sampling* samp, int32_t* accepted_len,
                                 int32_t* next_token, int32_t* accepted_nodes,
                                 const spec_debug* dbg) {
  g_err.clear();
  if (!samp) return fail(SPEC_ERR_INVALID, "null sampling parameters");
  return verify_impl(cfg, w, kv, nullptr, batch, sample_ids, tree_offsets, tree_tokens, tree_parents,
                     seq_lens, workspace, ws_bytes, stream, samp, accepted_len, next_token,
                     accepted_nodes, dbg);
}

SPEC_API int spec_verify_noalloc(const spec_model_config* cfg, const spec_weights* w,
                                 spec_kv* kv, int32_t batch, const int32_t* sample_ids,
                                 const int32_t* tree_offsets, const int32_t* tree_tokens,
                                 const int32_t* tree_parents, const int32_t* seq_lens,
                                 void* stream, int32_t* accepted_len, int32_t* next_token,
                                 int32_t* accepted_nodes, const spec_debug* dbg) {
  g_err.clear();
  return verify_impl(cfg, w, kv, nullptr, batch, sample_ids, tree_offsets, tree_tokens, tree_parents,
                     seq_lens, nullptr, 0, stream, nullptr, accepted_len, next_token,
                     accepted_nodes, dbg, true);
}

SPEC_API size_t spec_workspace_bytes_kv4(const spec_model_config* cfg, int32_t max_batch, int32_t max_tokens,
                                         int32_t max_pages, int32_t sampled) {
  std::string why;
  if (!cfg || max_batch < 1 || max_tokens < max_batch || max_pages < 1 || !config_ok(cfg, &why)) return 0;
  return ws_layout(cfg, max_batch, max_tokens, sampled != 0, max_pages).total;
}

SPEC_API int spec_verify_kv4(const spec_model_config* cfg, const spec_weights* w, spec_kv4* kv,
                             int32_t batch, const int32_t* sample_ids, const int32_t* tree_offsets,
                             const int32_t* tree_tokens, const int32_t* tree_parents,
                             const int32_t* seq_lens, void* workspace, size_t ws_bytes, void* stream,
                             const spec_sampling* samp, int32_t* accepted_len, int32_t* next_token,
                             int32_t* accepted_nodes, const spec_debug* dbg) {
  return guarded([&]() -> int {
    if (!kv) return fail(SPEC_ERR_INVALID, "null argument");
    return verify_impl(cfg, w, nullptr, kv, batch, sample_ids, tree_offsets, tree_tokens, tree_parents, seq_lens,
                       workspace, ws_bytes, stream, samp, accepted_len, next_token, accepted_nodes, dbg);
  });
}

SPEC_API size_t spec_workspace_bytes_w4(const spec_model_config* cfg, int32_t max_batch, int32_t max_tokens,
                                        int32_t max_pages, int32_t sampled) {
  std::string why;
  if (!cfg || max_batch < 1 || max_tokens < max_batch || max_pages < 0 || !config_ok(cfg, &why)) return 0;
  return ws_layout(cfg, max_batch, max_tokens, sampled != 0, max_pages, true).total;
}

SPEC_API int spec_verify_w4(const spec_model_config* cfg, const spec_weights_w4* w, spec_kv* kv, spec_kv4* kv4,
                            int32_t batch, const int32_t* sample_ids, const int32_t* tree_offsets,
                            const int32_t* tree_tokens, const int32_t* tree_parents, const int32_t* seq_lens,
                            void* workspace, size_t ws_bytes, void* stream, const spec_sampling* samp,
                            int32_t* accepted_len, int32_t* next_token, int32_t* accepted_nodes,
                            const spec_debug* dbg) {
  return guarded([&]() -> int {
    if (!w) return fail(SPEC_ERR_INVALID, "null argument");
    if (!kv == !kv4) return fail(SPEC_ERR_INVALID, "one pool: kv or kv4");
    return verify_impl(cfg, nullptr, kv, kv4, batch, sample_ids, tree_offsets, tree_tokens, tree_parents, seq_lens,
                       workspace, ws_bytes, stream, samp, accepted_len, next_token, accepted_nodes, dbg, false, w);
  });
}

SPEC_API int spec_kv_commit(spec_kv* kv, int32_t batch, const int32_t* sample_ids,
                            const int32_t* seq_lens, const int32_t* accepted_len,
                            const int32_t* accepted_nodes, int32_t* new_seq_lens, void* stream) {
  g_err.clear();
  if (!kv || !sample_ids || !seq_lens || !accepted_len || !accepted_nodes || !new_seq_lens)
    return fail(SPEC_ERR_INVALID, "null argument");
  if (batch < 1 || batch > kv->n) return fail(SPEC_ERR_INVALID, "batch %d out of range", batch);
  if (int rc = check_samples(kv, batch, sample_ids)) return rc;
  std::vector<SampleInfo> si(batch);
  for (int b = 0; b < batch; ++b) {
    const int id = sample_ids[b];
    if (seq_lens[b] < 0 || seq_lens[b] >= kv->cap[id])
      return fail(SPEC_ERR_CAPACITY, "seq_lens[%d] = %d outside capacity %d", b, seq_lens[b], kv->cap[id]);
    si[b] = SampleInfo{kv->base[id], kv->cap[id], seq_lens[b], 0, SPEC_MAX_TREE, 0, 0};
  }
  hipStream_t s = (hipStream_t)stream;
  void* ctl = (char*)kv->pool + kv->ctl_off;
  if (int rc = kv->ring.upload(si.data(), batch * sizeof(SampleInfo), ctl, s)) return rc;
  const spec_model_config& c = kv->cfg;
  HIP_TRY(timed(SPEC_K_COMMIT, s, [&] {
            return launch_compact((const SampleInfo*)ctl, batch, kv->pool, c.n_layers,
                                  c.n_kv_heads, c.head_dim, accepted_len, accepted_nodes,
                                  new_seq_lens, s);
          }),
          "compact");
  return SPEC_OK;
}

SPEC_API int spec_kv_reorder(spec_kv* kv, int32_t groups, int32_t width, const int32_t* sample_ids,
                             const int32_t* begin, const int32_t* end, const int32_t* parents, void* stream) {
  return guarded([&]() -> int {
    if (!kv) return fail(SPEC_ERR_INVALID, "null argument");
    if (int rc = check_reorder(kv->n, groups, width, sample_ids, begin, end, parents)) return rc;
    ReorderBeams beams;
    const int total = groups * width;
    const bool small = groups <= kInlineGroups && total <= kInlineBeams;
    // [groups], [groups * width]: at most 24 bytes per sample, which the control area has
    std::vector<char> blob(small ? 0 : groups * sizeof(ReorderGroup) + total * sizeof(ReorderBeam));
    ReorderGroup* group = small ? beams.groups_here : (ReorderGroup*)blob.data();
    ReorderBeam* beam = small ? beams.beams_here : (ReorderBeam*)(group + groups);
    int most = 0;
    for (int g = 0; g < groups; ++g) {
      most = std::max(most, end[g] - begin[g]);
      group[g] = ReorderGroup{begin[g], end[g], 0, 0};
      for (int j = 0; j < width; ++j) {
        const int id = sample_ids[g * width + j];
        if (end[g] > kv->cap[id])
          return fail(SPEC_ERR_CAPACITY, "group %d: positions up to %d exceed sample %d's capacity %d", g, end[g], id,
                      kv->cap[id]);
        if (kv->base[id] / 128 > 0xffffffffll) return fail(SPEC_ERR_UNSUPPORTED, "a pool of more than 1 TB");
        beam[g * width + j] = ReorderBeam{(uint32_t)(kv->base[id] / 128), kv->cap[id]};
      }
    }
    if (int rc = refuse_capture(stream)) return rc;
    if (most == 0 || width == 1) return SPEC_OK;
    hipStream_t s = (hipStream_t)stream;
    char* ctl = (char*)kv->pool + kv->ctl_off;
    beams.groups = small ? nullptr : (const ReorderGroup*)ctl;
    beams.beams = small ? nullptr : (const ReorderBeam*)(ctl + groups * sizeof(ReorderGroup));
    if (!small)
      if (int rc = kv->ring.upload(blob.data(), blob.size(), ctl, s)) return rc;
    const spec_model_config& c = kv->cfg;
    HIP_TRY(timed(SPEC_K_REORDER, s, [&] {
              return launch_reorder(beams, groups, width, most, kv->pool, c.n_layers, c.n_kv_heads,
                                    c.head_dim, parents, s);
            }),
            "reorder");
    return SPEC_OK;
  });
}

namespace {

// Validate a transfer request and build its per-sample descriptors.
int transfer_plan(const spec_kv* kv, int32_t n, const int32_t* sample_ids, const int32_t* tok_begin,
                  const int32_t* tok_end, std::vector<MigrateInfo>* info, int64_t* wg_per_slab,
                  int64_t* tok_total) {
  if (!kv || !sample_ids || !tok_begin || !tok_end) return fail(SPEC_ERR_INVALID, "null argument");
  if (n < 1 || n > kv->n) return fail(SPEC_ERR_INVALID, "n %d out of range", n);
  if (int rc = check_samples(kv, n, sample_ids)) return rc;
  const spec_model_config& c = kv->cfg;
  info->resize(n);
  int64_t wg = 0, tok = 0;
  for (int j = 0; j < n; ++j) {
    const int id = sample_ids[j];
    if (tok_begin[j] < 0 || tok_end[j] < tok_begin[j] || tok_end[j] > kv->cap[id])
      return fail(SPEC_ERR_CAPACITY, "token range [%d, %d) of sample %d outside capacity %d",
                  tok_begin[j], tok_end[j], id, kv->cap[id]);
    const int count = tok_end[j] - tok_begin[j];
    const int64_t chunks = kv_transfer_chunks(count, c.head_dim);
    (*info)[j] = MigrateInfo{kv->base[id], kv->cap[id], tok_begin[j], count, (int32_t)tok,
                             (int32_t)wg, (int32_t)chunks};
    wg += chunks * c.n_kv_heads;
    tok += count;
    if (wg > 0x7fffffff || tok > 0x7fffffff) return fail(SPEC_ERR_INVALID, "transfer too large");
  }
  *wg_per_slab = wg;
  *tok_total = tok;
  return SPEC_OK;
}

int transfer(bool to_buffer, spec_kv* kv, int32_t n, const int32_t* sample_ids,
             const int32_t* tok_begin, const int32_t* tok_end, void* buf, size_t buf_bytes,
             void* stream) {
  g_err.clear();
  std::vector<MigrateInfo> info;
  int64_t wg = 0, tok = 0;
  if (int rc = transfer_plan(kv, n, sample_ids, tok_begin, tok_end, &info, &wg, &tok)) return rc;
  if (!buf) return fail(SPEC_ERR_INVALID, "null buffer");
  if ((uintptr_t)buf % 16) return fail(SPEC_ERR_INVALID, "buffer not 16-byte aligned");
  const spec_model_config& c = kv->cfg;
  const size_t need = (size_t)tok * c.n_layers * 2 * c.n_kv_heads * c.head_dim * 2;
  if (buf_bytes < need)
    return fail(SPEC_ERR_CAPACITY, "transfer buffer holds %zu bytes, needs %zu", buf_bytes, need);
  if (wg == 0) return SPEC_OK;
  hipStream_t s = (hipStream_t)stream;
  void* ctl = (char*)kv->pool + kv->ctl_off;
  if (int rc = kv->ring.upload(info.data(), n * sizeof(MigrateInfo), ctl, s)) return rc;
  HIP_TRY(timed(SPEC_K_TRANSFER, s, [&] {
            return launch_kv_transfer(to_buffer, (const MigrateInfo*)ctl, n, wg, (int)tok, kv->pool,
                                      (bf16*)buf, c.n_layers, c.n_kv_heads, c.head_dim, s);
          }),
          to_buffer ? "kv pack" : "kv unpack");
  return SPEC_OK;
}

}  // namespace

SPEC_API size_t spec_kv_transfer_bytes(const spec_kv* kv, int32_t n, const int32_t* tok_begin,
                                       const int32_t* tok_end) {
  if (!kv || !tok_begin || !tok_end || n < 1) return 0;
  size_t tok = 0;
  for (int j = 0; j < n; ++j) {
    if (tok_end[j] < tok_begin[j] || tok_begin[j] < 0) return 0;
    tok += (size_t)(tok_end[j] - tok_begin[j]);
  }
  const spec_model_config& c = kv->cfg;
  return tok * c.n_layers * 2 * c.n_kv_heads * c.head_dim * 2;
}

SPEC_API int spec_kv_pack(spec_kv* kv, int32_t n, const int32_t* sample_ids,
                          const int32_t* tok_begin, const int32_t* tok_end, void* buf,
                          size_t buf_bytes, void* stream) {
  return transfer(true, kv, n, sample_ids, tok_begin, tok_end, buf, buf_bytes, stream);
}

SPEC_API int spec_kv_unpack(spec_kv* kv, int32_t n, const int32_t* sample_ids,
                            const int32_t* tok_begin, const int32_t* tok_end, const void* buf,
                            size_t buf_bytes, void* stream) {
  return transfer(false, kv, n, sample_ids, tok_begin, tok_end, const_cast<void*>(buf), buf_bytes,
                  stream);
}

SPEC_API int spec_profile_begin(int32_t kernel_class, int32_t max_launches) {
  if (kernel_class < 0 || kernel_class >= SPEC_K_COUNT || max_launches < 1)
    return fail(SPEC_ERR_INVALID, "bad profile request");
  for (auto e : g_prof.ev) (void)hipEventDestroy(e);
  g_prof.ev.assign(2 * (size_t)max_launches, nullptr);
  for (auto& e : g_prof.ev) HIP_TRY(hipEventCreate(&e), "profile event");
  g_prof.kind = kernel_class;
  g_prof.max = max_launches;
  g_prof.count = 0;
  g_prof.on = true;
  return SPEC_OK;
}

SPEC_API int spec_profile_end(float* total_ms, int32_t* launches) {
  if (!total_ms || !launches) return fail(SPEC_ERR_INVALID, "null argument");
  g_prof.on = false;
  float tot = 0.f;
  for (int i = 0; i < g_prof.count; ++i) {
    HIP_TRY(hipEventSynchronize(g_prof.ev[2 * i + 1]), "profile sync");
    float ms = 0.f;
    HIP_TRY(hipEventElapsedTime(&ms, g_prof.ev[2 * i], g_prof.ev[2 * i + 1]), "profile elapsed");
    tot += ms;
  }
  *total_ms = tot;
  *launches = g_prof.count;
  for (auto e : g_prof.ev) (void)hipEventDestroy(e);
  g_prof.ev.clear();
  g_prof.count = 0;
  return SPEC_OK;
}

SPEC_API int spec_gemm_plan(const spec_model_config* cfg, int32_t kernel_class, int32_t n_tokens,
                            int32_t* tile_rows, int32_t* tile_cols, int32_t* splits) {
  g_err.clear();
  if (!cfg || !tile_rows || !tile_cols || !splits) return fail(SPEC_ERR_INVALID, "null argument");
  std::string why;
  if (!config_ok(cfg, &why)) return fail(SPEC_ERR_UNSUPPORTED, "%s", why.c_str());
  if (kernel_class != SPEC_K_GEMM_QKV && kernel_class != SPEC_K_GEMM_O && kernel_class != SPEC_K_GEMM_GATE_UP &&
      kernel_class != SPEC_K_GEMM_DOWN && kernel_class != SPEC_K_LM_HEAD)
    return fail(SPEC_ERR_INVALID, "kernel class %d is not a product", kernel_class);
  if (n_tokens < 1) return fail(SPEC_ERR_INVALID, "n_tokens must be >= 1");
  const GemmPlan p = product_plan(cfg, kernel_class, n_tokens);
  *splits = p.splits;
  switch (p.shape) {
    case GEMM_FEW_ROWS: *tile_rows = 0, *tile_cols = 16; break;
    case GEMM_64x64: *tile_rows = 64, *tile_cols = 64; break;
    case GEMM_64x128: *tile_rows = 64, *tile_cols = 128; break;
    case GEMM_128x128: *tile_rows = 128, *tile_cols = 128; break;
    case GEMM_256x128: *tile_rows = 256, *tile_cols = 128; break;
    case GEMM_256x256: *tile_rows = 256, *tile_cols = 256; break;
  }
  return SPEC_OK;
}
