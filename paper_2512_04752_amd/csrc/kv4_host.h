// Host side of the 4-bit paged KV cache that the verify step shares.
#pragma once

#include <exception>
#include <new>
#include <vector>

#include "host.h"
#include "kv4.h"

// Library-owned part of a 4-bit KV pool: every sample's pages, how many samples
// use each page, and a staging ring for uploads (a verify step makes two and its
// commit one: two steps of them stay in flight).
struct spec_kv4 {
  spec_model_config cfg;
  int32_t n = 0;
  std::vector<std::vector<int32_t>> pages;
  std::vector<int32_t> uses;
  char* pool = nullptr;
  size_t ctl_off = 0;            // byte offset of the control area (commit descriptors)
  spec::StagingRing<6> ring;
};

// A planned step: what its launches take, pointing into the caller's workspace.
struct spec_kv4_step {
  spec_kv4* kv = nullptr;
  int n_rows = 0;
  spec::Kv4RowArgs rows;
  spec::Kv4AttnArgs attn;
};

namespace spec {

// Run the body of an entry point; no exception leaves it.
template <class F>
int guarded(F&& body) {
  clear_error();
  try {
    return body();
  } catch (const std::bad_alloc&) {
    return fail(SPEC_ERR_CAPACITY, "out of host memory");
  } catch (const std::exception& e) {
    return fail(SPEC_ERR_INVALID, "%s", e.what());
  }
}

// Uploads go through staging memory that the next calls reuse, so a captured one
// would replay another call's descriptors.
int refuse_capture(void* stream);

// The checks of a step's rows; parents NULL: runs.
int kv4_check_rows(const spec_kv4* kv, int32_t batch, const int32_t* sample_ids, const int32_t* offsets,
                   const int32_t* parents, const int32_t* seq_lens);
size_t kv4_step_bytes(const spec_model_config* cfg, int64_t batch, int64_t rows, int64_t pages);
// Pages that the step's keys lie in.
int64_t kv4_step_pages(const spec_kv4* kv, int32_t batch, const int32_t* offsets, const int32_t* seq_lens);
// Plan checked rows in `workspace` (kv4_step_bytes) and enqueue the upload and the
// trees' metadata.
int kv4_plan_step(spec_kv4* kv, int32_t batch, const int32_t* sample_ids, const int32_t* offsets,
                  const int32_t* parents, const int32_t* seq_lens, void* workspace, hipStream_t s,
                  const spec_debug& dbg, spec_kv4_step* st);
int kv4_append(const spec_kv4_step* st, int layer, const bf16* k, int64_t k_stride, const bf16* v, int64_t v_stride,
               int rotate, hipStream_t s);
// Rotated K/V laid out [K, V][kv head][row][head_dim] per sample, samples in order.
int kv4_append_blocks(const spec_kv4_step* st, int layer, const bf16* kv, hipStream_t s);
int kv4_attend(const spec_kv4_step* st, int layer, const bf16* q, int64_t q_stride, bf16* out, hipStream_t s);

}  // namespace spec
