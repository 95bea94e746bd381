// Host side of the choice of beams: checks, workspace and launch.
#include "beam.h"
#include "host.h"

using namespace spec;

namespace {

constexpr int64_t kMaxRows = 1 << 22;

// Shapes of a call into `a`; SPEC_OK or an error.
int shapes(int32_t groups, int32_t width, int32_t vocab, int32_t k, BeamArgs* a) {
  if (groups < 1 || vocab < 1) return fail(SPEC_ERR_INVALID, "%d groups, a vocabulary of %d", groups, vocab);
  if (width < 1 || width > kMaxBeams) return fail(SPEC_ERR_INVALID, "width %d outside 1 .. %d", width, kMaxBeams);
  if (k < 1 || k > kMaxBeams) return fail(SPEC_ERR_INVALID, "k %d outside 1 .. %d", k, kMaxBeams);
  if ((int64_t)groups * width > kMaxRows)
    return fail(SPEC_ERR_UNSUPPORTED, "%lld beams in one call, at most %lld", (long long)groups * width,
                (long long)kMaxRows);
  if (vocab > 1 << 30) return fail(SPEC_ERR_UNSUPPORTED, "a vocabulary of %d", vocab);
  a->groups = groups;
  a->width = width;
  a->vocab = vocab;
  a->k = k;
  return SPEC_OK;
}

}  // namespace

SPEC_API size_t spec_beam_workspace_bytes(int32_t groups, int32_t width, int32_t vocab, int32_t k) {
  size_t most = 0;
  for (const int is_bf16 : {0, 1}) {
    BeamArgs a{};
    if (shapes(groups, width, vocab, k, &a)) return 0;
    a.is_bf16 = is_bf16;
    plan_beam(&a);
    most = std::max(most, beam_scratch(&a, nullptr));
  }
  return most;
}

SPEC_API int spec_beam_select(const void* logits, int64_t row_stride, int32_t is_bf16, int32_t groups, int32_t width,
                              int32_t vocab, const float* scores, const int32_t* last_tokens, int32_t eos_token,
                              int32_t k, int32_t* parents, int32_t* tokens, float* new_scores, void* workspace,
                              size_t ws_bytes, void* stream) {
  clear_error();
  if (!logits || !scores || !parents || !tokens || !new_scores || !workspace)
    return fail(SPEC_ERR_INVALID, "null argument");
  BeamArgs a{};
  if (int rc = shapes(groups, width, vocab, k, &a)) return rc;
  if (is_bf16 != 0 && is_bf16 != 1) return fail(SPEC_ERR_INVALID, "bf16 must be 0 or 1");
  if ((uintptr_t)logits % (is_bf16 ? 2 : 4)) return fail(SPEC_ERR_INVALID, "logits not aligned to their type");
  if (row_stride < vocab) return fail(SPEC_ERR_INVALID, "row stride %lld below %d", (long long)row_stride, vocab);
  if (eos_token < -1 || eos_token >= vocab) return fail(SPEC_ERR_INVALID, "eos_token %d out of range", eos_token);
  if (eos_token >= 0 && !last_tokens) return fail(SPEC_ERR_INVALID, "an eos_token needs last_tokens");
  for (const void* p : {(const void*)scores, (const void*)last_tokens, (const void*)parents, (const void*)tokens,
                        (const void*)new_scores})
    if ((uintptr_t)p % 4) return fail(SPEC_ERR_INVALID, "an array is not 4-byte aligned");
  if ((uintptr_t)workspace % kAlign) return fail(SPEC_ERR_INVALID, "workspace not 256-byte aligned");
  a.logits = logits;
  a.row_stride = row_stride;
  a.is_bf16 = is_bf16;
  a.scores = scores;
  a.last = last_tokens;
  a.eos = eos_token;
  a.parents = parents;
  a.tokens = tokens;
  a.new_scores = new_scores;
  plan_beam(&a);
  const size_t need = beam_scratch(&a, (char*)workspace);
  if (ws_bytes < need) return fail(SPEC_ERR_WORKSPACE, "workspace %zu bytes, needs %zu", ws_bytes, need);
  hipStream_t s = (hipStream_t)stream;
  HIP_TRY(timed(SPEC_K_BEAM, s, [&] { return launch_beam(a, s); }), "beam choice");
  return SPEC_OK;
}
