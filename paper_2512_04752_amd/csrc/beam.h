// The choice of beams: kernel arguments and launcher prototypes.
#pragma once

#include "common.h"

namespace spec {

constexpr int kMaxBeams = SPEC_MAX_BEAMS;
static_assert(kMaxBeams == kWave, "a list is one entry per lane");

struct BeamArgs {
  const void* logits;       // row r of the groups * width at r * row_stride
  int64_t row_stride;
  int is_bf16;
  int groups, width, vocab, k;
  const float* scores;      // [groups][width]
  const int32_t* last;      // [groups][width], read when eos >= 0
  int eos;
  int32_t* parents;         // [groups][k]
  int32_t* tokens;
  float* new_scores;
  // Every row is cut into `segs` segments, of `seg` 16-byte vectors, one per wave.
  int segs, seg;
  double* sums;             // [rows][segs] sum of exp(z - top), and
  float* tops;              // [rows][segs] the segment's largest logit (or what stands for it)
  float* cand_z;            // [rows][segs][k] the segment's best logits, best first
  int32_t* cand_y;          // their tokens; -1 past the last
};

// segs and seg of a call.
void plan_beam(BeamArgs* a);
size_t beam_scratch(BeamArgs* a, char* base);   // carve the workspace (a->segs set); bytes
hipError_t launch_beam(const BeamArgs& a, hipStream_t s);

}  // namespace spec
