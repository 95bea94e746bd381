// The cache rows that follow the beams: descriptors and launcher prototypes.
#pragma once

#include "common.h"

namespace spec {

constexpr int kMaxReorder = SPEC_MAX_BEAMS;      // beams of a group

// One beam over the bf16 pool.
struct ReorderBeam {
  uint32_t block;       // the sample's block, in units of 256 bytes
  int32_t cap;          // positions per (layer, K/V, kv head)
};

// One group.
struct ReorderGroup {
  int32_t begin, end;
  int32_t pages;        // 4-bit pool: that the range touches, of every beam
  int32_t table;        // its first entry in the table: [width][pages] page ids
};
static_assert(sizeof(ReorderGroup) == 16, "ReorderGroup layout");

// Descriptors of a small call go along as kernel arguments (an upload takes the host 5 us, and
// the stream as long); of a larger one they lie in device memory.
constexpr int kInlineBeams = 288, kInlineGroups = 64, kInlinePages = 1216;
struct ReorderBeams {
  const ReorderGroup* groups;            // NULL: here
  const ReorderBeam* beams;
  ReorderGroup groups_here[kInlineGroups];
  ReorderBeam beams_here[kInlineBeams];
};
struct ReorderPages {
  const ReorderGroup* groups;            // NULL: here
  const int32_t* table;
  ReorderGroup groups_here[kInlineGroups];
  uint16_t table_here[kInlinePages];
};
static_assert(sizeof(ReorderBeams) < 3500 && sizeof(ReorderPages) < 3500, "kernel arguments");

// most: tokens of the longest range, or pages.
hipError_t launch_reorder(const ReorderBeams& beams, int groups, int width, int most, bf16* pool, int n_layers,
                          int n_kv_heads, int head_dim, const int32_t* parents, hipStream_t s);
hipError_t launch_kv4_reorder(const ReorderPages& info, int groups, int width, int most, char* pool,
                              int64_t page_bytes, int head_dim, const int32_t* parents, hipStream_t s);

}  // namespace spec
