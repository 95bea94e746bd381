// The 4-bit paged KV cache: layout, device descriptors and launcher prototypes.
#pragma once

#include "common.h"

namespace spec {

constexpr int kKv4Page = SPEC_KV4_PAGE;   // positions per page
static_assert(kKv4Page == 64, "two blocks of 32 keys, eight octets");

// One head of one layer in a page, see specverify.h: key codes, value codes, key
// scales, value scales.
constexpr __host__ __device__ int kv4_head_bytes(int hd) { return kKv4Page * (hd + hd / 32 + 2); }
constexpr __host__ __device__ int kv4_block_bytes(int hd) { return 16 * hd; }      // codes of 32 keys
constexpr __host__ __device__ int kv4_octet_bytes(int hd) { return 4 * hd; }       // value codes of 8 keys
constexpr __host__ __device__ int kv4_value_at(int hd) { return kKv4Page * hd / 2; }
constexpr __host__ __device__ int kv4_kscale_at(int hd) { return kKv4Page * hd; }
constexpr __host__ __device__ int kv4_vscale_at(int hd) { return kKv4Page * (hd + hd / 32); }

// Tables hold a page's place in units of 128 bytes, which every page and head is a
// multiple of (a shift instead of a 64-bit product where the attention looks it up).
constexpr int kKv4Unit = 128;
static_assert(kv4_head_bytes(64) % kKv4Unit == 0 && kv4_head_bytes(128) % kKv4Unit == 0, "page unit");
constexpr __host__ __device__ uint64_t kv4_page_offset(uint32_t page) { return (uint64_t)page * kKv4Unit; }

// Where a step's cache lies.  SampleInfo::kv_base is the sample's first entry in `table`.
struct Kv4View {
  char* pool;
  const uint32_t* table;         // each sample's pages in position order, kv4_page_offset()
  const SampleInfo* samples;
  int layer, n_kv_heads, head_dim;
};

// The rows of one sample that fall into one aligned group of eight positions
// [slot0, slot0 + 8): positions slot0 + lo .. slot0 + hi - 1.
struct Kv4Octet {
  uint32_t page;                 // of slot0, kv4_page_offset()
  int32_t slot0, lo, hi;
  int32_t row0;                  // row of slot0, which may lie before the sample's first
  int32_t tok0, ntok;            // the sample's rows
  int32_t pad;
};
static_assert(sizeof(Kv4Octet) == 32, "Kv4Octet layout");

struct Kv4RowArgs {
  Kv4View v;
  const Kv4Octet* octets;
  int n_octets;
  const TokInfo* toks;           // rows' positions (trees); NULL: a row's position is its slot
  const double* freq;            // [head_dim / 2] rotary frequencies
  bf16* k;                       // row r, head g at k + r * k_stride + g * head_dim
  bf16* val;
  int64_t k_stride, v_stride;
  int rotate;
  int blocks;                    // append: k holds [K, V][kv head][row][head_dim] per sample instead
};

// Quantise rows into the cache (k, val are read), or read them back (written).
hipError_t launch_kv4_append(const Kv4RowArgs& a, hipStream_t s);
hipError_t launch_kv4_read(const Kv4RowArgs& a, hipStream_t s);

// One attention work-group: four waves on up to 4 * wave_tiles tiles of 16 query rows
// of one (sample, kv head), from row row0 on, against keys [key0, key1).  It holds what
// the kernel needs of the sample, so that the first keys are two dependent loads away.
struct Kv4Item {
  int32_t kvh, row0, key0, key1, nsplit, part;
  int32_t waves;                 // waves that share wave_tiles row tiles: 4, 2 or 1; 0: no work
  int32_t seq_len, tok0, ntok;   // the sample's
  uint32_t pages;                // its first entry in the table
  int32_t pad[5];
};
static_assert(sizeof(Kv4Item) == 64, "Kv4Item layout");

// The key ranges of one row tile, to be merged.
struct Kv4Merge {
  int32_t kvh, row0, nsplit, part0;
  int32_t tok0, ntok;            // the sample's
  int32_t pad[2];
};
static_assert(sizeof(Kv4Merge) == 32, "Kv4Merge layout");

struct Kv4AttnArgs {
  Kv4View v;
  const bf16* q;                 // row r, query head i at q + r * q_stride + i * head_dim
  int64_t q_stride;
  const uint64_t* anc;           // [N][kAncWords] (trees); NULL: row i sees rows 0 .. i (runs)
  const Kv4Item* items;
  int n_items;
  int wave_tiles;                // row tiles of a wave: 1 or 2
  int once;                      // one row tile per sample and KV head: no key is read by two waves
  float* part_o;                 // [slots][16][head_dim], divided by its l
  float* part_ml;                // [slots][16][2]
  bf16* out;                     // [N][n_heads*head_dim]
  int n_heads;
  int group;                     // query heads per KV head
  uint32_t group_inv;            // ceil(2^32 / group): row / group = high word of row * group_inv
  const Kv4Merge* comb;
  int n_comb;
};
hipError_t launch_kv4_attention(const Kv4AttnArgs& a, hipStream_t s);

// One sample of a commit: the pages of positions from seq_len / 64 * 64 on.
struct Kv4CommitInfo {
  int32_t seq_len, cap;          // cap: positions the mapped pages hold
  int32_t pages[6];              // -1 past the mapped pages
};
static_assert(sizeof(Kv4CommitInfo) == 32, "Kv4CommitInfo layout");
hipError_t launch_kv4_compact(const Kv4CommitInfo* info, int batch, char* pool, int64_t page_bytes,
                              int n_layers, int n_kv_heads, int head_dim, const int32_t* accepted_len,
                              const int32_t* accepted_nodes, int32_t* new_seq_lens, hipStream_t s);

}  // namespace spec
