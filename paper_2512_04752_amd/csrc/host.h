// What the host sides of the C ABI share: error reporting, checks of shapes and
// sample ids, the pinned staging of per-call uploads and the kernel timing hooks.
#pragma once

#include <string.h>

#include <algorithm>
#include <string>
#include <vector>

#include "common.h"
#include "specverify.h"

#define SPEC_API extern "C" __attribute__((visibility("default")))

#define HIP_TRY(expr, what)               \
  do {                                    \
    hipError_t e_ = (expr);               \
    if (e_ != hipSuccess) return ::spec::hip_fail(e_, what); \
  } while (0)

namespace spec {

constexpr size_t kAlign = 256;
inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

// Record a message as the calling thread's spec_last_error() and return `code`.
int fail(int code, const char* fmt, ...);
int hip_fail(hipError_t e, const char* what);
void clear_error();

// Whether the library supports the shape; *why says what it does not.
bool config_ok(const spec_model_config* c, std::string* why);
bool same_config(const spec_model_config* a, const spec_model_config* b);
// Sample ids of a call: distinct and in [0, n).
int check_sample_ids(int n, int32_t batch, const int32_t* ids);

// Order attention items longest-first per XCD.  A kernel hands XCD x the items
// [x*per, (x+1)*per) in order.  Deal the groups of items that share a key range
// (adjacent, so they meet in one XCD's L2), longest first, to the XCD with the
// least work so far; pad every XCD's list to `per` with empty items (sample -1).
void deal_items(std::vector<AttnItem>& list);

// Process-wide kernel timing state (measurement only).
struct Profiler {
  bool on = false;
  int kind = -1, max = 0, count = 0;
  std::vector<hipEvent_t> ev;
};
extern Profiler g_prof;

template <class F>
hipError_t timed(int kind, hipStream_t s, F&& fn) {
  const bool rec = g_prof.on && g_prof.kind == kind && g_prof.count < g_prof.max;
  if (rec) {
    const hipError_t e = hipEventRecord(g_prof.ev[2 * g_prof.count], s);
    if (e != hipSuccess) return e;
  }
  const hipError_t e = fn();
  if (rec) {
    const hipError_t e2 = hipEventRecord(g_prof.ev[2 * g_prof.count + 1], s);
    ++g_prof.count;
    if (e2 != hipSuccess) return e2;
  }
  return e;
}

// A ring of N pinned buffers for per-call host->device uploads: the host waits
// only when it comes back to a buffer whose copy has not run yet.
template <int N>
struct StagingRing {
  struct Slot {
    void* host = nullptr;
    size_t size = 0;
    hipEvent_t ev = nullptr;
    bool pending = false;
  } slots[N];
  int next = 0;

  // Copy `bytes` of `src` to device `dst` through the next buffer.
  int upload(const void* src, size_t bytes, void* dst, hipStream_t s) {
    Slot& sl = slots[next];
    next = (next + 1) % N;
    if (sl.pending) {
      HIP_TRY(hipEventSynchronize(sl.ev), "staging wait");
      sl.pending = false;
    }
    if (sl.ev == nullptr) HIP_TRY(hipEventCreateWithFlags(&sl.ev, hipEventDisableTiming), "event");
    if (sl.size < bytes) {
      if (sl.host) HIP_TRY(hipHostFree(sl.host), "free staging");
      sl.host = nullptr;
      sl.size = 0;
      const size_t want = std::max(bytes, (size_t)1 << 20);
      HIP_TRY(hipHostMalloc(&sl.host, want, hipHostMallocDefault), "pinned staging");
      sl.size = want;
    }
    memcpy(sl.host, src, bytes);
    HIP_TRY(hipMemcpyAsync(dst, sl.host, bytes, hipMemcpyHostToDevice, s), "upload");
    HIP_TRY(hipEventRecord(sl.ev, s), "staging event");
    sl.pending = true;
    return SPEC_OK;
  }

  // Wait for the pending copies and free the buffers.
  int release() {
    int rc = SPEC_OK;
    for (auto& sl : slots) {
      if (sl.pending && hipEventSynchronize(sl.ev) != hipSuccess) rc = SPEC_ERR_HIP;
      if (sl.ev) (void)hipEventDestroy(sl.ev);
      if (sl.host) (void)hipHostFree(sl.host);
    }
    return rc;
  }
};

}  // namespace spec
