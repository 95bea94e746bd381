// Host side of the products with 4-bit weights: checks, plans and launches.
#include <algorithm>
#include <exception>
#include <new>

#include "host.h"
#include "w4.h"

using namespace spec;

namespace {

constexpr int kMaxDim = 1 << 24, kMaxN = 1 << 20;
constexpr int64_t kMaxStride = 1 << 28, kMaxOut = 1ll << 34;     // values

bool dims_ok(int32_t rows, int32_t cols) {
  return rows >= 1 && cols >= 1 && cols % 32 == 0 && rows <= kMaxDim && cols <= kMaxDim;
}

int check_dims(int32_t rows, int32_t cols) {
  if (rows < 1 || cols < 1) return fail(SPEC_ERR_INVALID, "a matrix of %d rows and %d columns", rows, cols);
  if (!dims_ok(rows, cols))
    return fail(SPEC_ERR_UNSUPPORTED, "%d x %d: columns must be a multiple of 32, both at most %d", rows, cols, kMaxDim);
  return SPEC_OK;
}

int check_data(const void* data) {
  if (!data) return fail(SPEC_ERR_INVALID, "null argument");
  if ((uintptr_t)data % kAlign) return fail(SPEC_ERR_INVALID, "matrix data not 256-byte aligned");
  return SPEC_OK;
}

// bf16 rows of `width` values `stride` apart, accessed 16 bytes at a time.
int check_rows(const char* what, const void* p, int64_t stride, int64_t width) {
  if (!p) return fail(SPEC_ERR_INVALID, "null argument");
  if ((uintptr_t)p % 16) return fail(SPEC_ERR_INVALID, "%s not 16-byte aligned", what);
  if (stride < width || stride % 8)
    return fail(SPEC_ERR_INVALID, "%s: row stride %lld must be a multiple of 8 and at least %lld", what,
                (long long)stride, (long long)width);
  return SPEC_OK;
}

int product(const spec_w4* m, const spec_w4* up, const void* x, int64_t x_stride, int32_t n, void* out,
            int64_t out_stride, int32_t kind, void* workspace, size_t ws_bytes, void* stream) {
  if (!m || !x || !out) return fail(SPEC_ERR_INVALID, "null argument");
  if (int rc = check_dims(m->rows, m->cols)) return rc;
  if (int rc = check_data(m->data)) return rc;
  if (up) {
    if (int rc = check_data(up->data)) return rc;
    if (up->rows != m->rows || up->cols != m->cols)
      return fail(SPEC_ERR_INVALID, "gate is %d x %d, up %d x %d", m->rows, m->cols, up->rows, up->cols);
  }
  if (kind != SPEC_W4_BF16 && kind != SPEC_W4_F32 && kind != SPEC_W4_ADD)
    return fail(SPEC_ERR_INVALID, "output kind %d", kind);
  if (n < 0) return fail(SPEC_ERR_INVALID, "n = %d", n);
  if (n > kMaxN) return fail(SPEC_ERR_UNSUPPORTED, "%d rows, at most %d in one call", n, kMaxN);
  if (int rc = check_rows("x", x, x_stride, m->cols)) return rc;
  if (x_stride > kMaxStride)
    return fail(SPEC_ERR_UNSUPPORTED, "x: row stride %lld, at most %lld", (long long)x_stride, (long long)kMaxStride);
  if ((int64_t)n * m->rows > kMaxOut)
    return fail(SPEC_ERR_UNSUPPORTED, "%d x %d outputs, at most %lld in one call", n, m->rows, (long long)kMaxOut);
  if (out_stride < m->rows) return fail(SPEC_ERR_INVALID, "out: row stride %lld below %d", (long long)out_stride, m->rows);
  if ((uintptr_t)out % (kind == SPEC_W4_BF16 ? 2 : 4)) return fail(SPEC_ERR_INVALID, "out not aligned to its type");
  const size_t need = w4_partial_bytes(m->rows, m->cols, n, up != nullptr);
  if (need) {
    if (!workspace || ws_bytes < need)
      return fail(SPEC_ERR_WORKSPACE, "workspace %zu bytes, needs %zu", workspace ? ws_bytes : 0, need);
    if ((uintptr_t)workspace % kAlign) return fail(SPEC_ERR_INVALID, "workspace not 256-byte aligned");
  }
  W4Args a{};
  a.plan = plan_w4(m->rows, m->cols, n, up != nullptr);
  a.w0 = (const char*)m->data;
  a.w1 = up ? (const char*)up->data : nullptr;
  a.rows = m->rows;
  a.cols = m->cols;
  a.x = (const bf16*)x;
  a.x_stride = x_stride;
  a.n = n;
  a.out = out;
  a.out_stride = out_stride;
  a.kind = kind;
  a.partial = (float*)workspace;
  hipStream_t s = (hipStream_t)stream;
  HIP_TRY(timed(SPEC_K_W4, s, [&] { return launch_w4(a, s); }), "w4 product");
  return SPEC_OK;
}

}  // namespace

SPEC_API size_t spec_w4_bytes(int32_t rows, int32_t cols) {
  if (!dims_ok(rows, cols)) return 0;
  return (size_t)((rows + kW4Rows - 1) / kW4Rows) * w4_tile_bytes(w4_col_tiles(cols));
}

SPEC_API int spec_w4_pack(const void* w, int64_t stride, int32_t rows, int32_t cols, void* data, size_t bytes,
                          void* stream) {
  clear_error();
  if (int rc = check_dims(rows, cols)) return rc;
  if (int rc = check_rows("w", w, stride, cols)) return rc;
  if (int rc = check_data(data)) return rc;
  const size_t need = spec_w4_bytes(rows, cols);
  if (bytes < need) return fail(SPEC_ERR_CAPACITY, "matrix data holds %zu bytes, needs %zu", bytes, need);
  HIP_TRY(launch_w4_pack((const bf16*)w, stride, rows, cols, (char*)data, (hipStream_t)stream), "w4 pack");
  return SPEC_OK;
}

SPEC_API int spec_w4_unpack(const spec_w4* m, void* w, int64_t stride, void* stream) {
  clear_error();
  if (!m) return fail(SPEC_ERR_INVALID, "null argument");
  if (int rc = check_dims(m->rows, m->cols)) return rc;
  if (int rc = check_data(m->data)) return rc;
  if (int rc = check_rows("w", w, stride, m->cols)) return rc;
  HIP_TRY(launch_w4_unpack((const char*)m->data, m->rows, m->cols, (bf16*)w, stride, (hipStream_t)stream), "w4 unpack");
  return SPEC_OK;
}

SPEC_API size_t spec_w4_workspace_bytes(int32_t rows, int32_t cols, int32_t max_n) {
  if (!dims_ok(rows, cols) || max_n < 1) return 0;
  size_t most = 0;
  for (int n = 1; n <= std::min<int>(max_n, kMostSplitRows); ++n)
    for (const bool pair : {false, true}) most = std::max(most, w4_partial_bytes(rows, cols, n, pair));
  return align_up(most);
}

SPEC_API size_t spec_w4_product_bytes(int32_t rows, int32_t cols, int32_t n, int32_t pair) {
  if (!dims_ok(rows, cols) || n < 1 || n > kMaxN || (pair != 0 && pair != 1)) return 0;
  return align_up(w4_partial_bytes(rows, cols, n, pair == 1));
}

SPEC_API int spec_w4_linear(const spec_w4* m, const void* x, int64_t x_stride, int32_t n, void* out,
                            int64_t out_stride, int32_t kind, void* workspace, size_t ws_bytes, void* stream) {
  clear_error();
  return product(m, nullptr, x, x_stride, n, out, out_stride, kind, workspace, ws_bytes, stream);
}

SPEC_API int spec_w4_gate_up(const spec_w4* gate, const spec_w4* up, const void* x, int64_t x_stride, int32_t n,
                             void* out, int64_t out_stride, void* workspace, size_t ws_bytes, void* stream) {
  clear_error();
  if (!up) return fail(SPEC_ERR_INVALID, "null argument");
  return product(gate, up, x, x_stride, n, out, out_stride, SPEC_W4_BF16, workspace, ws_bytes, stream);
}
