// What the entry points check of their arguments, and how they end.
#pragma once
#include "tslt.h"

#include <algorithm>

#include "error.h"
#include "rows.h"

namespace {

using tslt::fail;

inline int elem_bytes(tslt_dtype dt) { return dt == TSLT_F32 ? 4 : 2; }
inline bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// Rows of new tokens: 16 bytes at a time are read of each.
inline int check_rows(const char* who, const char* what, const tslt_rows* r, tslt_dtype dt) {
  if (!r || !r->data) return fail(TSLT_ERR_INVALID_ARG, "%s: null %s", who, what);
  const int64_t unit = 16 / elem_bytes(dt);
  if (!aligned(r->data, 16) || r->seq_stride % unit || r->token_stride % unit || r->head_stride % unit)
    return fail(TSLT_ERR_INVALID_ARG, "%s: rows of %s must begin at multiples of 16 bytes", who, what);
  return TSLT_OK;
}
// Rows of `width` elements that are written to lie apart: from the nearest of their dimensions to the farthest, each steps over all that those inside it span.
inline int check_distinct(const char* who, const char* what, const tslt_rows* r, int64_t B, int64_t n, int64_t heads, int64_t width) {
  typedef __int128 Wide;
  struct Dim { Wide stride; int64_t size; } d[3] = {{r->seq_stride, B}, {r->token_stride, n}, {r->head_stride, heads}};
  for (Dim& x : d) x.stride = x.size < 2 ? 0 : x.stride < 0 ? -x.stride : x.stride;
  std::sort(d, d + 3, [](const Dim& x, const Dim& y) { return x.stride < y.stride; });
  Wide span = width;
  for (const Dim& x : d) {
    if (x.size < 2) continue;
    if (x.stride < span) return fail(TSLT_ERR_INVALID_ARG, "%s: rows of %s must not lie on each other", who, what);
    span += x.stride * (x.size - 1);
  }
  return TSLT_OK;
}
inline bool valid_dtype(tslt_dtype dt) { return dt == TSLT_F32 || dt == TSLT_BF16 || dt == TSLT_F16; }
inline tslt::RowsView view(const tslt_rows* r) {
  return r ? tslt::RowsView{r->data, r->seq_stride, r->token_stride, r->head_stride} : tslt::RowsView{nullptr, 0, 0, 0};
}
// A launch has fewer than 2^32 threads (`threads` a workgroup; the calls that leave it out are bounded by their own checks or by HIP).
inline bool grid_fits(const char* who, int64_t blocks, int& code, int64_t threads = 1) {
  code = blocks > (threads == 1 ? 0x7FFFFFFF : 0xFFFFFFFF / threads) ? fail(TSLT_ERR_UNSUPPORTED, "%s: too many workgroups for one launch", who) : 0;
  return code == 0;
}
inline int launched(const char* who) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? TSLT_OK : tslt::hip_fail(e, who);
}

}  // namespace
