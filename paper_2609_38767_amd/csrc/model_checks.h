// Argument checks shared by the model-side entry points: sizes, rows, workspaces
// and what may not overlap.
#pragma once

#include <algorithm>
#include <initializer_list>

#include "api_common.h"
#include "dattri.h"

namespace dattri {

constexpr int64_t kMaxWidth = (int64_t)1 << 23;  // columns of a row (check_rows holds 256 rows below 4 GiB)

inline dattri_status elt_of(dattri_dtype dtype, int* elt) {
  if (dtype != DATTRI_F32 && dtype != DATTRI_BF16)
    return fail(DATTRI_E_DTYPE, "dtype %d is neither F32 nor BF16", (int)dtype);
  *elt = dtype == DATTRI_BF16 ? 2 : 4;
  return DATTRI_OK;
}

inline dattri_status check_width(const char* what, int64_t d) {
  if (d < 1) return fail(DATTRI_E_INVALID_ARG, "%s must be >= 1 (got %lld)", what, (long long)d);
  if (d > kMaxWidth) return fail(DATTRI_E_UNSUPPORTED, "%s=%lld exceeds 2^23", what, (long long)d);
  return DATTRI_OK;
}

inline dattri_status check_count(const char* what, int64_t n) {
  if (n < 0) return fail(DATTRI_E_INVALID_ARG, "%s must be >= 0 (got %lld)", what, (long long)n);
  if (n > INT32_MAX) return fail(DATTRI_E_UNSUPPORTED, "%s=%lld does not fit int32", what, (long long)n);
  return DATTRI_OK;
}

// A matrix argument of `rows` rows of `d` columns: its stride (0 = dense) and pointer.
inline dattri_status check_rows(const char* what, const void* p, int64_t* ld, int64_t rows, int64_t d, int elt, bool needed) {
  if (*ld < 0) return fail(DATTRI_E_INVALID_ARG, "row stride of %s must be >= 0", what);
  if (*ld == 0) *ld = d;
  if (*ld < d)
    return fail(DATTRI_E_INVALID_ARG, "row stride of %s (%lld) must be >= its width %lld", what, (long long)*ld,
                (long long)d);
  if (*ld >= kMaxBlockBytes || *ld * elt * 256 >= kMaxBlockBytes)
    return fail(DATTRI_E_UNSUPPORTED, "row stride of %s (%lld) too large (256 rows must stay below 4 GiB)", what,
                (long long)*ld);
  if (needed && rows > 0 && !p) return fail(DATTRI_E_INVALID_ARG, "%s is NULL", what);
  if ((uintptr_t)p % elt) return fail(DATTRI_E_INVALID_ARG, "%s is not aligned to its elements", what);
  return DATTRI_OK;
}

inline dattri_status check_workspace(const void* ws, size_t have, size_t need) {
  if (need == 0) return DATTRI_OK;
  if (!ws) return fail(DATTRI_E_WORKSPACE, "workspace is NULL (needs %zu bytes)", need);
  if ((uintptr_t)ws % kAlign) return fail(DATTRI_E_WORKSPACE, "workspace must be 256-byte aligned");
  if (have < need) return fail(DATTRI_E_WORKSPACE, "workspace has %zu bytes, needs %zu", have, need);
  return DATTRI_OK;
}

inline dattri_status check_act(dattri_act act) {
  if ((int)act < DATTRI_ACT_NONE || (int)act > DATTRI_ACT_SILU)
    return fail(DATTRI_E_INVALID_ARG, "unknown activation %d", (int)act);
  return DATTRI_OK;
}

// Both operands of a product readable in 16-byte pieces as far as pointers and
// strides go (the widths are known to the layout).
inline bool on_16(const void* a, int64_t lda, const void* b, int64_t ldb, int elt) {
  return (uintptr_t)a % 16 == 0 && (uintptr_t)b % 16 == 0 && (lda * elt) % 16 == 0 && (ldb * elt) % 16 == 0;
}

// The memory of an argument: `rows` pieces of `width` bytes, `stride` apart.
struct Span {
  const char* what;
  int64_t at, rows, width, stride;
  Span(const char* what_, const void* p, int64_t rows_, int64_t d, int64_t ld, int elt)
      : what(what_), at((int64_t)p), rows(p ? rows_ : 0), width(d * elt), stride(ld * elt) {}
  Span(const char* what_, const void* p, int64_t bytes) : Span(what_, p, bytes > 0, bytes, bytes, 1) {}
  int64_t end() const { return at + (rows - 1) * stride + width; }
  bool same(const Span& o) const { return at == o.at && width == o.width && (rows == 1 || stride == o.stride); }
};

// Whether two arguments share a byte.  Rows of one may lie between the other's
// (column ranges of one matrix), so where the ranges meet the rows decide.
inline bool overlap(const Span& a, const Span& b) {
  if (a.rows == 0 || b.rows == 0 || a.at >= b.end() || b.at >= a.end()) return false;
  if (a.rows == 1 && b.rows == 1) return true;
  if (a.rows > 1 && b.rows > 1 && a.stride == b.stride) {
    // b's row j starts `off` behind a's row j + k
    const int64_t by = b.at - a.at, k = by >= 0 ? by / a.stride : -((a.stride - 1 - by) / a.stride), off = by - k * a.stride;
    auto meet = [&](int64_t shift) { return std::max<int64_t>(0, shift) < std::min(a.rows, b.rows + shift); };
    return (off < a.width && meet(k)) || (a.stride - off < b.width && meet(k + 1));
  }
  // every row of the one with fewer against the first row of the other that ends behind its start
  const Span &f = a.rows <= b.rows ? a : b, &m = a.rows <= b.rows ? b : a;
  const int64_t first = std::max<int64_t>(0, (m.at - f.at - f.width) / f.stride);
  for (int64_t i = first; i < f.rows; ++i) {
    const int64_t u = f.at + i * f.stride, past = u - m.at - m.width;  // m's rows that end at u or before
    if (u >= m.end()) break;
    const int64_t j = past < 0 ? 0 : past / m.stride + 1;
    if (j < m.rows && m.at + j * m.stride < u + f.width) return true;
  }
  return false;
}

// What a call writes may not lie in what it reads or in what else it writes;
// `in_place`, where given, may be `out` itself, element by element.
inline dattri_status check_apart(const Span& out, std::initializer_list<Span> others, const Span* in_place = nullptr,
                          const Span* in_place2 = nullptr) {
  for (const Span& o : others)
    if (overlap(out, o)) return fail(DATTRI_E_INVALID_ARG, "%s overlaps %s", out.what, o.what);
  for (const Span* o : {in_place, in_place2})
    if (o && !out.same(*o) && overlap(out, *o))
      return fail(DATTRI_E_INVALID_ARG, "%s overlaps %s without being it", out.what, o->what);
  return DATTRI_OK;
}

}  // namespace dattri

#define TRY(expr)                                   \
  do {                                              \
    const dattri_status st_ = (expr);               \
    if (st_ != DATTRI_OK) return st_;               \
  } while (0)
