// Argument checks shared by the files that implement include/pblock.h's operators
// around the block, made on the host before any HIP call.  (Internal to each file.)
#pragma once

#include "abi.h"

#include <math.h>

#include <cmath>

#include <algorithm>

#include "kernels.h"

using pb::align256;
using pb::fail;
using pb::finish_launches;

namespace {

[[maybe_unused]] constexpr long long kMaxInt = 2147483647LL;
// Workgroups of 256 threads in a launch of fewer than 2^32 threads.
[[maybe_unused]] constexpr long long kMaxBlocks = 1LL << 24;

[[maybe_unused]] bool known(pb_dtype dt) { return dt == PB_BF16 || dt == PB_F32; }
[[maybe_unused]] size_t size_of(pb_dtype dt) { return dt == PB_BF16 ? 2 : 4; }
[[maybe_unused]] pb::Dt dt_of(pb_dtype dt) { return dt == PB_BF16 ? pb::Dt::BF16 : pb::Dt::F32; }

[[maybe_unused]] pb_status check_ptr(const void* p, size_t align, const char* name) {
  if (!p) return fail(PB_ERR_INVALID_ARG, "%s is NULL", name);
  if ((uintptr_t)p % align)
    return fail(PB_ERR_INVALID_ARG, "%s is not %zu-byte aligned", name, align);
  return PB_OK;
}
[[maybe_unused]] pb_status check_opt(const void* p, size_t align, const char* name) {
  return p ? check_ptr(p, align, name) : PB_OK;
}
[[maybe_unused]] pb_status check_ws(const void* ws, size_t bytes, size_t need) {
  if (!need) return PB_OK;
  if (!ws || (uintptr_t)ws % 256)
    return fail(PB_ERR_INVALID_ARG, "ws is NULL or not 256-byte aligned");
  if (bytes < need) return fail(PB_ERR_WORKSPACE, "ws_bytes=%zu < %zu needed", bytes, need);
  return PB_OK;
}

// Rows of `width` elements of `e` bytes, ld elements apart.
struct Span {
  const void* p;
  size_t ld, width;
  int64_t rows;
};
// Whether two such share memory.  Tensors apart as a whole, or of one leading dimension
// (whose rows may interleave), are told at once; else the rows of one are looked up among
// the other's, a few ns each.
[[maybe_unused]] bool overlap(const Span& a, const Span& b, size_t e) {
  if (!a.rows || !b.rows || !a.p || !b.p) return false;
  const Span &lo = (uintptr_t)a.p <= (uintptr_t)b.p ? a : b, &hi = &lo == &a ? b : a;
  const size_t off = ((uintptr_t)hi.p - (uintptr_t)lo.p) / e;  // elements from lo to hi
  if (off >= (size_t)(lo.rows - 1) * lo.ld + lo.width) return false;
  if (lo.rows > 1 && off % lo.ld < lo.width) return true;
  if (lo.ld == hi.ld || lo.rows == 1 || hi.rows == 1) {
    const size_t ld = lo.rows > 1 ? lo.ld : hi.ld, at = off % ld;
    return at < lo.width || ld - at < hi.width;
  }
  const Span &few = lo.rows < hi.rows ? lo : hi, &many = &few == &lo ? hi : lo;
  const int64_t first = &few == &hi ? (int64_t)off : -(int64_t)off;  // of few, from many's
  const int64_t ld = (int64_t)few.ld, width = (int64_t)few.width, ld2 = (int64_t)many.ld;
  const int64_t end = (many.rows - 1) * ld2 + (int64_t)many.width;
  for (int64_t r = first < 0 ? -first / ld : 0; r < few.rows && first + r * ld < end; ++r) {
    const int64_t at = first + r * ld;
    if (at + width <= 0) continue;
    // many's last row that begins before this one ends
    const int64_t k = std::min((at + width - 1) / ld2, many.rows - 1);
    if (k * ld2 + (int64_t)many.width > at) return true;
  }
  return false;
}
// A workspace (or other dense range) and the rows of an element of e bytes.
[[maybe_unused]] bool overlap(const void* ws, size_t bytes, const Span& x, size_t e) {
  return overlap(Span{ws, bytes, bytes, 1}, Span{x.p, x.ld * e, x.width * e, x.rows}, 1);
}

// A dense range of a call's memory.  An output may be an input where both are rows of
// the same size that the call reads before it writes them.
struct Range {
  const char* name;
  const void* p;
  size_t bytes;
  bool out, same;
};
template <size_t N>
pb_status check_apart(const Range (&r)[N]) {
  for (size_t i = 0; i < N; ++i)
    for (size_t j = 0; j < i; ++j) {
      const Range &a = r[i], &b = r[j];
      if (!a.p || !b.p || !(a.out || b.out)) continue;
      if (a.p == b.p && a.same && b.same && !(a.out && b.out)) continue;
      const uintptr_t pa = (uintptr_t)a.p, pb = (uintptr_t)b.p;
      if (pa < pb + b.bytes && pb < pa + a.bytes)
        return fail(PB_ERR_INVALID_ARG, "%s and %s overlap", a.name, b.name);
    }
  return PB_OK;
}

// A call without any element: as finish_launches(), but no HIP call is made.
[[maybe_unused]] pb_status nothing_to_do() {
  pb::clear_error();
  return PB_OK;
}

#define PB_CHECK(expr)                      \
  do {                                      \
    const pb_status st_ = (expr);           \
    if (st_ != PB_OK) return st_;           \
  } while (0)

}  // namespace
