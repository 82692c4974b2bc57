// Rows of heads as the serving calls take them: x[t * ld + h * hs + c], channels side by side.
#pragma once
#include <algorithm>

#include "cafeq_common.hpp"

namespace cafeq {

inline bool aligned_to(const void* p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

struct HeadRows {
  const void* p;
  int64_t n, ld, heads, hs, d;
  int size;      // bytes an element
  int64_t width() const { return (heads - 1) * hs + d; }        // elements of a token, first to last
  int64_t length() const { return (n - 1) * ld + d; }           // of a head over all tokens
  int64_t extent() const { return ((n - 1) * ld + width()) * size; }
  // whether no element has two places: tokens behind each other, or heads
  bool plain() const {
    if (ld < 0 || hs < 0) return false;
    return ((heads == 1 || hs >= d) && (n == 1 || ld >= width())) || ((n == 1 || ld >= d) && (heads == 1 || hs >= length()));
  }
  bool same(const HeadRows& o) const { return p == o.p && (n == 1 || ld == o.ld) && (heads == 1 || hs == o.hs) && heads == o.heads; }
};

// Whether two of them may share memory.  Slices side by side of rows with one leading dimension do not; what is not seen to be apart counts as
// sharing.
inline bool may_share(const HeadRows& a, const HeadRows& b) {
  if (!a.p || !b.p || a.n < 1 || b.n < 1) return false;
  const auto p = reinterpret_cast<uintptr_t>(a.p), q = reinterpret_cast<uintptr_t>(b.p);
  if (p >= q + uint64_t(b.extent()) || q >= p + uint64_t(a.extent())) return false;
  auto cross = [&](int64_t step, int64_t wa, int64_t wb, bool more) {
    // runs of wa and wb elements, both every `step` of them
    if (!more || step <= 0 || wa > step || wb > step) return true;
    const uint64_t s = uint64_t(step) * a.size;
    const uint64_t off = p > q ? (s - (p - q) % s) % s : (q - p) % s;     // where b's runs begin behind a's
    return off < uint64_t(wa) * a.size || off + uint64_t(wb) * b.size > s;
  };
  if (a.size == b.size && a.ld == b.ld && !cross(a.ld, a.width(), b.width(), a.n > 1)) return false;
  if (a.size == b.size && a.hs == b.hs && !cross(a.hs, a.length(), b.length(), a.heads > 1)) return false;
  return true;
}

}  // namespace cafeq
