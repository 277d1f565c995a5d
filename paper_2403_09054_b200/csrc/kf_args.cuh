// Host-side checks of arguments that the context-free entry points share (kf_api_ops.cu, kf_api_pages.cu).
#pragma once

#include <cstddef>
#include <cstdint>
#include <initializer_list>

namespace kf {
namespace args {

constexpr size_t ALIGN = 256;
inline size_t align_up(size_t x) { return (x + ALIGN - 1) / ALIGN * ALIGN; }
inline bool misaligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }
// Whether [a, a + n) and [b, b + m) share a byte.
inline bool overlap(const void* a, uint64_t n, const void* b, uint64_t m) {
  const uint64_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a && b && x < y + m && y < x + n;
}
// A tensor of a call.  `rows` > 1: that many rows of `bytes`, `stride` bytes apart; what lies between them is not the call's.
struct Range {
  const void* at;
  uint64_t bytes, rows = 1, stride = 0;
  uint64_t extent() const { return (rows - 1) * stride + bytes; }
};
// [a][b] rows of d 16-bit values (strides in elements) that lie apart from one another, as rows at one stride where that says it all: single rows, or
// what belongs to one of the outer dimension.
inline Range rows_of(const void* at, int64_t a, int64_t stride_a, int64_t b, int64_t stride_b, int d) {
  const uint64_t A = (uint64_t)a, B = (uint64_t)b, sa = 2 * (uint64_t)stride_a, sb = 2 * (uint64_t)stride_b, row = 2 * (uint64_t)d;
  if (a == 1 || sa == B * sb) return {at, row, A * B, sb};
  if (b == 1 || sb == A * sa) return {at, row, A * B, sa};
  return sa >= sb ? Range{at, (B - 1) * sb + row, A, sa} : Range{at, (A - 1) * sa + row, B, sb};
}
// Whether one of the rows of `a` shares a byte with the extent of `b`, or with one of its rows where they come at the same stride, given that
// the two extents share one.
inline bool touches(const Range& a, const Range& b) {
  if (a.rows == 1 || a.stride <= a.bytes) return true;
  if (b.rows > 1 && b.stride == a.stride) {
    const int64_t apart = (int64_t)(reinterpret_cast<uintptr_t>(b.at) - reinterpret_cast<uintptr_t>(a.at)) % (int64_t)a.stride;
    const uint64_t from = (uint64_t)(apart < 0 ? apart + (int64_t)a.stride : apart);
    return from < a.bytes || from + b.bytes > a.stride;
  }
  const uint64_t base = reinterpret_cast<uintptr_t>(a.at), x = reinterpret_cast<uintptr_t>(b.at);
  const uint64_t begin = x > base ? x - base : 0, end = x + b.extent() - base;     // of b, from the first row on
  return begin % a.stride < a.bytes || end > (begin / a.stride + 1) * a.stride;
}
// Whether something that the call writes shares memory with another of its tensors.  Every pair of extents without a branch
// (this runs for every token and layer): two meet where both differences are negative; one that is absent ends before everything.
inline bool conflict(std::initializer_list<Range> writes, std::initializer_list<Range> reads) {
  constexpr int MOST = 16;
  uint64_t from[MOST], to[MOST];
  int n = 0;
  auto add = [&](const Range& r) {
    from[n] = reinterpret_cast<uintptr_t>(r.at);
    to[n] = r.at ? from[n] + r.extent() : 0;
    ++n;
  };
  for (const Range& r : writes) add(r);
  const int written = n;
  for (const Range& r : reads) add(r);
  uint64_t meet = 0;
  for (int i = 0; i < written; ++i)
    for (int j = i + 1; j < n; ++j) meet |= (from[j] - to[i]) & (from[i] - to[j]);
  if (meet >> 63 == 0) return false;
  auto range = [&](int i) { return i < written ? writes.begin()[i] : reads.begin()[i - written]; };
  for (int i = 0; i < written; ++i)
    for (int j = i + 1; j < n; ++j)
      if (from[j] < to[i] && from[i] < to[j] && touches(range(j), range(i))) return true;
  return false;
}
inline bool head_dim_ok(int d) { return d == 64 || d == 128 || d == 256; }

}  // namespace args
}  // namespace kf
