// Rows of bytes that lie on one another: calls refuse outputs over what they read (host).
#pragma once

#include <stdint.h>

#include <algorithm>
#include <utility>

namespace seedq {

__extension__ typedef __int128 Wide;  // strides are the caller's: products of any of them

// n0 x n1 rows of `bytes` bytes, s0 and s1 bytes apart; counts of one or more.
struct ByteRows {
  Wide at, n0, s0, n1, s1, bytes;
};
inline ByteRows byte_rows(const void *p, Wide bytes, Wide n0 = 1, Wide s0 = 0, Wide n1 = 1, Wide s1 = 0) {
  ByteRows r{(Wide)(uintptr_t)p, n0, s0, n1, s1, bytes};
  // strides of zero for single rows, upwards, the larger first
  if (r.n0 == 1) r.s0 = 0;
  if (r.n1 == 1) r.s1 = 0;
  if (r.s0 < 0) r.at += (r.n0 - 1) * r.s0, r.s0 = -r.s0;
  if (r.s1 < 0) r.at += (r.n1 - 1) * r.s1, r.s1 = -r.s1;
  if (r.n0 == 1 || (r.n1 > 1 && r.s0 < r.s1)) std::swap(r.n0, r.n1), std::swap(r.s0, r.s1);
  return r;
}

// What a search of interleaved rows may take; beyond it they count as overlapping.
constexpr int64_t kOverlapSteps = 1 << 20;

// Whether two different rows have a byte in common.
inline bool overlaps_itself(const ByteRows &r) {
  if (r.n0 > 1 && r.s0 < r.bytes) return true;
  if (r.n1 > 1 && r.s1 < r.bytes) return true;
  if (r.n0 == 1 || (r.n1 - 1) * r.s1 + r.bytes <= r.s0) return false;
  // i steps of the larger stride against j of the smaller
  if (std::min(r.n0, r.n1) > kOverlapSteps) return true;
  if (r.n0 <= r.n1) {
    for (Wide i = 1; i < r.n0; ++i) {
      const Wide j = i * r.s0 / r.s1;
      for (Wide k = j; k <= j + 1 && k < r.n1; ++k)
        if (k * r.s1 - i * r.s0 < r.bytes && i * r.s0 - k * r.s1 < r.bytes) return true;
    }
  } else {
    for (Wide j = 1; j < r.n1; ++j) {
      const Wide i = j * r.s1 / r.s0;
      for (Wide k = std::max<Wide>(i, 1); k <= i + 1 && k < r.n0; ++k)
        if (j * r.s1 - k * r.s0 < r.bytes && k * r.s0 - j * r.s1 < r.bytes) return true;
    }
  }
  return false;
}

// The same bytes in fewer rows, where rows touch or lie evenly.
inline ByteRows joined_rows(ByteRows r) {
  if (r.n1 > 1 && r.s1 <= r.bytes) r.bytes += (r.n1 - 1) * r.s1, r.n1 = 1, r.s1 = 0;
  if (r.n1 > 1 && r.s0 == r.n1 * r.s1) r.n0 *= r.n1, r.s0 = r.s1, r.n1 = 1, r.s1 = 0;
  if (r.n1 == 1 && r.n0 > 1 && r.s0 <= r.bytes) r.bytes += (r.n0 - 1) * r.s0, r.n0 = 1, r.s0 = 0;
  return r;
}

// Whether two sets of rows have a byte in common.
inline bool overlap(const ByteRows &x, const ByteRows &y) {
  auto end = [](const ByteRows &r) { return r.at + (r.n0 - 1) * r.s0 + (r.n1 - 1) * r.s1 + r.bytes; };
  if (end(x) <= y.at || end(y) <= x.at) return false;
  const ByteRows a = joined_rows(x), b = joined_rows(y);
  // k in [low, high] with -a.bytes < d + k s < b.bytes
  auto meet = [&](Wide d, Wide s, Wide low, Wide high) {
    if (s == 0) return -a.bytes < d && d < b.bytes;
    const Wide least = -a.bytes - d;  // the first k behind it
    const Wide k = std::max(low, (least >= 0 ? least / s : -((-least + s - 1) / s)) + 1);
    return k <= high && d + k * s < b.bytes;
  };
  const bool even = a.n0 == 1 || b.n0 == 1 || a.s0 == b.s0;
  Wide steps = 0;
  for (Wide i = 0; i < a.n1; ++i)
    for (Wide j = 0; j < b.n1; ++j) {
      const Wide d = a.at + i * a.s1 - (b.at + j * b.s1);
      steps += even ? 1 : a.n0 + b.n0;
      if (steps > kOverlapSteps) return true;
      if (even) {
        if (meet(d, a.n0 == 1 ? b.s0 : a.s0, b.n0 == 1 ? 0 : -(b.n0 - 1), a.n0 == 1 ? 0 : a.n0 - 1)) return true;
        continue;
      }
      for (Wide k = 0, l = 0; k < a.n0 && l < b.n0;) {
        const Wide p = d + k * a.s0, q = l * b.s0;
        if (p + a.bytes <= q) ++k;
        else if (q + b.bytes <= p) ++l;
        else return true;
      }
    }
  return false;
}

}  // namespace seedq
