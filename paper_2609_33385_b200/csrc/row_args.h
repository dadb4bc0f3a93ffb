// Host checks of row-strided arguments that the entry points without a context share.
#pragma once
#include <cstddef>
#include <cstdint>

namespace oled {

inline bool off_boundary(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

// No array's rows are further apart than this (elements): the last row's offset stays in 64 bits for every array that memory can hold.
constexpr int64_t kMaxStride = 1ll << 36;
inline bool stride_ok(int64_t stride, int64_t width) { return stride >= width && stride <= kMaxStride; }

// `rows` rows of `width` bytes, `stride` bytes apart.
struct RowRange {
  const void* p;
  int64_t stride, width, rows;
};
// Do two arrays share a byte?  Columns of one buffer, whose rows interleave, do not.
inline bool rows_overlap(const RowRange& a, const RowRange& b) {
  if (a.p == nullptr || b.p == nullptr || a.rows <= 0 || b.rows <= 0 || a.width <= 0 || b.width <= 0) return false;
  const auto a0 = reinterpret_cast<uintptr_t>(a.p), b0 = reinterpret_cast<uintptr_t>(b.p);
  const uintptr_t a1 = a0 + (uintptr_t)((a.rows - 1) * a.stride + a.width), b1 = b0 + (uintptr_t)((b.rows - 1) * b.stride + b.width);
  if (a1 <= b0 || b1 <= a0) return false;
  if (a.stride == b.stride && a.stride > 0) {
    const int64_t d = (int64_t)((b0 - a0) % (uintptr_t)a.stride), e = (int64_t)((a0 - b0) % (uintptr_t)a.stride);
    const int64_t ahead = b0 >= a0 ? d : (e == 0 ? 0 : a.stride - e);  // b's column within a's rows
    return !(ahead >= a.width && ahead + b.width <= a.stride);
  }
  return true;
}
inline bool same_rows(const RowRange& a, const RowRange& b) { return a.p == b.p && a.stride == b.stride && a.width == b.width; }

}  // namespace oled
