// Regions of device memory that entry points compare before a launch.
#pragma once

#include <cstdint>

namespace aecct {

// `rows` rows of `width` bytes, `pitch` bytes apart.
struct Span {
  const void *p;
  int64_t rows, width, pitch;
  uintptr_t begin() const { return (uintptr_t)p; }
  uintptr_t end() const { return rows > 0 && width > 0 ? begin() + (uintptr_t)((rows - 1) * pitch + width) : begin(); }
};
inline bool same(const Span &a, const Span &b) {
  return a.p == b.p && a.width == b.width && (a.pitch == b.pitch || a.rows <= 1);
}
// Whether two regions may share a byte: their spans do, unless both are columns of rows of one pitch that lie side by side.
inline bool overlap(const Span &a, const Span &b) {
  if (!a.p || !b.p || a.begin() >= b.end() || b.begin() >= a.end()) return false;
  if (a.pitch != b.pitch || a.pitch <= 0) return true;
  const uintptr_t pitch = (uintptr_t)a.pitch;
  const uintptr_t off = b.begin() >= a.begin() ? (b.begin() - a.begin()) % pitch
                                               : (pitch - (a.begin() - b.begin()) % pitch) % pitch;
  return !(off >= (uintptr_t)a.width && off + (uintptr_t)b.width <= pitch);
}

}  // namespace aecct
