// Checks of the buffers of a call (host).
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace sgmv {

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// A device buffer of a call; none at all where `at` is nullptr.
struct Span {
  const void* at;
  size_t bytes;
};
inline bool overlap(const Span& a, const Span& b) {
  const uintptr_t from = reinterpret_cast<uintptr_t>(a.at), to = reinterpret_cast<uintptr_t>(b.at);
  return a.at != nullptr && b.at != nullptr && (to - from < a.bytes || from - to < b.bytes);
}

}  // namespace sgmv
