// Checks, on the host, of what a call may not let overlap (cmc_prefill.cu, cmc_attn_weighted.cu, cmc_evict.cu).
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace cmc {

// Memory that a call reads or writes (at NULL: none).
struct Range {
  const void* at;
  size_t bytes;
};
inline bool meet(const Range& a, const Range& b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.at), y = reinterpret_cast<uintptr_t>(b.at);
  return a.at && b.at && a.bytes && b.bytes && x < y + b.bytes && y < x + a.bytes;
}
inline bool same(const Range& a, const Range& b) { return a.at == b.at && a.bytes == b.bytes; }
// Whether one of `a` meets one of `b`, or another of `a`.
template <int N, int M>
inline bool any_meet(const Range (&a)[N], const Range (&b)[M]) {
  for (int i = 0; i < N; ++i)
    for (int j = 0; j < M; ++j)
      if (meet(a[i], b[j])) return true;
  return false;
}
template <int N>
inline bool any_meet(const Range (&a)[N]) {
  for (int i = 0; i < N; ++i)
    for (int j = 0; j < i; ++j)
      if (meet(a[i], a[j])) return true;
  return false;
}

}  // namespace cmc
