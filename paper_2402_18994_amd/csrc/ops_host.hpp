// Host arithmetic that the entry points of snn_ops.h share (no HIP).
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "../../include/snn_ops.h"

namespace snn {

inline bool aligned(const void *p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
inline size_t rup256(size_t n) { return (n + 255) & ~(size_t)255; }

// Whether the rows of a tensor of T steps of B sequences can be taken `vec` elements of `size` bytes at a time.
inline bool rows_take(const snn_rows &r, int T, int B, int vec, size_t size) {
  return !r.p || (aligned(r.p, vec * size) && (T <= 1 || r.stride_t % vec == 0) && (B <= 1 || r.stride_b % vec == 0));
}

}  // namespace snn
