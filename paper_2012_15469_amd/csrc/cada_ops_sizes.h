// Sizes and alignments of the operators' arguments, on the host.
#pragma once

#include <cstddef>
#include <cstdint>

#include "cada_ops.h"

namespace cada {

constexpr size_t kOpsAlign = 256;
inline size_t ops_align(size_t x) { return (x + kOpsAlign - 1) / kOpsAlign * kOpsAlign; }
inline size_t type_bytes(int type) { return type == CADA_BF16 ? 2 : 4; }
inline bool aligned16(const void *p, int64_t ld, size_t elem) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (ld * (int64_t)elem) % 16 == 0; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace cada
