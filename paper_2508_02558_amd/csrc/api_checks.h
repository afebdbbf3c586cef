// What the entry points check their arguments with.
#pragma once

#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include "sdllm.h"

namespace sdllm {

constexpr size_t kAlign = 256;
constexpr float kLog2e = 1.4426950408889634f;
inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
inline int elem_size(int dtype) { return dtype == SDLLM_BF16 ? 2 : 4; }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline bool strides_ok(const int64_t* st, int esize) {
  for (int i = 0; i < 3; ++i)
    if (st[i] < 0 || (st[i] * esize) % 16 != 0) return false;
  return true;
}

inline bool row_stride_ok(const int64_t* st, int d) { return st[2] >= d; }

// the fields of a shape that say what is done to a head
int32_t check_qk_shape(const sdllm_qk_shape_t* s);

}  // namespace sdllm
