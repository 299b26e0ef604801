// Checks of arguments that the C entry points on rows of logits share.  Host code only.
#pragma once

#include <stdint.h>

#include "rtopk.h"
#include "rtopk_shape.hpp"

namespace rtopk {
namespace checks {

inline uintptr_t addr(const void* p) { return reinterpret_cast<uintptr_t>(p); }

struct Buffer {
  const void* p;
  uint64_t bytes, align;
  bool written;
};

// RTOPK_OK, or what is wrong with the buffers: alignment, or bytes that a written one shares with another.
template <int C>
int check_buffers(const Buffer (&b)[C]) {
  for (const Buffer& x : b)
    if (!is_aligned(addr(x.p), x.align)) return RTOPK_ERR_MISALIGNED;
  for (int i = 0; i < C; ++i)
    for (int j = i + 1; j < C; ++j)
      if ((b[i].written || b[j].written) && b[i].p && b[j].p && ranges_overlap(addr(b[i].p), b[i].bytes, addr(b[j].p), b[j].bytes))
        return RTOPK_ERR_OVERLAP;
  return RTOPK_OK;
}

inline uint64_t size_of(int dtype) { return dtype == RTOPK_F32 ? 4 : 2; }
inline bool is_type(int dtype) { return dtype == RTOPK_F32 || dtype == RTOPK_F16 || dtype == RTOPK_BF16; }

}  // namespace checks
}  // namespace rtopk
