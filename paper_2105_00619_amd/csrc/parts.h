// How a reduction is cut into parts.
#pragma once
#include <stdint.h>

#if defined(__HIPCC__)
#define OSEQ_PARTS_FN __host__ __device__ __forceinline__
#else
#define OSEQ_PARTS_FN inline
#endif

namespace oseq {

// K values in at most `wanted` parts of whole slots of 64; a part's values are [first, end).  K up to 2^31 - 256: its
// parts' ends are no sums of two numbers near it, which wrap.
struct Parts {
  int K, size, count;
  OSEQ_PARTS_FN int first(int part) const { return part * size; }
  OSEQ_PARTS_FN int end(int part) const { const int left = K - part * size; return part * size + (left < size ? left : size); }
};
inline Parts parts_of(int K, int wanted) {
  const int64_t slots = ((int64_t)K + 63) / 64;
  const int64_t size = (slots + wanted - 1) / wanted * 64;
  return Parts{K, (int)size, (int)(((int64_t)K + size - 1) / size)};
}

}  // namespace oseq
