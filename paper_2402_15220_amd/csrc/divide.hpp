// Division by a number fixed for a call, for the kernels that number the tiles
// and units of chunks.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace ca {

// x / n for 0 <= x by a product with the rounded-up inverse; exact while x n
// stays below 2^32 (windowed calls: kWindowChunk).
__device__ __forceinline__ uint32_t inverse32(int n) {
  return n > 1 ? 0xffffffffu / static_cast<unsigned>(n) + 1u : 0u;
}
__device__ __forceinline__ int divide32(int x, int n, uint32_t inv) {
  return n == 1 ? x : static_cast<int>(__umulhi(static_cast<unsigned>(x), inv));
}

}  // namespace ca
