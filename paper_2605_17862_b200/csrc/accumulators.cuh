// How a tile's contraction is cut into accumulators: blocks [done, accumulator_end) share one, then it is taken out and added up in fp32.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define FOPD_EVERYWHERE __host__ __device__ __forceinline__
#else
#define FOPD_EVERYWHERE inline
#endif

namespace fopd {

// Blocks of 64 to an accumulator at most, whatever is summed: the last bits that 16,384 terms lose are below 2^-14 of their sum, and a
// wait for one accumulator is short whatever the length of the contraction.
constexpr int kLongChunk = 256;

// Of `blocks` blocks the first `small` are of products with planes of what roundings left (2^-11 or 2^-8 of the others: one long
// accumulator after another is exact enough); the others are taken out every `chunk` (at most kLongChunk).
FOPD_EVERYWHERE int accumulator_end(int done, int small, int blocks, int chunk) {
  if (done < small) return small - done < kLongChunk ? small : done + kLongChunk;
  return blocks - done < chunk ? blocks : done + chunk;
}

}  // namespace fopd
