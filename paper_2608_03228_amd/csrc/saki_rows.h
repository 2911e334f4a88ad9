// How the kernels over packed prompts find the rows of a work-group.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "saki_topk.h"

namespace saki_dev {

// Block `x` of `rows` rows of the packed prompts.  The rows of one KV head are
// (token, one of its G query heads) pairs, token after token; a prompt's blocks
// start at floor(first row / rows) + b, which leaves each prompt its own ones
// (with gaps), so that a block finds its prompt by a search of the offsets.
struct Block {
  int b, start, len, row0;  // prompt, its first token and length, first row in it; len = 0: none
};
__device__ __forceinline__ Block find_block(const int* cu, int B, int T, int x, int G, int rows) {
  auto at = [&](int b) { return min(max(cu[b], 0), T); };
  int lo = 0, n = B;  // the prompt is one of lo .. lo + n - 1: a wave tells 64 parts of them apart at once
  while (n > 1) {
    const int step = (n + kWave - 1) / kWave, i = (int)(threadIdx.x % kWave) * step;
    const bool below = i < n && (long long)at(lo + i) * G / rows + lo + i <= x;
    const uint64_t which = __ballot(below);  // none: the block lies before the first prompt
    const int part = which ? (63 - __builtin_clzll(which)) * step : 0;
    n = min(n - part, step);
    lo += part;
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  Block r;
  r.b = lo;
  r.start = at(lo);
  r.len = max(at(lo + 1) - r.start, 0);
  const long long row0 = (x - ((long long)r.start * G / rows + lo)) * rows;
  if (row0 < 0 || row0 >= (long long)r.len * G) r.len = 0;
  r.row0 = (int)row0;
  return r;
}

}  // namespace saki_dev
