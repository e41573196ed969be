// gfx950 kernel of the masks and depths of drafted trees (cp_tree_build).
#include <hip/hip_runtime.h>

#include "device_common.h"
#include "tree.h"

namespace cp {

// A thread takes a token and walks up: its ancestors' numbers fall, so the words of its
// mask are finished one after the other, from the token's own down, and each is written
// once. The parents of the tree are in LDS (a number that is no earlier token's ends the
// walk, so that every walk ends). Bound by its launch and the longest walk: a step is one
// LDS round trip, some 50 ns. One tree of 8 tokens 1.5 us, eight of 61 4 us.
__global__ __launch_bounds__(kTreeThreads) void tree_kernel(const TreeArgs a) {
  extern __shared__ int32_t up[];
  const int r = sorted_search(a.n_req, blockIdx.x, [&](int i) { return a.req[i].block_begin; });
  const TreeArgs::Req &rq = a.req[r];
  const uint32_t t0 = (blockIdx.x - rq.block_begin) * kTreeThreads, t1 = min(rq.n, t0 + kTreeThreads);
  for (uint32_t i = threadIdx.x; i < t1; i += kTreeThreads) up[i] = a.parents[rq.tok0 + i];
  __syncthreads();
  const uint32_t t = t0 + threadIdx.x;
  if (t >= t1) return;
  uint32_t *const row = a.mask + (uint64_t)(rq.tok0 + t) * (uint32_t)a.words;
  int32_t w = a.words - 1, depth = -1;
  uint32_t bits = 0, at = t;
  for (;;) {
    const int32_t word = (int32_t)(at / 32);
    while (w > word) {
      row[w--] = bits;
      bits = 0;
    }
    bits |= 1u << (at % 32);
    ++depth;
    const int32_t next = up[at];
    if (next < 0 || (uint32_t)next >= at) break;
    at = (uint32_t)next;
  }
  while (w >= 0) {
    row[w--] = bits;
    bits = 0;
  }
  a.depth[rq.tok0 + t] = depth;
}

hipError_t launch_tree(const TreeArgs &a, hipStream_t stream) {
  if (a.n_blocks <= 0) return hipSuccess;
  uint32_t most = 0;
  for (int i = 0; i < a.n_req; ++i) most = a.req[i].n > most ? a.req[i].n : most;
  hipLaunchKernelGGL(tree_kernel, dim3((uint32_t)a.n_blocks), dim3(kTreeThreads), most * sizeof(int32_t), stream, a);
  return hipGetLastError();
}

}  // namespace cp
