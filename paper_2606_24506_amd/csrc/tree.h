// Masks and depths of drafted trees (cp_tree_build): launch records shared by the host
// (api.cpp) and the kernel (tree_kernels.hip).
#pragma once

#include <stdint.h>

namespace cp {

constexpr int kTreeThreads = 256;
constexpr int kMaxTreesPerLaunch = 64;

struct TreeArgs {
  const int32_t *parents;
  uint32_t *mask;
  int32_t *depth;
  int32_t words, n_req, n_blocks, pad;
  struct Req {
    uint32_t tok0, n;      // its first token in the arrays, and how many
    uint32_t block_begin;  // its first workgroup
    uint32_t pad;
  } req[kMaxTreesPerLaunch];
};
static_assert(sizeof(TreeArgs) <= 3776, "tree kernel arguments too large");

}  // namespace cp
