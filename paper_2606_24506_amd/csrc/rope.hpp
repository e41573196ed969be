// Rotary positions: the handle behind cp_rope and the records its kernels
// take (rope.cpp, rope_kernels.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <vector>

#include "crosspool.h"
#include "kargs.h"

struct cp_rope {
  int device = -1;  // -1: host only
  int32_t rot = 0;  // rotated elements of a head
  int32_t layout = CP_ROPE_HALF;
  float magnitude = 1.f;
  std::vector<double> turns;    // full turns per position, one per pair
  double *dev_turns = nullptr;  // the same in device memory
};

namespace cp {

constexpr int kRopeThreads = 256;
constexpr int kMaxRopeParts = 16;  // tensors in one launch

// The rotation as the kernels see it.
struct RopeK {
  const double *turns;
  float magnitude;
  int32_t pairs;        // rot / 2
  int32_t interleaved;  // pairs (2i, 2i + 1) instead of (i, i + pairs)
  int32_t inverse;
};

// One tensor [tokens][heads][width]; strides in elements.
struct RopePart {
  const void *src;
  void *dst;
  int64_t src_tok, src_head, dst_tok, dst_head;
  int32_t heads, width, offset, vec;  // vec: every 16-byte access is aligned
};

struct RopeArgs {
  RopeK rope;
  const int32_t *pos;  // NULL: first + token
  int64_t first, n_tokens;
  int32_t n_parts, tokens;  // tokens per workgroup
  RopePart part[kMaxRopeParts];
  int32_t item0[kMaxRopeParts + 1];  // first work item of each part among one token's
};
static_assert(sizeof(RopeArgs) <= 3776, "rope kernel arguments too large");

inline RopeK rope_k(const cp_rope &r, bool inverse) {
  return RopeK{r.dev_turns, r.magnitude, r.rot / 2, r.layout == CP_ROPE_INTERLEAVED, inverse};
}

}  // namespace cp
