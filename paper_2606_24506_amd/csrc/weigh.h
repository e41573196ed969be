// Weights that queries give to cached tokens (cp_attn_weights): launch records shared by
// the host planner (api.cpp) and the kernels (weigh_kernels.hip).
#pragma once

#include <stdint.h>

#include "extend.h"
#include "kargs.h"

namespace cp {

// Kernels, chosen per request by the model's geometry and its rows (a query token and a
// query head of one KV head).
//   kWVec   vector: one thread per key, any geometry.
//   kWFew*  matrix cores, at most 16 rows: bound by reading K.
//   kWRows* matrix cores, keys in registers, blocks of rows streamed past them.
// 64 and 128: GQA / MHA of that head_dim; Mla: latent 512 and rotary part 64.
enum : int32_t { kWVec = 0, kWFew64, kWFew128, kWFewMla, kWRows64, kWRows128, kWRowsMla, kWKinds };

constexpr int kWeighThreads = 256;
constexpr int kWeighBlock = 64;  // rows of a block
// Keys of a workgroup.
constexpr int32_t weigh_tile_keys(int32_t kind) {
  return kind == kWFew64 ? 512 : kind == kWFewMla ? 128 : 256;
}

struct WeighReq {
  const float *old;  // this layer's rows of the sums so far (NULL: none)
  float *sum;        // ... and of the result
  int64_t old_head, sum_head;
  uint64_t ws;           // splits > 1: the first partial sum, [split][KV head][ctx]
  uint32_t unit_begin;   // first workgroup
  uint32_t pte_base, ctx, n_q, prefix;
  uint32_t tok0;         // its first query token in the call's arrays
  uint32_t tiles, splits;  // of keys, and of the rows of a tile
};
constexpr int kWeighMaxReq = 40;

struct WeighArgs {
  const uint8_t *pool;
  const uint32_t *pte;
  const uint16_t *q;
  const float *lse;
  float *ws;
  const float *slopes;
  const int32_t *doc_begin;
  float decay;
  float softcap, score_mul, cap_mul, cap_edge, cap_k[kTanhTerms];  // as ExtArgs
  uint32_t window, page_magic, g_magic;
  int32_t n_req, n_units;
  GeomK g;
  WeighReq req[kWeighMaxReq];
};
static_assert(sizeof(WeighArgs) <= 3776, "weight kernel arguments too large");

struct WeighJoinArgs {
  const float *ws;
  float decay;
  int32_t n_req, n_blocks, hkv;
  struct Req {
    const float *old;
    float *sum;
    int64_t old_head, sum_head;
    uint64_t ws;
    uint32_t block_begin, ctx, splits, pad;
  } req[kWeighMaxReq];
};
static_assert(sizeof(WeighJoinArgs) <= 3776, "weight join arguments too large");

}  // namespace cp
