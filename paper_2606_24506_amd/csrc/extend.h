// Attention of token chunks (cp_attn_extend): launch records shared by the
// host planner (api.cpp) and the kernels (extend_kernels.hip), and the device
// helpers of those kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kargs.h"

namespace cp {

// Kernels, chosen per call by the model's geometry and its rows per KV head.
//   kXVec    vector: one wave per row, any geometry.
//   kXRows*  matrix cores, GQA / MHA of head_dim 64 or 128: tiles of 128 rows.
//   kXSome*  the same with 32 rows, the four waves taking keys in turn.
//   kXFew*   ... with 16 rows.
//   kXMla    matrix cores, MLA with latent 512 and rotary part 64: 128 rows.
enum : int32_t { kXVec = 0, kXRows64, kXRows128, kXSome64, kXSome128, kXFew64, kXFew128, kXMla, kXKinds };

constexpr int kExtThreads = 256;
// Rows (a token and a query head of one KV head) of a tile, and keys of one
// step, of each kernel.
constexpr int32_t ext_tile_rows(int32_t kind) {
  return kind == kXVec ? 4 : kind == kXSome64 || kind == kXSome128 ? 32 : kind == kXFew64 || kind == kXFew128 ? 16 : 128;
}
constexpr int32_t ext_tile_keys(int32_t kind) {
  return kind >= kXSome64 && kind <= kXFew128 ? 128 : kind == kXMla ? 32 : 64;
}

// tanh(x) = x + x sum_{k > 0} kTanh[k] x^2k, to 4.2e-8 of its value under kCapEdge (in
// exact arithmetic): a least-squares fit, reweighted towards its largest relative error.
constexpr int kTanhTerms = 4;
constexpr float kTanh[kTanhTerms] = {1.f, -3.33326690e-01f, 1.32999740e-01f, -4.91567400e-02f};
constexpr float kCapEdge = 0.35f;

constexpr int kExtMaxReq = 40;  // items of a launch, and requests of its shared ones

// One item: a request, or a part of it. Requests that share leading pages
// (forks) and stand next to each other are taken apart: the shared keys are one
// item, whose rows are those of all of them, and the keys behind are an item of each.
struct ExtReq {
  uint32_t unit_begin;  // first workgroup of the item (a multiple of 8)
  uint32_t pte_base;    // page-table entries of the plane
  uint32_t ctx, n_q;    // context, and how many of its last tokens ask
  uint32_t prefix;
  uint32_t tok0;        // its first query token in the call's arrays
  uint32_t n_tok;       // query tokens (n_q, or those of all members)
  uint32_t key_lo, key_hi;  // the item's keys
  uint32_t tiles;       // row tiles per KV head
  uint32_t splits;      // key ranges per tile
  uint32_t split0, all; // the first of its ranges among all of its rows', and how many those have
  uint16_t member0, members;  // of ExtArgs::member (members 0: a request of its own)
  uint64_t ws_row;      // first partial row (all > 1)
};
struct ExtMember {
  uint32_t ctx, n_q, prefix, pad;
};

struct ExtArgs {
  const uint8_t *pool;
  const uint32_t *pte;
  const uint16_t *q;
  uint16_t *out;
  float *lse;
  float *ws_o;  // partial outputs, normalised: [row][split][d_v]
  float *ws_l;  // partial log-sum-exp (base 2): [row][split]
  const float *slopes;
  const int32_t *doc_begin;
  float softcap;
  // Scores from products, in units of log2 e: product * score_mul, or capped
  // cap_mul * tanh(product * score_mul); while |product| < cap_edge the latter is
  // product * sum_k cap_k[k] product^2k.
  float score_mul, cap_mul, cap_edge, cap_k[kTanhTerms];
  uint32_t window;
  uint32_t page_magic;  // page_divide
  int32_t n_req, n_units;
  GeomK g;
  ExtReq req[kExtMaxReq];
  ExtMember member[kExtMaxReq];
};
static_assert(sizeof(ExtArgs) <= 3776, "extend kernel arguments too large");

struct ExtMergeArgs {
  const float *ws_o, *ws_l;
  uint16_t *out;
  float *lse;
  int32_t n_req, d_v, lanes, pad;  // lanes: ranges of a row taken at once
  struct Req {
    uint32_t row_begin, rows;  // rows of the launch before, and of, these requests
    uint64_t ws_row;
    uint64_t out_row;
    uint32_t splits, pad;
  } req[kMaxReqPerLaunch];
};
static_assert(sizeof(ExtMergeArgs) <= 3776, "extend merge arguments too large");

// floor(2^32 / P), for page_divide on the device.
inline uint32_t page_magic(int32_t page_tokens) {
  return page_tokens == 1 ? 0xFFFFFFFFu : (uint32_t)((1ull << 32) / (uint32_t)page_tokens);
}

}  // namespace cp
