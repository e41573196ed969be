// Requests that keep some of their tokens (cp_request_keep, cp_kv_evict): launch records
// shared by the host (api.cpp) and the kernels (compact_kernels.hip).
#pragma once

#include <stdint.h>

#include "kargs.h"

namespace cp {

constexpr int kMaxMoveReq = 28;    // requests of one launch
constexpr int kMoveEntMax = 288;   // kept tokens that one launch of cp_request_keep carries
constexpr int kEvictMaxReq = 14;
constexpr int kEvictEntMax = 448;  // new page-table entries that one launch of the choice carries
constexpr int kSelectThreads = 1024;
constexpr int kKeepThreads = 256, kKeepCols = 16, kKeepUnroll = 4;     // cp_request_keep
constexpr int kMoveThreads = 1024, kMoveCols = 8, kMoveUnroll = 8;     // evictions in place
// ... where workgroups of kMoveCols columns are at most a quarter of the card's CUs: twice as
// many read every line twice, and pay only while CUs are idle. (Evictions of 16 K to 2 K
// tokens, 8 heads of 128, by requests, us with eight columns and with four: one, 32 workgroups,
// 33.4 and 30.9; two, 64, 35.5 and 34.4; three, 96, 42.3 and 43.6; four 49 and 49; six 51 and
// 62. In 4 layers of 4 heads of 64, 4 K tokens: 32 23.8 and 23.8; 96 26.3 and 26.3; 192 29.4
// and 32.5.)
constexpr int kMoveFewCols = 4;
constexpr int kApartThreads = 256, kApartUnroll = 4;                   // ... into pages of their own
// Rows of a workgroup of those (segs: 16-byte pieces of a row).
constexpr uint32_t apart_rows(uint32_t segs) {
  const uint32_t r = (uint32_t)(kApartThreads * kApartUnroll) / segs;
  return r < 1 ? 1 : r;
}

// Rows of one request, in every layer: row first + k becomes what row first + list[k] was,
// k0 <= k < n.
struct MoveReq {
  const uint32_t *src;  // page-table entries of the rows read, and from layer to layer
  const int32_t *list;  // NULL: MoveArgs::ent
  int64_t list_head, list_layer;
  uint32_t src_plane;
  uint32_t dst_base, dst_plane;  // entries of the pages written, in MoveArgs::pte
  uint32_t first, k0, n, rows;   // rows: tokens of the request before (list entries are less)
  uint32_t ent0;                 // list == NULL: its entries from k0 on
  uint32_t block_begin, per_layer;  // workgroups of one layer
  uint32_t model, pad;
};
struct MoveArgs {
  uint8_t *pool;
  const uint32_t *pte;
  int32_t n_req, n_blocks;
  uint32_t page_magic, pad;
  GeomK geom[kMaxLaunchModels];
  MoveReq req[kMaxMoveReq];
  uint32_t ent[kMoveEntMax];
};
static_assert(sizeof(MoveReq) == 80, "move record");

// One request of the choice: per layer and KV head the `keep` tokens of `n` that stay.
struct EvictReq {
  const float *old;
  float *sum;     // NULL: the sums stay as they are
  int32_t *list;  // out, [layer][head][keep] by these strides
  int64_t old_head, old_layer, sum_head, sum_layer, list_head, list_layer;
  uint32_t *tab;  // entries as they were, [layer][tab_n], of requests whose pages are replaced (NULL: none)
  uint32_t n, keep;
  uint32_t first, last;  // kept anyway
  uint32_t block_begin, layers, hkv, tab_n;
  uint32_t pte_base, plane;  // of the request in the page table
  uint32_t page0, pages;     // entries replaced: pages [page0, page0 + pages) of every layer
  uint32_t ent, pad;         // ... whose new ones are EvictArgs::ent[ent + layer * pages ...] (kNoWs: written later)
};
struct EvictArgs {
  uint32_t *pte;
  int32_t n_req, n_blocks;
  EvictReq req[kEvictMaxReq];
  uint32_t ent[kEvictEntMax];
};

// The choice's search for the k-th largest of a row's numbers (32 bits each, in the order
// of the weights): those that it may still be, and which of them it is from the largest on.
struct Search {
  uint32_t lo, hi, need;
};
constexpr int kBins = 2048;  // counters of a pass: number x is counted by (x - lo) >> search_shift
constexpr int search_shift(const Search &x) {
  const int bits = 32 - __builtin_clz(x.hi - x.lo);  // lo < hi
  return bits > 11 ? bits - 11 : 0;
}
// Behind a pass that found it in counter `bin`, which holds `in_bin`, as the left-th largest of
// those. Does another pass have to follow? Each leaves a 2^11-th of the range, so that three are
// the most whatever they count: none found it (in_bin 0) in a row that is written
// meanwhile, and the search ends with what it has.
constexpr bool search_narrow(Search *x, uint32_t bin, uint32_t left, uint32_t in_bin) {
  if (in_bin == 0) return false;
  const uint32_t rest = (1u << search_shift(*x)) - 1u, lo = x->lo + bin * (rest + 1);
  if (left == in_bin) {  // every number of the counter is among the k: all above lo - 1 are
    *x = Search{lo - 1, lo - 1, 0};
    return false;
  }
  *x = Search{lo, x->hi - lo < rest ? x->hi : lo + rest, left};
  return x->lo < x->hi;
}
static_assert(sizeof(MoveArgs) <= 3776 && sizeof(EvictArgs) <= 3776, "compaction kernel arguments too large");

}  // namespace cp
