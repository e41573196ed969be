// Device helpers of the kernels of attention of token chunks (extend_kernels.hip,
// extend_rows.hip, extend_mla.hip).
//
// A row is a query token t and one of the g query heads of a KV head: row r of
// a request is token r / g, head r % g. A work unit is a tile of consecutive rows
// of one KV head over one range of keys. Row r at position p sees keys [lo, hi):
//   hi = max(p + 1, prefix),  lo = max(p - window + 1, doc_begin, 0).
// In a tree row r stands at p = base + depth, base = context - n_q, and sees keys
// [min(lo, base), base) and those of the n_q behind that its mask names.
// One pass over the keys keeps, per row, the running maximum m and sum l of
// 2^(s - m) in fp32 (s: scores times log2 e) and the output sums; where a tile's
// keys are cut into ranges, ext_merge_kernel joins their results.
#pragma once

#include <hip/hip_runtime.h>

#include "decode_mfma.h"
#include "device_common.h"
#include "extend.h"

namespace cp {


typedef unsigned int u32x4e __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2e __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float kLog2e = 1.4426950408889634f;

// x / P and the remainder for any page size: the estimate by the magic factor
// floor(2^32 / P) is at most one too small.
CP_DEV uint32_t page_divide(uint32_t x, uint32_t P, uint32_t magic, uint32_t *rest) {
  uint32_t q = __umulhi(x, magic), r = x - q * P;
  if (r >= P) {
    q += 1;
    r -= P;
  }
  *rest = r;
  return q;
}

// Unit of a request's workgroup b of n: workgroups are dealt to the eight XCDs in
// turn, and consecutive units (which share KV) go to one XCD, whose L2 they then
// share. Request by request, so that the XCDs get equal parts of long and short
// ones: over the launch as a whole, three prompts of 16K, 9K and 4K tokens left
// the XCDs of the short one idle for half the time.
CP_DEV uint32_t xcd_unit(uint32_t b, uint32_t n) {
  const uint32_t per = n / 8, rem = n % 8, x = b % 8;
  return x * per + min(x, rem) + b / 8;
}

// tanh to 7e-7 of its value. Under kCapEdge a polynomial in x^2 fitted to tanh(x) / x
// (kTanh, 2e-7 with its roundings; 1 - 2 / (e^2x + 1) loses what the difference cancels,
// and scores far under the cap are the usual case), above it the quotient, which is
// worst just above the edge: there e^2x = 2.0 is off by 2e-7 of itself (argument 8e-8,
// exponential one last place, 1.2e-7), the quotient 0.66 by 3.1e-7 (2/3 of that, the
// sum 6e-8, the reciprocal one last place), which is 6.2e-7 of the difference 0.34.
CP_DEV float tanh_large(float x) {
  const float a = __builtin_fabsf(x);
  const float t = 1.f - 2.f * __builtin_amdgcn_rcpf(fast_exp2(a * (2.f * kLog2e)) + 1.f);
  return __builtin_copysignf(t, x);
}
CP_DEV float cap_tanh(float x) {
  const float y = x * x;
  float p = kTanh[kTanhTerms - 1];
#pragma unroll
  for (int k = kTanhTerms - 2; k > 0; --k) p = __builtin_fmaf(p, y, kTanh[k]);
  return __builtin_fabsf(x) < kCapEdge ? __builtin_fmaf(x * y, p, x) : tanh_large(x);  // NaN: the second, NaN too
}

// How a kernel's scores are formed (a kernel for each, for their registers
// and instructions): products times a factor (left to the exponent's fma);
// capped; capped or not, with slopes. The same with trees: products times a
// factor, and anything else.
enum : int { kModePlain = 0, kModeCap, kModeAny, kModeTree, kModeTreeAny };
constexpr bool is_tree(int mode) { return mode >= kModeTree; }
constexpr bool is_plain(int mode) { return mode == kModePlain || mode == kModeTree; }
constexpr bool is_any(int mode) { return mode == kModeAny || mode == kModeTreeAny; }

struct Unit {
  const ExtReq *rq;
  uint32_t kvh, tile, split;
  bool none;  // one of the workgroups up to the next multiple of 8
};
CP_DEV Unit find_unit(const ExtArgs &a) {
  const int r = sorted_search(a.n_req, blockIdx.x, [&](int i) { return a.req[i].unit_begin; });
  const ExtReq &rq = a.req[r];
  const uint32_t per_head = rq.tiles * rq.splits, n = per_head * (uint32_t)a.g.hkv, b = blockIdx.x - rq.unit_begin;
  const uint32_t w = xcd_unit(b, n), kvh = w / per_head, u = w - kvh * per_head;
  // later tiles see more keys: they start first
  return Unit{&rq, kvh, rq.tiles - 1 - u / rq.splits, u % rq.splits, b >= n};
}

// What a row sees, and where its results go.
struct Row {
  uint32_t pos, lo, hi;  // lo == hi: nothing
  uint32_t head;         // of all query heads
  uint64_t tok;          // query token of the call
  uint32_t base;         // every key before it is behind the row: its own place + 1, or its tree's first
  uint32_t n_q, tok0;    // trees: their tokens, and the first of those in the call
};
template <bool TREE>
CP_DEV Row row_of(const ExtArgs &a, const ExtReq &rq, uint32_t kvh, uint32_t r) {
  const uint32_t g = (uint32_t)a.g.g, rows = rq.n_tok * g, rc = min(r, rows - 1);
  uint32_t t = rc / g, ctx = rq.ctx, n_q = rq.n_q, prefix = rq.prefix;
  Row x;
  x.tok = (uint64_t)rq.tok0 + t;
  x.head = kvh * g + (rc - t * g);
  for (uint32_t k = 0; k < rq.members; ++k) {  // the member whose token it is
    const ExtMember &m = a.member[rq.member0 + k];
    ctx = m.ctx;
    n_q = m.n_q;
    prefix = m.prefix;
    if (t < n_q) break;
    t -= n_q;
  }
  x.pos = ctx - n_q + t;
  x.base = x.pos + 1;
  if constexpr (TREE) {
    x.base = ctx - n_q;
    x.n_q = n_q;
    x.tok0 = (uint32_t)x.tok - t;
    x.pos = x.base + min((uint32_t)a.tree_depth[x.tok], n_q - 1);
    x.hi = min(ctx, rq.key_hi);
  } else {
    x.hi = min(max(x.pos + 1, min(prefix, ctx)), rq.key_hi);
  }
  x.lo = a.window && x.pos >= a.window ? x.pos - a.window + 1 : 0u;
  if (a.doc_begin) {
    const int32_t d = a.doc_begin[x.tok];
    if (d > 0) x.lo = max(x.lo, (uint32_t)d);
  }
  if (TREE) x.lo = min(x.lo, x.base);
  x.lo = max(x.lo, rq.key_lo);
  if (x.lo >= x.hi) x.lo = x.hi = 0;
  return x;  // rows past the last repeat it (their results are not stored)
}

// A row of a tree, formed afresh in the few steps that ask: what is kept of it through the
// loop costs registers that the kernels have not.
CP_DEV Row tree_row(const ExtArgs &a, const ExtReq &rq, uint32_t kvh, uint32_t r) {
  asm volatile("" : "+v"(r));
  return row_of<true>(a, rq, kvh, r);
}
struct RowAt {  // what tree_row takes
  const ExtReq *rq;
  uint32_t kvh, r;
};
// Which of the N <= 64 keys from k0 on it sees. Only steps that reach into the tree ask, so
// that a tree costs what a chunk of as many tokens costs (eight of 61 tokens behind 1 to 16 K,
// 32 heads over 8: 54 us, 0.6 PFLOP/s, bound as there).
template <int N>
CP_DEV uint64_t tree_bits(const ExtArgs &a, const Row &x, uint32_t k0) {
  uint64_t b = ~0ull;
  if (k0 + N > x.base) {
    const uint32_t *const m = a.tree_mask + x.tok * (uint32_t)a.tree_words;
    const uint32_t before = k0 < x.base ? x.base - k0 : 0u, first = k0 < x.base ? 0u : k0 - x.base;  // before < N
    const uint32_t w = first / 32, sh = first % 32, n = (uint32_t)a.tree_words;
    const uint32_t w0 = w < n ? m[w] : 0u, w1 = w + 1 < n ? m[w + 1] : 0u, w2 = w + 2 < n ? m[w + 2] : 0u;
    b = (uint64_t)w0 | (uint64_t)w1 << 32;
    if (sh) b = b >> sh | (uint64_t)w2 << (64 - sh);
    if (before) b = b << before | ((1ull << before) - 1);
  }
  const uint32_t lo = x.lo > k0 ? min(x.lo - k0, 64u) : 0u, hi = x.hi > k0 ? min(x.hi - k0, 64u) : 0u;
  if (hi < 64) b &= (1ull << hi) - 1;
  return lo < 64 ? b >> lo << lo : 0;
}
// Where key j stands.
CP_DEV uint32_t tree_pos(const ExtArgs &a, const Row &x, uint32_t j) {
  if (j < x.base) return j;
  const uint32_t i = min(j - x.base, x.n_q - 1);  // (keys past the context are hidden)
  return x.base + min((uint32_t)a.tree_depth[x.tok0 + i], x.n_q - 1);
}

// Stores of a row's result: NORMAL to the call's arrays, or a range's part.
CP_DEV uint64_t part_row(const ExtArgs &a, const ExtReq &rq, const Row &x, uint32_t split) {
  return (rq.ws_row + (x.tok - rq.tok0) * (uint32_t)a.g.hq + x.head) * rq.all + rq.split0 + split;
}

// product * sum_k cap_k product^2k: the capped score, in units of log2 e, of a
// product under cap_edge. less: subtracted in the last step.
template <class A>
CP_DEV float small_cap(const A &a, float s, float less) {
  const float y = s * s;
  float p = a.cap_k[kTanhTerms - 1];
#pragma unroll
  for (int k = kTanhTerms - 2; k >= 0; --k) p = __builtin_fmaf(p, y, a.cap_k[k]);
  return __builtin_fmaf(s, p, -less);
}
template <int N, class A>
CP_DEV bool all_small(const A &a, const float (&s)[N]) {
  float big = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) big = __builtin_fmaxf(big, __builtin_fabsf(s[i]));
  return __builtin_amdgcn_ballot_w64(big >= a.cap_edge) == 0;  // (a NaN is not: the polynomial keeps it too)
}

// Scores of N keys of one row, from products to units of log2 e. Element i is
// key k0 + at(i); behind: no key is past the position of any row of the wave, or in its tree.
template <int MODE, int N, class A, class F>
CP_DEV void shape_scores(const A &a, const RowAt &row, float (&s)[N], float slope, const Row &x, uint32_t k0,
                         bool behind, F at) {
  const uint32_t pos = x.pos;
  if (MODE == kModeCap || a.softcap > 0.f) {
    if (all_small(a, s)) {
#pragma unroll
      for (int i = 0; i < N; ++i) s[i] = small_cap(a, s[i], 0.f);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) s[i] = cap_tanh(s[i] * a.score_mul) * a.cap_mul;
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] *= a.score_mul;
  }
  if constexpr (is_any(MODE)) {
    if (behind) {  // slope * (pos - key) in two steps
      const float far = (float)(pos - k0);
#pragma unroll
      for (int i = 0; i < N; ++i) s[i] = __builtin_fmaf(-slope, far - (float)at(i), s[i]);
    } else {
      Row t{};
      if constexpr (is_tree(MODE)) t = tree_row(a, *row.rq, row.kvh, row.r);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (is_tree(MODE)) __builtin_amdgcn_sched_barrier(0);  // one load at once, for the registers
        uint32_t key = k0 + at(i);
        if constexpr (is_tree(MODE)) key = tree_pos(a, t, key);
        s[i] = __builtin_fmaf(-slope, (float)(max(key, pos) - min(key, pos)), s[i]);
      }
    }
  }
}

// Scores of N keys of one row, with those out of sight made -inf, and their
// maximum in units of log2 e. hide: some row of the wave does not see some of
// the keys; bits: of a tree, the row's tree_bits from k0 on. Where it can, it
// leaves the products as they are (returns true), for weight() to scale or cap
// and take the reference off in one go.
template <int MODE, int N, class A, class B, class F>
CP_DEV bool scores_of(const A &a, const RowAt &row, float (&s)[N], float slope, const Row &x, uint32_t k0,
                      bool behind, bool hide, B bits, F at, float *top) {
  bool raw = is_plain(MODE) || (MODE == kModeCap && !hide && all_small(a, s));
  if (!raw) shape_scores<MODE, N>(a, row, s, slope, x, k0, behind, at);
  if (hide) {
    const uint32_t lo = x.lo - k0, n = x.hi - x.lo;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (is_tree(MODE) ? !(bits >> at(i) & 1) : (uint32_t)at(i) - lo >= n) s[i] = -INFINITY;
  }
  float t = s[0];
#pragma unroll
  for (int i = 1; i < N; ++i) t = __builtin_fmaxf(t, s[i]);
  if (is_plain(MODE)) t *= a.score_mul;
  if (MODE == kModeCap && raw) t = small_cap(a, t, 0.f);
  *top = t;
  return raw;
}

// 2^(score - ref) of N elements in order: each(i, weight of i, weight of i + 1)
template <int MODE, int N, class A, class E>
CP_DEV void weights(const A &a, const float (&s)[N], bool raw, float ref, E each) {
  if (is_plain(MODE)) {
#pragma unroll
    for (int i = 0; i < N; i += 2)
      each(i, fast_exp2(__builtin_fmaf(s[i], a.score_mul, -ref)), fast_exp2(__builtin_fmaf(s[i + 1], a.score_mul, -ref)));
  } else if (MODE == kModeCap && raw) {
#pragma unroll
    for (int i = 0; i < N; i += 2) each(i, fast_exp2(small_cap(a, s[i], ref)), fast_exp2(small_cap(a, s[i + 1], ref)));
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 2) each(i, fast_exp2(s[i] - ref), fast_exp2(s[i + 1] - ref));
  }
}

// Of some rows: the first key that any sees and the last plus one, the keys that
// every one sees (a row that sees none: none), and the first key that is not behind
// every one.
struct Sight {
  uint32_t lo, hi, all_lo, all_hi, behind;
};
// Of a wave whose lanes with equal low bits (2 TOP values) hold one row.
template <int TOP, bool TREE>
CP_DEV Sight wave_sight(const Row &x) {
  const bool some = x.lo < x.hi;
  Sight s{some ? x.lo : 0xFFFFFFFFu, x.hi, x.lo, TREE ? min(x.hi, x.base) : x.hi, x.base};
#pragma unroll
  for (int o = TOP; o > 0; o >>= 1) {
    s.lo = min(s.lo, (uint32_t)__shfl_xor((int)s.lo, o, 64));
    s.hi = max(s.hi, (uint32_t)__shfl_xor((int)s.hi, o, 64));
    s.all_lo = max(s.all_lo, (uint32_t)__shfl_xor((int)s.all_lo, o, 64));
    s.all_hi = min(s.all_hi, (uint32_t)__shfl_xor((int)s.all_hi, o, 64));
    s.behind = min(s.behind, (uint32_t)__shfl_xor((int)s.behind, o, 64));
  }
  s.lo = __builtin_amdgcn_readfirstlane(min(s.lo, s.hi));
  s.hi = __builtin_amdgcn_readfirstlane(s.hi);
  s.all_lo = __builtin_amdgcn_readfirstlane(s.all_lo);
  s.all_hi = __builtin_amdgcn_readfirstlane(s.all_hi);
  s.behind = __builtin_amdgcn_readfirstlane(s.behind);
  return s;
}
// Of a workgroup's waves (barriers inside).
template <int WAVES>
CP_DEV Sight group_sight(const Sight &own, int wave, int lane, uint32_t (*shared)[4]) {
  if (lane == 0) {
    // a wave that sees nothing has no first key
    shared[wave][0] = own.lo < own.hi ? own.lo : 0xFFFFFFFFu;
    shared[wave][1] = own.hi;
    shared[wave][2] = own.all_lo;
    shared[wave][3] = own.all_hi;
  }
  __syncthreads();
  Sight s = own;
  s.lo = 0xFFFFFFFFu;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    s.lo = min(s.lo, shared[w][0]);
    s.hi = max(s.hi, shared[w][1]);
    s.all_lo = max(s.all_lo, shared[w][2]);
    s.all_hi = min(s.all_hi, shared[w][3]);
  }
  s.lo = __builtin_amdgcn_readfirstlane(min(s.lo, s.hi));
  s.hi = __builtin_amdgcn_readfirstlane(s.hi);
  s.all_lo = __builtin_amdgcn_readfirstlane(s.all_lo);
  s.all_hi = __builtin_amdgcn_readfirstlane(s.all_hi);
  __syncthreads();
  return s;
}

// Direct loads from the pool to LDS (completion is awaited with wait_vm).
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
// 16 bytes a lane from base + offset to LDS at lds_base + 16 lane; with the
// non-temporal policy where KV is read once.
template <bool NT>
CP_DEV void row_load_lds(uint64_t base, uint32_t offset, uint32_t lds_base) {
  lds_base = __builtin_amdgcn_readfirstlane(lds_base);
  if constexpr (NT)
    asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dwordx4 %0, %2 nt" ::"v"(offset), "s"(lds_base), "s"(base)
                 : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dwordx4 %0, %2" ::"v"(offset), "s"(lds_base), "s"(base)
                 : "memory", "m0");
}
// The same, every lane with an address of its own.
template <bool NT>
CP_DEV void lane_load_lds(uint64_t addr, uint32_t lds_base) {
  lds_base = __builtin_amdgcn_readfirstlane(lds_base);
  if constexpr (NT)
    asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dwordx4 %0, off nt" ::"v"(addr), "s"(lds_base) : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(addr), "s"(lds_base) : "memory", "m0");
}
// Four bytes a lane, every lane with an address of its own, to LDS at lds_base + 4 lane.
CP_DEV void dword_load_lds(uint64_t addr, uint32_t lds_base) {
  lds_base = __builtin_amdgcn_readfirstlane(lds_base);
  asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dword %0, off" ::"v"(addr), "s"(lds_base) : "memory", "m0");
}
#pragma clang diagnostic pop

CP_DEV float other_half(float x) {
  auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float((threadIdx.x & 32) ? p[0] : p[1]);
}

// Does any of eight bf16 numbers have the exponent of infinities and NaN?
CP_DEV bool any_special(u32x4e w) {
  bool x = false;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    x = x || (w[i] & 0x7F80u) == 0x7F80u || (w[i] & 0x7F800000u) == 0x7F800000u;
  return x;
}
// Eight bf16 numbers with those made 0.
CP_DEV u32x4e without_special(u32x4e w) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if ((w[i] & 0x7F80u) == 0x7F80u) w[i] &= 0xFFFF0000u;
    if ((w[i] & 0x7F800000u) == 0x7F800000u) w[i] &= 0xFFFFu;
  }
  return w;
}
// 1.0 where a number is infinite with this sign (1: negative) or NaN, else 0.
CP_DEV bf16x8 special_ones(bf16x8 v, uint32_t sign) {
  u32x4e w = __builtin_bit_cast(u32x4e, v);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t r = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t x = (w[i] >> (16 * h)) & 0xFFFFu;
      const bool nan = (x & 0x7FFFu) > 0x7F80u, inf = (x & 0x7FFFu) == 0x7F80u;
      if (nan || (inf && (x >> 15) == sign)) r |= 0x3F80u << (16 * h);
    }
    w[i] = r;
  }
  return __builtin_bit_cast(bf16x8, w);
}

}  // namespace cp
