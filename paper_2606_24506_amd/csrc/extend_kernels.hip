// gfx950 kernels of attention of token chunks over the pool (cp_attn_extend).
//
// A row is a query token t and one of the g query heads of a KV head: row r of
// a request is token r / g, head r % g. A work unit is a tile of consecutive rows
// of one KV head over one range of keys. Row r at position p sees keys [lo, hi):
//   hi = max(p + 1, prefix),  lo = max(p - window + 1, doc_begin, 0).
// One pass over the keys keeps, per row, the running maximum m and sum l of
// 2^(s - m) in fp32 (s: scores times log2 e) and the output sums; where a tile's
// keys are cut into ranges, ext_merge_kernel joins their results.
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

// The unit of a workgroup: consecutive units (which share KV) go to one XCD, whose
// L2 they then share; workgroups are dealt to the eight XCDs in turn.
CP_DEV uint32_t xcd_unit(uint32_t b, uint32_t n) {
  const uint32_t per = n / 8, rem = n % 8, x = b % 8;
  return x * per + min(x, rem) + b / 8;
}

// tanh to 1.2e-7 of its value: below 0.6 a polynomial (1 - 2 / (e^2x + 1) loses what
// the difference cancels; scores far under the cap are the usual case), fitted
// to tanh(x) / x in x^2.
CP_DEV float tanh_small(float x) {
  const float y = x * x;
  float p = -5.875653302e-03f;
  p = __builtin_fmaf(p, y, 2.078145661e-02f);
  p = __builtin_fmaf(p, y, -5.378023840e-02f);
  p = __builtin_fmaf(p, y, 1.333189099e-01f);
  p = __builtin_fmaf(p, y, -3.333329714e-01f);
  return __builtin_fmaf(x * y, p, x);
}
CP_DEV float tanh_large(float x) {
  const float a = __builtin_fabsf(x);
  const float t = 1.f - 2.f * __builtin_amdgcn_rcpf(fast_exp2(a * (2.f * kLog2e)) + 1.f);
  return __builtin_copysignf(t, x);
}
CP_DEV float cap_tanh(float x) {
  const float s = tanh_small(x), l = tanh_large(x);
  return __builtin_fabsf(x) < 0.6f ? s : l;  // NaN: the second, NaN too
}

struct Unit {
  const ExtReq *rq;
  uint32_t kvh, tile, split;
};
CP_DEV Unit find_unit(const ExtArgs &a) {
  const uint32_t v = xcd_unit(blockIdx.x, (uint32_t)a.n_units);
  const int r = sorted_search(a.n_req, v, [&](int i) { return a.req[i].unit_begin; });
  const ExtReq &rq = a.req[r];
  const uint32_t w = v - rq.unit_begin, per_head = rq.tiles * rq.splits;
  const uint32_t kvh = w / per_head, u = w - kvh * per_head;
  // later tiles see more keys: they start first
  return Unit{&rq, kvh, rq.tiles - 1 - u / rq.splits, u % rq.splits};
}

// What a row sees, and where its results go.
struct Row {
  uint32_t pos, lo, hi;  // lo == hi: nothing
  uint32_t head;         // of all query heads
  uint64_t tok;          // query token of the call
};
CP_DEV Row row_of(const ExtArgs &a, const ExtReq &rq, uint32_t kvh, uint32_t r) {
  const uint32_t g = (uint32_t)a.g.g, rows = rq.n_q * g, rc = min(r, rows - 1);
  const uint32_t t = rc / g;
  Row x;
  x.tok = (uint64_t)rq.tok0 + t;
  x.head = kvh * g + (rc - t * g);
  x.pos = rq.ctx - rq.n_q + t;
  x.hi = max(x.pos + 1, min(rq.prefix, rq.ctx));
  x.lo = a.window && x.pos >= a.window ? x.pos - a.window + 1 : 0u;
  if (a.doc_begin) {
    const int32_t d = a.doc_begin[x.tok];
    if (d > 0) x.lo = max(x.lo, (uint32_t)d);
  }
  if (x.lo >= x.hi) x.lo = x.hi = 0;
  return x;  // rows past the last repeat it (their results are not stored)
}

// Stores of a row's result: NORMAL to the call's arrays, or a range's part.
CP_DEV uint64_t part_row(const ExtArgs &a, const ExtReq &rq, const Row &x, uint32_t split) {
  return (rq.ws_row + (x.tok - rq.tok0) * (uint32_t)a.g.hq + x.head) * rq.splits + split;
}

// ------------------------------------------------------------ vector path

// One wave per row, for every geometry: a lane per key for the scores (its K row
// read in 16-byte pieces), then lanes across the columns for the sums, key after
// key, keys out of sight skipped. Bound by the vector unit and the per-lane row
// reads; it serves the geometries without a matrix kernel.
template <int E>  // V columns per lane
__global__ __launch_bounds__(kExtThreads) void extend_vec_kernel(const ExtArgs a) {
  extern __shared__ float qs[];  // [4][d_k]
  const Unit un = find_unit(a);
  const ExtReq &rq = *un.rq;
  const GeomK &g = a.g;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t r = un.tile * 4 + wave;
  if (r >= rq.n_q * (uint32_t)g.g) return;  // no barrier below: waves are on their own
  const Row x = row_of(a, rq, un.kvh, r);
  const uint32_t dk = (uint32_t)g.d_k, P = (uint32_t)g.page_tokens;
  float *const qw = qs + wave * dk;
  const uint16_t *const qrow = a.q + (x.tok * (uint32_t)g.hq + x.head) * dk;
  for (uint32_t i = lane; i < dk; i += 64) qw[i] = bf16_to_f32(qrow[i]);
  const float slope = a.slopes ? a.slopes[x.head] * kLog2e : 0.f;
  const float s1 = a.softcap > 0.f ? a.scale / a.softcap : a.scale * kLog2e, s2 = a.softcap * kLog2e;
  // bytes from the page to K and V of slot 0, and from slot to slot
  const uint64_t kof = g.kind == 0 ? 0 : (uint64_t)un.kvh * 4 * P * dk, vof = g.kind == 0 ? 0 : kof + 2ull * P * dk;
  const uint32_t n = x.hi - x.lo;
  const uint32_t b = x.lo + (uint32_t)((uint64_t)n * un.split / rq.splits),
                 e = x.lo + (uint32_t)((uint64_t)n * (un.split + 1) / rq.splits);
  float m = -INFINITY, l = 0.f, o[E];
#pragma unroll
  for (int i = 0; i < E; ++i) o[i] = 0.f;
  for (uint32_t k0 = b; k0 < e; k0 += 64) {
    const uint32_t key = k0 + lane;
    const bool see = key < e;
    float s = -INFINITY;
    uint64_t row = 0;
    if (see) {
      uint32_t slot;
      const uint32_t pg = page_divide(key, P, a.page_magic, &slot);
      const uint64_t page = (uint64_t)a.pte[rq.pte_base + pg] << 8;
      row = page + (uint64_t)slot * dk * 2;
      const u32x4e *const kp = reinterpret_cast<const u32x4e *>(a.pool + row + kof);
      float acc = 0.f;
      for (uint32_t c = 0; c < dk / 8; ++c) {
        const u32x4e w = kp[c];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          acc = __builtin_fmaf(__uint_as_float(w[i] << 16), qw[8 * c + 2 * i], acc);
          acc = __builtin_fmaf(__uint_as_float(w[i] & 0xFFFF0000u), qw[8 * c + 2 * i + 1], acc);
        }
      }
      s = acc * s1;
      if (a.softcap > 0.f) s = cap_tanh(s) * s2;
      if (a.slopes) s -= slope * (float)(max(x.pos, key) - min(x.pos, key));
    }
    const float mn = fmaxf(m, wave_max(s)), base = mn == -INFINITY ? 0.f : mn;
    const float al = fast_exp2(m - base);
    const float p = see ? fast_exp2(s - base) : 0.f;
    m = mn;
    l = l * al + wave_sum(p);
#pragma unroll
    for (int i = 0; i < E; ++i) o[i] *= al;
    const uint32_t cnt = min(64u, e - k0);
    for (uint32_t j = 0; j < cnt; ++j) {
      const float pj = __shfl(p, (int)j, 64);
      const uint64_t rj = (uint64_t)(uint32_t)__shfl((int)(uint32_t)row, (int)j, 64) |
                          (uint64_t)(uint32_t)__shfl((int)(uint32_t)(row >> 32), (int)j, 64) << 32;
      const uint16_t *const v = reinterpret_cast<const uint16_t *>(a.pool + rj + vof) + lane * E;
#pragma unroll
      for (int i = 0; i < E; ++i) o[i] = __builtin_fmaf(pj, bf16_to_f32(v[i]), o[i]);
    }
  }
  const bool none = l == 0.f;  // (all scores NaN: l is NaN, and so are the results)
  const float inv = none ? 0.f : 1.f / l;
  const float lse = none ? -INFINITY : m + fast_log2(l);
  if (rq.splits > 1) {
    const uint64_t pr = part_row(a, rq, x, un.split);
#pragma unroll
    for (int i = 0; i < E; ++i) a.ws_o[pr * (uint32_t)g.d_v + lane * E + i] = none ? 0.f : o[i] * inv;
    if (lane == 0) a.ws_l[pr] = lse;
  } else {
    const uint64_t orow = x.tok * (uint32_t)g.hq + x.head;
#pragma unroll
    for (int i = 0; i < E; ++i)
      a.out[orow * (uint32_t)g.d_v + lane * E + i] = (uint16_t)f32_to_bf16(none ? 0.f : o[i] * inv);
    if (lane == 0) a.lse[orow] = lse * kLn2;
  }
}

// --------------------------------------------- matrix path, head_dim 64 / 128

// Scores are computed transposed, S^T = K Q^T by 32x32x16 products: a lane
// then holds scores of one row (its column, lane % 32), 16 of every 32 keys, and
// the other half of the wave the other 16. So the softmax runs inside lanes, and the
// same registers, rounded, are the operand P^T of O^T = V^T P^T, the products'
// contraction taking keys in the order that the first left them in:
// of 16 keys, half h of the wave has keys 4 h + {0..3} and 8 + 4 h + {0..3}. V^T
// comes from LDS by transposing reads.
//
// LDS rows are not padded but their 16-byte pieces swapped by the row number:
// K reads touch 16 rows at one piece (all 16 pieces of a 256-byte line), V
// reads four rows at four pieces.
//
// RW = 4: 128 rows, a wave for every 32, all over the same 64 keys a step; the
// next step's keys travel through registers while this one's are worked on.
// RW = 1: 32 rows, every wave with 32 keys of its own a step (few rows: bound
// by reading KV); the waves' sums join at the end.
template <int D, int RW>
struct ExtCfg {
  static constexpr int KW = RW == 4 ? 64 : 32;          // keys of a wave's step
  static constexpr int KEYS = RW == 4 ? 64 : 128;       // keys of a workgroup's step
  static constexpr int ROW = 2 * D;                     // bytes
  static constexpr int CPR = D / 8;                     // 16-byte pieces of a row
  static constexpr int TILE = KW * ROW;                 // bytes of K (or V) of a step of a wave's keys
  static constexpr int BUFS = RW == 4 ? 2 : 4;          // double buffer, or one for each wave
  static constexpr int LOADERS = RW == 4 ? 256 : 64;    // threads that fill one
  static constexpr int RPI = LOADERS / CPR;             // rows that they fill at once
  static constexpr int NL = KW / RPI;                   // 16-byte loads of K (and of V) of a thread
  static constexpr int KB = KW / 32;                    // blocks of 32 keys
  static constexpr int NP = RW == 4 ? 1 : 2;            // bf16 parts of a probability
  static constexpr int LDS = 2 * TILE * BUFS;
  static_assert(RW == 4 || LDS >= 4 * 32 * D * 4, "the join reuses the tiles");
};

// Swapped piece numbers: 16 rows at one piece (K), 4 rows at 4 neighbouring pieces (V).
template <int D>
CP_DEV int k_piece(int row, int c) {
  return D == 128 ? c ^ (row & 15) : c ^ ((row >> 1) & 7);
}
template <int D>
CP_DEV int v_piece(int row, int c) {
  return D == 128 ? c ^ (4 * (row & 3)) : c ^ (4 * ((row >> 1) & 1));
}

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

// Of eight bf16 numbers: 1.0 where the number is infinite with this sign or
// NaN, else 0 (SIGN 0 or 1); and the numbers with those made 0.
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
CP_DEV bf16x8 without_special(bf16x8 v) {
  u32x4e w = __builtin_bit_cast(u32x4e, v);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if ((w[i] & 0x7F80u) == 0x7F80u) w[i] &= 0xFFFF0000u;
    if ((w[i] & 0x7F800000u) == 0x7F800000u) w[i] &= 0xFFFFu;
  }
  return __builtin_bit_cast(bf16x8, w);
}

template <int D, int RW>
__global__ __launch_bounds__(kExtThreads, 2) void extend_kernel(const ExtArgs a) {
  using C = ExtCfg<D, RW>;
  constexpr int KS = D / 16, DB = D / 32;
  __shared__ __attribute__((aligned(16))) char lds[C::LDS];
  __shared__ uint32_t bounds[4][4];  // per wave: lowest lo, highest hi, highest lo, lowest hi of its rows
  __shared__ uint32_t special[2][4];  // RW 4: per buffer and wave, V held an infinity or NaN
  __shared__ float stats[2][4][32];   // RW 1: the waves' m and l
  const Unit un = find_unit(a);
  const ExtReq &rq = *un.rq;
  const GeomK &g = a.g;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5, c16 = lane & 15, grp = (lane >> 4) & 1;
  const uint32_t P = (uint32_t)g.page_tokens;

  // ---- this lane's row and what the tile sees
  const uint32_t r = un.tile * (32 * RW) + (RW == 4 ? 32 * wave : 0) + col;
  const Row x = row_of(a, rq, un.kvh, r);
  const bool some = x.lo < x.hi;
  uint32_t mn_lo = some ? x.lo : 0xFFFFFFFFu, mx_hi = x.hi, mx_lo = x.lo, mn_hi = some ? x.hi : 0u;
  // a row that sees nothing keeps tiles from counting as seen in full
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    mn_lo = min(mn_lo, (uint32_t)__shfl_xor((int)mn_lo, o, 64));
    mx_hi = max(mx_hi, (uint32_t)__shfl_xor((int)mx_hi, o, 64));
    mx_lo = max(mx_lo, (uint32_t)__shfl_xor((int)mx_lo, o, 64));
    mn_hi = min(mn_hi, (uint32_t)__shfl_xor((int)mn_hi, o, 64));
  }
  mn_lo = __builtin_amdgcn_readfirstlane(mn_lo);
  mx_hi = __builtin_amdgcn_readfirstlane(mx_hi);
  mx_lo = __builtin_amdgcn_readfirstlane(mx_lo);
  mn_hi = __builtin_amdgcn_readfirstlane(mn_hi);
  uint32_t key_lo = mn_lo, key_hi = mx_hi, all_lo = mx_lo, all_hi = mn_hi;  // of the workgroup
  if (RW == 4) {
    if (lane == 0) {
      bounds[wave][0] = mn_lo;
      bounds[wave][1] = mx_hi;
      bounds[wave][2] = mx_lo;
      bounds[wave][3] = mn_hi;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      key_lo = min(key_lo, bounds[w][0]);
      key_hi = max(key_hi, bounds[w][1]);
      all_lo = max(all_lo, bounds[w][2]);
      all_hi = min(all_hi, bounds[w][3]);
    }
    key_lo = __builtin_amdgcn_readfirstlane(key_lo);
    key_hi = __builtin_amdgcn_readfirstlane(key_hi);
    all_lo = __builtin_amdgcn_readfirstlane(all_lo);
    all_hi = __builtin_amdgcn_readfirstlane(all_hi);
  }
  if (key_lo > key_hi) key_lo = key_hi;  // nothing at all
  // steps of the unit: whole steps from a multiple of KEYS on
  const uint32_t first = key_lo / C::KEYS, last = (key_hi + C::KEYS - 1) / C::KEYS, steps = last - first;
  const uint32_t s0 = first + (uint32_t)((uint64_t)steps * un.split / rq.splits),
                 s1 = first + (uint32_t)((uint64_t)steps * (un.split + 1) / rq.splits);

  // ---- Q^T: lane holds row `col`, dims 16 ks + 8 half .. + 7
  bf16x8 qf[KS];
  {
    const uint16_t *const qrow = a.q + (x.tok * (uint32_t)g.hq + x.head) * D + 8 * half;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const bf16x8 *>(qrow + 16 * ks);
  }
  const bool cap = a.softcap > 0.f;
  const float sc1 = cap ? a.scale / a.softcap : a.scale * kLog2e, sc2 = a.softcap * kLog2e;
  const float slope = a.slopes ? a.slopes[x.head] * kLog2e : 0.f;

  float m = -INFINITY, l = 0.f;
  f32x16 o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.f;

  // ---- loads: thread takes piece lc of rows lr, lr + RPI, ...
  const int lt = RW == 4 ? (int)threadIdx.x : lane, lc = lt % C::CPR, lr = lt / C::CPR;
  const uint8_t *const head_base = a.pool + (uint64_t)un.kvh * (4ull * P * D) + 16 * lc;
  u32x4e kreg[C::NL], vreg[C::NL];
  // keys of step s: RW 4, [64 s, + 64); RW 1, wave w has [128 s + 32 w, + 32)
  auto base_of = [&](uint32_t s) { return s * C::KEYS + (RW == 4 ? 0u : 32u * wave); };
  uint32_t pte[C::NL], slot[C::NL];
  auto load_ptes = [&](uint32_t s) {
#pragma unroll
    for (int i = 0; i < C::NL; ++i) {
      const uint32_t key = base_of(s) + lr + C::RPI * i;
      const uint32_t pg = page_divide(key, P, a.page_magic, &slot[i]);
      pte[i] = key >= key_lo && key < key_hi ? a.pte[rq.pte_base + pg] : 0u;
    }
  };
  auto load_keys = [&](uint32_t s) {
#pragma unroll
    for (int i = 0; i < C::NL; ++i) {
      const uint32_t key = base_of(s) + lr + C::RPI * i;
      kreg[i] = vreg[i] = u32x4e{0u, 0u, 0u, 0u};
      if (key >= key_lo && key < key_hi) {
        const uint8_t *const kp = head_base + ((uint64_t)pte[i] << 8) + slot[i] * C::ROW;
        kreg[i] = *reinterpret_cast<const u32x4e *>(kp);
        vreg[i] = *reinterpret_cast<const u32x4e *>(kp + (uint64_t)P * C::ROW);
      }
    }
  };
  // Are there keys of step s that some row of the workgroup does not see?
  auto mixed = [&](uint32_t s) {
    const uint32_t b = base_of(s);
    return b < all_lo || b + C::KW > all_hi;
  };
  uint32_t own_special = 0;  // RW 1
  auto store_keys = [&](int buf, uint32_t s) {
    char *const kt = lds + buf * (2 * C::TILE), *const vt = kt + C::TILE;
#pragma unroll
    for (int i = 0; i < C::NL; ++i) {
      const int row = lr + C::RPI * i;
      *reinterpret_cast<u32x4e *>(kt + row * C::ROW + 16 * k_piece<D>(row, lc)) = kreg[i];
      *reinterpret_cast<u32x4e *>(vt + row * C::ROW + 16 * v_piece<D>(row, lc)) = vreg[i];
    }
    uint32_t sp = 0;
    if (mixed(s)) {
      bool any = false;
#pragma unroll
      for (int i = 0; i < C::NL; ++i) any = any || any_special(vreg[i]);
      sp = __builtin_amdgcn_ballot_w64(any) != 0;
    }
    if (RW == 4) {
      if (lane == 0) special[buf][wave] = sp;
    } else {
      own_special = sp;
    }
  };

  // ---- one step over the keys in a buffer
  auto compute = [&](int buf, uint32_t s) {
    const uint32_t b0 = base_of(s);
    if (b0 >= mx_hi || b0 + C::KW <= mn_lo) return;  // out of this wave's sight
    const char *const kt = lds + buf * (2 * C::TILE), *const vt = kt + C::TILE;
    f32x16 sc[C::KB];
#pragma unroll
    for (int kb = 0; kb < C::KB; ++kb) {
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[kb][i] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const int row = 32 * kb + col;
        const bf16x8 kf = *reinterpret_cast<const bf16x8 *>(kt + row * C::ROW + 16 * k_piece<D>(row, 2 * ks + half));
        sc[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[ks], sc[kb], 0, 0, 0);
      }
    }
    // scores: key 32 kb + 8 (i / 4) + 4 half + i % 4 of the step
    auto key_at = [&](int kb, int i) { return b0 + 32 * kb + 8 * (i / 4) + 4 * half + i % 4; };
    if (cap) {
      float big = 0.f;
#pragma unroll
      for (int kb = 0; kb < C::KB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          sc[kb][i] *= sc1;
          big = __builtin_fmaxf(big, __builtin_fabsf(sc[kb][i]));
        }
      // (a NaN does not raise `big`: the polynomial keeps it as well)
      if (__builtin_amdgcn_ballot_w64(big >= 0.6f)) {
#pragma unroll
        for (int kb = 0; kb < C::KB; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) sc[kb][i] = cap_tanh(sc[kb][i]) * sc2;
      } else {
#pragma unroll
        for (int kb = 0; kb < C::KB; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) sc[kb][i] = tanh_small(sc[kb][i]) * sc2;
      }
    } else {
#pragma unroll
      for (int kb = 0; kb < C::KB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[kb][i] *= sc1;
    }
    if (a.slopes) {
#pragma unroll
      for (int kb = 0; kb < C::KB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const uint32_t key = key_at(kb, i);
          sc[kb][i] = __builtin_fmaf(-slope, (float)(max(key, x.pos) - min(key, x.pos)), sc[kb][i]);
        }
    }
    const bool hide = b0 < mx_lo || b0 + C::KW > mn_hi;  // keys that some row of the wave does not see
    if (hide) {
#pragma unroll
      for (int kb = 0; kb < C::KB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const uint32_t key = key_at(kb, i);
          if (key < x.lo || key >= x.hi) sc[kb][i] = -INFINITY;
        }
    }
    float t = sc[0][0];
#pragma unroll
    for (int kb = 0; kb < C::KB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) t = __builtin_fmaxf(t, sc[kb][i]);
    // the reference moves when some row's maximum passes it by 2^kLazy
    if (__builtin_amdgcn_ballot_w64(t > m + kLazy || (m == -INFINITY && t > m))) {
      const float mt = __builtin_fmaxf(t, other_half(t));
      const float mn = mt > m + kLazy || m == -INFINITY ? __builtin_fmaxf(mt, m) : m;
      const float al = mn == -INFINITY ? 1.f : fast_exp2(m - mn);
      m = mn;
      l *= al;
#pragma unroll
      for (int d = 0; d < DB; ++d) o[d] *= al;
    }
    const float ref = m == -INFINITY ? 0.f : m;
    uint32_t pw[C::NP][C::KB][8];  // two probabilities each, operand order
#pragma unroll
    for (int kb = 0; kb < C::KB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; i += 2) {
        const float p0 = fast_exp2(sc[kb][i] - ref), p1 = fast_exp2(sc[kb][i + 1] - ref);
        l += p0 + p1;
        if constexpr (C::NP == 1) {
          pw[0][kb][i / 2] = pack_bf16x2(p0, p1);
        } else {
          // leading 8 bits, and the rest rounded: together 16 bits and a half step
          const uint32_t h0 = __float_as_uint(p0) & 0xFFFF0000u, h1 = __float_as_uint(p1) & 0xFFFF0000u;
          pw[0][kb][i / 2] = upper_halves(h0, h1);
          // (kept above zero: an infinite V times 0 would be NaN)
          pw[1][kb][i / 2] = pack_bf16x2(__builtin_fmaxf(p0 - __uint_as_float(h0), 1e-37f),
                                         __builtin_fmaxf(p1 - __uint_as_float(h1), 1e-37f));
        }
      }
    // V^T of 16 keys and block d of 32 columns
    auto v_frag = [&](int kb, int ks, int d) {
      s16x4 f[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int row = 32 * kb + 16 * ks + 8 * h + 4 * half + (c16 >> 2);
        const int c = 4 * d + 2 * grp + ((c16 >> 1) & 1);
        f[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(
            vt + row * C::ROW + 16 * v_piece<D>(row, c) + 8 * (c16 & 1)));
      }
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(f[0], f[1], 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto p_frag = [&](int part, int kb, int ks) {
      return __builtin_bit_cast(bf16x8, u32x4e{pw[part][kb][4 * ks], pw[part][kb][4 * ks + 1], pw[part][kb][4 * ks + 2],
                                               pw[part][kb][4 * ks + 3]});
    };
    bool odd = RW == 4 ? false : own_special != 0;
    if (RW == 4 && hide) odd = (special[buf][0] | special[buf][1] | special[buf][2] | special[buf][3]) != 0;
    if (__builtin_expect(!(odd && hide), 1)) {
#pragma unroll
      for (int kb = 0; kb < C::KB; ++kb)
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
          for (int d = 0; d < DB; ++d) {
            const bf16x8 vf = v_frag(kb, ks, d);
#pragma unroll
            for (int part = 0; part < C::NP; ++part)
              o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, p_frag(part, kb, ks), o[d], 0, 0, 0);
          }
    } else {
      // V has infinities or NaN and not every row sees every key: 0 times
      // those is no 0. They are taken out of the products; which rows see one
      // is a product of ones, and those rows' sums get it added.
#pragma unroll
      for (int d = 0; d < DB; ++d) {
        f32x16 up, down;
#pragma unroll
        for (int i = 0; i < 16; ++i) up[i] = down[i] = 0.f;
#pragma unroll
        for (int kb = 0; kb < C::KB; ++kb)
#pragma unroll
          for (int ks = 0; ks < 2; ++ks) {
            const bf16x8 vf = v_frag(kb, ks, d), plain = without_special(vf);
#pragma unroll
            for (int part = 0; part < C::NP; ++part)
              o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(plain, p_frag(part, kb, ks), o[d], 0, 0, 0);
            u32x4e seen;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const uint32_t k0 = key_at(kb, 8 * ks + 2 * k), k1 = k0 + 1;
              seen[k] = (k0 >= x.lo && k0 < x.hi ? 0x3F80u : 0u) | (k1 >= x.lo && k1 < x.hi ? 0x3F800000u : 0u);
            }
            up = __builtin_amdgcn_mfma_f32_32x32x16_bf16(special_ones(vf, 0u), __builtin_bit_cast(bf16x8, seen), up, 0, 0, 0);
            down = __builtin_amdgcn_mfma_f32_32x32x16_bf16(special_ones(vf, 1u), __builtin_bit_cast(bf16x8, seen), down, 0, 0, 0);
          }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          if (up[i] > 0.f) o[d][i] += INFINITY;
          if (down[i] > 0.f) o[d][i] -= INFINITY;
        }
      }
    }
  };

  // ---- the steps
  if (RW == 4) {
    if (s0 < s1) {
      load_ptes(s0);
      load_keys(s0);
      store_keys(0, s0);
      if (s0 + 1 < s1) load_ptes(s0 + 1);
    }
    __syncthreads();
#pragma unroll 1
    for (uint32_t s = s0; s < s1; ++s) {
      const int buf = (s - s0) & 1;
      if (s + 1 < s1) {
        load_keys(s + 1);
        if (s + 2 < s1) load_ptes(s + 2);
      }
      compute(buf, s);
      if (s + 1 < s1) store_keys(buf ^ 1, s + 1);
      __syncthreads();
    }
  } else {
    if (s0 < s1) {
      load_ptes(s0);
      load_keys(s0);
      if (s0 + 1 < s1) load_ptes(s0 + 1);
    }
#pragma unroll 1
    for (uint32_t s = s0; s < s1; ++s) {
      store_keys(wave, s);
      if (s + 1 < s1) {
        load_keys(s + 1);
        if (s + 2 < s1) load_ptes(s + 2);
      }
      // a wave's LDS operations run in order: its reads follow its writes
      __builtin_amdgcn_wave_barrier();
      compute(wave, s);
      __builtin_amdgcn_wave_barrier();
    }
  }

  // ---- results: column d = 32 db + 8 (i / 4) + 4 half + i % 4 of row `col`
  l += other_half(l);
  if (RW == 4) {
    if (r >= rq.n_q * (uint32_t)g.g) return;
    const bool none = l == 0.f;  // (all scores NaN: l is NaN, and so are the results)
    const float inv = none ? 0.f : 1.f / l, lse = none ? -INFINITY : m + fast_log2(l);
    if (rq.splits > 1) {
      const uint64_t pr = part_row(a, rq, x, un.split);
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const f32x4 w = {o[d][i] * inv, o[d][i + 1] * inv, o[d][i + 2] * inv, o[d][i + 3] * inv};
          *reinterpret_cast<f32x4 *>(a.ws_o + pr * D + 32 * d + 2 * i + 4 * half) = none ? f32x4{0.f, 0.f, 0.f, 0.f} : w;
        }
      if (half == 0) a.ws_l[pr] = lse;
    } else {
      const uint64_t orow = x.tok * (uint32_t)g.hq + x.head;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const uint2 w = bf16x4_bits(o[d][i] * inv, o[d][i + 1] * inv, o[d][i + 2] * inv, o[d][i + 3] * inv);
          *reinterpret_cast<uint2 *>(a.out + orow * D + 32 * d + 2 * i + 4 * half) = none ? uint2{0u, 0u} : w;
        }
      if (half == 0) a.lse[orow] = lse * kLn2;
    }
  } else {
    __syncthreads();  // every wave is done with its tile
    float *const part = reinterpret_cast<float *>(lds) + wave * (32 * D);  // [column][row]
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) part[(32 * d + 8 * (i / 4) + 4 * half + i % 4) * 32 + col] = o[d][i];
    if (half == 0) {
      stats[0][wave][col] = m;
      stats[1][wave][col] = l;
    }
    __syncthreads();
    // thread: row t % 32, D / 8 columns
    constexpr int NC = D / 8;
    const int row = threadIdx.x & 31, c0 = (threadIdx.x >> 5) * NC;
    const uint32_t rr = un.tile * 32 + row;
    if (rr >= rq.n_q * (uint32_t)g.g) return;
    const Row y = row_of(a, rq, un.kvh, rr);
    float mt = stats[0][0][row];
#pragma unroll
    for (int w = 1; w < 4; ++w) mt = __builtin_fmaxf(mt, stats[0][w][row]);
    const float ref = mt == -INFINITY ? 0.f : mt;
    float f[4], lt4 = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      f[w] = fast_exp2(stats[0][w][row] - ref);
      lt4 += f[w] * stats[1][w][row];
    }
    const bool none = lt4 == 0.f;
    const float inv = none ? 0.f : 1.f / lt4, lse = none ? -INFINITY : mt + fast_log2(lt4);
    float v[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      float acc = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w)  // a wave that saw nothing of the row has nothing to add
        if (f[w] > 0.f) acc += f[w] * reinterpret_cast<const float *>(lds)[w * 32 * D + (c0 + c) * 32 + row];
      v[c] = acc * inv;
    }
    if (rq.splits > 1) {
      const uint64_t pr = part_row(a, rq, y, un.split);
#pragma unroll
      for (int c = 0; c < NC; c += 4)
        *reinterpret_cast<f32x4 *>(a.ws_o + pr * D + c0 + c) = f32x4{v[c], v[c + 1], v[c + 2], v[c + 3]};
      if (c0 == 0) a.ws_l[pr] = lse;
    } else {
      const uint64_t orow = y.tok * (uint32_t)g.hq + y.head;
#pragma unroll
      for (int c = 0; c < NC; c += 4)
        *reinterpret_cast<uint2 *>(a.out + orow * D + c0 + c) = bf16x4_bits(v[c], v[c + 1], v[c + 2], v[c + 3]);
      if (c0 == 0) a.lse[orow] = lse * kLn2;
    }
  }
}

// ----------------------------------------------------------------- join

// One wave per row: weights 2^(lse_s - max) of the ranges, then the columns.
__global__ __launch_bounds__(kExtThreads) void ext_merge_kernel(const ExtMergeArgs a) {
  const int lane = threadIdx.x & 63;
  const uint32_t row = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = sorted_search(a.n_req, row, [&](int i) { return a.req[i].row_begin; });
  const ExtMergeArgs::Req &rq = a.req[r];
  const uint32_t i = row - rq.row_begin;
  if (i >= rq.rows) return;
  const uint64_t pr = (rq.ws_row + i) * rq.splits;
  float mx = -INFINITY;
  for (uint32_t s = lane; s < rq.splits; s += 64) mx = fmaxf(mx, a.ws_l[pr + s]);
  mx = wave_max(mx);
  const float ref = mx == -INFINITY ? 0.f : mx;
  float sum = 0.f;
  for (uint32_t s = lane; s < rq.splits; s += 64) sum += fast_exp2(a.ws_l[pr + s] - ref);
  sum = wave_sum(sum);
  const bool none = sum == 0.f;
  const float inv = none ? 0.f : 1.f / sum;
  const uint32_t dv = (uint32_t)a.d_v;
  for (uint32_t c = lane; c < dv; c += 64) {
    float acc = 0.f;
    for (uint32_t s = 0; s < rq.splits; ++s) {
      const float w = fast_exp2(a.ws_l[pr + s] - ref);
      if (w > 0.f) acc = __builtin_fmaf(w, a.ws_o[(pr + s) * dv + c], acc);
    }
    a.out[(rq.out_row + i) * dv + c] = (uint16_t)f32_to_bf16(acc * inv);
  }
  if (lane == 0) a.lse[rq.out_row + i] = none ? -INFINITY : (mx + fast_log2(sum)) * kLn2;
}

hipError_t launch_extend(const ExtArgs &a, int32_t kind, hipStream_t stream) {
  const dim3 grid((uint32_t)a.n_units), block(kExtThreads);
  switch (kind) {
    case kXVec: {
      const size_t lds = 4 * (size_t)a.g.d_k * sizeof(float);
      switch (a.g.d_v / 64) {
        case 1: hipLaunchKernelGGL(extend_vec_kernel<1>, grid, block, lds, stream, a); break;
        case 2: hipLaunchKernelGGL(extend_vec_kernel<2>, grid, block, lds, stream, a); break;
        case 4: hipLaunchKernelGGL(extend_vec_kernel<4>, grid, block, lds, stream, a); break;
        default: hipLaunchKernelGGL(extend_vec_kernel<8>, grid, block, lds, stream, a); break;
      }
      break;
    }
    case kXRows64: hipLaunchKernelGGL((extend_kernel<64, 4>), grid, block, 0, stream, a); break;
    case kXRows128: hipLaunchKernelGGL((extend_kernel<128, 4>), grid, block, 0, stream, a); break;
    case kXFew64: hipLaunchKernelGGL((extend_kernel<64, 1>), grid, block, 0, stream, a); break;
    case kXFew128: hipLaunchKernelGGL((extend_kernel<128, 1>), grid, block, 0, stream, a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

hipError_t launch_ext_merge(const ExtMergeArgs &a, uint32_t rows, hipStream_t stream) {
  if (rows == 0) return hipSuccess;
  hipLaunchKernelGGL(ext_merge_kernel, dim3((rows + 3) / 4), dim3(kExtThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace cp
