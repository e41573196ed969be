// gfx950 kernels of the weights that queries give to cached tokens (cp_attn_weights):
//   sum[h][j] = decay old[h][j] + sum over rows that see j of e^(s_j - lse),
// a row being a query token and a query head of KV head h, and lse what the attention of
// these queries left. A score and an exponential for every pair, no maximum and no second
// product: each key's sum is its own, so a workgroup owns keys and takes rows in order.
// Sums are held in 32 bits and added in an order that the call's lengths alone decide.
#include <hip/hip_runtime.h>

#include "extend_device.h"
#include "weigh.h"

namespace cp {

namespace {

struct WeighUnit {
  const WeighReq *rq;
  uint32_t kvh, tile, split;
  bool none;
};
CP_DEV WeighUnit weigh_unit(const WeighArgs &a) {
  const int r = sorted_search(a.n_req, blockIdx.x, [&](int i) { return a.req[i].unit_begin; });
  const WeighReq &rq = a.req[r];
  const uint32_t per_head = rq.tiles * rq.splits, n = per_head * (uint32_t)a.g.hkv, b = blockIdx.x - rq.unit_begin;
  // (units of one KV head share its queries, in one XCD's L2)
  const uint32_t w = xcd_unit(b, n), kvh = w / per_head, u = w - kvh * per_head;
  return WeighUnit{&rq, kvh, u / rq.splits, u % rq.splits, b >= n};
}

// A row: what it sees, its log-sum-exp in units of log2 e and its slope.
struct WeighRow {
  Row x;
  float ref, slope;
};
// What of a row comes from memory: asked for a block ahead, looked at a block later.
struct RowLoads {
  float lse, slope;
  int32_t doc;
};
struct RowAddr {
  uint32_t t;     // query token of the request
  uint64_t tok;   // ... of the call
  uint32_t head;  // of all query heads
};
CP_DEV RowAddr row_addr(const WeighArgs &a, const WeighReq &rq, uint32_t kvh, uint32_t r) {
  uint32_t j;
  RowAddr x;
  x.t = page_divide(min(r, rq.n_q * (uint32_t)a.g.g - 1), (uint32_t)a.g.g, a.g_magic, &j);
  x.tok = (uint64_t)rq.tok0 + x.t;
  x.head = kvh * (uint32_t)a.g.g + j;
  return x;
}
CP_DEV RowLoads row_loads(const WeighArgs &a, const RowAddr &x) {
  RowLoads l;
  l.lse = a.lse[x.tok * (uint32_t)a.g.hq + x.head];
  l.doc = a.doc_begin ? a.doc_begin[x.tok] : 0;
  l.slope = a.slopes ? a.slopes[x.head] : 0.f;
  return l;
}
CP_DEV WeighRow weigh_row(const WeighArgs &a, const WeighReq &rq, const RowAddr &at, const RowLoads &l, uint32_t r) {
  WeighRow w;
  w.x.tok = at.tok;
  w.x.head = at.head;
  w.x.pos = rq.ctx - rq.n_q + at.t;
  w.x.hi = max(w.x.pos + 1, min(rq.prefix, rq.ctx));
  w.x.lo = a.window && w.x.pos >= a.window ? w.x.pos - a.window + 1 : 0u;
  if (l.doc > 0) w.x.lo = max(w.x.lo, (uint32_t)l.doc);
  w.ref = l.lse * kLog2e;
  w.slope = l.slope * kLog2e;
  // rows past the last, and those that saw nothing, give nothing
  if (r >= rq.n_q * (uint32_t)a.g.g || w.x.lo >= w.x.hi || l.lse == -INFINITY) {
    w.x.lo = w.x.hi = 0;
    w.ref = 0.f;
  }
  return w;
}

// Blocks of rows of which some may see keys [k0, k1), and this unit's part of them.
struct Blocks {
  uint32_t from, to;
};
CP_DEV Blocks weigh_blocks(const WeighArgs &a, const WeighReq &rq, uint32_t k0, uint32_t k1, uint32_t split) {
  const uint32_t g = (uint32_t)a.g.g, base = rq.ctx - rq.n_q;
  uint32_t t0 = min(rq.prefix, rq.ctx) > k0 || k0 <= base ? 0u : k0 - base, t1 = rq.n_q;
  if (a.window) {  // position p sees keys > p - window
    const uint64_t end = (uint64_t)k1 + a.window - 1;
    t1 = end <= base ? 0u : (uint32_t)min((uint64_t)t1, end - base);
  }
  if (t0 >= t1) return Blocks{0, 0};
  const uint32_t b0 = t0 * g / kWeighBlock, b1 = (t1 * g + kWeighBlock - 1) / kWeighBlock, n = b1 - b0;
  return Blocks{b0 + (uint32_t)((uint64_t)n * split / rq.splits), b0 + (uint32_t)((uint64_t)n * (split + 1) / rq.splits)};
}

CP_DEV void put_sum(const WeighArgs &a, const WeighReq &rq, uint32_t kvh, uint32_t split, uint32_t key, float v) {
  if (rq.splits > 1) {
    a.ws[rq.ws + ((uint64_t)split * (uint32_t)a.g.hkv + kvh) * rq.ctx + key] = v;
    return;
  }
  const float *const o = rq.old ? rq.old + (int64_t)kvh * rq.old_head + key : nullptr;
  rq.sum[(int64_t)kvh * rq.sum_head + key] = o ? __builtin_fmaf(a.decay, *o, v) : v;
}

// A row whose log-sum-exp is NaN gives NaN to what it sees, and to nothing else.
template <int N, class F>
CP_DEV float nan_row(float (&s)[N], float ref, const Row &x, uint32_t k0, F at) {
  if (__builtin_expect(__builtin_amdgcn_ballot_w64(ref != ref) == 0, 1)) return ref;
  if (ref == ref) return ref;
#pragma unroll
  for (int i = 0; i < N; ++i) s[i] = k0 + at(i) >= x.lo && k0 + at(i) < x.hi ? ref : -INFINITY;
  return 0.f;
}

// Sums over the 16 lanes of a DPP row, in every lane.
template <int CTRL>
CP_DEV float dpp_add(float x) {
  return x + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, 0xF, 0xF, false));
}
CP_DEV float row_sum_16(float x) {
  return dpp_add<0x121>(dpp_add<0x122>(dpp_add<0x124>(dpp_add<0x128>(x))));  // row_ror 8, 4, 2, 1
}

}  // namespace

// --------------------------------------------------------------- few rows

// At most 16 rows: S^T = K Q^T by 16x16x32 products, a lane holding 16 bytes of one key's row
// of the first operand. All of a wave's keys are asked for at once. Rows of 256 bytes come in
// loads of 1 KiB that follow each other in memory, kept in no cache, and each block of 16 is
// turned into operands through LDS of the wave's own, without a barrier; others are loaded as
// operands, every line by two loads. A lane then has four keys of one row; the rows' sum is
// over 16 lanes. Bound by reading K: 8 requests of 32 K tokens, 8 heads of 128, 90 us (6.0 TB/s;
// loaded as operands 104, those uncached 111); heads of 64, 128 K tokens 213 (5.0 TB/s, turned
// 215); latent, 32 of 32 K 235 (5.1 TB/s; uncached 283, turned 295: fewer waves).
template <int DK>
struct FewCfg {
  static constexpr int NB = weigh_tile_keys(DK == 128 ? kWFew128 : DK == 64 ? kWFew64 : kWFewMla) / 64;  // blocks of a wave
  static constexpr int ROW = 2 * DK, LOADS = 16 * ROW / 1024;
  static constexpr bool TURN = DK == 128;
  static_assert(!TURN || ROW == 256, "sixteen pieces of 16 bytes a row");
};

template <int DK, int MODE>
__global__ __launch_bounds__(kWeighThreads) void weigh_few_kernel(const WeighArgs a) {
  using C = FewCfg<DK>;
  constexpr int KS = DK / 32, NB = C::NB;
  __shared__ __attribute__((aligned(16))) char lds[C::TURN ? 4 * 16 * C::ROW : 16];
  const WeighUnit un = weigh_unit(a);
  if (un.none) return;
  const WeighReq &rq = *un.rq;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, quad = lane >> 4;
  const uint32_t P = (uint32_t)a.g.page_tokens, b0 = (un.tile * 4 + wave) * (16 * NB);
  if (b0 >= rq.ctx) return;  // (no barrier below)
  uint32_t at[NB], slot[NB];
#pragma unroll
  for (int n = 0; n < NB; ++n) {  // keys past the context: the last one (their sums are not stored)
    const uint32_t pg = page_divide(min(b0 + 16 * n + col, rq.ctx - 1), P, a.page_magic, &slot[n]);
    at[n] = a.pte[rq.pte_base + pg];
  }
  bf16x8 qf[KS];
  const RowAddr ra = row_addr(a, rq, un.kvh, col);
  const WeighRow w = weigh_row(a, rq, ra, row_loads(a, ra), col);
  {
    const uint16_t *const qrow = a.q + (w.x.tok * (uint32_t)a.g.hq + w.x.head) * DK + 8 * quad;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const bf16x8 *>(qrow + 32 * ks);
  }
  const uint8_t *const head = a.pool + (DK == 576 ? 0ull : (uint64_t)un.kvh * (4ull * P * DK));
  u32x4e kf[NB][C::LOADS];
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    const uint64_t row_at = (uint64_t)(uintptr_t)head + ((uint64_t)at[n] << 8) + (uint64_t)slot[n] * C::ROW;  // of key `col`
    const int lo = (int)(uint32_t)row_at, hi = (int)(uint32_t)(row_at >> 32);
#pragma unroll
    for (int i = 0; i < C::LOADS; ++i) {
      if (C::TURN) {  // row 4 i + quad, piece col
        const int key = 4 * (4 * i + quad);
        const uint64_t from = (uint64_t)(uint32_t)__builtin_amdgcn_ds_bpermute(key, hi) << 32 |
                              (uint32_t)__builtin_amdgcn_ds_bpermute(key, lo);
        kf[n][i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4e *>(from) + col);
      } else {
        kf[n][i] = reinterpret_cast<const u32x4e *>(row_at)[4 * i + quad];
      }
    }
  }
  char *const mine = lds + wave * (16 * C::ROW);
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    const uint32_t k0 = b0 + 16 * n;
    if (k0 >= rq.ctx) return;
    if constexpr (C::TURN) {  // (pieces swapped by the row: 16 rows at one piece meet no bank twice)
#pragma unroll
      for (int i = 0; i < C::LOADS; ++i)
        *reinterpret_cast<u32x4e *>(mine + (4 * i + quad) * C::ROW + 16 * (col ^ (4 * i + quad))) = kf[n][i];
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        kf[n][ks] = *reinterpret_cast<const u32x4e *>(mine + col * C::ROW + 16 * ((4 * ks + quad) ^ col));
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    f32x4 sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[n][ks]), qf[ks], sc, 0, 0, 0);
    auto &flat = reinterpret_cast<float(&)[4]>(sc);
    const bool hide = __builtin_amdgcn_ballot_w64(w.x.lo > k0 || w.x.hi < k0 + 16) != 0;
    const bool behind = MODE == kModeAny && __builtin_amdgcn_ballot_w64(w.x.pos + 1 < k0 + 16) == 0;
    float top;
    auto key_of = [](int i) { return i; };
    const bool raw = scores_of<MODE, 4>(a, RowAt{}, flat, w.slope, w.x, k0 + 4 * quad, behind, hide, 0u, key_of, &top);
    float v[4];
    weights<MODE, 4>(a, flat, raw, nan_row(flat, w.ref, w.x, k0 + 4 * quad, key_of), [&](int i, float p0, float p1) {
      v[i] = p0;
      v[i + 1] = p1;
    });
    float mine = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float s = row_sum_16(v[i]);
      mine = col == i ? s : mine;
    }
    const uint32_t key = k0 + 4 * quad + col;
    if (col < 4 && key < rq.ctx) put_sum(a, rq, un.kvh, 0, key, mine);
  }
}

// --------------------------------------------------------------- many rows

// K in registers (the products' first operand), queries and their log-sum-exps streamed past
// them through LDS, a ring of steps of 64 rows (MLA 32). Scores are transposed as in the
// attention kernels: a lane holds one row's scores, and adds their exponentials to sums of its
// own, one for every key; the lanes' sums meet at the end. Turns of 16 rows, 16x16x32 products.
// head_dim 64 and 128: 64 keys a wave, three workgroups a CU (LDS: a ring of three steps for
// 128). A score costs a multiply-add, an exponential and an addition, 16 cycles a wave for 64
// of them, and its products 16 too (head_dim 128): plain scores are one turn behind their
// products, so that the vector unit and the matrix cores work at once (the compiler left to
// itself starts the exponentials when the products are done), and masks are looked at only
// where some row of a step does not see some key. Bound by the products with the vector work
// in their shadow: the last 5,000 tokens of 8 K and of 5 K, 32 heads over 8, 364 to 385 us, 0.9
// PFLOP/s where a large library product reaches 1.39; without the exponentials 320, without
// the products 190, without new queries 350. 32 rows by 32x32x16 products took 655 us where
// these take 450; an inner loop without a moved register, its turns apart from those with a
// mask, took as long.
// MLA: 32 keys a wave, 144 registers, whose few scores leave registers to read fragments
// ahead. LDS bounds it with the matrix cores: a fragment of 1 KiB feeds 32 cycles of products.
// 64 rows past 256 keys take 5 us (0.97 PFLOP/s with every CU full); 64 tokens of four contexts
// of 22 K in all, 16 heads, 41 us, of which a third goes to 174 units on 256 CUs.
template <int DK>
struct WeighCfg {
  static constexpr bool MLA = DK == 576;
  static constexpr int KB = MLA ? 2 : 4;           // blocks of 16 keys of a wave
  static constexpr int RT = 16;                    // rows of a turn, and keys of a block
  static constexpr int THREADS = MLA ? 512 : 256, WAVES = THREADS / 64;
  static constexpr int KW = RT * KB, KEYS = KW * WAVES;
  static constexpr int KD = 32;                    // dims of a product
  static constexpr int KS = DK / KD;
  static constexpr int EB = 4;                     // scores of a lane and block
  static constexpr int LAT = MLA ? 1024 : 2 * DK;  // bytes of a row in LDS (latent part), and behind all of those
  static constexpr int ROT = MLA ? 128 : 0;        // ... of its rotary part
  static constexpr int STEP = MLA ? 32 : 64, TURNS = STEP / RT;  // rows between two barriers
  static constexpr int TILE = STEP * (LAT + ROT) + 256;          // bytes of a step: queries, and 64 log-sum-exps
  static constexpr int RING = DK == 128 ? 3 : 4;  // (three workgroups a CU)
  // pieces of 16 bytes, swapped by the row so that 16 rows at one piece meet no bank twice
  static CP_DEV int lat_piece(int row, int c) { return LAT == 128 ? c ^ ((row >> 1) & 7) : c ^ (row & 15); }
  static CP_DEV int rot_piece(int row, int c) { return c ^ ((row >> 1) & 7); }
};

template <int DK, int MODE>
__global__ __launch_bounds__(WeighCfg<DK>::THREADS, DK == 576 ? 2 : 3) void weigh_rows_kernel(const WeighArgs a) {
  using C = WeighCfg<DK>;
  typedef float scores_t __attribute__((ext_vector_type(C::EB)));
  constexpr int KB = C::KB, KS = C::KS, NE = C::EB * KB, TURNS = C::TURNS, STEP = C::STEP;
  constexpr bool BEHIND = MODE == kModePlain && !C::MLA;  // exponentials a turn behind
  __shared__ __attribute__((aligned(16))) char lds[C::RING * C::TILE];
  const WeighUnit un = weigh_unit(a);
  if (un.none) return;
  const WeighReq &rq = *un.rq;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane % C::RT, part = lane / C::RT;  // row of a turn; which dims, and keys
  const uint32_t P = (uint32_t)a.g.page_tokens, g = (uint32_t)a.g.g, hq = (uint32_t)a.g.hq;
  const uint32_t t0 = un.tile * C::KEYS, b0 = t0 + wave * C::KW;
  const Blocks bl = weigh_blocks(a, rq, t0, min(t0 + C::KEYS, rq.ctx), un.split);
  // steps of rows (a block's last may lie past the last row)
  const uint32_t from = bl.from * (kWeighBlock / STEP), to = min(bl.to * (kWeighBlock / STEP), (rq.n_q * g + STEP - 1) / STEP);

  // ---- K: lane holds key RT kb + col, dims KD ks + 8 part .. + 7
  bf16x8 kf[KB][KS];
  if (from < to) {
    const uint8_t *const head = a.pool + (C::MLA ? 0ull : (uint64_t)un.kvh * (4ull * P * DK)) + 16 * part;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      uint32_t slot;
      const uint32_t pg = page_divide(min(b0 + C::RT * kb + col, rq.ctx - 1), P, a.page_magic, &slot);
      const u32x4e *const k = reinterpret_cast<const u32x4e *>(head + ((uint64_t)a.pte[rq.pte_base + pg] << 8) +
                                                              (uint64_t)slot * (2 * DK));
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        kf[kb][ks] = __builtin_bit_cast(bf16x8, k[ks * (C::KD / 8)]);
    }
  }

  // ---- places of rows. Row r of a step is `off(r)` rows of the call's queries behind the
  // step's first where steps end with tokens or a token's heads are all of one KV head's;
  // otherwise, and in the last step, each is looked up (rows past the last repeat it).
  const uint32_t last_full = rq.n_q * g / STEP;  // steps from here on are not whole
  const bool even = a.g.hkv == 1 || STEP % g == 0;
  auto off = [&](uint32_t row) {
    if (a.g.hkv == 1) return row;
    uint32_t j;
    const uint32_t t = page_divide(row, g, a.g_magic, &j);
    return t * hq + j;
  };
  auto first_row = [&](uint32_t st) {  // of the call's queries
    return a.g.hkv == 1 ? (uint64_t)rq.tok0 * hq + (uint64_t)st * STEP
                        : ((uint64_t)rq.tok0 + (uint64_t)st * (STEP / g)) * hq + un.kvh * g;
  };
  // a step's queries and log-sum-exps go to LDS directly: N instructions of RPI rows for each
  // wave, MLA's rotary parts by the first waves, and the same 64 numbers by every wave (one
  // count of loads in flight for all)
  constexpr int CPR = C::LAT / 16, RPI = CPR >= 64 ? 1 : 64 / CPR, N = STEP / RPI / C::WAVES;
  constexpr int ROTW = C::ROT > 0 ? STEP / 8 : 0;  // waves with an instruction of eight rotary rows
  constexpr int NO = C::MLA ? 1 : N;  // (MLA: a wave's latent rows, one an instruction, follow each other)
  uint32_t qoff[NO], roff = 0, loff;  // bytes from the step's first row to this lane's pieces; rows, to its own
#pragma unroll
  for (int i = 0; i < NO; ++i) {
    const int row = (wave * N + i) * RPI + lane / CPR;
    qoff[i] = off(row) * (2 * DK) + (C::MLA ? 0 : 16 * C::lat_piece(row, lane % CPR));
  }
  if (C::MLA) {
    const int row = (8 * wave + lane / 8) % STEP;
    roff = off(row) * (2 * DK) + C::LAT + 16 * C::rot_piece(row, lane % 8);
  }
  loff = off(lane % STEP);
  auto issue = [&](uint32_t st) {
    const uint32_t tile = lds_addr(lds) + (st - from) % C::RING * C::TILE;
    const bool whole = even && st < last_full;
    const uint64_t base = (uint64_t)(uintptr_t)a.q + first_row(st) * (2ull * DK);
    auto place = [&](uint32_t row) {
      const RowAddr x = row_addr(a, rq, un.kvh, st * STEP + row);
      return x.tok * hq + x.head;
    };
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int row0 = (wave * N + i) * RPI, row = row0 + lane / CPR;
      if (whole && C::MLA)
        row_load_lds<false>(base + (uint64_t)(row0 * (2 * DK)), 16u * C::lat_piece(row0, lane), tile + row0 * C::LAT);
      else if (whole)
        row_load_lds<false>(base, qoff[C::MLA ? 0 : i], tile + row0 * C::LAT);
      else
        lane_load_lds<false>((uint64_t)(uintptr_t)a.q + place(row) * (2ull * DK) + 16 * C::lat_piece(row, lane % CPR),
                             tile + row0 * C::LAT);
    }
    if (wave < ROTW) {
      const int row = 8 * wave + lane / 8;
      if (whole)
        row_load_lds<false>(base, roff, tile + STEP * C::LAT + 8 * wave * C::ROT);
      else
        lane_load_lds<false>((uint64_t)(uintptr_t)a.q + place(row) * (2ull * DK) + C::LAT + 16 * C::rot_piece(row, lane % 8),
                             tile + STEP * C::LAT + 8 * wave * C::ROT);
    }
    dword_load_lds((uint64_t)(uintptr_t)a.lse + 4 * (whole ? first_row(st) + loff : place(lane % STEP)),
                   tile + STEP * (C::LAT + C::ROT));
  };

  float acc[NE];
#pragma unroll
  for (int i = 0; i < NE; ++i) acc[i] = 0.f;
  // element i: key b0 + 4 part + key_of(i)
  auto key_of = [](int i) { return 16 * (i / 4) + i % 4; };

  // Does every row of a step see every key of this wave (documents aside)?
  auto all_seen = [&](uint32_t st) {
    uint32_t rest;
    const uint32_t r0 = st * STEP, base = rq.ctx - rq.n_q;
    const uint32_t p0 = base + page_divide(r0, g, a.g_magic, &rest), p1 = base + page_divide(r0 + STEP - 1, g, a.g_magic, &rest);
    return st < last_full && !a.doc_begin && b0 + C::KW <= max(p0 + 1, min(rq.prefix, rq.ctx)) &&
           (a.window == 0 || p1 < b0 + a.window);
  };
  // fragments of a turn's queries: row `col`, dims KD ks + 8 part
  auto q_frag = [&](const char *qt, int turn, int ks) {
    const int row = C::RT * turn + col, c = ks * (C::KD / 8) + part;
    return *reinterpret_cast<const bf16x8 *>(
        C::MLA && ks * (C::KD / 8) >= 64 ? qt + STEP * C::LAT + row * C::ROT + 16 * C::rot_piece(row, c - 64)
                                         : qt + row * C::LAT + 16 * C::lat_piece(row, c));
  };
  // products of a turn; after(e) follows the e-th of KS KB
  auto products = [&](const char *qt, int turn, scores_t (&sc)[KB], auto after) {
    constexpr int AHEAD = C::MLA ? 4 : 1;
    bf16x8 qf[AHEAD + 1];
#pragma unroll
    for (int ks = 0; ks < AHEAD; ++ks) qf[ks] = q_frag(qt, turn, ks);
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < C::EB; ++i) sc[kb][i] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if (ks + AHEAD < KS) qf[(ks + AHEAD) % (AHEAD + 1)] = q_frag(qt, turn, ks + AHEAD);
      if (C::MLA) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        sc[kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[kb][ks], qf[ks % (AHEAD + 1)], sc[kb], 0, 0, 0);
        after(ks * KB + kb);
      }
    }
  };
  // Scores in the form that their exponentials take, those out of sight -inf, and the
  // reference that comes off. easy: every row sees every key, and has a log-sum-exp.
  auto shape = [&](scores_t (&sc)[KB], uint32_t st, int turn, float lse, bool easy, bool *raw) {
    auto &flat = reinterpret_cast<float(&)[NE]>(sc);
    float top;
    if (__builtin_expect(easy && MODE == kModePlain, 1)) {
      *raw = true;
      return lse * kLog2e;
    }
    const uint32_t r = st * STEP + C::RT * turn + col;
    const RowAddr at = row_addr(a, rq, un.kvh, r);
    RowLoads l;
    l.lse = lse;
    l.doc = a.doc_begin ? a.doc_begin[at.tok] : 0;
    l.slope = MODE == kModeAny && a.slopes ? a.slopes[at.head] : 0.f;
    const WeighRow w = weigh_row(a, rq, at, l, r);
    const bool hide = !easy && __builtin_amdgcn_ballot_w64(w.x.lo > b0 || w.x.hi < b0 + C::KW) != 0;
    const bool behind = MODE == kModeAny && __builtin_amdgcn_ballot_w64(w.x.pos + 1 < b0 + C::KW) == 0;
    *raw = scores_of<MODE, NE>(a, RowAt{}, flat, w.slope, w.x, b0 + 4 * part, behind, hide, 0u, key_of, &top);
    return nan_row(flat, w.ref, w.x, b0 + 4 * part, key_of);
  };

  for (uint32_t st = from; st < to && st < from + C::RING - 1; ++st) issue(st);
  // K is there from here on: the compiler's own waits, inside the loop, would drain blocks in flight
#pragma unroll
  for (int kb = 0; kb < KB; ++kb)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(kf[kb][ks]));
  scores_t held[2][KB];  // BEHIND: a turn's scores, and those of the one before
  float held_ref = 0.f;
  if (BEHIND) {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < C::EB; ++i) held[1][kb][i] = -INFINITY;
  }
  static_assert(TURNS % 2 == 0, "turns alternate");
#pragma unroll 1
  for (uint32_t st = from; st < to; ++st) {
    // own loads of this step have landed once at most the later steps' remain
    constexpr int L = N + 1, LATER = C::RING - 2;
    if (to - st <= LATER) wait_vm<0>();
    else if (wave < ROTW) wait_vm<LATER * (L + 1)>();
    else wait_vm<LATER * L>();
    __syncthreads();  // this step is there for every wave; the one before is done with
    if (st + C::RING - 1 < to) issue(st + C::RING - 1);
    const char *const qt = lds + (st - from) % C::RING * C::TILE;
    const float *const lse_of = reinterpret_cast<const float *>(qt + STEP * (C::LAT + C::ROT)) + col;
    float lse[TURNS];
    bool none = false;
#pragma unroll
    for (int t = 0; t < TURNS; ++t) {
      lse[t] = lse_of[C::RT * t];
      none = none || !(lse[t] > -INFINITY);
    }
    const bool easy = all_seen(st) && __builtin_amdgcn_ballot_w64(none) == 0;
    if constexpr (BEHIND) {
#pragma unroll
      for (int t = 0; t < TURNS; ++t) {
        constexpr int EACH = NE / (KS * KB);
        bool raw;
        auto &prev = reinterpret_cast<float(&)[NE]>(held[(t & 1) ^ 1]);
        float p[EACH] = {};
        __builtin_amdgcn_sched_barrier(0);
        // an exponential's sum is taken a product later, when it is there
        products(qt, t, held[t & 1], [&](int e) {
#pragma unroll
          for (int i = 0; i < EACH; ++i) {
            if (e > 0) {
              acc[(e - 1) * EACH + i] += p[i];
              asm volatile("" : "+v"(acc[(e - 1) * EACH + i]));  // here, and not where the loop ends
            }
            p[i] = fast_exp2(__builtin_fmaf(prev[e * EACH + i], a.score_mul, -held_ref));
          }
          __builtin_amdgcn_sched_barrier(0);
        });
#pragma unroll
        for (int i = 0; i < EACH; ++i) acc[NE - EACH + i] += p[i];
        held_ref = shape(held[t & 1], st, t, lse[t], easy, &raw);
      }
    } else {
#pragma unroll 1
      for (int t = 0; t < TURNS; ++t) {
        bool raw;
        scores_t sc[KB];
        float mine = lse[0];
#pragma unroll
        for (int u = 1; u < TURNS; ++u) mine = t == u ? lse[u] : mine;
        products(qt, t, sc, [](int) {});
        const float ref = shape(sc, st, t, mine, easy, &raw);
        weights<MODE, NE>(a, reinterpret_cast<float(&)[NE]>(sc), raw, ref, [&](int i, float p0, float p1) {
          acc[i] += p0;
          acc[i + 1] += p1;
        });
      }
    }
  }
  if constexpr (BEHIND) {
    auto &prev = reinterpret_cast<float(&)[NE]>(held[1]);
#pragma unroll
    for (int i = 0; i < NE; ++i) acc[i] += fast_exp2(__builtin_fmaf(prev[i], a.score_mul, -held_ref));
  }

  // ---- the lanes' sums of a key: the RT lanes of one part
#pragma unroll
  for (int kb = 0; kb < KB; ++kb) {
    float mine = 0.f;
#pragma unroll
    for (int i = 0; i < C::EB; ++i) {
      const float s = row_sum_16(acc[C::EB * kb + i]);
      mine = (col & 15) == i ? s : mine;
    }
    const int i = col & 15;
    const uint32_t key = b0 + 4 * part + key_of(C::EB * kb + (i < C::EB ? i : 0));
    if (col < C::EB && key < rq.ctx) put_sum(a, rq, un.kvh, un.split, key, mine);
  }
}

// ------------------------------------------------------------ vector path

// A thread per key, eight rows at a time from LDS, for every geometry. Bound by the vector
// unit and each thread's own row reads (a block of 64 rows takes 20 us and more); it serves the
// geometries without a matrix kernel.
__global__ __launch_bounds__(kWeighThreads) void weigh_vec_kernel(const WeighArgs a) {
  constexpr int R = 8;
  extern __shared__ float qs[];  // [R][d_k]
  __shared__ WeighRow ws[R];
  const WeighUnit un = weigh_unit(a);
  if (un.none) return;
  const WeighReq &rq = *un.rq;
  const uint32_t dk = (uint32_t)a.g.d_k, P = (uint32_t)a.g.page_tokens, g = (uint32_t)a.g.g, rows = rq.n_q * g;
  const uint32_t t0 = un.tile * kWeighThreads, key = t0 + threadIdx.x;
  const Blocks bl = weigh_blocks(a, rq, t0, min(t0 + kWeighThreads, rq.ctx), un.split);
  uint32_t slot;
  const uint32_t pg = page_divide(min(key, rq.ctx - 1), P, a.page_magic, &slot);
  const u32x4e *const k = reinterpret_cast<const u32x4e *>(
      a.pool + ((uint64_t)a.pte[rq.pte_base + pg] << 8) + (a.g.kind == 0 ? 0ull : (uint64_t)un.kvh * 4 * P * dk) +
      (uint64_t)slot * (2 * dk));
  float sum = 0.f;
  const uint32_t r1 = min(bl.to * kWeighBlock, rows);
  for (uint32_t r0 = bl.from * kWeighBlock; r0 < r1; r0 += R) {
    __syncthreads();
    if (threadIdx.x < R) {
      const RowAddr ra = row_addr(a, rq, un.kvh, r0 + threadIdx.x);
      ws[threadIdx.x] = weigh_row(a, rq, ra, row_loads(a, ra), r0 + threadIdx.x);
    }
    for (uint32_t i = threadIdx.x; i < R * dk; i += kWeighThreads) {
      uint32_t j;
      const uint32_t row = i / dk, t = page_divide(min(r0 + row, rows - 1), g, a.g_magic, &j);
      qs[i] = bf16_to_f32(a.q[(((uint64_t)rq.tok0 + t) * (uint32_t)a.g.hq + un.kvh * g + j) * dk + (i - row * dk)]);
    }
    __syncthreads();
    float acc[R];
#pragma unroll
    for (int i = 0; i < R; ++i) acc[i] = 0.f;
    for (uint32_t c = 0; c < dk / 8; ++c) {
      const u32x4e x = k[c];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float lo = __uint_as_float(x[e] << 16), hi = __uint_as_float(x[e] & 0xFFFF0000u);
#pragma unroll
        for (int i = 0; i < R; ++i)
          acc[i] = __builtin_fmaf(hi, qs[i * dk + 8 * c + 2 * e + 1], __builtin_fmaf(lo, qs[i * dk + 8 * c + 2 * e], acc[i]));
      }
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const WeighRow &w = ws[i];
      float s = acc[i] * a.score_mul;
      if (a.softcap > 0.f) s = cap_tanh(s) * a.cap_mul;
      if (a.slopes) s -= w.slope * (float)(max(w.x.pos, key) - min(w.x.pos, key));
      if (key >= w.x.lo && key < w.x.hi) sum += fast_exp2(s - w.ref);
    }
  }
  if (key < rq.ctx) put_sum(a, rq, un.kvh, un.split, key, sum);
}

// ------------------------------------------------------------------- join

// The parts of keys whose rows were cut, in order. A thread per KV head and key. Bound by its
// launch (13 K tokens of 8 heads in 8 parts: 5 us).
__global__ __launch_bounds__(kWeighThreads) void weigh_join_kernel(const WeighJoinArgs a) {
  const int r = sorted_search(a.n_req, blockIdx.x, [&](int i) { return a.req[i].block_begin; });
  const WeighJoinArgs::Req &rq = a.req[r];
  const uint64_t i = (uint64_t)(blockIdx.x - rq.block_begin) * kWeighThreads + threadIdx.x, n = (uint64_t)a.hkv * rq.ctx;
  if (i >= n) return;
  const uint32_t h = (uint32_t)(i / rq.ctx), key = (uint32_t)(i - (uint64_t)h * rq.ctx);
  float v = 0.f;
  for (uint32_t s = 0; s < rq.splits; ++s) v += a.ws[rq.ws + s * n + i];
  const float *const o = rq.old ? rq.old + (int64_t)h * rq.old_head + key : nullptr;
  rq.sum[(int64_t)h * rq.sum_head + key] = o ? __builtin_fmaf(a.decay, *o, v) : v;
}

namespace {
template <int DK, bool FEW>
void launch_matrix(const WeighArgs &a, hipStream_t stream) {
  const dim3 grid((uint32_t)a.n_units), block(kWeighThreads);
  if constexpr (FEW) {
    if (a.slopes)
      hipLaunchKernelGGL((weigh_few_kernel<DK, kModeAny>), grid, block, 0, stream, a);
    else if (a.softcap > 0.f)
      hipLaunchKernelGGL((weigh_few_kernel<DK, kModeCap>), grid, block, 0, stream, a);
    else
      hipLaunchKernelGGL((weigh_few_kernel<DK, kModePlain>), grid, block, 0, stream, a);
  } else {
    const dim3 wide(WeighCfg<DK>::THREADS);
    if (a.slopes)
      hipLaunchKernelGGL((weigh_rows_kernel<DK, kModeAny>), grid, wide, 0, stream, a);
    else if (a.softcap > 0.f)
      hipLaunchKernelGGL((weigh_rows_kernel<DK, kModeCap>), grid, wide, 0, stream, a);
    else
      hipLaunchKernelGGL((weigh_rows_kernel<DK, kModePlain>), grid, wide, 0, stream, a);
  }
}
}  // namespace

hipError_t launch_weigh(const WeighArgs &a, int32_t kind, hipStream_t stream) {
  switch (kind) {
    case kWVec:
      hipLaunchKernelGGL(weigh_vec_kernel, dim3((uint32_t)a.n_units), dim3(kWeighThreads), 8 * (size_t)a.g.d_k * sizeof(float),
                         stream, a);
      break;
    case kWFew64: launch_matrix<64, true>(a, stream); break;
    case kWFew128: launch_matrix<128, true>(a, stream); break;
    case kWFewMla: launch_matrix<576, true>(a, stream); break;
    case kWRows64: launch_matrix<64, false>(a, stream); break;
    case kWRows128: launch_matrix<128, false>(a, stream); break;
    case kWRowsMla: launch_matrix<576, false>(a, stream); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

hipError_t launch_weigh_join(const WeighJoinArgs &a, hipStream_t stream) {
  if (a.n_blocks <= 0) return hipSuccess;
  hipLaunchKernelGGL(weigh_join_kernel, dim3((uint32_t)a.n_blocks), dim3(kWeighThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace cp
