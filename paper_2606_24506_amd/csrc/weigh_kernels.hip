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

// At most 16 rows: S^T = K Q^T by 16x16x32 products, K from the pool straight to the
// operand's registers (a lane holds 16 bytes of one key's row), all of a wave's keys asked
// for at once. A lane has four keys of one row; the rows' sum is over 16 lanes.
template <int DK, int MODE>
__global__ __launch_bounds__(kWeighThreads) void weigh_few_kernel(const WeighArgs a) {
  constexpr int KS = DK / 32, NB = DK == 128 ? 4 : DK == 64 ? 8 : 2;  // blocks of 16 keys of a wave
  const WeighUnit un = weigh_unit(a);
  if (un.none) return;
  const WeighReq &rq = *un.rq;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, quad = lane >> 4;
  const uint32_t P = (uint32_t)a.g.page_tokens, b0 = (un.tile * 4 + wave) * (16 * NB);
  if (b0 >= rq.ctx) return;  // (no barrier below)
  const uint8_t *const head = a.pool + (DK == 576 ? 0ull : (uint64_t)un.kvh * (4ull * P * DK)) + 16 * quad;
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
  u32x4e kf[NB][KS];
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    const u32x4e *const k = reinterpret_cast<const u32x4e *>(head + ((uint64_t)at[n] << 8) + (uint64_t)slot[n] * (2 * DK));
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) kf[n][ks] = __builtin_nontemporal_load(k + 4 * ks);
  }
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    const uint32_t k0 = b0 + 16 * n;
    if (k0 >= rq.ctx) return;
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

// K in registers (32 or 64 keys of a wave, the 32x32x16 products' first operand), queries
// streamed past them through LDS in blocks of 32 rows, one block ahead. Scores are
// transposed as in the attention kernels: a lane holds one row's scores, and adds their
// exponentials to sums of its own, one for every key; the lanes' sums meet at the end.
template <int DK>
struct WeighCfg {
  static constexpr int KB = DK == 576 ? 1 : 2;   // blocks of 32 keys of a wave
  static constexpr int KW = 32 * KB, WAVES = kWeighThreads / 64, KEYS = KW * WAVES;
  static constexpr int KS = DK / 16;
  static constexpr int LAT = DK == 576 ? 1024 : 2 * DK;  // bytes of a row in LDS (latent part), and behind all of those
  static constexpr int ROT = DK == 576 ? 128 : 0;        // ... of its rotary part
  static constexpr int TILE = kWeighBlock * (LAT + ROT);
  // pieces of 16 bytes, swapped by the row so that 16 rows at one piece meet no bank twice
  static CP_DEV int lat_piece(int row, int c) { return LAT == 128 ? c ^ ((row >> 1) & 7) : c ^ (row & 15); }
  static CP_DEV int rot_piece(int row, int c) { return c ^ ((row >> 1) & 7); }
};

// (capped and sloped scores beside 144 registers of an MLA key: one wave a SIMD, or they spill)
template <int DK, int MODE>
__global__ __launch_bounds__(kWeighThreads, DK == 576 && MODE != kModePlain ? 1 : 2) void weigh_rows_kernel(const WeighArgs a) {
  using C = WeighCfg<DK>;
  constexpr int KB = C::KB, KS = C::KS, NE = 16 * KB;
  __shared__ __attribute__((aligned(16))) char lds[2 * C::TILE];
  const WeighUnit un = weigh_unit(a);
  if (un.none) return;
  const WeighReq &rq = *un.rq;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;
  const uint32_t P = (uint32_t)a.g.page_tokens, t0 = un.tile * C::KEYS, b0 = t0 + wave * C::KW;
  const Blocks bl = weigh_blocks(a, rq, t0, min(t0 + C::KEYS, rq.ctx), un.split);

  // ---- K: lane holds key 32 kb + col, dims 16 ks + 8 half .. + 7
  bf16x8 kf[KB][KS];
  if (bl.from < bl.to) {
    const uint8_t *const head = a.pool + (DK == 576 ? 0ull : (uint64_t)un.kvh * (4ull * P * DK)) + 16 * half;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      uint32_t slot;
      const uint32_t pg = page_divide(min(b0 + 32 * kb + col, rq.ctx - 1), P, a.page_magic, &slot);
      const u32x4e *const k = reinterpret_cast<const u32x4e *>(head + ((uint64_t)a.pte[rq.pte_base + pg] << 8) +
                                                              (uint64_t)slot * (2 * DK));
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) kf[kb][ks] = __builtin_bit_cast(bf16x8, __builtin_nontemporal_load(k + 2 * ks));
    }
  }

  // ---- a block's queries go to LDS directly; rows past the last repeat it
  auto query = [&](uint32_t r) {
    const RowAddr x = row_addr(a, rq, un.kvh, r);
    return (uint64_t)(uintptr_t)a.q + (x.tok * (uint32_t)a.g.hq + x.head) * (2ull * DK);
  };
  auto issue = [&](uint32_t blk, int buf) {
    const uint32_t to = lds_addr(lds) + buf * C::TILE;
    constexpr int CPR = C::LAT / 16, RPI = CPR >= 64 ? 1 : 64 / CPR, N = kWeighBlock / RPI / C::WAVES;
#pragma unroll
    for (int i = 0; i < N; ++i) {  // a wave's instruction: RPI rows
      const int row0 = (wave * N + i) * RPI, row = row0 + lane / CPR;
      lane_load_lds<false>(query(blk * kWeighBlock + row) + 16 * C::lat_piece(row, lane % CPR), to + row0 * C::LAT);
    }
    if constexpr (C::ROT > 0) {
      const int row = 8 * wave + lane / 8;
      lane_load_lds<false>(query(blk * kWeighBlock + row) + C::LAT + 16 * C::rot_piece(row, lane % 8),
                           to + kWeighBlock * C::LAT + 8 * wave * C::ROT);
    }
  };
  float acc[NE];
#pragma unroll
  for (int i = 0; i < NE; ++i) acc[i] = 0.f;

  auto loads = [&](uint32_t blk) { return row_loads(a, row_addr(a, rq, un.kvh, blk * kWeighBlock + col)); };
  RowLoads next{};
  if (bl.from < bl.to) next = loads(bl.from);
  // a wait the compiler sees for K: its own would drain blocks in flight
  __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
  if (bl.from < bl.to) issue(bl.from, 0);
#pragma unroll 1
  for (uint32_t blk = bl.from; blk < bl.to; ++blk) {
    const int buf = (blk - bl.from) & 1;
    const uint32_t r = blk * kWeighBlock + col;
    const WeighRow w = weigh_row(a, rq, row_addr(a, rq, un.kvh, r), next, r);
    const Row &x = w.x;
    wait_vm<0>();
    __syncthreads();  // this block is there for every wave; the one before is done with
    if (blk + 1 < bl.to) {
      next = loads(blk + 1);
      issue(blk + 1, buf ^ 1);
    }
    if (__builtin_amdgcn_ballot_w64(x.lo < b0 + C::KW && x.hi > b0)) {
      const char *const qt = lds + buf * C::TILE;
      f32x16 sc[KB];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[kb][i] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const int c = 2 * ks + half;
        const char *const at = DK == 576 && ks >= 32 ? qt + kWeighBlock * C::LAT + col * C::ROT + 16 * C::rot_piece(col, c - 64)
                                                     : qt + col * C::LAT + 16 * C::lat_piece(col, c);
        const bf16x8 qf = *reinterpret_cast<const bf16x8 *>(at);
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) sc[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[kb][ks], qf, sc[kb], 0, 0, 0);
      }
      // element i of block kb: key b0 + 32 kb + 8 (i / 4) + 4 half + i % 4
      auto &flat = reinterpret_cast<float(&)[NE]>(sc);
      const bool hide = __builtin_amdgcn_ballot_w64(x.lo > b0 || x.hi < b0 + C::KW) != 0;
      const bool behind = MODE == kModeAny && __builtin_amdgcn_ballot_w64(x.pos + 1 < b0 + C::KW) == 0;
      float top;
      auto key_of = [](int i) { return 32 * (i / 16) + 8 * (i % 16 / 4) + i % 4; };
      const bool raw = scores_of<MODE, NE>(a, RowAt{}, flat, w.slope, x, b0 + 4 * half, behind, hide, 0u, key_of, &top);
      weights<MODE, NE>(a, flat, raw, nan_row(flat, w.ref, x, b0 + 4 * half, key_of), [&](int i, float p0, float p1) {
        acc[i] += p0;
        acc[i + 1] += p1;
      });
    }
  }

  // ---- the lanes' sums of a key: 32 lanes of one half
#pragma unroll
  for (int kb = 0; kb < KB; ++kb) {
    float mine = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float s = row_sum_16(acc[16 * kb + i]);
      const auto o = __builtin_amdgcn_permlane16_swap(__float_as_uint(s), __float_as_uint(s), false, false);
      s = __uint_as_float(o[0]) + __uint_as_float(o[1]);
      mine = (col & 15) == i ? s : mine;
    }
    const int i = col & 15;
    const uint32_t key = b0 + 32 * kb + 8 * (i / 4) + 4 * half + i % 4;
    if (col < 16 && key < rq.ctx) put_sum(a, rq, un.kvh, un.split, key, mine);
  }
}

// ------------------------------------------------------------ vector path

// A thread per key, eight rows at a time from LDS, for every geometry. Bound by the vector
// unit and each thread's own row reads; it serves the geometries without a matrix kernel.
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

// The parts of keys whose rows were cut, in order. A thread per KV head and key.
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
    if (a.slopes)
      hipLaunchKernelGGL((weigh_rows_kernel<DK, kModeAny>), grid, block, 0, stream, a);
    else if (a.softcap > 0.f)
      hipLaunchKernelGGL((weigh_rows_kernel<DK, kModeCap>), grid, block, 0, stream, a);
    else
      hipLaunchKernelGGL((weigh_rows_kernel<DK, kModePlain>), grid, block, 0, stream, a);
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
