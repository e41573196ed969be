// gfx950 kernel of attention of token chunks for MLA with a 512-wide latent and a
// 64-wide rotary part, on the matrix cores.
#include <hip/hip_runtime.h>

#include "extend_device.h"

namespace cp {

// A tile is 128 rows, eight waves of 16, two to a SIMD: a wave keeps its queries
// (18 fragments) and all 512 columns of its output sums in registers. A step is
// 32 keys, a 36 KiB piece of LDS that serves K (576 wide) and V (its first 512
// columns). Scores are transposed (S^T = K Q^T, 16x16x32 products: a lane holds
// four of every 16 keys of its row) and, rounded, are the operand P^T of O^T =
// V^T P^T in place. A fragment of 1 KiB feeds 16 rows, 16 cycles of a product:
// four SIMDs ask for the 256 bytes a cycle that LDS gives (544 KiB a step, 2,180 cycles
// of LDS and as many of products). With every CU full (two requests of 16 K keys, the
// last 2,048 tokens of each, 16 heads; warm) they reach 961 TFLOP/s, and 1,087 with 128
// heads and 512 tokens; where half of the CUs run short contexts the matrix cores are
// 41% busy, LDS 42%, the vector unit 38%: a step's scores, softmax and sums are a chain
// that two waves a SIMD cover in part. 32 rows a wave would halve the reads, but
// their sums and queries do not fit in registers.
// Probabilities are rounded to one bf16 part (2.0e-3 from 64 bits instead of 1.7e-3):
// with a second part, a second product for every fragment of V, prompts of 1,024 tokens
// took 353 us instead of 285, and drafts of 5 tokens 58 instead of 50.
//
// KV goes from the pool to LDS directly, NBUF - 1 steps ahead, a load for a row's
// latent part and one for eight rows' rotary parts. The lane for a 16-byte place of
// LDS loads the piece that belongs there: the pieces of latent row r are swapped by
// 2 r mod 16, those of rotary row r by r & 6, and both the reads of K (16 rows at
// one piece) and of V (8 rows at two) meet no bank twice.
struct ExtMla {
  static constexpr int DK = 576, DV = 512, KEYS = 32, WAVES = 8;
  static constexpr int ROW = 2 * DK, MROW = 2 * DV, RROW = ROW - MROW;  // bytes: in the pool; latent; rotary
  static constexpr int RING = KEYS * MROW;  // a step's latent part, the rotary part behind it
  static constexpr int TILE = KEYS * ROW;   // 36 KiB
  static constexpr int NBUF = 3;
  static constexpr int KS = DK / 32, DB = DV / 16;
  static constexpr int MLOADS = KEYS / WAVES;  // latent rows of a wave; waves 0 to 3 load eight rotary rows each too
  static constexpr int PTAB = 1024;            // page-table entries kept in LDS
  static constexpr int OFF_TAB = NBUF * TILE;
  static constexpr int LDS = OFF_TAB + 4 * PTAB;
  static_assert(MROW == 1024 && RROW == 128 && LDS + 512 <= 163840, "LDS budget");
};
CP_DEV int latent_swap(int row) { return (2 * row) & 15; }
CP_DEV int rotary_swap(int row) { return row & 6; }

template <int MODE, bool NT>
__global__ __launch_bounds__(64 * ExtMla::WAVES, 2) void extend_mla_kernel(const ExtArgs a) {
  using C = ExtMla;
  __shared__ __attribute__((aligned(16))) char lds[C::LDS];
  __shared__ uint32_t shared_u[C::WAVES][4];
  uint32_t *const ptab = reinterpret_cast<uint32_t *>(lds + C::OFF_TAB);
  const Unit un = find_unit(a);
  if (un.none) return;
  const ExtReq &rq = *un.rq;
  const GeomK &g = a.g;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, quad = lane >> 4;
  const uint32_t P = (uint32_t)g.page_tokens, rows = rq.n_tok * (uint32_t)g.g;

  const uint32_t r = un.tile * 128 + 16 * wave + col;
  auto row_now = [&] { return un.tile * 128 + 16 * wave + (uint32_t)lane_ids().col; };
  const bool busy = un.tile * 128 + 16 * wave < rows;  // else the wave only loads
  const Row x = row_of<is_tree(MODE)>(a, rq, un.kvh, r);
  const Sight ws = wave_sight<8, is_tree(MODE)>(x);
  const Sight gs = group_sight<C::WAVES>(ws, wave, lane, shared_u);
  const uint32_t first = gs.lo / C::KEYS, last = (gs.hi + C::KEYS - 1) / C::KEYS, steps = last - first;
  const uint32_t s0 = first + (uint32_t)((uint64_t)steps * un.split / rq.splits),
                 s1 = first + (uint32_t)((uint64_t)steps * (un.split + 1) / rq.splits);

  // ---- loads
  uint32_t tab0 = 0, tab_n = 0;  // pages whose entries are in LDS: [tab0, tab0 + tab_n)
  auto issue = [&](uint32_t s) {
    uint32_t slot, rest;
    const uint32_t lo = min(max(s * C::KEYS, gs.lo), gs.hi - 1), hi = min(s * C::KEYS + C::KEYS, gs.hi) - 1;
    const uint32_t pl = page_divide(lo, P, a.page_magic, &rest), ph = page_divide(max(hi, lo), P, a.page_magic, &rest);
    if (pl < tab0 || ph >= tab0 + tab_n) {  // (at most once in 31 steps; every wave is here)
      __syncthreads();
      tab0 = pl;
      tab_n = C::PTAB;
      const uint32_t end = page_divide(gs.hi - 1, P, a.page_magic, &rest);
      for (uint32_t i = threadIdx.x; i < C::PTAB; i += 64 * C::WAVES) ptab[i] = a.pte[rq.pte_base + min(tab0 + i, end)];
      __syncthreads();
    }
    // lane i looks key i up; out of sight, the nearest in sight (the lane is
    // counted afresh: what follows from it is formed here, not kept through the loop)
    const int ln = lane_ids().lane;
    const uint32_t key = min(max(s * C::KEYS + (ln & 31), gs.lo), gs.hi - 1);
    const uint32_t pte = ptab[page_divide(key, P, a.page_magic, &slot) - tab0];
    slot *= C::ROW;
    const uint32_t buf = lds_addr(lds) + ((s - s0) % C::NBUF) * C::TILE;
#pragma unroll
    for (int j = 0; j < C::MLOADS; ++j) {
      const int row = C::MLOADS * wave + j;
      const uint64_t base = (uint64_t)(uintptr_t)a.pool + ((uint64_t)(uint32_t)__builtin_amdgcn_readlane(pte, row) << 8) +
                            (uint32_t)__builtin_amdgcn_readlane(slot, row);
      row_load_lds<NT>(base, 16u * (uint32_t)(ln ^ latent_swap(row)), buf + row * C::MROW);
    }
    if (wave < 4) {
      const int row = 8 * wave + (ln >> 3);
      const uint64_t base = (uint64_t)(uintptr_t)a.pool + ((uint64_t)(uint32_t)__shfl((int)pte, row, 64) << 8) +
                            (uint32_t)__shfl((int)slot, row, 64) + C::MROW + 16 * ((ln & 7) ^ rotary_swap(row));
      lane_load_lds<NT>(base, buf + C::RING + 8 * wave * C::RROW);
    }
  };

  // ---- Q^T: lane holds row `col`, dims 32 ks + 8 quad .. + 7
  bf16x8 qf[C::KS];
  {
    const uint16_t *const qrow = a.q + (x.tok * (uint32_t)g.hq + x.head) * C::DK + 8 * quad;
#pragma unroll
    for (int ks = 0; ks < C::KS; ++ks) qf[ks] = *reinterpret_cast<const bf16x8 *>(qrow + 32 * ks);
  }
  const float slope = is_any(MODE) && a.slopes ? a.slopes[x.head] * kLog2e : 0.f;
  // a wait the compiler sees: its own at the first use would drain the steps in flight
  __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);

  float m = -INFINITY, l = 0.f;
  f32x4 o[C::DB];
#pragma unroll
  for (int d = 0; d < C::DB; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};

  // LDS byte offsets in a step's tile, formed afresh in each step (kept through the loop
  // they would cost 13 registers). K of keys 16 u + col, dims 32 ks + 8 quad: latent at
  // k[ks % 4] + 256 (ks / 4) + 16 u rows, rotary (ks 16, 17) at r ^ 64 (ks - 16) + 16 u
  // rows.
  struct KAt {
    uint32_t k[4], r;
  };
  auto k_at = [] {
    const LaneIds L = lane_ids();
    KAt x;
    x.r = (uint32_t)(C::RING + L.col * C::RROW + 16 * (L.quad ^ rotary_swap(L.col)));
#pragma unroll
    for (int k = 0; k < 4; ++k) x.k[k] = (uint32_t)(L.col * C::MROW + 16 * ((4 * k + L.quad) ^ latent_swap(L.col)));
    return x;
  };
  // V^T of a step's keys 4 quad + {0..3} and 16 on, and block d of 16 columns
  auto v_frag = [&](const char *tb, const LaneIds &L, int d) {
    const int vr = 4 * L.quad + (L.col >> 2);
    const char *const at = tb + vr * C::MROW + 8 * (L.col & 1) +
                           16 * ((2 * (d % 8) + ((L.col >> 1) & 1)) ^ latent_swap(vr)) + 256 * (d / 8);
    s16x4 f[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
      f[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(at + 16 * h * C::MROW));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(f[0], f[1], 0, 1, 2, 3, 4, 5, 6, 7));
  };
  // Does some row of the workgroup not see some key of step s?
  auto mixed = [&](uint32_t s) { return s * C::KEYS < gs.all_lo || s * C::KEYS + C::KEYS > gs.all_hi; };
  uint32_t sp_first = 0xFFFFFFFFu, sp_last = 0;

  for (uint32_t s = s0; s < s1 && s < s0 + C::NBUF - 1; ++s) issue(s);
#pragma unroll 1
  for (uint32_t s = s0; s < s1; ++s) {
    // own loads of step s have landed once at most the next step's remain
    if (s + 1 == s1) wait_vm<0>();
    else if (wave < 4) wait_vm<5>();
    else wait_vm<4>();
    __syncthreads();  // step s is there for every wave; step s - 1 is done with
    if (s + C::NBUF - 1 < s1) issue(s + C::NBUF - 1);
    char *const tb = lds + ((s - s0) % C::NBUF) * C::TILE;
    const bool mix = mixed(s);
    const uint32_t k0 = s * C::KEYS + 4 * quad;  // element (u, i): key k0 + 16 u + i
    f32x4 sc[2];
    if (busy) {
#pragma unroll
      for (int u = 0; u < 2; ++u) sc[u] = f32x4{0.f, 0.f, 0.f, 0.f};
      // fragments are read KD products ahead, in this order (left to itself the
      // compiler reads one or two ahead, and the products wait for LDS)
      constexpr int KD = 4;
      bf16x8 kf[KD + 1];
      const KAt at = k_at();
      auto kread = [&](int e) {
        const int ks = e / 2, u = e % 2;
        return *reinterpret_cast<const bf16x8 *>(
            tb + (ks < 16 ? at.k[ks % 4] + 256 * (ks / 4) + 16 * u * C::MROW : (at.r ^ (64 * (ks - 16))) + 16 * u * C::RROW));
      };
#pragma unroll
      for (int e = 0; e < KD; ++e) kf[e] = kread(e);
#pragma unroll
      for (int e = 0; e < 2 * C::KS; ++e) {
        if (e + KD < 2 * C::KS) kf[(e + KD) % (KD + 1)] = kread(e + KD);
        __builtin_amdgcn_sched_barrier(0);
        sc[e % 2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[e % (KD + 1)], qf[e / 2], sc[e % 2], 0, 0, 0);
      }
    }
    if (mix) {
      // infinities and NaN of V stay out of the products (0 times those is
      // no 0): they are made 0 in LDS once every wave has its scores, and
      // the steps that had any are gone through again at the end
      __syncthreads();
      bool any = false;
      for (int e = threadIdx.x; e < C::RING / 16; e += 64 * C::WAVES) {
        u32x4e *const w = reinterpret_cast<u32x4e *>(tb) + e;
        if (any_special(*w)) {
          any = true;
          *w = without_special(*w);
        }
      }
      if (__builtin_amdgcn_ballot_w64(any)) {
        sp_first = min(sp_first, s);
        sp_last = s;
      }
      __syncthreads();
    }
    if (!busy) continue;
    // the first fragments of V arrive during the softmax
    constexpr int VD = MODE == kModeTreeAny ? 2 : 4;  // (with 4 a query fragment would spill)
    bf16x8 vf[VD + 1];
    const LaneIds vl = lane_ids();
#pragma unroll
    for (int d = 0; d < VD; ++d) vf[d] = v_frag(tb, vl, d);
    __builtin_amdgcn_sched_barrier(0);
    auto &flat = reinterpret_cast<float(&)[8]>(sc);
    float t;
    uint32_t bits = 0;
    if (is_tree(MODE) && mix) bits = (uint32_t)(tree_bits<C::KEYS>(a, tree_row(a, rq, un.kvh, row_now()), s * C::KEYS) >> (4 * quad));
    const bool raw = scores_of<MODE, 8>(a, RowAt{&rq, un.kvh, row_now()}, flat, slope, x, k0, s * C::KEYS + C::KEYS <= ws.behind, mix, bits,
                                        [](int i) { return 16 * (i / 4) + i % 4; }, &t);
    if (__builtin_amdgcn_ballot_w64(t > m + kLazy || (m == -INFINITY && t > m))) {
      const float mt = xor_max_16_32(t);
      const float mn = mt > m + kLazy || m == -INFINITY ? __builtin_fmaxf(mt, m) : m;
      const float al = mn == -INFINITY ? 1.f : fast_exp2(m - mn);
      m = mn;
      l *= al;
#pragma unroll
      for (int d = 0; d < C::DB; ++d) o[d] *= al;
    }
    const float ref = m == -INFINITY ? 0.f : m;
    uint32_t pw[4];
    weights<MODE, 8>(a, flat, raw, ref, [&](int i, float p0, float p1) {
      l += p0 + p1;
      pw[i / 2] = pack_bf16x2(p0, p1);
    });
    const bf16x8 pf = __builtin_bit_cast(bf16x8, u32x4e{pw[0], pw[1], pw[2], pw[3]});
#pragma unroll
    for (int d = 0; d < C::DB; ++d) {
      if (d + VD < C::DB) vf[(d + VD) % (VD + 1)] = v_frag(tb, vl, d + VD);
      __builtin_amdgcn_sched_barrier(0);
      o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[d % (VD + 1)], pf, o[d], 0, 0, 0);
    }
  }

  // ---- infinities and NaN of V that not every row sees: which rows see one is a
  // product of ones, and their sums get it added
  __syncthreads();
  if (lane == 0) {
    shared_u[wave][0] = sp_first;
    shared_u[wave][1] = sp_last;
  }
  __syncthreads();
  uint32_t from = 0xFFFFFFFFu, to = 0;
#pragma unroll
  for (int w = 0; w < C::WAVES; ++w) {
    from = min(from, shared_u[w][0]);
    to = max(to, shared_u[w][1]);
  }
  from = __builtin_amdgcn_readfirstlane(from);
  to = __builtin_amdgcn_readfirstlane(to);
  if (__builtin_expect(from <= to, 0)) {
#pragma unroll 1
    for (uint32_t s = from; s <= to; ++s) {
      if (!mixed(s)) continue;
      __syncthreads();
      issue(s);
      wait_vm<0>();
      __syncthreads();
      if (!busy) continue;
      const char *const tb = lds + ((s - s0) % C::NBUF) * C::TILE;
      const uint32_t k0 = s * C::KEYS + 4 * quad, lo = x.lo - k0, n = x.hi - x.lo;
      const uint64_t bits = is_tree(MODE) ? tree_bits<C::KEYS>(a, tree_row(a, rq, un.kvh, row_now()), s * C::KEYS) >> (4 * quad) : ~0ull;
      const LaneIds vl = lane_ids();
      u32x4e seen;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t e = 16 * (k / 2) + 2 * (k % 2);
        seen[k] = ((is_tree(MODE) ? bits >> e & 1 : e - lo < n) ? 0x3F80u : 0u) |
                  ((is_tree(MODE) ? bits >> (e + 1) & 1 : e + 1 - lo < n) ? 0x3F800000u : 0u);
      }
#pragma unroll
      for (int d = 0; d < C::DB; ++d)
#pragma unroll 1
        for (uint32_t sign = 0; sign < 2; ++sign) {
          f32x4 hit = {0.f, 0.f, 0.f, 0.f};
          hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(special_ones(v_frag(tb, vl, d), sign),
                                                        __builtin_bit_cast(bf16x8, seen), hit, 0, 0, 0);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (hit[i] > 0.f) o[d][i] += sign ? -INFINITY : INFINITY;
          __builtin_amdgcn_sched_barrier(0);
        }
    }
  }

  // ---- results: columns 16 d + 4 quad + {0..3} of row `col`
  l = xor_sum_16_32(l);
  if (r >= rows) return;
  const bool none = l == 0.f;  // (all scores NaN: l is NaN, and so are the results)
  const float inv = none ? 0.f : 1.f / l, lse = none ? -INFINITY : m + fast_log2(l);
  if (rq.all > 1) {
    const uint64_t pr = part_row(a, rq, x, un.split);
    if (quad == 0) a.ws_l[pr] = lse;
    if (none) return;  // (the join takes no sums of such a range)
#pragma unroll
    for (int d = 0; d < C::DB; ++d)
      *reinterpret_cast<f32x4 *>(a.ws_o + pr * C::DV + 16 * d + 4 * quad) = o[d] * inv;
  } else {
    const uint64_t orow = x.tok * (uint32_t)g.hq + x.head;
#pragma unroll
    for (int d = 0; d < C::DB; ++d) {
      const uint2 w = bf16x4_bits(o[d][0] * inv, o[d][1] * inv, o[d][2] * inv, o[d][3] * inv);
      *reinterpret_cast<uint2 *>(a.out + orow * C::DV + 16 * d + 4 * quad) = none ? uint2{0u, 0u} : w;
    }
    if (quad == 0) a.lse[orow] = lse * kLn2;
  }
}

namespace {
template <bool NT>
void launch_mla(const ExtArgs &a, hipStream_t stream) {
  const dim3 grid((uint32_t)a.n_units), block(64 * ExtMla::WAVES);
  if (a.tree_mask && (a.slopes || a.softcap > 0.f))
    hipLaunchKernelGGL((extend_mla_kernel<kModeTreeAny, NT>), grid, block, 0, stream, a);
  else if (a.tree_mask)
    hipLaunchKernelGGL((extend_mla_kernel<kModeTree, NT>), grid, block, 0, stream, a);
  else if (a.slopes)
    hipLaunchKernelGGL((extend_mla_kernel<kModeAny, NT>), grid, block, 0, stream, a);
  else if (a.softcap > 0.f)
    hipLaunchKernelGGL((extend_mla_kernel<kModeCap, NT>), grid, block, 0, stream, a);
  else
    hipLaunchKernelGGL((extend_mla_kernel<kModePlain, NT>), grid, block, 0, stream, a);
}
}  // namespace

void launch_extend_mla(const ExtArgs &a, hipStream_t stream) {
  // one tile per request: its KV is read once
  bool once = true;
  for (int i = 0; i < a.n_req; ++i) once = once && a.req[i].tiles == 1;
  once ? launch_mla<true>(a, stream) : launch_mla<false>(a, stream);
}

}  // namespace cp
