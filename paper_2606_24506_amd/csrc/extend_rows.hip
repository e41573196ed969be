// gfx950 kernels of attention of token chunks for GQA and MHA of head_dim 64 and
// 128, on the matrix cores.
#include <hip/hip_runtime.h>

#include "extend_device.h"

namespace cp {

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
// next step's keys go to LDS directly while this one's are worked on (through
// registers, the loads' shuffles and LDS stores were a fifth of the vector unit's
// work, and 40 registers). Bound by the vector unit (exponentials, cap) and the
// matrix cores, which overlap only as far as two workgroups a CU take turns; LDS reads
// for 32 rows (1 KiB a product of 32 cycles, four SIMDs, at 256 bytes a cycle) take half
// as long as the products. Two requests of 16 K keys, the last 2,048 tokens of each, 32
// query heads over 8, the card warm: 936 TFLOP/s plain, 813 under a cap of 50, 797
// sloped; 16 over 4 heads of head_dim 64 759, 576, 568. (From idle the clock is lower
// for some 10 ms. Steps measured there: 886 plain, 782 capped, 774 sloped; with no
// fragments read ahead 847, 730, 718; with loads through registers too 810, 726, 732.
// Steps of 32 keys and three workgroups a CU: 660 sloped.) A cap of the scores' size
// takes the tangent's other form: 555 under a cap of 2.
// Probabilities are rounded to one bf16 part, off by at most 2^-8 of themselves, as the
// outputs are: these are 2.0e-3 to 2.4e-3 from 64 bits instead of 1.6e-3 to 1.8e-3 (the
// root of the mean square, of the values'). Two parts (RW = 1) took 1,304 us instead of 1,008 on capped prompts
// of 16 K, 9 K and 4 K tokens, and 47 instead of 40 on packed documents of 700.
// RW = 1: 32 rows, every wave with 32 keys of its own a step (few rows: bound
// by reading KV); the waves' sums join at the end. Its loads pass through
// registers, because a wave's keys are its own and no barrier is needed.
template <int D, int RW>
struct ExtCfg {
  static constexpr int KW = RW == 4 ? 64 : 32;        // keys of a wave's step
  static constexpr int KEYS = RW == 4 ? 64 : 128;     // keys of a workgroup's step
  static constexpr int ROW = 2 * D;                   // bytes
  static constexpr int CPR = D / 8;                   // 16-byte pieces of a row
  static constexpr int TILE = KW * ROW;               // bytes of K (or V) of a step of a wave's keys
  static constexpr int BUFS = RW == 4 ? 2 : 4;        // double buffer, or one for each wave
  static constexpr int RPI = 64 / CPR;                // rows that a wave loads at once
  static constexpr int NL = KW / RPI;                 // 16-byte loads of K (and of V) of a thread (RW 1)
  static constexpr int KB = KW / 32;                  // blocks of 32 keys
  static constexpr int NP = RW == 4 ? 1 : 2;          // bf16 parts of a probability
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

// What a probability has behind its leading 8 bits h, with its last bit set: an infinite V
// that is seen times a part that is 0 would be NaN. (A floor of 1e-37 instead gave
// hidden keys, and those that weigh less, that much of a large V. The last bit of 0 is
// 2^-149, which the rounding to bf16 drops: what weighs nothing stays at nothing.)
CP_DEV float low_part(float p, uint32_t h) { return __uint_as_float(__float_as_uint(p) | 1u) - __uint_as_float(h); }

// Results of a tile of ROWS rows from its four waves' m, l and sums (parts: [wave][column]
// [row] in LDS). A thread takes D ROWS / 256 columns of one row.
template <int D, int ROWS>
CP_DEV void join_waves(const ExtArgs &a, const ExtReq &rq, const Unit &un, const float *parts,
                       const float (&stats)[2][4][ROWS]) {
  constexpr int NC = D * ROWS / kExtThreads;
  const int row = threadIdx.x % ROWS, c0 = threadIdx.x / ROWS * NC;
  const uint32_t r = un.tile * ROWS + row;
  if (r >= rq.n_tok * (uint32_t)a.g.g) return;
  const Row y = row_of(a, rq, un.kvh, r);
  float mt = stats[0][0][row];
#pragma unroll
  for (int w = 1; w < 4; ++w) mt = __builtin_fmaxf(mt, stats[0][w][row]);
  const float ref = mt == -INFINITY ? 0.f : mt;
  float f[4], sum = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    f[w] = fast_exp2(stats[0][w][row] - ref);
    sum += f[w] * stats[1][w][row];
  }
  const bool none = sum == 0.f;
  const float inv = none ? 0.f : 1.f / sum, lse = none ? -INFINITY : mt + fast_log2(sum);
  float v[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    float acc = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w)  // a wave that saw nothing of the row has nothing to add; sums of weight 0 may be NaN
      if (stats[0][w][row] != -INFINITY) acc += f[w] * parts[w * ROWS * D + (c0 + c) * ROWS + row];
    v[c] = acc * inv;
  }
  if (rq.all > 1) {
    const uint64_t pr = part_row(a, rq, y, un.split);
    if (c0 == 0) a.ws_l[pr] = lse;
    if (none) return;  // (the join takes no sums of such a range)
#pragma unroll
    for (int c = 0; c < NC; c += 4)
      *reinterpret_cast<f32x4 *>(a.ws_o + pr * D + c0 + c) = f32x4{v[c], v[c + 1], v[c + 2], v[c + 3]};
  } else {
    const uint64_t orow = y.tok * (uint32_t)a.g.hq + y.head;
#pragma unroll
    for (int c = 0; c < NC; c += 4)
      *reinterpret_cast<uint2 *>(a.out + orow * D + c0 + c) = bf16x4_bits(v[c], v[c + 1], v[c + 2], v[c + 3]);
    if (c0 == 0) a.lse[orow] = lse * kLn2;
  }
}

template <int D, int RW, int MODE>
__global__ __launch_bounds__(kExtThreads, 2) void extend_rows_kernel(const ExtArgs a) {
  using C = ExtCfg<D, RW>;
  constexpr int KS = D / 16, DB = D / 32;
  __shared__ __attribute__((aligned(16))) char lds[C::LDS];
  __shared__ uint32_t shared_u[4][4];
  __shared__ float stats[2][4][32];  // RW 1: the waves' m and l
  const Unit un = find_unit(a);
  if (un.none) return;
  const ExtReq &rq = *un.rq;
  const GeomK &g = a.g;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5, c16 = lane & 15, grp = (lane >> 4) & 1;
  const uint32_t P = (uint32_t)g.page_tokens;

  // ---- this lane's row, what its wave sees, and what the workgroup sees
  const uint32_t r = un.tile * (32 * RW) + (RW == 4 ? 32 * wave : 0) + col;
  const Row x = row_of(a, rq, un.kvh, r);
  const Sight ws = wave_sight<16>(x);
  const Sight gs = RW == 4 ? group_sight<4>(ws, wave, lane, shared_u) : ws;
  // steps of the unit: whole steps from a multiple of KEYS on
  const uint32_t first = gs.lo / C::KEYS, last = (gs.hi + C::KEYS - 1) / C::KEYS, steps = last - first;
  const uint32_t s0 = first + (uint32_t)((uint64_t)steps * un.split / rq.splits),
                 s1 = first + (uint32_t)((uint64_t)steps * (un.split + 1) / rq.splits);

  // ---- Q^T: lane holds row `col`, dims 16 ks + 8 half .. + 7
  bf16x8 qf[KS];
  {
    const uint16_t *const qrow = a.q + (x.tok * (uint32_t)g.hq + x.head) * D + 8 * half;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const bf16x8 *>(qrow + 16 * ks);
  }
  const float slope = MODE == kModeAny && a.slopes ? a.slopes[x.head] * kLog2e : 0.f;

  float m = -INFINITY, l = 0.f;
  f32x16 o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.f;

  // ---- loads. RW 1: a lane takes piece lc of rows lr, lr + RPI, ... of a step. Lane
  // i of every wave looks key i up, a step ahead; keys out of sight are looked up
  // as the nearest one in sight (they are hidden below, and never stale memory).
  const int lc = lane % C::CPR, lr = lane / C::CPR;
  const uint8_t *const head_base = a.pool + (uint64_t)un.kvh * (4ull * P * D) + 16 * lc;
  u32x4e kreg[C::NL], vreg[C::NL];
  // keys of step s: RW 4, [64 s, + 64); RW 1, wave w has [128 s + 32 w, + 32)
  auto base_of = [&](uint32_t s) { return s * C::KEYS + (RW == 4 ? 0u : 32u * wave); };
  uint32_t key_pte = 0, key_slot = 0;
  auto look_up = [&](uint32_t s) {
    const uint32_t key = min(max(base_of(s) + (lane & (C::KW - 1)), gs.lo), gs.hi - 1);
    key_pte = a.pte[rq.pte_base + page_divide(key, P, a.page_magic, &key_slot)];
  };
  auto load_v = [&](int i, const uint8_t *kp) {
    const u32x4e *const p = reinterpret_cast<const u32x4e *>(kp + (uint64_t)P * C::ROW);
    vreg[i] = __builtin_nontemporal_load(p);
  };
  auto row_ptr = [&](int i) {
    const int row = lr + C::RPI * i;
    const uint32_t pte = (uint32_t)__shfl((int)key_pte, row, 64), slot = (uint32_t)__shfl((int)key_slot, row, 64);
    return head_base + ((uint64_t)pte << 8) + slot * C::ROW;
  };
  auto load_keys = [&] {
#pragma unroll
    for (int i = 0; i < C::NL; ++i) {
      const uint8_t *const kp = row_ptr(i);
      const u32x4e *const p = reinterpret_cast<const u32x4e *>(kp);
      kreg[i] = __builtin_nontemporal_load(p);
    }
  };
  // RW 1 asks for the next V once the scores' registers are free: 64 registers of
  // loads in flight beside them do not fit
  auto load_values = [&] {
#pragma unroll
    for (int i = 0; i < C::NL; ++i) load_v(i, row_ptr(i));
  };
  // RW 4: a wave's quarter of a step straight to LDS, 1 KiB a load. The lane for a
  // 16-byte place of LDS loads the piece that belongs there (the swaps undo themselves).
  auto issue = [&](int buf, bool keys, bool values) {
    const uint32_t kt = lds_addr(lds) + buf * (2 * C::TILE), vt = kt + C::TILE;
    const uint32_t ln = (uint32_t)lane_ids().lane;  // (counted afresh: formed here, not kept through the loop)
    const uint32_t row0 = wave * (C::KW / 4), r0 = row0 + ln / C::CPR, p = ln % C::CPR;
    constexpr int N = C::KW / 4 / C::RPI;
    // rows of 256 bytes have one number for page and slot, in units of the page table
    const uint32_t key_at = C::ROW == 256 ? key_pte + key_slot : key_pte;
    uint32_t at[N], slot[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      at[i] = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * (r0 + C::RPI * i), (int)key_at);
      slot[i] = C::ROW == 256 ? 0u : (uint32_t)__builtin_amdgcn_ds_bpermute(4 * (r0 + C::RPI * i), (int)key_slot);
    }
    const uint64_t head = (uint64_t)(uintptr_t)a.pool + (uint64_t)un.kvh * (4ull * P * D);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t row = r0 + C::RPI * i, to = (row0 + C::RPI * i) * C::ROW;
      const uint64_t base = head + ((uint64_t)at[i] << 8);
      const uint32_t in_page = slot[i] * C::ROW;
      if (keys) lane_load_lds<false>(base + (in_page + 16u * k_piece<D>(row, p)), kt + to);
      if (values) lane_load_lds<false>(base + (uint64_t)P * C::ROW + (in_page + 16u * v_piece<D>(row, p)), vt + to);
    }
  };
  // Are there keys of step s that some row of the workgroup does not see? Then
  // infinities and NaN of V stay out of the products (0 times those is no
  // 0), and the steps that had any are gone through again at the end.
  auto mixed = [&](uint32_t s) {
    const uint32_t b = base_of(s);
    return b < gs.all_lo || b + C::KW > gs.all_hi;
  };
  uint32_t sp_first = 0xFFFFFFFFu, sp_last = 0;
  auto note_special = [&](uint32_t s, bool any) {
    if (!__builtin_amdgcn_ballot_w64(any)) return false;
    sp_first = min(sp_first, s);
    sp_last = s;
    return true;
  };
  auto clean_values = [&](int buf, uint32_t s) {  // RW 4, in LDS
    bool any = false;
    for (int e = threadIdx.x; e < C::TILE / 16; e += kExtThreads) {
      u32x4e *const w = reinterpret_cast<u32x4e *>(lds + buf * (2 * C::TILE) + C::TILE) + e;
      if (any_special(*w)) {
        any = true;
        *w = without_special(*w);
      }
    }
    note_special(s, any);
    __syncthreads();
  };
  auto store_keys = [&](int buf, uint32_t s) {  // RW 1
    char *const kt = lds + buf * (2 * C::TILE), *const vt = kt + C::TILE;
    if (mixed(s)) {
      bool any = false;
#pragma unroll
      for (int i = 0; i < C::NL; ++i) any = any || any_special(vreg[i]);
      if (note_special(s, any)) {
#pragma unroll
        for (int i = 0; i < C::NL; ++i) vreg[i] = without_special(vreg[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < C::NL; ++i) {
      const int row = lr + C::RPI * i;
      *reinterpret_cast<u32x4e *>(kt + row * C::ROW + 16 * k_piece<D>(row, lc)) = kreg[i];
      *reinterpret_cast<u32x4e *>(vt + row * C::ROW + 16 * v_piece<D>(row, lc)) = vreg[i];
    }
  };
  // V^T of 16 keys and block d of 32 columns
  auto v_frag = [&](const char *vt, int kb, int ks, int d) {
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

  // ---- one step over the keys in a buffer
  constexpr int AHEAD = RW == 1 ? 0 : D == 128 ? 4 : 2;  // (6 and 2: the same; 4 with head_dim 64: 1% slower)
  auto compute = [&](int buf, uint32_t s, bool more) {
    const uint32_t b0 = base_of(s);
    if (b0 >= ws.hi || b0 + C::KW <= ws.lo) {  // out of this wave's sight
      if (RW == 1 && more) load_values();
      return;
    }
    const char *const kt = lds + buf * (2 * C::TILE), *const vt = kt + C::TILE;
    f32x16 sc[C::KB];
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int kb = 0; kb < C::KB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[kb][i] = 0.f;
    // fragments are read KD products ahead, in this order (left to itself the compiler
    // reads one or two ahead, and the products wait for LDS)
    constexpr int KD = AHEAD, NKF = KS * C::KB;
    bf16x8 kf[KD + 1];
    auto kread = [&](int e) {
      const int row = 32 * (e % C::KB) + col;
      return *reinterpret_cast<const bf16x8 *>(kt + row * C::ROW + 16 * k_piece<D>(row, 2 * (e / C::KB) + half));
    };
#pragma unroll
    for (int e = 0; e < KD; ++e) kf[e] = kread(e);
#pragma unroll
    for (int e = 0; e < NKF; ++e) {
      if (e + KD < NKF) kf[(e + KD) % (KD + 1)] = kread(e + KD);
      if (RW == 4) __builtin_amdgcn_sched_barrier(0);
      sc[e % C::KB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[e % (KD + 1)], qf[e / C::KB], sc[e % C::KB], 0, 0, 0);
    }
    __builtin_amdgcn_s_setprio(0);
    // the first fragments of V arrive during the softmax
    constexpr int VD = AHEAD, NVF = 2 * C::KB * DB;
    bf16x8 vf[VD + 1];
    auto vread = [&](int e) { return v_frag(vt, e / (2 * DB), e / DB % 2, e % DB); };
    if (RW == 4) {
#pragma unroll
      for (int e = 0; e < VD; ++e) vf[e] = vread(e);
      __builtin_amdgcn_sched_barrier(0);
    }
    // element i of block kb: key b0 + 32 kb + 8 (i / 4) + 4 half + i % 4
    const uint32_t k0 = b0 + 4 * half;
    const bool hide = b0 < ws.all_lo || b0 + C::KW > ws.all_hi;
    auto &flat = reinterpret_cast<float(&)[16 * C::KB]>(sc);
    float t;
    const bool raw = scores_of<MODE, 16 * C::KB>(a, flat, slope, x, k0, b0 + C::KW <= ws.pos + 1, hide,
                                                 [](int i) { return 32 * (i / 16) + 8 * (i % 16 / 4) + i % 4; }, &t);
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
    weights<MODE, 16 * C::KB>(a, flat, raw, ref, [&](int i, float p0, float p1) {
      l += p0 + p1;
      if constexpr (C::NP == 1) {
        pw[0][i / 16][i % 16 / 2] = pack_bf16x2(p0, p1);
      } else {
        // leading 8 bits, and the rest rounded: together 16 bits and a half step
        const uint32_t h0 = __float_as_uint(p0) & 0xFFFF0000u, h1 = __float_as_uint(p1) & 0xFFFF0000u;
        pw[0][i / 16][i % 16 / 2] = upper_halves(h0, h1);
        pw[1][i / 16][i % 16 / 2] = pack_bf16x2(low_part(p0, h0), low_part(p1, h1));
      }
    });
    if (RW == 1 && more) load_values();
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int e = 0; e < NVF; ++e) {
      if (e + VD < NVF) vf[(e + VD) % (VD + 1)] = vread(e + VD);
      if (RW == 4) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int part = 0; part < C::NP; ++part) {
        const uint32_t *const w = &pw[part][e / (2 * DB)][4 * (e / DB % 2)];
        o[e % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            vf[e % (VD + 1)], __builtin_bit_cast(bf16x8, u32x4e{w[0], w[1], w[2], w[3]}), o[e % DB], 0, 0, 0);
      }
    }
    __builtin_amdgcn_s_setprio(0);
  };

  // ---- the steps
  if constexpr (RW == 4) {
    // a wait the compiler sees for what it has loaded: its own would drain steps in flight
    if (s0 < s1) look_up(s0);
    __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
    if (s0 < s1) issue(0, true, true);
    if (s0 + 1 < s1) look_up(s0 + 1);
  } else if (s0 < s1) {
    look_up(s0);
    load_keys();
    load_values();
    if (s0 + 1 < s1) look_up(s0 + 1);
  }
#pragma unroll 1
  for (uint32_t s = s0; s < s1; ++s) {
    const bool more = s + 1 < s1;
    if constexpr (RW == 4) {
      const int buf = (s - s0) & 1;
      __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
      __syncthreads();  // step s is there for every wave; step s - 1 is done with
      if (more) {
        issue(buf ^ 1, true, true);
        if (s + 2 < s1) look_up(s + 2);
      }
      if (mixed(s)) clean_values(buf, s);
      compute(buf, s, more);
    } else {
      store_keys(wave, s);
      if (more) load_keys();
      // a wave's LDS operations run in order: its reads follow its writes
      __builtin_amdgcn_wave_barrier();
      compute(wave, s, more);
      if (s + 2 < s1) look_up(s + 2);
      __builtin_amdgcn_wave_barrier();
    }
  }

  // ---- infinities and NaN of V that not every row sees: which rows see one is a
  // product of ones, and their sums get it added
  if (RW == 4) {
    __syncthreads();
    if (lane == 0) {
      shared_u[wave][0] = sp_first;
      shared_u[wave][1] = sp_last;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      sp_first = min(sp_first, shared_u[w][0]);
      sp_last = max(sp_last, shared_u[w][1]);
    }
  }
  sp_first = __builtin_amdgcn_readfirstlane(sp_first);
  sp_last = __builtin_amdgcn_readfirstlane(sp_last);
  if (__builtin_expect(sp_first <= sp_last, 0)) {
#pragma unroll 1
    for (uint32_t s = sp_first; s <= sp_last; ++s) {
      if (!mixed(s)) continue;
      char *const vt = lds + (RW == 4 ? C::TILE : wave * (2 * C::TILE));
      look_up(s);
      if constexpr (RW == 4) {
        issue(0, false, true);
        wait_vm<0>();
        __syncthreads();
      } else {
#pragma unroll
        for (int i = 0; i < C::NL; ++i) {
          const int row = lr + C::RPI * i;
          load_v(i, row_ptr(i));
          *reinterpret_cast<u32x4e *>(vt + row * C::ROW + 16 * v_piece<D>(row, lc)) = vreg[i];
        }
      }
      __builtin_amdgcn_wave_barrier();
      const uint32_t k0 = base_of(s) + 4 * half, lo = x.lo - k0, n = x.hi - x.lo;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll 1
        for (uint32_t sign = 0; sign < 2; ++sign) {
          f32x16 hit;
#pragma unroll
          for (int i = 0; i < 16; ++i) hit[i] = 0.f;
#pragma unroll
          for (int kb = 0; kb < C::KB; ++kb)
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
              u32x4e seen;
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const uint32_t e = 32 * kb + 16 * ks + 8 * (k / 2) + 2 * (k % 2);
                seen[k] = (e - lo < n ? 0x3F80u : 0u) | (e + 1 - lo < n ? 0x3F800000u : 0u);
              }
              hit = __builtin_amdgcn_mfma_f32_32x32x16_bf16(special_ones(v_frag(vt, kb, ks, d), sign),
                                                            __builtin_bit_cast(bf16x8, seen), hit, 0, 0, 0);
            }
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (hit[i] > 0.f) o[d][i] += sign ? -INFINITY : INFINITY;
        }
      if (RW == 4) __syncthreads();
      __builtin_amdgcn_wave_barrier();
    }
  }

  // ---- results: column d = 32 db + 8 (i / 4) + 4 half + i % 4 of row `col`
  l += other_half(l);
  if (RW == 4) {
    if (r >= rq.n_tok * (uint32_t)g.g) return;
    const bool none = l == 0.f;  // (all scores NaN: l is NaN, and so are the results)
    const float inv = none ? 0.f : 1.f / l, lse = none ? -INFINITY : m + fast_log2(l);
    if (rq.all > 1) {
      const uint64_t pr = part_row(a, rq, x, un.split);
      if (half == 0) a.ws_l[pr] = lse;
      if (none) return;  // (the join takes no sums of such a range)
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          *reinterpret_cast<f32x4 *>(a.ws_o + pr * D + 32 * d + 2 * i + 4 * half) =
              f32x4{o[d][i] * inv, o[d][i + 1] * inv, o[d][i + 2] * inv, o[d][i + 3] * inv};
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
    join_waves<D, 32>(a, rq, un, reinterpret_cast<const float *>(lds), stats);
  }
}

// At most 16 rows a KV head (single tokens of groups to 16 heads): bound by reading
// KV. As RW = 1 above, but by 16x16x32 products, which leave a lane 8 scores of 32
// keys and not 16, half of them of rows that are not there: the vector unit's
// work for one row a tile halves, and so do the registers of queries and
// sums: capped single tokens over 480 MB of KV take 85 us with the join (89 by RW = 1;
// 6.1 TB/s in the kernel), sloped ones over 537 MB 86 (104; 6.7 TB/s). Lanes are (row
// `col` of 16, quarter `quad`); pieces of LDS rows are swapped so that K reads (16 rows at one piece) and V reads (8 rows at two) meet no bank
// twice.
template <int D>
struct ExtFew {
  static constexpr int KW = 32, KEYS = 128, ROW = 2 * D, CPR = D / 8, TILE = KW * ROW;
  static constexpr int RPI = 64 / CPR, NL = KW / RPI;
  static constexpr int KS = D / 32, DB = D / 16;
  static constexpr int LDS = 8 * TILE;
  static_assert(LDS >= 4 * 16 * D * 4, "the join reuses the tiles");
};
template <int D>
CP_DEV int few_piece(int row, int c) {
  return c ^ (D == 128 ? (2 * row) & 15 : row & 6);
}

template <int D, int MODE>
__global__ __launch_bounds__(kExtThreads, 2) void extend_few_kernel(const ExtArgs a) {
  using C = ExtFew<D>;
  __shared__ __attribute__((aligned(16))) char lds[C::LDS];
  __shared__ float stats[2][4][16];  // the waves' m and l
  const Unit un = find_unit(a);
  if (un.none) return;
  const ExtReq &rq = *un.rq;
  const GeomK &g = a.g;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, quad = lane >> 4;
  const uint32_t P = (uint32_t)g.page_tokens;

  const Row x = row_of(a, rq, un.kvh, un.tile * 16 + col);
  const Sight gs = wave_sight<8>(x);  // every wave has the same rows
  const uint32_t first = gs.lo / C::KEYS, last = (gs.hi + C::KEYS - 1) / C::KEYS, steps = last - first;
  const uint32_t s0 = first + (uint32_t)((uint64_t)steps * un.split / rq.splits),
                 s1 = first + (uint32_t)((uint64_t)steps * (un.split + 1) / rq.splits);

  // ---- loads, as in extend_rows_kernel
  const int lc = lane % C::CPR, lr = lane / C::CPR;
  const uint8_t *const head_base = a.pool + (uint64_t)un.kvh * (4ull * P * D) + 16 * lc;
  u32x4e kreg[C::NL], vreg[C::NL];
  auto base_of = [&](uint32_t s) { return s * C::KEYS + 32u * wave; };
  uint32_t key_pte = 0, key_slot = 0;
  auto look_up = [&](uint32_t s) {
    const uint32_t key = min(max(base_of(s) + (lane & 31), gs.lo), gs.hi - 1);
    key_pte = a.pte[rq.pte_base + page_divide(key, P, a.page_magic, &key_slot)];
  };
  auto row_ptr = [&](int i) {
    const int row = lr + C::RPI * i;
    const uint32_t pte = (uint32_t)__shfl((int)key_pte, row, 64), slot = (uint32_t)__shfl((int)key_slot, row, 64);
    return reinterpret_cast<const u32x4e *>(head_base + ((uint64_t)pte << 8) + slot * C::ROW);
  };
  auto load_keys = [&] {
#pragma unroll
    for (int i = 0; i < C::NL; ++i) {
      const u32x4e *const kp = row_ptr(i);
      kreg[i] = __builtin_nontemporal_load(kp);
      vreg[i] = __builtin_nontemporal_load(kp + P * C::CPR);
    }
  };
  if (s0 < s1) look_up(s0);

  bf16x8 qf[C::KS];
  {
    const uint16_t *const qrow = a.q + (x.tok * (uint32_t)g.hq + x.head) * D + 8 * quad;
#pragma unroll
    for (int ks = 0; ks < C::KS; ++ks) qf[ks] = *reinterpret_cast<const bf16x8 *>(qrow + 32 * ks);
  }
  const float slope = MODE == kModeAny && a.slopes ? a.slopes[x.head] * kLog2e : 0.f;
  float m = -INFINITY, l = 0.f;
  f32x4 o[C::DB];
#pragma unroll
  for (int d = 0; d < C::DB; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};

  char *const kt = lds + wave * (2 * C::TILE), *const vt = kt + C::TILE;
  auto mixed = [&](uint32_t s) {
    const uint32_t b = base_of(s);
    return b < gs.all_lo || b + C::KW > gs.all_hi;
  };
  uint32_t sp_first = 0xFFFFFFFFu, sp_last = 0;
  auto store_v = [&] {
#pragma unroll
    for (int i = 0; i < C::NL; ++i) {
      const int row = lr + C::RPI * i;
      *reinterpret_cast<u32x4e *>(vt + row * C::ROW + 16 * few_piece<D>(row, lc)) = vreg[i];
    }
  };
  auto store_keys = [&](uint32_t s) {
    if (mixed(s)) {
      bool any = false;
#pragma unroll
      for (int i = 0; i < C::NL; ++i) any = any || any_special(vreg[i]);
      if (__builtin_amdgcn_ballot_w64(any)) {
        sp_first = min(sp_first, s);
        sp_last = s;
#pragma unroll
        for (int i = 0; i < C::NL; ++i) vreg[i] = without_special(vreg[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < C::NL; ++i) {
      const int row = lr + C::RPI * i;
      *reinterpret_cast<u32x4e *>(kt + row * C::ROW + 16 * few_piece<D>(row, lc)) = kreg[i];
    }
    store_v();
  };
  // V^T of a step's keys 4 quad + {0..3} and 16 on, and block d of 16 columns
  auto v_frag = [&](int d) {
    const int vr = 4 * quad + (col >> 2);
    s16x4 f[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
      f[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(
          vt + (vr + 16 * h) * C::ROW + 16 * few_piece<D>(vr + 16 * h, 2 * d + ((col >> 1) & 1)) + 8 * (col & 1)));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(f[0], f[1], 0, 1, 2, 3, 4, 5, 6, 7));
  };

  if (s0 < s1) {
    load_keys();
    if (s0 + 1 < s1) look_up(s0 + 1);
  }
#pragma unroll 1
  for (uint32_t s = s0; s < s1; ++s) {
    store_keys(s);
    if (s + 1 < s1) {
      load_keys();
      if (s + 2 < s1) look_up(s + 2);
    }
    // a wave's LDS operations run in order: its reads follow its writes
    __builtin_amdgcn_wave_barrier();
    const uint32_t b0 = base_of(s), k0 = b0 + 4 * quad;  // element (u, i): key k0 + 16 u + i
    if (b0 < gs.hi && b0 + C::KW > gs.lo) {
      f32x4 sc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
      for (int ks = 0; ks < C::KS; ++ks)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int row = 16 * u + col;
          const bf16x8 kf = *reinterpret_cast<const bf16x8 *>(kt + row * C::ROW + 16 * few_piece<D>(row, 4 * ks + quad));
          sc[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[ks], sc[u], 0, 0, 0);
        }
      auto &flat = reinterpret_cast<float(&)[8]>(sc);
      float t;
      const bool raw = scores_of<MODE, 8>(a, flat, slope, x, k0, b0 + C::KW <= gs.pos + 1, mixed(s),
                                          [](int i) { return 16 * (i / 4) + i % 4; }, &t);
      // the reference moves when some row's maximum passes it by 2^kLazy
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
      uint32_t pw[2][4];
      weights<MODE, 8>(a, flat, raw, ref, [&](int i, float p0, float p1) {
        l += p0 + p1;
        // leading 8 bits, and the rest rounded: together 16 bits and a half step
        const uint32_t h0 = __float_as_uint(p0) & 0xFFFF0000u, h1 = __float_as_uint(p1) & 0xFFFF0000u;
        pw[0][i / 2] = upper_halves(h0, h1);
        pw[1][i / 2] = pack_bf16x2(low_part(p0, h0), low_part(p1, h1));
      });
#pragma unroll
      for (int d = 0; d < C::DB; ++d) {
        const bf16x8 vf = v_frag(d);
#pragma unroll
        for (int part = 0; part < 2; ++part)
          o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              vf, __builtin_bit_cast(bf16x8, u32x4e{pw[part][0], pw[part][1], pw[part][2], pw[part][3]}), o[d], 0, 0, 0);
      }
    }
    __builtin_amdgcn_wave_barrier();
  }

  // ---- infinities and NaN of V that not every row sees (as in extend_rows_kernel)
  sp_first = __builtin_amdgcn_readfirstlane(sp_first);
  sp_last = __builtin_amdgcn_readfirstlane(sp_last);
  if (__builtin_expect(sp_first <= sp_last, 0)) {
#pragma unroll 1
    for (uint32_t s = sp_first; s <= sp_last; ++s) {
      if (!mixed(s)) continue;
      look_up(s);
#pragma unroll
      for (int i = 0; i < C::NL; ++i) vreg[i] = row_ptr(i)[P * C::CPR];
      store_v();
      __builtin_amdgcn_wave_barrier();
      const uint32_t k0 = base_of(s) + 4 * quad, lo = x.lo - k0, n = x.hi - x.lo;
      u32x4e seen;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t e = 16 * (k / 2) + 2 * (k % 2);
        seen[k] = (e - lo < n ? 0x3F80u : 0u) | (e + 1 - lo < n ? 0x3F800000u : 0u);
      }
#pragma unroll
      for (int d = 0; d < C::DB; ++d)
#pragma unroll 1
        for (uint32_t sign = 0; sign < 2; ++sign) {
          f32x4 hit = {0.f, 0.f, 0.f, 0.f};
          hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(special_ones(v_frag(d), sign), __builtin_bit_cast(bf16x8, seen),
                                                        hit, 0, 0, 0);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (hit[i] > 0.f) o[d][i] += sign ? -INFINITY : INFINITY;
        }
      __builtin_amdgcn_wave_barrier();
    }
  }

  // ---- the waves' sums joined: columns 16 d + 4 quad + {0..3} of row `col`
  l = xor_sum_16_32(l);
  __syncthreads();  // every wave is done with its tile
  float *const part = reinterpret_cast<float *>(lds) + wave * (16 * D);  // [column][row]
#pragma unroll
  for (int d = 0; d < C::DB; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) part[(16 * d + 4 * quad + i) * 16 + col] = o[d][i];
  if (quad == 0) {
    stats[0][wave][col] = m;
    stats[1][wave][col] = l;
  }
  __syncthreads();
  join_waves<D, 16>(a, rq, un, reinterpret_cast<const float *>(lds), stats);
}

namespace {
template <int D, int RW>
void launch_rows(const ExtArgs &a, hipStream_t stream) {
  const dim3 grid((uint32_t)a.n_units), block(kExtThreads);
  if (a.slopes)
    hipLaunchKernelGGL((extend_rows_kernel<D, RW, kModeAny>), grid, block, 0, stream, a);
  else if (a.softcap > 0.f)
    hipLaunchKernelGGL((extend_rows_kernel<D, RW, kModeCap>), grid, block, 0, stream, a);
  else
    hipLaunchKernelGGL((extend_rows_kernel<D, RW, kModePlain>), grid, block, 0, stream, a);
}
template <int D>
void launch_few(const ExtArgs &a, hipStream_t stream) {
  const dim3 grid((uint32_t)a.n_units), block(kExtThreads);
  if (a.slopes)
    hipLaunchKernelGGL((extend_few_kernel<D, kModeAny>), grid, block, 0, stream, a);
  else if (a.softcap > 0.f)
    hipLaunchKernelGGL((extend_few_kernel<D, kModeCap>), grid, block, 0, stream, a);
  else
    hipLaunchKernelGGL((extend_few_kernel<D, kModePlain>), grid, block, 0, stream, a);
}
}  // namespace

void launch_extend_rows(const ExtArgs &a, int32_t kind, hipStream_t stream) {
  switch (kind) {
    case kXRows64: return launch_rows<64, 4>(a, stream);
    case kXRows128: return launch_rows<128, 4>(a, stream);
    case kXSome64: return launch_rows<64, 1>(a, stream);
    case kXSome128: return launch_rows<128, 1>(a, stream);
    case kXFew64: return launch_few<64>(a, stream);
    default: return launch_few<128>(a, stream);
  }
}

}  // namespace cp
