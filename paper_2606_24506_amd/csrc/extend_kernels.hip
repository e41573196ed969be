// gfx950 kernels of attention of token chunks over the pool (cp_attn_extend):
// the vector kernel, the join of key ranges, and the launches.
#include <hip/hip_runtime.h>

#include "extend_device.h"

namespace cp {

void launch_extend_rows(const ExtArgs &a, int32_t kind, hipStream_t stream);
void launch_extend_mla(const ExtArgs &a, hipStream_t stream);

// ------------------------------------------------------------ vector path

// One wave per row, for every geometry: a lane per key for the scores (its K row
// read in 16-byte pieces), then lanes across the columns for the sums, key after
// key, keys out of sight skipped. Bound by the vector unit and the per-lane row
// reads; it serves the geometries without a matrix kernel.
template <int E>  // V columns per lane
__global__ __launch_bounds__(kExtThreads) void extend_vec_kernel(const ExtArgs a) {
  extern __shared__ float qs[];  // [4][d_k]
  const Unit un = find_unit(a);
  if (un.none) return;
  const ExtReq &rq = *un.rq;
  const GeomK &g = a.g;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t r = un.tile * 4 + wave;
  if (r >= rq.n_tok * (uint32_t)g.g) return;  // no barrier below: waves are on their own
  const Row x = a.tree_mask ? row_of<true>(a, rq, un.kvh, r) : row_of<false>(a, rq, un.kvh, r);
  const uint32_t dk = (uint32_t)g.d_k, P = (uint32_t)g.page_tokens;
  float *const qw = qs + wave * dk;
  const uint16_t *const qrow = a.q + (x.tok * (uint32_t)g.hq + x.head) * dk;
  for (uint32_t i = lane; i < dk; i += 64) qw[i] = bf16_to_f32(qrow[i]);
  const float slope = a.slopes ? a.slopes[x.head] * kLog2e : 0.f;
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
    bool see = key < e;
    if (a.tree_mask && see && key >= x.base) see = tree_bits<1>(a, x, key) & 1;
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
      s = acc * a.score_mul;
      if (a.softcap > 0.f) s = cap_tanh(s) * a.cap_mul;
      if (a.slopes) {
        const uint32_t at = a.tree_mask ? tree_pos(a, x, key) : key;
        s -= slope * (float)(max(x.pos, at) - min(x.pos, at));
      }
    }
    const float mn = fmaxf(m, wave_max(s)), base = mn == -INFINITY ? 0.f : mn;
    const float al = fast_exp2(m - base);
    const float p = see ? fast_exp2(s - base) : 0.f;
    m = mn;
    l = l * al + wave_sum(p);
#pragma unroll
    for (int i = 0; i < E; ++i) o[i] *= al;
    const uint32_t cnt = min(64u, e - k0);
    const uint64_t seen = __builtin_amdgcn_ballot_w64(see);
    for (uint32_t j = 0; j < cnt; ++j) {
      if (!(seen >> j & 1)) continue;  // of a tree
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
  if (rq.all > 1) {
    const uint64_t pr = part_row(a, rq, x, un.split);
    if (lane == 0) a.ws_l[pr] = lse;
    if (none) return;  // (the join takes no sums of such a range)
#pragma unroll
    for (int i = 0; i < E; ++i) a.ws_o[pr * (uint32_t)g.d_v + lane * E + i] = o[i] * inv;
  } else {
    const uint64_t orow = x.tok * (uint32_t)g.hq + x.head;
#pragma unroll
    for (int i = 0; i < E; ++i)
      a.out[orow * (uint32_t)g.d_v + lane * E + i] = (uint16_t)f32_to_bf16(none ? 0.f : o[i] * inv);
    if (lane == 0) a.lse[orow] = lse * kLn2;
  }
}

// ----------------------------------------------------------------- join

// Weights 2^(lse_s - max) of a row's ranges, then the columns: a thread takes four
// columns of every `lanes`-th range, four loads in flight, with a running maximum as
// over keys; the lanes' sums meet in LDS. A workgroup takes 256 / (d_v / 4 *
// lanes) rows. Bound by its launch and a row's chain of loads: 4.6 to 5 us behind
// single tokens, 9 for 80 rows of 512 columns.
__global__ __launch_bounds__(kExtThreads) void ext_merge_kernel(const ExtMergeArgs a) {
  __shared__ float part[4][kExtThreads];
  __shared__ float stat[2][kExtThreads];
  const uint32_t dv4 = (uint32_t)a.d_v / 4, lanes = (uint32_t)a.lanes, per_row = dv4 * lanes;
  const uint32_t sub = threadIdx.x / per_row, t = threadIdx.x - sub * per_row, c = t % dv4, ln = t / dv4;
  const uint32_t row = blockIdx.x * (kExtThreads / per_row) + sub;
  // the request of each thread's row: rows of a workgroup may belong to two
  int r = 0;
  while (r + 1 < a.n_req && a.req[r + 1].row_begin <= row) ++r;
  const ExtMergeArgs::Req &rq = a.req[r];
  const uint32_t i = row - rq.row_begin;
  const bool valid = i < rq.rows;
  const uint64_t pr = (rq.ws_row + (valid ? i : 0u)) * rq.splits;
  const uint32_t n = valid ? rq.splits : 0u;
  float m = -INFINITY, sum = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  const f32x4 *const o = reinterpret_cast<const f32x4 *>(a.ws_o) + pr * dv4 + c;
  for (uint32_t s0 = ln; s0 < n; s0 += 4 * lanes) {
    f32x4 v[4];
    float e[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const uint32_t s = s0 + u * lanes;
      e[u] = s < n ? a.ws_l[pr + s] : -INFINITY;
      v[u] = s < n ? o[(uint64_t)s * dv4] : f32x4{0.f, 0.f, 0.f, 0.f};
    }
    float mn = m;
#pragma unroll
    for (int u = 0; u < 4; ++u) mn = fmaxf(mn, e[u]);
    const float ref = mn == -INFINITY ? 0.f : mn, al = fast_exp2(m - ref);
    m = mn;
    sum *= al;
    acc *= al;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float w = fast_exp2(e[u] - ref);
      sum += w;
      // (a range that saw nothing has nothing to add, and wrote no sums; those of weight 0 may be NaN)
      if (e[u] != -INFINITY) acc += w * v[u];
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) part[k][threadIdx.x] = acc[k];
  stat[0][threadIdx.x] = m;
  stat[1][threadIdx.x] = sum;
  __syncthreads();
  if (!valid || ln != 0) return;
  float mx = m;
  for (uint32_t k = 1; k < lanes; ++k) mx = fmaxf(mx, stat[0][threadIdx.x + k * dv4]);
  const float ref = mx == -INFINITY ? 0.f : mx, own = fast_exp2(m - ref);
  sum *= own;
  acc *= own;
  for (uint32_t k = 1; k < lanes; ++k) {
    const uint32_t at = threadIdx.x + k * dv4;
    const float w = fast_exp2(stat[0][at] - ref);
    sum += w * stat[1][at];
#pragma unroll
    for (int q = 0; q < 4; ++q) acc[q] += w * part[q][at];
  }
  const bool none = sum == 0.f;
  const float inv = none ? 0.f : 1.f / sum;
  const uint64_t orow = rq.out_row + i;
  *reinterpret_cast<uint2 *>(a.out + orow * (uint32_t)a.d_v + 4 * c) =
      bf16x4_bits(acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
  if (c == 0) a.lse[orow] = none ? -INFINITY : (mx + fast_log2(sum)) * kLn2;
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
    case kXRows64:
    case kXRows128:
    case kXSome64:
    case kXSome128:
    case kXFew64:
    case kXFew128: launch_extend_rows(a, kind, stream); break;
    case kXMla: launch_extend_mla(a, stream); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

// few_lanes (trees): no more lanes of a row than it takes to fill the card, kJoinThreads
// threads in all: their sums' way through LDS costs more than a row's own chain then.
constexpr uint64_t kJoinThreads = 1 << 19;
hipError_t launch_ext_merge(const ExtMergeArgs &in, uint32_t rows, uint32_t most_splits, bool few_lanes, hipStream_t stream) {
  if (rows == 0) return hipSuccess;
  ExtMergeArgs a = in;
  const int dv4 = a.d_v / 4;
  a.lanes = 1;
  while (a.lanes * 2 * dv4 <= kExtThreads && (uint32_t)a.lanes < most_splits &&
         (!few_lanes || (uint64_t)rows * (uint64_t)(dv4 * a.lanes) < kJoinThreads))
    a.lanes *= 2;
  const uint32_t per = (uint32_t)(kExtThreads / (dv4 * a.lanes));
  hipLaunchKernelGGL(ext_merge_kernel, dim3((rows + per - 1) / per), dim3(kExtThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace cp
