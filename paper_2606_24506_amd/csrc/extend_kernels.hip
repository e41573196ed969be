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
      s = acc * a.score_mul;
      if (a.softcap > 0.f) s = cap_tanh(s) * a.cap_mul;
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
    case kXRows64:
    case kXRows128:
    case kXFew64:
    case kXFew128: launch_extend_rows(a, kind, stream); break;
    case kXMla: launch_extend_mla(a, stream); break;
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
