// gfx950 kernels of rotary positions: rotation of strided tensors, and the
// append that rotates keys on their way into the pool.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "device_common.h"
#include "rope_device.h"

namespace cp {

typedef unsigned int u32x4r __attribute__((ext_vector_type(4)));

// Elements as floats and back, one rounding.
template <bool F32>
struct RopeElem {
  using T = uint16_t;
  static constexpr int V = 8;  // per 16 bytes
  CP_DEV static float get(u32x4r w, int i) { return __uint_as_float(i & 1 ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16); }
  CP_DEV static u32x4r pack(const float (&x)[8]) {
    u32x4r w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = f32_to_bf16(x[2 * i]) | (f32_to_bf16(x[2 * i + 1]) << 16);
    return w;
  }
  CP_DEV static float load(const T *p) { return bf16_to_f32(*p); }
  CP_DEV static void store(T *p, float x) { *p = (T)f32_to_bf16(x); }
};
template <>
struct RopeElem<true> {
  using T = float;
  static constexpr int V = 4;
  CP_DEV static float get(u32x4r w, int i) { return __uint_as_float(w[i]); }
  CP_DEV static u32x4r pack(const float (&x)[4]) {
    return u32x4r{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
  }
  CP_DEV static float load(const T *p) { return *p; }
  CP_DEV static void store(T *p, float x) { *p = x; }
};

// Item `it` of one token and part: item j of a head is a rotated piece (both
// halves' pieces, or a piece of whole pairs) or, behind those, a copied one.
template <bool F32>
CP_DEV void rope_item(const RopeArgs &a, const RopePart &p, int64_t tok, uint32_t it, const float2 *turn) {
  using E = RopeElem<F32>;
  using T = typename E::T;
  constexpr int V = E::V;
  const uint32_t pairs = (uint32_t)a.rope.pairs, rot = 2 * pairs;
  const bool half = !a.rope.interleaved, copies = p.src != p.dst;
  const uint32_t step = p.vec ? V : 1;
  const uint32_t turning = half ? pairs / step : (p.vec ? rot / V : pairs);
  const uint32_t per_head = turning + (copies ? ((uint32_t)p.width - rot) / step : 0u);
  const uint32_t head = it / per_head, j = it - head * per_head;
  const T *const s = (const T *)p.src + tok * p.src_tok + (int64_t)head * p.src_head;
  T *const d = (T *)p.dst + tok * p.dst_tok + (int64_t)head * p.dst_head;
  if (j >= turning) {  // unrotated: before the offset or behind the rotated elements
    uint32_t e = (j - turning) * step;
    if (e >= (uint32_t)p.offset) e += rot;
    if (p.vec)
      *(u32x4r *)(d + e) = *(const u32x4r *)(s + e);
    else
      d[e] = s[e];
    return;
  }
  const T *const sr = s + p.offset;
  T *const dr = d + p.offset;
  if (!p.vec) {
    const uint32_t e0 = half ? j : 2 * j, e1 = half ? j + pairs : 2 * j + 1;
    const float x = E::load(sr + e0), y = E::load(sr + e1);
    E::store(dr + e0, rope_first(x, y, turn[j]));
    E::store(dr + e1, rope_second(x, y, turn[j]));
  } else if (half) {
    const u32x4r x = __builtin_nontemporal_load((const u32x4r *)(sr + j * V)),
                 y = __builtin_nontemporal_load((const u32x4r *)(sr + pairs + j * V));
    float u[V], w[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float2 t = turn[j * V + i];
      u[i] = rope_first(E::get(x, i), E::get(y, i), t);
      w[i] = rope_second(E::get(x, i), E::get(y, i), t);
    }
    *(u32x4r *)(dr + j * V) = E::pack(u);
    *(u32x4r *)(dr + pairs + j * V) = E::pack(w);
  } else {
    const u32x4r x = *(const u32x4r *)(sr + j * V);
    float u[V];
#pragma unroll
    for (int i = 0; i < V; i += 2) {
      const float2 t = turn[(j * V + i) / 2];
      u[i] = rope_first(E::get(x, i), E::get(x, i + 1), t);
      u[i + 1] = rope_second(E::get(x, i), E::get(x, i + 1), t);
    }
    *(u32x4r *)(dr + j * V) = E::pack(u);
  }
}

// A workgroup takes a.tokens tokens (as many as make about one (token, pair)
// for each thread, so that a sine is computed once per token and pair, not once per
// head) and a slice of their work items.
template <bool F32>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(const RopeArgs a) {
  extern __shared__ float2 turn[];  // [tokens][pairs]
  const uint32_t pairs = (uint32_t)a.rope.pairs;
  const int64_t tok0 = (int64_t)blockIdx.x * a.tokens;
  const uint32_t nt = (uint32_t)min((int64_t)a.tokens, a.n_tokens - tok0);
  for (uint32_t i = threadIdx.x; i < nt * pairs; i += kRopeThreads) {
    const uint32_t t = i / pairs;
    const int64_t pos = a.pos ? (int64_t)a.pos[tok0 + t] : a.first + tok0 + t;
    turn[i] = rope_turn(a.rope, pos, (int32_t)(i - t * pairs));
  }
  __syncthreads();
  const uint32_t items = (uint32_t)a.item0[a.n_parts];
  for (uint32_t i = blockIdx.y * kRopeThreads + threadIdx.x; i < nt * items; i += gridDim.y * kRopeThreads) {
    const uint32_t t = i / items, it = i - t * items;
    int p = 0;
    while (p + 1 < a.n_parts && it >= (uint32_t)a.item0[p + 1]) ++p;
    rope_item<F32>(a, a.part[p], tok0 + t, it - (uint32_t)a.item0[p], turn + t * pairs);
  }
}

hipError_t launch_rope(const RopeArgs &in, int32_t items, bool f32, hipStream_t stream) {
  RopeArgs a = in;
  // fewer tokens where the items of one would pass 2^31 / tokens
  a.tokens = (int32_t)std::max<int64_t>(1, std::min<int64_t>({kRopeThreads / a.rope.pairs, a.n_tokens, 0x3FFFFFFF / items}));
  const int64_t rounds = ((int64_t)a.tokens * items + kRopeThreads - 1) / kRopeThreads;
  const size_t lds = (size_t)a.tokens * a.rope.pairs * sizeof(float2);
  const int64_t size = f32 ? 4 : 2;
  for (int64_t done = 0; done < in.n_tokens;) {
    const int64_t blocks = (in.n_tokens - done + a.tokens - 1) / a.tokens;
    // few tokens: one round of items per workgroup (latency); many: up to eight, for
    // fewer sines (us with one and with eight: 4 tokens of 40 heads 5.3 and 7.8, 8,192
    // of them 42 and 37; but 5,001 tokens of 16 heads with 64 of 576 elements 8.3 and 9.6)
    const int64_t per = blocks * rounds <= 2048 ? 1 : 8, slices = std::min<int64_t>(65535, (rounds + per - 1) / per);
    // (a launch has less than 2^32 threads)
    const int64_t most = std::max<int64_t>(1, ((1 << 24) - 1) / slices), now = std::min(blocks, most);
    a.n_tokens = std::min(in.n_tokens - done, now * a.tokens);
    a.first = in.first + done;
    a.pos = in.pos ? in.pos + done : nullptr;
    for (int i = 0; i < a.n_parts; ++i) {
      a.part[i].src = (const char *)in.part[i].src + done * in.part[i].src_tok * size;
      a.part[i].dst = (char *)in.part[i].dst + done * in.part[i].dst_tok * size;
    }
    const dim3 grid((uint32_t)now, (uint32_t)slices);
    if (f32)
      hipLaunchKernelGGL(rope_kernel<true>, grid, dim3(kRopeThreads), lds, stream, a);
    else
      hipLaunchKernelGGL(rope_kernel<false>, grid, dim3(kRopeThreads), lds, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    done += a.n_tokens;
  }
  return hipSuccess;
}

// ------------------------------------------------------- append, rotated

// Rows [block R, block R + R) of one item as in the plain append; every thread
// writes one 16-byte segment at a time. A segment of rotated elements needs
// their partners too: its own neighbours (interleaved), or the segment half a
// rotation away, which another thread of the workgroup reads as its own.
__global__ __launch_bounds__(kCopyThreads) void kv_append_rope_kernel(const AppendArgs a, const RopeK rope) {
  extern __shared__ float2 turn[];  // [rows][pairs]
  const int r = sorted_search(a.n_req, blockIdx.x, [&](int i) { return a.req[i].block_begin; });
  const AppReq &rq = a.req[r];
  const GeomK &g = a.geom[rq.model];
  const uint32_t P = (uint32_t)g.page_tokens, R = copy_rows_per_block((uint32_t)g.row_elems);
  const uint32_t row0 = (blockIdx.x - rq.block_begin) * R, row1 = min(rq.n_new, row0 + R), nrows = row1 - row0;
  const uint32_t first_new = (rq.old_len + P - 1) / P;
  if (rq.ent != kNoEnt) {
    const uint32_t pg = (rq.old_len + row0 + P - 1) / P + threadIdx.x;
    if (pg <= (rq.old_len + row1 - 1) / P) a.pte[rq.pte_base + pg] = a.ent[rq.ent + (pg - first_new)];
  }
  auto pte_of = [&](uint32_t pg) {
    return rq.ent != kNoEnt && pg >= first_new ? a.ent[rq.ent + (pg - first_new)] : a.pte[rq.pte_base + pg];
  };
  const uint32_t pairs = (uint32_t)rope.pairs, rot = 2 * pairs;
  const uint32_t pos0 = rq.old_len + row0;
  const int64_t first = (int64_t)rq.old_len + rq.dropped;
  const int32_t *const depth = a.depth ? a.depth + rq.src_off / (uint32_t)g.row_elems + row0 : nullptr;
  for (uint32_t i = threadIdx.x; i < nrows * pairs; i += kCopyThreads) {
    const uint32_t t = i / pairs;
    const int64_t at = first + (depth ? min((uint32_t)depth[t], rq.n_new - 1) : row0 + t);
    turn[i] = rope_turn(rope, at, (int32_t)(i - t * pairs));
  }
  __syncthreads();
  const uint32_t nseg = (uint32_t)g.row_elems / 8, total = nrows * nseg;
  const uint16_t *const rows = a.rows + rq.src_off + (uint64_t)row0 * (uint32_t)g.row_elems;
  // keys: heads of d elements from e_key on, rotated from head_off on
  const uint32_t d = (uint32_t)g.d_k, kelems = g.kind == 0 ? d : (uint32_t)g.hkv * d;
  const uint32_t head_off = g.kind == 0 ? (uint32_t)g.d_v : 0u;
  for (uint32_t i = threadIdx.x; i < total; i += kCopyThreads) {
    const uint32_t row = i / nseg, seg = i - row * nseg, e = seg * 8;
    const uint32_t pos = pos0 + row, pg = pos / P;
    const uint16_t *const src = rows + (uint64_t)row * (uint32_t)g.row_elems;
    u32x4r x = *(const u32x4r *)(src + e);
    if (e < kelems) {
      const uint32_t in_head = e % d;  // the segment's first element in its head
      const float2 *const tr = turn + row * pairs;
      if (in_head >= head_off && in_head < head_off + rot) {
        const uint32_t c = in_head - head_off;  // ... and among the rotated ones
        float y[8];
        if (rope.interleaved) {
#pragma unroll
          for (int k = 0; k < 8; k += 2) {
            const float u = RopeElem<false>::get(x, k), w = RopeElem<false>::get(x, k + 1);
            const float2 t = c + k < rot ? tr[(c + k) / 2] : float2{1.f, 0.f};
            y[k] = c + k < rot ? rope_first(u, w, t) : u;
            y[k + 1] = c + k < rot ? rope_second(u, w, t) : w;
          }
        } else if (pairs % 8 == 0) {
          const bool upper = c >= pairs;
          const u32x4r z = *(const u32x4r *)(src + (upper ? e - pairs : e + pairs));
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float u = RopeElem<false>::get(x, k), w = RopeElem<false>::get(z, k);
            const float2 t = tr[upper ? c - pairs + k : c + k];
            y[k] = upper ? rope_second(w, u, t) : rope_first(u, w, t);
          }
        } else {  // halves that end inside segments
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const uint32_t ck = c + k;
            const float u = RopeElem<false>::get(x, k);
            if (ck >= rot)
              y[k] = u;
            else if (ck >= pairs)
              y[k] = rope_second(bf16_to_f32(src[e + k - pairs]), u, tr[ck - pairs]);
            else
              y[k] = rope_first(u, bf16_to_f32(src[e + k + pairs]), tr[ck]);
          }
        }
        u32x4r o = RopeElem<false>::pack(y);
        if (c + 8 > rot) {  // the unrotated rest keeps its bits
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (c + 2 * k >= rot) o[k] = x[k];
        }
        x = o;
      }
    }
    *(u32x4r *)(a.pool + ((uint64_t)pte_of(pg) << 8) + row_seg_offset(g, pos - pg * P, seg)) = x;
  }
}

hipError_t launch_append_rope(const AppendArgs &a, const RopeK &rope, hipStream_t stream) {
  if (a.n_blocks <= 0) return hipSuccess;
  uint32_t rows = 1;
  for (int m = 0; m < kMaxLaunchModels && a.geom[m].row_elems; ++m)
    rows = std::max(rows, copy_rows_per_block((uint32_t)a.geom[m].row_elems));
  const size_t lds = (size_t)rows * rope.pairs * sizeof(float2);
  hipLaunchKernelGGL(kv_append_rope_kernel, dim3(a.n_blocks), dim3(kCopyThreads), lds, stream, a, rope);
  return hipGetLastError();
}

}  // namespace cp
