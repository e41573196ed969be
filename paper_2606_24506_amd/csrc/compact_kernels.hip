// gfx950 kernels of requests that keep some of their tokens: the choice of the heaviest
// (cp_kv_evict) and the moves of their rows (cp_request_keep, cp_kv_evict).
#include <hip/hip_runtime.h>

#include "compact.h"
#include "decode_mfma.h"
#include "device_common.h"

namespace cp {

typedef unsigned int u32x4m __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------------ choice

namespace {

constexpr int kSelWaves = kSelectThreads / 64;
constexpr int kBins = 2048;

// Numbers in the order of floats: NaN below all, -0 as 0.
CP_DEV uint32_t order_key(float f) {
  const uint32_t u = __float_as_uint(f + 0.f);
  if ((u & 0x7FFFFFFFu) > 0x7F800000u) return 0u;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// The threshold of the k heaviest: all above `above` are among them, and the first `equal`
// of those that are it.
struct Cut {
  uint32_t key, equal;
};

}  // namespace

// A workgroup per layer and KV head. The k-th largest of the middle's sums is found by
// counting: each pass spreads the numbers between the smallest and the largest that are
// still possible over 2,048 counters (in the order of floats, which spreads sums of any
// scale) and keeps the counter that holds the k-th; after at most three passes it holds one
// value. Then every wave takes a piece of the row in order and writes the numbers that
// stay, in their order. The row is read again in each pass: from L2, as fast as LDS would
// give it, and of any length. Bound by those passes of one workgroup.
__global__ __launch_bounds__(kSelectThreads) void evict_select_kernel(const EvictArgs a) {
  __shared__ uint32_t hist[kBins];
  __shared__ uint32_t part[2][kSelWaves];
  __shared__ uint32_t found[4];  // lo, hi, still needed, exact
  const int r = sorted_search(a.n_req, blockIdx.x, [&](int i) { return a.req[i].block_begin; });
  const EvictReq &rq = a.req[r];
  const uint32_t b = blockIdx.x - rq.block_begin, layer = b / rq.hkv, head = b - layer * rq.hkv;
  const uint32_t tid = threadIdx.x;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  // ---- the entries of pages that are replaced, as they were, and their new ones
  if (head == 0 && rq.tab) {
    uint32_t *const pte = a.pte + rq.pte_base + layer * rq.plane;
    for (uint32_t i = tid; i < rq.tab_n; i += kSelectThreads) rq.tab[(uint64_t)layer * rq.tab_n + i] = pte[i];
    __syncthreads();
    if (rq.ent != kNoWs)
      for (uint32_t i = tid; i < rq.pages; i += kSelectThreads) pte[rq.page0 + i] = a.ent[rq.ent + layer * rq.pages + i];
  }

  const float *const w = rq.old + (int64_t)layer * rq.old_layer + (int64_t)head * rq.old_head;
  int32_t *const list = rq.list + (int64_t)layer * rq.list_layer + (int64_t)head * rq.list_head;
  const uint32_t m0 = rq.first, m1 = rq.n - rq.last, need0 = rq.keep - rq.first - rq.last;

  // ---- smallest and largest
  uint32_t lo = 0xFFFFFFFFu, hi = 0;
  for (uint32_t i = m0 + tid; i < m1; i += kSelectThreads) {
    const uint32_t k = order_key(w[i]);
    lo = min(lo, k);
    hi = max(hi, k);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    lo = min(lo, (uint32_t)__shfl_xor((int)lo, o, 64));
    hi = max(hi, (uint32_t)__shfl_xor((int)hi, o, 64));
  }
  if (lane == 0) {
    part[0][wave] = lo;
    part[1][wave] = hi;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSelWaves; ++i) {
    lo = min(lo, part[0][i]);
    hi = max(hi, part[1][i]);
  }
  Cut cut{hi, need0};  // (nothing to find where none, or all, of the middle stay)
  if (need0 == m1 - m0) cut = Cut{0, need0};
  if (need0 > 0 && need0 < m1 - m0) {
    uint32_t need = need0;
    while (lo < hi) {
      const int bits = 32 - __builtin_clz(hi - lo), s = bits > 11 ? bits - 11 : 0;
      for (uint32_t i = tid; i < kBins; i += kSelectThreads) hist[i] = 0;
      __syncthreads();
      for (uint32_t i0 = m0; i0 < m1; i0 += kSelectThreads) {
        const uint32_t i = i0 + tid;
        const uint32_t k = i < m1 ? order_key(w[i]) : 0u;
        const bool in = i < m1 && k >= lo && k <= hi;
        const uint32_t bin = (k - lo) >> s;
        // (many equal numbers: one addition for those of the wave's first)
        const uint64_t some = __builtin_amdgcn_ballot_w64(in);
        if (some) {
          const uint32_t lead = (uint32_t)__builtin_amdgcn_readlane((int)bin, __builtin_ctzll(some));
          const uint64_t same = __builtin_amdgcn_ballot_w64(in && bin == lead);
          if (lane == __builtin_ctzll(some)) atomicAdd(&hist[lead], (uint32_t)__builtin_popcountll(same));
          if (in && bin != lead) atomicAdd(&hist[bin], 1u);
        }
      }
      __syncthreads();
      // counters from the largest down: a thread has two
      const uint32_t h0 = hist[kBins - 1 - 2 * tid], h1 = hist[kBins - 2 - 2 * tid];
      uint32_t sum = h0 + h1;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const uint32_t x = (uint32_t)__shfl_up((int)sum, o, 64);
        if (lane >= o) sum += x;
      }
      if (lane == 63) part[0][wave] = sum;
      __syncthreads();
      uint32_t before = sum - h0 - h1;
      for (int i = 0; i < wave; ++i) before += part[0][i];
      if (before < need && need <= before + h0 + h1) {
        const bool first = need <= before + h0;
        const uint32_t bin = kBins - 1 - 2 * tid - (first ? 0u : 1u), left = need - before - (first ? 0u : h0);
        const uint32_t nlo = lo + (bin << s);
        found[0] = nlo;
        found[1] = min(hi, nlo + ((1u << s) - 1u));
        found[2] = left;
        found[3] = left == (first ? h0 : h1);  // every number of the counter is among them
      }
      __syncthreads();
      lo = found[0];
      hi = found[1];
      need = found[2];
      if (found[3] && lo > 0) {
        lo = hi = lo - 1;
        need = 0;
      }
      __syncthreads();
    }
    cut = Cut{lo, need};
  }

  // ---- the numbers that stay, in order: pieces of the middle, one for each wave
  const uint32_t m = m1 - m0, each = ((m + kSelWaves - 1) / kSelWaves + 63) / 64 * 64;
  const uint32_t s0 = min(m1, m0 + wave * each), s1 = min(m1, s0 + each);
  uint32_t above = 0, equal = 0;
  for (uint32_t i0 = s0; i0 < s1; i0 += 64) {
    const uint32_t i = i0 + lane;
    const uint32_t k = i < s1 ? order_key(w[i]) : 0u;
    above += (uint32_t)__builtin_popcountll(__builtin_amdgcn_ballot_w64(i < s1 && k > cut.key));
    equal += (uint32_t)__builtin_popcountll(__builtin_amdgcn_ballot_w64(i < s1 && k == cut.key));
  }
  if (need0 == 0) above = 0;
  __syncthreads();
  if (lane == 0) {
    part[0][wave] = above;
    part[1][wave] = equal;
  }
  __syncthreads();
  uint32_t at = rq.first, eq = 0;
  for (int i = 0; i < wave; ++i) {
    at += part[0][i];
    eq += part[1][i];
  }
  at += min(eq, cut.equal);
  const uint64_t below = (1ull << lane) - 1;
  if (need0 > 0)
    for (uint32_t i0 = s0; i0 < s1; i0 += 64) {
      const uint32_t i = i0 + lane;
      const uint32_t k = i < s1 ? order_key(w[i]) : 0u;
      const uint64_t be = __builtin_amdgcn_ballot_w64(i < s1 && k == cut.key);
      const bool take = i < s1 && (k > cut.key || (k == cut.key && eq + (uint32_t)__builtin_popcountll(be & below) < cut.equal));
      const uint64_t bt = __builtin_amdgcn_ballot_w64(take);
      if (take) list[at + (uint32_t)__builtin_popcountll(bt & below)] = (int32_t)i;
      at += (uint32_t)__builtin_popcountll(bt);
      eq += (uint32_t)__builtin_popcountll(be);
    }
  for (uint32_t i = tid; i < rq.first; i += kSelectThreads) list[i] = (int32_t)i;
  for (uint32_t i = tid; i < rq.last; i += kSelectThreads) list[rq.keep - rq.last + i] = (int32_t)(rq.n - rq.last + i);

  // ---- the sums of those that stay; they may take the place of the old ones: what a step
  // reads lies at or behind what it writes
  if (!rq.sum) return;
  constexpr int U = 8;
  float *const out = rq.sum + (int64_t)layer * rq.sum_layer + (int64_t)head * rq.sum_head;
  __syncthreads();
  for (uint32_t c = 0; c < rq.keep; c += U * kSelectThreads) {
    float v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t k = c + u * kSelectThreads + tid;
      v[u] = k < rq.keep ? w[list[k]] : 0.f;
    }
    __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
    __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t k = c + u * kSelectThreads + tid;
      if (k < rq.keep) out[k] = v[u];
    }
  }
  __syncthreads();
  for (uint32_t i = rq.keep + tid; i < rq.n; i += kSelectThreads) out[i] = 0.f;
}

// ------------------------------------------------------------------- moves

// A 16-byte column of a row: which KV head's list it goes by.
CP_DEV uint32_t column_head(const GeomK &g, uint32_t seg) {
  return g.kind == 0 ? 0u : seg * 8 / (uint32_t)g.d_k % (uint32_t)g.hkv;
}

// Rows in place: a workgroup owns COLS columns of 16 bytes of one layer and takes the rows
// that stay in order, THREADS / COLS * UNROLL at once: all are read before any is written,
// and those of later steps lie behind what this one writes (list entries rise: entry k is at
// least k). So no workgroup waits for another. Bound by the round trips of a step where
// there are few workgroups.
template <int THREADS, int COLS, int UNROLL>
__global__ __launch_bounds__(THREADS) void move_kernel(const MoveArgs a) {
  constexpr uint32_t RPI = THREADS / COLS;
  const int r = sorted_search(a.n_req, blockIdx.x, [&](int i) { return a.req[i].block_begin; });
  const MoveReq &rq = a.req[r];
  const GeomK &g = a.geom[rq.model];
  const uint32_t b = blockIdx.x - rq.block_begin, layer = b / rq.per_layer, P = (uint32_t)g.page_tokens;
  const uint32_t seg = (b - layer * rq.per_layer) * COLS + threadIdx.x % COLS, row = threadIdx.x / COLS;
  const bool mine = seg < (uint32_t)g.row_elems / 8;
  const int32_t *const list =
      rq.list ? rq.list + (int64_t)layer * rq.list_layer + (int64_t)column_head(g, mine ? seg : 0u) * rq.list_head : nullptr;
  const uint32_t *const src = rq.src + (uint64_t)layer * rq.src_plane, *const dst = a.pte + rq.dst_base + layer * rq.dst_plane;
#pragma unroll 1
  for (uint32_t base = rq.k0; base < rq.n; base += RPI * UNROLL) {
    u32x4m v[UNROLL];
    uint64_t to[UNROLL];
    bool moves[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const uint32_t k = base + u * RPI + row;
      moves[u] = mine && k < rq.n;
      if (!moves[u]) continue;
      const uint32_t s = rq.first + min(list ? (uint32_t)list[k] : a.ent[rq.ent0 + (k - rq.k0)], rq.rows - 1);
      const uint32_t d = rq.first + k, sp = src[s / P], dp = dst[d / P];
      moves[u] = s != d || sp != dp;
      to[u] = ((uint64_t)dp << 8) + row_seg_offset(g, d % P, seg);
      if (moves[u]) v[u] = *reinterpret_cast<const u32x4m *>(a.pool + ((uint64_t)sp << 8) + row_seg_offset(g, s % P, seg));
    }
    __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
    __syncthreads();
#pragma unroll
    for (int u = 0; u < UNROLL; ++u)
      if (moves[u]) *reinterpret_cast<u32x4m *>(a.pool + to[u]) = v[u];
  }
}

// Rows that go to pages which nothing of the call reads: in any order.
__global__ __launch_bounds__(kApartThreads) void move_apart_kernel(const MoveArgs a) {
  const int r = sorted_search(a.n_req, blockIdx.x, [&](int i) { return a.req[i].block_begin; });
  const MoveReq &rq = a.req[r];
  const GeomK &g = a.geom[rq.model];
  const uint32_t b = blockIdx.x - rq.block_begin, layer = b / rq.per_layer, P = (uint32_t)g.page_tokens;
  const uint32_t nseg = (uint32_t)g.row_elems / 8;
  const uint64_t i0 = (uint64_t)(b - layer * rq.per_layer) * (kApartThreads * kApartUnroll) + threadIdx.x,
                 total = (uint64_t)(rq.n - rq.k0) * nseg;
  const uint32_t *const src = rq.src + (uint64_t)layer * rq.src_plane, *const dst = a.pte + rq.dst_base + layer * rq.dst_plane;
  u32x4m v[kApartUnroll];
  uint64_t to[kApartUnroll];
#pragma unroll
  for (int u = 0; u < kApartUnroll; ++u) {
    const uint64_t i = i0 + u * kApartThreads;
    if (i >= total) continue;
    const uint32_t row = (uint32_t)(i / nseg), seg = (uint32_t)(i - (uint64_t)row * nseg), d = rq.k0 + row;
    const int32_t *const list = rq.list + (int64_t)layer * rq.list_layer + (int64_t)column_head(g, seg) * rq.list_head;
    const uint32_t s = min((uint32_t)list[d], rq.rows - 1);
    to[u] = ((uint64_t)dst[d / P] << 8) + row_seg_offset(g, d % P, seg);
    v[u] = __builtin_nontemporal_load(
        reinterpret_cast<const u32x4m *>(a.pool + ((uint64_t)src[s / P] << 8) + row_seg_offset(g, s % P, seg)));
  }
#pragma unroll
  for (int u = 0; u < kApartUnroll; ++u)
    if (i0 + u * kApartThreads < total) *reinterpret_cast<u32x4m *>(a.pool + to[u]) = v[u];
}

hipError_t launch_evict_select(const EvictArgs &a, hipStream_t stream) {
  if (a.n_blocks <= 0) return hipSuccess;
  hipLaunchKernelGGL(evict_select_kernel, dim3((uint32_t)a.n_blocks), dim3(kSelectThreads), 0, stream, a);
  return hipGetLastError();
}

// how: 0 short lists in the arguments, 1 in place, 2 apart
hipError_t launch_moves(const MoveArgs &a, int how, hipStream_t stream) {
  if (a.n_blocks <= 0) return hipSuccess;
  const dim3 grid((uint32_t)a.n_blocks);
  if (how == 0)
    hipLaunchKernelGGL((move_kernel<kKeepThreads, kKeepCols, kKeepUnroll>), grid, dim3(kKeepThreads), 0, stream, a);
  else if (how == 1)
    hipLaunchKernelGGL((move_kernel<kMoveThreads, kMoveCols, kMoveUnroll>), grid, dim3(kMoveThreads), 0, stream, a);
  else
    hipLaunchKernelGGL(move_apart_kernel, grid, dim3(kApartThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace cp
