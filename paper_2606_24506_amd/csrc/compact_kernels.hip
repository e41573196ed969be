// gfx950 kernels of requests that keep some of their tokens: the choice of the heaviest
// (cp_kv_evict) and the moves of their rows (cp_request_keep, cp_kv_evict).
#include <hip/hip_runtime.h>

#include "compact.h"
#include "decode_mfma.h"
#include "extend_device.h"
#include "device_common.h"

namespace cp {

typedef unsigned int u32x4m __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------------ choice

namespace {

constexpr int kSelWaves = kSelectThreads / 64;
constexpr uint32_t kCands = 2048;  // numbers still possible that fit LDS

// Numbers in the order of floats, from 1 on: NaN (1) below all, -0 as 0. 0 is no number.
CP_DEV uint32_t order_key(float f) {
  const float x = f + 0.f;
  const uint32_t u = __float_as_uint(x), k = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
  return x == x ? k : 1u;
}

// The threshold of the k heaviest: all above `above` are among them, and the first `equal`
// of those that are it.
struct Cut {
  uint32_t key, equal;
};

}  // namespace

// A workgroup per layer and KV head, a wave for every piece of the row. The k-th largest of
// the middle's sums is found by counting: each pass spreads the numbers between the
// smallest and the largest that are still possible over 2,048 counters (in the order of
// floats, which spreads sums of any scale) and keeps the counter that holds the k-th; after
// at most three passes it holds one value (compact.h: also of a row that is written
// meanwhile, which gives some list, in bounds). Then every wave writes the numbers of its
// piece that stay, in their order.
// R > 0: the row in registers, R numbers a thread (rows of up to 1,024 R); 0: read again in
// each pass, eight loads in flight. Bound by the passes of one workgroup: rows of 5,000 numbers
// 12 us, of 16 K 14, of 64 K 35 (107 when each pass read them all again), of 128 K, which are
// read again, 50 to 70.
template <int R>
__global__ __launch_bounds__(kSelectThreads) void evict_select_kernel(const EvictArgs a) {
  __shared__ uint32_t hist[kBins];
  __shared__ uint32_t part[2][kSelWaves];
  __shared__ uint32_t found[4];  // the counter, which of its numbers, how many it holds (0: no counter); candidates
  __shared__ uint32_t cand[kCands];
  const int r = sorted_search(a.n_req, blockIdx.x, [&](int i) { return a.req[i].block_begin; });
  const EvictReq &rq = a.req[r];
  const uint32_t b = blockIdx.x - rq.block_begin, layer = b / rq.hkv, head = b - layer * rq.hkv;
  const uint32_t tid = threadIdx.x;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const float *const w = rq.old + (int64_t)layer * rq.old_layer + (int64_t)head * rq.old_head;
  int32_t *const list = rq.list + (int64_t)layer * rq.list_layer + (int64_t)head * rq.list_head;
  const uint32_t m0 = rq.first, m1 = rq.n - rq.last, m = m1 - m0, need0 = rq.keep - rq.first - rq.last;
  // this wave's piece of the middle
  const uint32_t each = ((m + kSelWaves - 1) / kSelWaves + 63) / 64 * 64;
  const uint32_t s0 = min(m1, m0 + wave * each), s1 = min(m1, s0 + each);
  uint32_t key[R > 0 ? R : 1];
  if constexpr (R > 0) {
    float x[R];
    if (s0 < s1) {
#pragma unroll
      for (int j = 0; j < R; ++j) x[j] = w[min(s0 + 64 * j + lane, s1 - 1)];
    }
#pragma unroll
    for (int j = 0; j < R; ++j) key[j] = s0 + 64 * j + lane < s1 ? order_key(x[j]) : 0u;
  }
  // f(the number of the first lane's, keys), in order; whole waves. Lanes behind the last
  // number of a piece have a key of 0.
  auto each_of = [&](auto f) {
    if constexpr (R > 0) {
      constexpr int G = R < 8 ? R : 8;
#pragma unroll
      for (int j0 = 0; j0 < R; j0 += G)
        if (s0 + 64 * j0 < s1) {
#pragma unroll
          for (int j = j0; j < j0 + G; ++j) f(s0 + 64 * j, key[j]);
        }
    } else {
      for (uint32_t i0 = s0; i0 < s1; i0 += 64 * 8) {
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = w[min(i0 + 64 * j + lane, s1 - 1)];
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (i0 + 64 * j < s1) f(i0 + 64 * j, i0 + 64 * j + lane < s1 ? order_key(x[j]) : 0u);
      }
    }
  };

  // ---- the entries of pages that are replaced, as they were, and their new ones
  if (head == 0 && rq.tab) {
    uint32_t *const pte = a.pte + rq.pte_base + layer * rq.plane;
    for (uint32_t i = tid; i < rq.tab_n; i += kSelectThreads) rq.tab[(uint64_t)layer * rq.tab_n + i] = pte[i];
    __syncthreads();
    if (rq.ent != kNoWs)
      for (uint32_t i = tid; i < rq.pages; i += kSelectThreads) pte[rq.page0 + i] = a.ent[rq.ent + layer * rq.pages + i];
  }

  // ---- smallest and largest
  uint32_t lo = 0xFFFFFFFFu, hi = 0;  // lo: less 1, so that a key of 0 is no smallest
  each_of([&](uint32_t, uint32_t k) {
    lo = min(lo, k - 1);
    hi = max(hi, k);
  });
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
  lo = __builtin_amdgcn_readfirstlane(lo + 1);
  hi = __builtin_amdgcn_readfirstlane(hi);
  Cut cut{need0 == m ? 0u : hi, 0u};  // (nothing to find where none, or all, of the middle stay)
  if (need0 > 0 && need0 < m) {
    Search x{lo, hi, need0};
    bool few = false;  // the numbers still possible are `cand`, found[3] of them
    for (bool more = lo < hi; more;) {
      const int s = search_shift(x);
      for (uint32_t i = tid; i < kBins; i += kSelectThreads) hist[i] = 0;
      if (tid == 0) found[2] = 0;
      __syncthreads();
      // (as many may be the smallest, tokens that nothing looked at: counted by the wave)
      if (few) {
        for (uint32_t i = tid; i < min(found[3], kCands); i += kSelectThreads)
          if (cand[i] - x.lo <= x.hi - x.lo) atomicAdd(&hist[(cand[i] - x.lo) >> s], 1u);
      } else {
        uint32_t least = 0;
        each_of([&](uint32_t, uint32_t k) {
          const uint32_t off = k - x.lo;
          least += (uint32_t)__builtin_popcountll(__builtin_amdgcn_ballot_w64(off == 0));
          if (off - 1 < x.hi - x.lo) atomicAdd(&hist[off >> s], 1u);
        });
        if (lane == 0 && least) atomicAdd(&hist[0], least);
      }
      __syncthreads();
      // counters from the largest down: a thread has two
      const uint32_t h0 = hist[kBins - 1 - 2 * tid], h1 = hist[kBins - 2 - 2 * tid];
      uint32_t sum = h0 + h1;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const uint32_t y = (uint32_t)__shfl_up((int)sum, o, 64);
        if (lane >= o) sum += y;
      }
      if (lane == 63) part[0][wave] = sum;
      __syncthreads();
      uint32_t before = sum - h0 - h1;
      for (int i = 0; i < wave; ++i) before += part[0][i];
      if (before < x.need && x.need <= before + h0 + h1) {
        const bool first = x.need <= before + h0;
        found[0] = kBins - 1 - 2 * tid - (first ? 0u : 1u);
        found[1] = x.need - before - (first ? 0u : h0);
        found[2] = first ? h0 : h1;
      }
      __syncthreads();
      const uint32_t in_bin = __builtin_amdgcn_readfirstlane(found[2]);
      more = search_narrow(&x, __builtin_amdgcn_readfirstlane(found[0]), __builtin_amdgcn_readfirstlane(found[1]), in_bin);
      if (more && !few && in_bin <= kCands) {  // those of the counter, in any order
        if (tid == 0) found[3] = 0;
        __syncthreads();
        each_of([&](uint32_t, uint32_t k) {
          if (k - x.lo <= x.hi - x.lo) cand[atomicAdd(&found[3], 1u) % kCands] = k;
        });
        few = true;
      }
      __syncthreads();
    }
    cut = Cut{x.lo, x.need};
  }

  // ---- the numbers that stay, in order
  uint32_t above = 0, equal = 0;
  each_of([&](uint32_t, uint32_t k) {
    above += (uint32_t)__builtin_popcountll(__builtin_amdgcn_ballot_w64(k > cut.key));
    if (cut.equal) equal += (uint32_t)__builtin_popcountll(__builtin_amdgcn_ballot_w64(k == cut.key));
  });
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
  at = __builtin_amdgcn_readfirstlane(at + min(eq, cut.equal));
  eq = __builtin_amdgcn_readfirstlane(eq);
  const uint32_t end = rq.keep - rq.last;
  auto below = [](uint64_t mask) {
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0u));
  };
  auto put = [&](uint32_t i0, bool take) {
    const uint64_t bt = __builtin_amdgcn_ballot_w64(take);
    const uint32_t to = at + below(bt);
    if (take && to < end) list[to] = (int32_t)(i0 + lane);  // (always, unless the sums change meanwhile)
    at += (uint32_t)__builtin_popcountll(bt);
  };
  if (need0 > 0 && cut.equal == 0)
    each_of([&](uint32_t i0, uint32_t k) { put(i0, k > cut.key); });
  else if (need0 > 0)
    each_of([&](uint32_t i0, uint32_t k) {  // the first of those that are equal, whatever wave has them
      const uint64_t be = __builtin_amdgcn_ballot_w64(k == cut.key);
      put(i0, k > cut.key || (k == cut.key && eq + below(be) < cut.equal));
      eq += (uint32_t)__builtin_popcountll(be);
    });
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
    int32_t from[U];
#pragma unroll
    for (int u = 0; u < U; ++u) from[u] = list[min(c + u * kSelectThreads + tid, rq.keep - 1)];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = w[min((uint32_t)from[u], rq.n - 1)];  // (all written, unless the sums change)
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

namespace {
// A 16-byte column of a row: which KV head's list it goes by, and the bytes from its page
// to it in slot 0 and from slot to slot.
struct Column {
  uint32_t head, step;
  uint64_t at;
};
CP_DEV Column column_of(const GeomK &g, uint32_t seg) {
  if (g.kind == 0) return Column{0u, (uint32_t)g.d_k * 2, 16ull * seg};
  const uint32_t per = (uint32_t)g.d_k / 8, part = seg / per, hkv = (uint32_t)g.hkv, v = part >= hkv;
  const uint32_t h = part - v * hkv;
  return Column{h, (uint32_t)g.d_k * 2, (uint64_t)(2 * h + v) * (uint32_t)g.page_tokens * ((uint32_t)g.d_k * 2) + 16 * (seg - part * per)};
}
}  // namespace

// Rows in place: a workgroup owns COLS columns of 16 bytes of one layer and takes the rows
// that stay in order, THREADS / COLS * UNROLL at once: all are read before any is written,
// and those of later steps lie behind what this one writes (list entries rise: entry k is at
// least k). So no workgroup waits for another. Bound by the round trips of a step (list,
// page table, row), each asked for by all of a thread's rows at once: 2,048 of 16 K and 1,125
// of 9 K tokens, 8 heads of 128, 11 us (13 MB, read twice and written; 142 with one row in flight),
// half of four 4 K contexts in 16 layers 205 (5.2 TB/s);
// accepted paths of 4 requests 3 us, 31 with the lists' loads in a row.
template <int THREADS, int COLS, int UNROLL>
__global__ __launch_bounds__(THREADS) void move_kernel(const MoveArgs a) {
  constexpr uint32_t RPI = THREADS / COLS;
  const int r = sorted_search(a.n_req, blockIdx.x, [&](int i) { return a.req[i].block_begin; });
  const MoveReq &rq = a.req[r];
  const GeomK &g = a.geom[rq.model];
  const uint32_t b = blockIdx.x - rq.block_begin, layer = b / rq.per_layer, P = (uint32_t)g.page_tokens;
  const uint32_t seg = (b - layer * rq.per_layer) * COLS + threadIdx.x % COLS, row = threadIdx.x / COLS;
  const bool mine = seg < (uint32_t)g.row_elems / 8;
  const Column c = column_of(g, mine ? seg : 0u);
  const int32_t *const list = rq.list ? rq.list + (int64_t)layer * rq.list_layer + (int64_t)c.head * rq.list_head
                                      : reinterpret_cast<const int32_t *>(a.ent) + rq.ent0 - rq.k0;
  const uint32_t *const src = rq.src + (uint64_t)layer * rq.src_plane, *const dst = a.pte + rq.dst_base + layer * rq.dst_plane;
#pragma unroll 1
  for (uint32_t base = rq.k0; base < rq.n; base += RPI * UNROLL) {
    uint32_t from[UNROLL], to[UNROLL], fs[UNROLL], ts[UNROLL];
    u32x4m v[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {  // (threads without a row repeat the last one)
      const uint32_t k = min(base + u * RPI + row, rq.n - 1);
      from[u] = rq.first + min((uint32_t)list[k], rq.rows - 1);
      to[u] = rq.first + k;
    }
    bool moves[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      moves[u] = from[u] != to[u];
      from[u] = src[page_divide(from[u], P, a.page_magic, &fs[u])];
      to[u] = dst[page_divide(to[u], P, a.page_magic, &ts[u])];
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      moves[u] = (moves[u] || from[u] != to[u]) && mine && base + u * RPI + row < rq.n;
      v[u] = *reinterpret_cast<const u32x4m *>(a.pool + ((uint64_t)from[u] << 8) + c.at + (uint64_t)fs[u] * c.step);
    }
    __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
    __syncthreads();
#pragma unroll
    for (int u = 0; u < UNROLL; ++u)
      if (moves[u]) *reinterpret_cast<u32x4m *>(a.pool + ((uint64_t)to[u] << 8) + c.at + (uint64_t)ts[u] * c.step) = v[u];
  }
}

// Rows that go to pages which nothing of the call reads: in any order, 16 KiB or a row a
// workgroup. Bound by memory: 27 K of 107 K latent rows, 31 MB read and written, 14 us (4.5 TB/s).
__global__ __launch_bounds__(kApartThreads) void move_apart_kernel(const MoveArgs a) {
  constexpr int U = kApartUnroll;
  const int r = sorted_search(a.n_req, blockIdx.x, [&](int i) { return a.req[i].block_begin; });
  const MoveReq &rq = a.req[r];
  const GeomK &g = a.geom[rq.model];
  const uint32_t b = blockIdx.x - rq.block_begin, layer = b / rq.per_layer, P = (uint32_t)g.page_tokens;
  const uint32_t nseg = (uint32_t)g.row_elems / 8, R = apart_rows(nseg);
  const uint32_t d0 = rq.k0 + (b - layer * rq.per_layer) * R, total = min(R, rq.n - d0) * nseg;
  const int32_t *const lists = rq.list + (int64_t)layer * rq.list_layer;
  const uint32_t *const src = rq.src + (uint64_t)layer * rq.src_plane, *const dst = a.pte + rq.dst_base + layer * rq.dst_plane;
  for (uint32_t i0 = threadIdx.x; i0 < total; i0 += U * kApartThreads) {
    uint32_t from[U], to[U], ts[U];
    uint64_t at[U];
    u32x4m v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {  // (threads without a piece repeat the last one)
      const uint32_t i = min(i0 + u * kApartThreads, total - 1), row = i / nseg, d = d0 + row;
      const Column c = column_of(g, i - row * nseg);
      at[u] = c.at;
      from[u] = min((uint32_t)lists[(int64_t)c.head * rq.list_head + d], rq.rows - 1);
      to[u] = dst[page_divide(d, P, a.page_magic, &ts[u])];
    }
    const uint32_t step = (uint32_t)g.d_k * 2;
    uint32_t fs[U];
#pragma unroll
    for (int u = 0; u < U; ++u) from[u] = src[page_divide(from[u], P, a.page_magic, &fs[u])];
#pragma unroll
    for (int u = 0; u < U; ++u)
      v[u] = __builtin_nontemporal_load(
          reinterpret_cast<const u32x4m *>(a.pool + ((uint64_t)from[u] << 8) + at[u] + (uint64_t)fs[u] * step));
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i0 + u * kApartThreads < total)
        *reinterpret_cast<u32x4m *>(a.pool + ((uint64_t)to[u] << 8) + at[u] + (uint64_t)ts[u] * step) = v[u];
  }
}

hipError_t launch_evict_select(const EvictArgs &a, hipStream_t stream) {
  if (a.n_blocks <= 0) return hipSuccess;
  uint32_t most = 0;
  for (int i = 0; i < a.n_req; ++i) most = a.req[i].n > most ? a.req[i].n : most;
  const dim3 grid((uint32_t)a.n_blocks), block(kSelectThreads);
  if (most <= 4 * kSelectThreads)
    hipLaunchKernelGGL(evict_select_kernel<4>, grid, block, 0, stream, a);
  else if (most <= 16 * kSelectThreads)
    hipLaunchKernelGGL(evict_select_kernel<16>, grid, block, 0, stream, a);
  else if (most <= 64 * kSelectThreads)
    hipLaunchKernelGGL(evict_select_kernel<64>, grid, block, 0, stream, a);
  else
    hipLaunchKernelGGL(evict_select_kernel<0>, grid, block, 0, stream, a);
  return hipGetLastError();
}

// how: 0 short lists in the arguments, 1 in place, 2 apart, 3 in place with few workgroups
hipError_t launch_moves(const MoveArgs &a, int how, hipStream_t stream) {
  if (a.n_blocks <= 0) return hipSuccess;
  const dim3 grid((uint32_t)a.n_blocks);
  if (how == 0)
    hipLaunchKernelGGL((move_kernel<kKeepThreads, kKeepCols, kKeepUnroll>), grid, dim3(kKeepThreads), 0, stream, a);
  else if (how == 1)
    hipLaunchKernelGGL((move_kernel<kMoveThreads, kMoveCols, kMoveUnroll>), grid, dim3(kMoveThreads), 0, stream, a);
  else if (how == 3)
    hipLaunchKernelGGL((move_kernel<kMoveThreads, kMoveFewCols, kMoveUnroll>), grid, dim3(kMoveThreads), 0, stream, a);
  else
    hipLaunchKernelGGL(move_apart_kernel, grid, dim3(kApartThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace cp
