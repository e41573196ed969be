// Rotary positions (cp_rope_*, declared in include/crosspool.h): frequency
// tables, argument checks and launches.
#include "rope.hpp"

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include "status.hpp"

namespace cp {
hipError_t launch_rope(const RopeArgs &a, int32_t items, bool f32, hipStream_t stream);
}  // namespace cp

using namespace cp;

namespace {

struct DeviceScope {
  int prev = -1;
  bool active = false;
  explicit DeviceScope(int dev) {
    if (hipGetDevice(&prev) == hipSuccess && prev != dev) active = hipSetDevice(dev) == hipSuccess;
  }
  ~DeviceScope() {
    if (active) (void)hipSetDevice(prev);
  }
};

constexpr double kTwoPi = 6.283185307179586476925286766559;

// Angles per position; "" or what is wrong with the description.
const char *angles_of(const cp_rope_desc &d, std::vector<double> *out) {
  const int32_t half = d.rot_dim / 2;
  out->resize((size_t)half);
  if (d.scaling == CP_ROPE_TABLE) {
    if (!d.table) return "null table";
    std::copy_n(d.table, half, out->begin());
  } else {
    if (!(d.base > 0)) return "base must be > 0";
    if (d.scaling != CP_ROPE_PLAIN && !(d.factor > 0)) return "factor must be > 0";
    double base = d.base;
    if (d.scaling == CP_ROPE_NTK) {
      if (d.rot_dim < 4) return "NTK scaling needs rot_dim >= 4";
      base *= std::pow(d.factor, (double)d.rot_dim / (d.rot_dim - 2));
    }
    if (d.scaling == CP_ROPE_PARTS && !(d.orig_len > 0 && d.low_turns < d.high_turns))
      return "PARTS scaling needs orig_len > 0 and low_turns < high_turns";
    for (int32_t i = 0; i < half; ++i) {
      double f = std::pow(base, -2.0 * i / d.rot_dim);
      if (d.scaling == CP_ROPE_LINEAR) f /= d.factor;
      if (d.scaling == CP_ROPE_PARTS) {
        const double r = d.orig_len * f / kTwoPi;
        const double w = std::min(1.0, std::max(0.0, (r - d.low_turns) / (d.high_turns - d.low_turns)));
        f = f * w + f / d.factor * (1.0 - w);
      }
      (*out)[(size_t)i] = f;
    }
  }
  for (double f : *out)
    if (!std::isfinite(f)) return "an angle is not finite";
  return "";
}

// Do two of the rows of `width` elements at t S + h H meet (t < tokens, h < heads)?
bool rows_overlap(int64_t tokens, int64_t heads, int64_t S, int64_t H, int64_t width) {
  typedef __int128 wide;
  if (tokens < 1 || (heads > 1 && H < width) || (tokens > 1 && S < width)) return tokens > 0;
  if (heads == 1 || tokens == 1) return false;
  if ((wide)S >= (wide)H * (heads - 1) + width || (wide)H >= (wide)S * (tokens - 1) + width) return false;
  // neither stride steps over all of the other's rows: the tokens next to every head
  for (int64_t h = 1; h < heads; ++h)
    for (wide at = (wide)h * H, t = at / S, end = t + 2; t < end; ++t)
      if (t < tokens && at - t * S < width && t * S - at < width) return true;
  return false;
}

}  // namespace

extern "C" {

cp_status cp_rope_create(const cp_rope_desc *d, int32_t device, cp_rope **out) {
  if (!d || !out) return fail(CP_EINVAL, "null argument");
  *out = nullptr;
  if (d->rot_dim < 2 || d->rot_dim > 1024 || d->rot_dim % 2) return fail(CP_EINVAL, "rot_dim must be even, in [2, 1024]");
  if (d->layout != CP_ROPE_HALF && d->layout != CP_ROPE_INTERLEAVED) return fail(CP_EINVAL, "unknown layout %d", d->layout);
  if (d->scaling < CP_ROPE_PLAIN || d->scaling > CP_ROPE_TABLE) return fail(CP_EINVAL, "unknown scaling %d", d->scaling);
  if (!std::isfinite(d->magnitude)) return fail(CP_EINVAL, "magnitude must be finite");
  std::vector<double> turns;
  const cp_status rc = guarded([&]() -> cp_status {
    const char *e = angles_of(*d, &turns);
    return *e ? fail(CP_EINVAL, "%s", e) : CP_OK;
  });
  if (rc) return rc;
  cp_rope *r = new (std::nothrow) cp_rope();
  if (!r) return fail(CP_ENOMEM, "host allocation failed");
  r->turns.swap(turns);
  for (double &t : r->turns) t /= kTwoPi;
  r->rot = d->rot_dim;
  r->layout = d->layout;
  r->magnitude = d->magnitude == 0 ? 1.f : (float)d->magnitude;
  r->device = device;
  if (device >= 0) {
    int ndev = 0;
    if (hipGetDeviceCount(&ndev) != hipSuccess || device >= ndev) {
      delete r;
      return fail(CP_EINVAL, "device %d not present", device);
    }
    DeviceScope g(device);
    const size_t bytes = r->turns.size() * sizeof(double);
    if (hipMalloc((void **)&r->dev_turns, bytes) != hipSuccess) {
      delete r;
      (void)hipGetLastError();
      return fail(CP_ENOMEM, "allocation of the frequency table failed");
    }
    const hipError_t he = hipMemcpy(r->dev_turns, r->turns.data(), bytes, hipMemcpyHostToDevice);
    if (he != hipSuccess) {
      (void)hipFree(r->dev_turns);
      delete r;
      return fail(CP_EHIP, "frequency table copy: %s", hipGetErrorString(he));
    }
  } else {
    r->device = -1;
  }
  *out = r;
  return CP_OK;
}

cp_status cp_rope_destroy(cp_rope *r) {
  if (!r) return fail(CP_EINVAL, "null rope");
  if (r->dev_turns) {
    DeviceScope g(r->device);
    (void)hipFree(r->dev_turns);
  }
  delete r;
  return CP_OK;
}

cp_status cp_rope_angles(const cp_rope *r, double *angles) {
  if (!r || !angles) return fail(CP_EINVAL, "null argument");
  for (size_t i = 0; i < r->turns.size(); ++i) angles[i] = r->turns[i] * kTwoPi;
  return CP_OK;
}

cp_status cp_rope_apply(const cp_rope *r, int32_t n_tensors, const cp_rope_tensor *t, int64_t n_tokens,
                        const int32_t *positions, int64_t first, int32_t inverse, void *hip_stream) {
  if (!r) return fail(CP_EINVAL, "null rope");
  if (n_tensors < 1 || n_tensors > kMaxRopeParts) return fail(CP_EINVAL, "1 to %d tensors per call", kMaxRopeParts);
  if (!t) return fail(CP_EINVAL, "null tensors");
  if (n_tokens < 0 || n_tokens > 0x7FFFFFFF) return fail(CP_EINVAL, "n_tokens out of range");
  if (first > (1ll << 52) || first < -(1ll << 52)) return fail(CP_EINVAL, "first position out of range");
  RopeArgs a{};
  a.rope = rope_k(*r, inverse != 0);
  a.pos = positions;
  a.first = first;
  a.n_tokens = n_tokens;
  a.n_parts = n_tensors;
  int32_t items = 0;
  for (int32_t i = 0; i < n_tensors; ++i) {
    const cp_rope_tensor &x = t[i];
    if (x.dtype != CP_ROPE_BF16 && x.dtype != CP_ROPE_F32) return fail(CP_EINVAL, "tensor %d: unknown dtype %d", i, x.dtype);
    if (x.dtype != t[0].dtype) return fail(CP_EINVAL, "tensors of one call have one dtype");
    if (x.heads < 1 || x.heads > 65536 || x.width < 1 || x.width > 65536)
      return fail(CP_EINVAL, "tensor %d: heads and width must be in [1, 65536]", i);
    if (x.offset < 0 || x.offset > x.width - r->rot)
      return fail(CP_EINVAL, "tensor %d: rotated elements [%d, %d) outside the width %d", i, x.offset,
                  x.offset + r->rot, x.width);
    if (x.src_token < 0 || x.src_head < 0 || x.dst_token < 0 || x.dst_head < 0)
      return fail(CP_EINVAL, "tensor %d: negative stride", i);
    if (n_tokens > 0 && (!x.src || !x.dst)) return fail(CP_EINVAL, "tensor %d: null pointer", i);
    for (int32_t k = 0; k < i && n_tokens > 0; ++k)  // their workgroups run in no order
      if (x.dst == t[k].dst || x.dst == t[k].src || x.src == t[k].dst)
        return fail(CP_EINVAL, "tensors %d and %d: one writes where the other begins", k, i);
    const bool in_place = x.src == x.dst;
    if (in_place && ((n_tokens > 1 && x.src_token != x.dst_token) || (x.heads > 1 && x.src_head != x.dst_head)))
      return fail(CP_EINVAL, "tensor %d: in place needs the same strides", i);
    if (rows_overlap(n_tokens, x.heads, x.dst_token, x.dst_head, x.width))
      return fail(CP_EINVAL, "tensor %d: heads or tokens of dst overlap", i);
    const int64_t es = x.dtype == CP_ROPE_F32 ? 4 : 2, v = 16 / es;
    if ((uintptr_t)x.src % es || (uintptr_t)x.dst % es) return fail(CP_EINVAL, "tensor %d: misaligned elements", i);
    RopePart &p = a.part[i];
    p = RopePart{x.src, x.dst, x.src_token, x.src_head, x.dst_token, x.dst_head, x.heads, x.width, x.offset, 0};
    // the vector form: whole 16-byte pieces on both sides of every boundary
    auto odd = [&](int64_t e) { return e % v != 0; };
    p.vec = !((uintptr_t)x.src % 16 || (uintptr_t)x.dst % 16 || (n_tokens > 1 && (odd(x.src_token) || odd(x.dst_token))) ||
              (x.heads > 1 && (odd(x.src_head) || odd(x.dst_head))) || odd(x.offset) || odd(x.width) ||
              odd(r->layout == CP_ROPE_HALF ? r->rot / 2 : r->rot));
    // work items of a token: per head the rotated ones (a piece of each half,
    // or a piece of whole pairs), then, out of place, the copied pieces
    const int64_t step = p.vec ? v : 1;
    const int64_t turn = r->layout == CP_ROPE_HALF ? r->rot / 2 / step : (p.vec ? r->rot / v : r->rot / 2);
    const int64_t copy = in_place ? 0 : (x.width - r->rot) / step;
    a.item0[i] = items;
    if ((int64_t)items + (turn + copy) * x.heads > 0x3FFFFFFF) return fail(CP_EINVAL, "too many elements per token");
    items += (int32_t)((turn + copy) * x.heads);
  }
  for (int32_t i = n_tensors; i <= kMaxRopeParts; ++i) a.item0[i] = items;
  if (r->device < 0) return fail(CP_ESTATE, "host-only rotation");
  if (n_tokens == 0) return CP_OK;
  DeviceScope g(r->device);
  const hipError_t e = launch_rope(a, items, t[0].dtype == CP_ROPE_F32, (hipStream_t)hip_stream);
  if (e != hipSuccess) return fail(CP_EHIP, "rope launch: %s", hipGetErrorString(e));
  return CP_OK;
}

}  // extern "C"
