// A stand-in for the HIP runtime calls of the library's host side, for tests of its
// error paths on the CPU: device memory is host memory, kernels do not run, and the
// test chooses which launch or asynchronous copy fails. Loaded with RTLD_GLOBAL
// ahead of the library, so that the library's calls bind to it.
#include <cstdint>
#include <cstdlib>
#include <cstring>

typedef int hipError_t;
typedef void *hipStream_t;
struct dim3_t {
  uint32_t x, y, z;
};

namespace {
int g_fail_in = 0;   // the n-th launch or asynchronous copy from now on fails (0: none)
int g_last = 0;      // hipGetLastError
int g_launches = 0;
int g_no_memory = 0;  // device allocations fail
constexpr int kLaunchFailure = 719;
int step() {
  if (g_fail_in > 0 && --g_fail_in == 0) return g_last = kLaunchFailure;
  return 0;
}
}  // namespace

extern "C" {
void fake_fail_in(int n) { g_fail_in = n; }
void fake_no_memory(int on) { g_no_memory = on; }
void fake_leave_error(int e) { g_last = e; }
int fake_launches() { return g_launches; }

hipError_t hipGetDeviceCount(int *n) { return *n = 1, 0; }
hipError_t hipGetDevice(int *d) { return *d = 0, 0; }
hipError_t hipSetDevice(int) { return 0; }
hipError_t hipDeviceGetAttribute(int *v, int, int) { return *v = 256, 0; }
hipError_t hipDeviceSynchronize() { return 0; }
hipError_t hipMalloc(void **p, size_t n) {
  if (g_no_memory) return g_last = 2;
  return (*p = calloc(1, n)) ? 0 : 2;
}
hipError_t hipFree(void *p) { return free(p), 0; }
hipError_t hipHostMalloc(void **p, size_t n, unsigned) { return hipMalloc(p, n); }
hipError_t hipHostFree(void *p) { return free(p), 0; }
hipError_t hipMemset(void *p, int v, size_t n) { return memset(p, v, n), 0; }
hipError_t hipMemcpy(void *d, const void *s, size_t n, int) { return memcpy(d, s, n), 0; }
hipError_t hipMemcpyAsync(void *d, const void *s, size_t n, int, hipStream_t) {
  if (const int e = step()) return e;
  return memcpy(d, s, n), 0;
}
hipError_t hipGetLastError() {
  const int e = g_last;
  g_last = 0;
  return e;
}
hipError_t __hipPushCallConfiguration(dim3_t, dim3_t, size_t, hipStream_t) { return 0; }
hipError_t __hipPopCallConfiguration(dim3_t *grid, dim3_t *block, size_t *lds, hipStream_t *stream) {
  *grid = *block = dim3_t{1, 1, 1};
  return *lds = 0, *stream = nullptr, 0;
}
hipError_t hipLaunchKernel(const void *, dim3_t, dim3_t, void **, size_t, hipStream_t) {
  ++g_launches;
  return step();
}
hipError_t hipExtLaunchKernel(const void *, dim3_t, dim3_t, void **, size_t, hipStream_t, void *, void *, int) {
  ++g_launches;
  return step();
}
}
