// The stand-in of fake_hip.cpp with a look at what is launched, and, where the test asks
// for it, asynchronous copies that run late: when the host waits for an event behind
// them or for the device, as behind earlier work of a stream.
#define hipMemcpyAsync prompt_copy
#define hipDeviceSynchronize prompt_synchronize
#define hipLaunchKernel quiet_launch
#include "fake_hip.cpp"
#undef hipMemcpyAsync
#undef hipDeviceSynchronize
#undef hipLaunchKernel

#include <deque>
#include <string>

#include "compact.h"

namespace {
struct Copy {
  void *to;
  const void *from;
  std::string meant;  // what was there when the copy was asked for
  long number;
};
std::deque<Copy> g_queue;
long g_enqueued = 0, g_waits = 0, g_changed = 0;
bool g_late = false;
int g_capturing = 0;
void (*g_launched)(const void *args) = nullptr;
void run_to(long number) {
  while (!g_queue.empty() && g_queue.front().number <= number) {
    const Copy c = g_queue.front();
    g_queue.pop_front();
    g_changed += memcmp(c.from, c.meant.data(), c.meant.size()) != 0;
    memcpy(c.to, c.from, c.meant.size());
  }
}
}  // namespace

extern "C" {
void late_copies(int on) { g_late = on; }
void capturing(int on) { g_capturing = on; }
long changed_copies() { return g_changed; }  // that ran with other bytes than they were asked for with
long copies() { return g_enqueued; }
void watch_launches(void (*f)(const void *)) { g_launched = f; }
long host_waits() { return g_waits; }

hipError_t hipMemcpyAsync(void *d, const void *s, size_t n, int kind, hipStream_t st) {
  if (!g_late) return prompt_copy(d, s, n, kind, st);
  if (const int e = step()) return e;
  g_queue.push_back(Copy{d, s, std::string(static_cast<const char *>(s), n), ++g_enqueued});
  return 0;
}
hipError_t hipDeviceSynchronize() { return ++g_waits, run_to(g_enqueued), 0; }
hipError_t hipStreamSynchronize(hipStream_t) { return ++g_waits, run_to(g_enqueued), 0; }
hipError_t hipStreamIsCapturing(hipStream_t, int *status) { return *status = g_capturing, 0; }
hipError_t hipLaunchKernel(const void *, dim3_t, dim3_t, void **args, size_t, hipStream_t) {
  ++g_launches;
  if (g_launched) g_launched(args[0]);
  return step();
}

// The rows that a launch of cp_request_keep moves: {first entry of the request's pages, place,
// token}, at most `room` of them; returns how many.
int kept_rows(const void *args, int64_t (*out)[3], int room) {
  const auto &a = *static_cast<const cp::MoveArgs *>(args);
  int n = 0;
  for (int r = 0; r < a.n_req; ++r)
    for (uint32_t k = a.req[r].k0; k < a.req[r].n && n < room; ++k, ++n) {
      out[n][0] = a.req[r].dst_base;
      out[n][1] = k;
      out[n][2] = a.ent[a.req[r].ent0 + k - a.req[r].k0];
    }
  return n;
}
}
