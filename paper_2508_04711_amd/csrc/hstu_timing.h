// Optional per-launch timing (hstu_debug_timing_begin/end): thread-local, off by default.
#pragma once
#include <hip/hip_runtime.h>

#include <vector>

namespace hstu {

struct Timing {
  bool on = false;
  std::vector<hipEvent_t> start, stop;
  std::vector<int> kind;
  size_t used = 0;
};
extern thread_local Timing g_timing;  // (hstu_api.hip)

struct TimedLaunch {
  hipStream_t stream;
  bool active;
  TimedLaunch(int kind, hipStream_t s) : stream(s), active(false) {
    Timing& t = g_timing;
    if (t.on && t.used < t.start.size()) {
      active = true;
      t.kind[t.used] = kind;
      (void)hipEventRecord(t.start[t.used], stream);
    }
  }
  ~TimedLaunch() {
    if (active) {
      Timing& t = g_timing;
      (void)hipEventRecord(t.stop[t.used], stream);
      ++t.used;
    }
  }
};

}  // namespace hstu
