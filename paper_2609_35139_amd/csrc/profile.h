// Per-launch timing of the entry points (cr_profile_*; internal to the library).
#pragma once
#include <hip/hip_runtime_api.h>

#include <atomic>
#include <mutex>
#include <string>
#include <vector>

#include "launch.h"

namespace cr {

struct Profiler {
  std::mutex mu;
  std::vector<hipEvent_t> ev;        // 2 per launch slot
  std::vector<std::string> cls;      // class of each used slot
  std::vector<char> valid;           // the slot's events were recorded
  int used = 0;
  std::atomic<bool> on{false};       // read without the lock on every launch
};
inline Profiler& prof() {
  static Profiler p;
  return p;
}

// Launch `f` on stream s, bracketed by events when profiling is enabled.
// While a slot is in use the profiler's lock is held, so a concurrent
// cr_profile_enable cannot destroy its events; a stage that fails leaves its
// slot marked invalid (its events may never be recorded).
template <typename F>
hipError_t timed(const char* name, hipStream_t s, F&& f) {
  Profiler& P = prof();
  if (!P.on) return f();
  std::unique_lock<std::mutex> g(P.mu);
  if (!P.on || P.used >= (int)P.ev.size() / 2) {
    g.unlock();
    return f();
  }
  const int slot = P.used++;
  P.cls.emplace_back(name);
  P.valid.push_back(0);
  const hipEvent_t e0 = P.ev[2 * slot], e1 = P.ev[2 * slot + 1];
  LaunchEvents& le = launch_events();
  le.start = e0;
  le.stop = e1;
  hipError_t e = f();
  if (e == hipSuccess && le.start) {   // the stage launched nothing: an empty interval
    e = hipEventRecord(e0, s);
    if (e == hipSuccess) e = hipEventRecord(e1, s);
  }
  le = LaunchEvents{};
  P.valid[slot] = e == hipSuccess;
  return e;
}

// Inside an entry point: a failed launch ends it with CR_ERR_LAUNCH.
#define CR_TRY(...)                                 \
  do {                                            \
    if ((__VA_ARGS__) != hipSuccess) return CR_ERR_LAUNCH; \
  } while (0)

}  // namespace cr
