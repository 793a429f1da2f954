// Stand-ins for the launchers of the operators that keep an answer going, for
// the host-only sanitizer build: every launcher fails without touching its
// arguments.
#include "../../paper_2609_35139_amd/csrc/answer.h"

namespace cr {

LaunchEvents& launch_events() {
  static thread_local LaunchEvents le;
  return le;
}
hipError_t copy_table(const int32_t*, int, int*, hipStream_t) { return hipErrorInvalidValue; }
template <typename T>
hipError_t weigh(const WeighArgs&, const WeighTable&, hipStream_t) { return hipErrorInvalidValue; }
hipError_t choose(const ChooseArgs&, hipStream_t) { return hipErrorInvalidValue; }
hipError_t compact(const CompactArgs&, hipStream_t) { return hipErrorInvalidValue; }
template <typename T>
hipError_t sample(const SampleArgs&, hipStream_t) { return hipErrorInvalidValue; }

#define STUBS(T)                                                                  \
  template hipError_t weigh<T>(const WeighArgs&, const WeighTable&, hipStream_t); \
  template hipError_t sample<T>(const SampleArgs&, hipStream_t);
STUBS(bf16)
STUBS(float)
#undef STUBS

}  // namespace cr
