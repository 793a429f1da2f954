// Stand-ins for the launchers of the paged-cache operators, for the host-only
// sanitizer build: every launcher fails without touching its arguments.
#include "../../paper_2609_35139_amd/csrc/serve.h"

namespace cr {

LaunchEvents& launch_events() {
  static thread_local LaunchEvents le;
  return le;
}
hipError_t copy_table(const int32_t*, int, int*, hipStream_t) { return hipErrorInvalidValue; }
template <typename T>
hipError_t append_kv(const AppendArgs&, const KeyRope&, const int32_t*, hipStream_t) {
  return hipErrorInvalidValue;
}
template <typename T>
hipError_t attend(const AttendArgs&, const SeqTable&, hipStream_t) { return hipErrorInvalidValue; }
template <typename T>
hipError_t attend_merge(const AttendArgs&, const SharedParts&, const SeqTable&, int, hipStream_t) {
  return hipErrorInvalidValue;
}

#define STUBS(T)                                                                              \
  template hipError_t append_kv<T>(const AppendArgs&, const KeyRope&, const int32_t*,        \
                                   hipStream_t);                                             \
  template hipError_t attend<T>(const AttendArgs&, const SeqTable&, hipStream_t);             \
  template hipError_t attend_merge<T>(const AttendArgs&, const SharedParts&, const SeqTable&, \
                                      int, hipStream_t);
STUBS(bf16)
STUBS(float)
#undef STUBS

}  // namespace cr
