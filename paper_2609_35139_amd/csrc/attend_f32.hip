// Attention over a paged cache, f32 storage.
#include "attend_kernel.h"

namespace cr {
template hipError_t attend<float>(const AttendArgs&, const SeqTable&, hipStream_t);
template hipError_t attend_merge<float>(const AttendArgs&, const SharedParts&, const SeqTable&, int,
                                      hipStream_t);
}  // namespace cr
