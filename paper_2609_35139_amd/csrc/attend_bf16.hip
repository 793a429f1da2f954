// Attention over a paged cache, bf16 storage.
#include "attend_kernel.h"

namespace cr {
template hipError_t attend<bf16>(const AttendArgs&, const SeqTable&, hipStream_t);
template hipError_t attend_merge<bf16>(const AttendArgs&, const SharedParts&, const SeqTable&, int,
                                      hipStream_t);
}  // namespace cr
