// Attention over a paged cache in 4 bits, few rows, bf16 (sc_packed_attend.h).
#include "sc_packed_attend.h"

namespace sc {

hipError_t launch_packed_few_bf16(const PackedAttendParams& p, int waves, int whole_pages, hipStream_t stream) {
  return waves == 8 ? launch_packed_dim<1, 8, false>(p, whole_pages, stream) : launch_packed_dim<1, 4, false>(p, whole_pages, stream);
}

}  // namespace sc
