// Attention over a paged cache in 4 bits, few rows, fp32 (sc_packed_attend.h).
#include "sc_packed_attend.h"

namespace sc {

hipError_t launch_packed_few_f32(const PackedAttendParams& p, int waves, int whole_pages, hipStream_t stream) {
  return waves == 8 ? launch_packed_dim<2, 8, false>(p, whole_pages, stream) : launch_packed_dim<2, 4, false>(p, whole_pages, stream);
}

}  // namespace sc
