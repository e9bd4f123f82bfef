// Attention over a paged cache in 4 bits, many rows, fp32 (sc_packed_attend.h).
#include "sc_packed_attend.h"

namespace sc {

hipError_t launch_packed_many_f32(const PackedAttendParams& p, int whole_pages, hipStream_t stream) { return launch_packed_dim<2, kPackedManyWaves, true>(p, whole_pages, stream); }

}  // namespace sc
