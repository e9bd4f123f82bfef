// Attention over a paged cache in 4 bits, many rows of bf16, heads above kPackedWideDim (sc_packed_attend.h).
#include "sc_packed_attend.h"

namespace sc {

hipError_t launch_packed_many_bf16(const PackedAttendParams& p, int whole_pages, hipStream_t stream) { return launch_packed<8, 1, kPackedManyWaves, true>(p, whole_pages, stream); }

}  // namespace sc
