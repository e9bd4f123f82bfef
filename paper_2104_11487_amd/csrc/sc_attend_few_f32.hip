// Attention over the paged cache, few rows, fp32 (sc_attend_few.h).
#include "sc_attend_few.h"

namespace sc {

hipError_t launch_attend_few_f32(const AttendParams& p, hipStream_t stream) { return launch_few_dim<float>(p, stream); }

}  // namespace sc
