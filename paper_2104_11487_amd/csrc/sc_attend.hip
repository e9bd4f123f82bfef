// Attention over the paged cache, many rows at once, bf16 (sc_attend_wide.h).
#include "sc_attend_wide.h"

namespace sc {

hipError_t launch_attend_wide_bf16(const AttendParams& p, int uniform_pages, hipStream_t stream) {
  return launch_wide_dim<uint16_t>(p, uniform_pages, stream);
}

}  // namespace sc
