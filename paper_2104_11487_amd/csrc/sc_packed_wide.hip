// Attention over a paged cache in 4 bits, many rows at once, bf16 (sc_packed_wide.h).
#include "sc_packed_wide.h"

namespace sc {

hipError_t launch_packed_wide_bf16(const PackedAttendParams& p, hipStream_t stream) {
  const bool twice = p.a.log_rows > log_packed_wide_rows(p.a.dim);
  if (p.a.dim <= 32) return twice ? launch_packed_wide<32, 2>(p, stream) : launch_packed_wide<32, 1>(p, stream);
  if (p.a.dim <= 64) return twice ? launch_packed_wide<64, 2>(p, stream) : launch_packed_wide<64, 1>(p, stream);
  if (p.a.dim <= 96) return launch_packed_wide<96, 1>(p, stream);
  if (p.a.dim <= 128) return launch_packed_wide<128, 1>(p, stream);
  if (p.a.dim <= 192) return launch_packed_wide<192, 1>(p, stream);
  return launch_packed_wide<256, 1>(p, stream);
}

}  // namespace sc
