// Attention over the paged cache, few rows (sc_attend_few.h), and the join of the chunks that keys were split into.
#include "sc_attend_few.h"

#pragma clang fp contract(off)

namespace sc {

namespace {

constexpr int kJoinWaves = 4;

// One workgroup a row (token, query head): its chunks' references, sums and outputs, joined in chunk order. The chunks are
// dealt to lane groups of dim / 4 lanes (a power of two), whose shares are then added in order.
template <typename T>
__global__ void __launch_bounds__(64 * kJoinWaves) attend_join_kernel(AttendParams p) {
  constexpr int kMost = 64 * kJoinWaves / 8;  // lane groups at the least head dimension
  __shared__ floatx4 shares[64 * kJoinWaves];
  __shared__ float sums[kMost];
  const int token = (int)blockIdx.x / p.q_heads, h = (int)blockIdx.x - token * p.q_heads;
  const int b = owner_of(p.c.row_start, p.c.batch, token);
  if (b >= p.c.batch) return;
  int at, first;
  Sequence s;
  Shape o;
  if (!find_units(p, b, 1, &at, &s, &o, &first) || o.splits <= 1) return;
  const int row = (token - s.start) * p.group + h % p.group;
  if (token < s.start || row >= s.n * p.group) return;
  const int tile = row >> p.log_rows;
  const int64_t unit = (int64_t)first + (int64_t)(h / p.group) * o.tiles * o.splits + (int64_t)(o.tiles - 1 - tile) * o.splits;
  if (unit + o.splits > p.units) return;
  const int rows = 1 << p.log_rows;
  const int64_t part0 = unit * rows + (row - (tile << p.log_rows));

  int width = 8;
  while (width * 4 < p.dim) width *= 2;  // lanes of a group: 8..64
  const int group = (int)threadIdx.x / width, groups = 64 * kJoinWaves / width, e = ((int)threadIdx.x & (width - 1)) * 4;

  float top = kNegInf;
  for (int i = threadIdx.x & 63; i < o.splits; i += 64) top = fmaxf(top, p.part_ml[(part0 + (int64_t)i * rows) * 2]);
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));

  floatx4 v{0.0f, 0.0f, 0.0f, 0.0f};
  float total = 0.0f;
  for (int i = group; i < o.splits; i += groups) {
    const int64_t part = part0 + (int64_t)i * rows;
    const floatx2 ml = *reinterpret_cast<const floatx2*>(p.part_ml + part * 2);
    if (ml.x != kNegInf) {
      const float f = __builtin_amdgcn_exp2f(ml.x - top);
      total += ml.y * f;
      if (e < p.dim) {
        const floatx4 x = *reinterpret_cast<const floatx4*>(p.part_o + part * p.dim + e);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] += x[k] * f;
      }
    }
  }
  shares[threadIdx.x] = v;
  if (e == 0) sums[group] = total;
  __syncthreads();
  if (group > 0 || e >= p.dim) return;
  for (int g = 1; g < min(groups, o.splits); ++g) {
    const floatx4 x = shares[g * width + (int)threadIdx.x];
    total += sums[g];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] += x[k];
  }
  const float inv = total == 0.0f ? 0.0f : 1.0f / total;
  char* to = p.out + ((int64_t)token * p.o_token + (int64_t)h * p.o_head) * (int64_t)sizeof(T);
  if constexpr (sizeof(T) == 2) *reinterpret_cast<u32x2*>(to + e * 2) = u32x2{pack2(v[0] * inv, v[1] * inv), pack2(v[2] * inv, v[3] * inv)};
  else *reinterpret_cast<floatx4*>(to + e * 4) = floatx4{v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv};
  if (p.lse && e == 0)
    p.lse[(int64_t)token * p.q_heads + h] = total == 0.0f ? kNegInf : (top + __builtin_amdgcn_logf(total)) * 0.69314718055994531f;
}

}  // namespace

int few_waves_of(int elem_bytes, int dim) {
  const int tile = pow2_at_least(dim * elem_bytes < 64 ? 64 : dim * elem_bytes) * (elem_bytes == 2 ? 32 : 16);
  return tile * 4 * 8 <= 131072 ? 8 : 131072 / (tile * 4);
}

hipError_t launch_attend_few_bf16(const AttendParams& p, hipStream_t stream) { return launch_few_dim<uint16_t>(p, stream); }

hipError_t launch_attend_join(const AttendParams& p, int elem_bytes, hipStream_t stream) {
  const dim3 grid((unsigned)(p.c.tokens * p.q_heads)), block(64 * kJoinWaves);
  if (elem_bytes == 2) attend_join_kernel<uint16_t><<<grid, block, 0, stream>>>(p);
  else attend_join_kernel<float><<<grid, block, 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace sc
