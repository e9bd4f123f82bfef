// Attention over the paged cache, few rows (sc_attend_few.h), and the join of the chunks that keys were split into.
#include "sc_attend_few.h"

#pragma clang fp contract(off)

namespace sc {

namespace {

constexpr int kJoinWaves = 4;

// One workgroup a row (token, query head): its parts' references, sums and outputs, joined in the order of their keys. The parts' weights
// go to LDS, 256 at a time; the parts are dealt to groups of dim / 4 lanes (a power of two), whose shares are then added in order.
// SHARES: the parts of the few-rows kernel, otherwise those of the wide kernel.
template <typename T, bool SHARES>
__global__ void __launch_bounds__(64 * kJoinWaves) attend_join_kernel(AttendParams p) {
  constexpr int kThreads = 64 * kJoinWaves;
  __shared__ floatx4 shares[kThreads];
  __shared__ float weights[kThreads], tops[kJoinWaves], sums[kJoinWaves];
  const int token = (int)blockIdx.x / p.q_heads, h = (int)blockIdx.x - token * p.q_heads;
  int b;
  Sequence s;
  Shape o;
  int64_t first;
  const Units<SHARES> units(p);
  if (!units.find(token, true, &b, &s, &o, &first)) return;
  const int head = h / p.group, row = (token - s.start) * p.group + (h - head * p.group);
  const int tile = row >> p.log_rows, rows = 1 << p.log_rows;
  const int64_t unit = first + ((int64_t)head * o.tiles + (o.tiles - 1 - tile)) * o.parts;
  int64_t slot0 = unit;  // the first part's slot; the next ones follow, `step` apart
  int parts = o.parts, step = 1, skip = 0;
  if constexpr (SHARES) {
    // workgroups w0 .. w1 held the item's units; each one's part is its first (slot 2 w), but where the share began before the item,
    // which only the first of them can, its last (2 w + 1)
    const Shares all = shares_of(p, units.all);
    const int w0 = all.holder(unit), w1 = all.holder(unit + o.parts - 1);
    parts = w1 - w0 + 1, step = 2;
    slot0 = 2 * (int64_t)w0;
    skip = all.at(w0) < unit ? 1 : 0;
  }
  if (parts <= 1 || slot0 + (int64_t)parts * step > p.slots) return;
  const int in_tile = row - (tile << p.log_rows);
  auto part_at = [&](int i) { return (slot0 + (int64_t)i * step + (i == 0 ? skip : 0)) * rows + in_tile; };
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;

  int width = 8;
  while (width * 4 < p.dim) width *= 2;  // lanes of a group: 8..64
  const int group = tid / width, groups = kThreads / width, e = (tid & (width - 1)) * 4;

  float top = kNegInf;
  for (int i = tid; i < parts; i += kThreads) top = fmaxf(top, p.part_ml[part_at(i) * 2]);
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  if (lane == 0) tops[wave] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kJoinWaves; ++w) top = fmaxf(top, tops[w]);

  floatx4 v{0.0f, 0.0f, 0.0f, 0.0f};
  float total = 0.0f;
  for (int i0 = 0; i0 < parts; i0 += kThreads) {
    const int n = min(parts - i0, kThreads);
    if (i0 > 0) __syncthreads();
    if (tid < n) {
      const floatx2 ml = *reinterpret_cast<const floatx2*>(p.part_ml + part_at(i0 + tid) * 2);
      weights[tid] = join_weight(ml.x, top);
      total += ml.y * weights[tid];
    }
    __syncthreads();
    if (e < p.dim) {
#pragma unroll 4
      for (int i = group; i < n; i += groups) {
        const floatx4 y = *reinterpret_cast<const floatx4*>(p.part_o + part_at(i0 + i) * p.dim + e);
        const float f = weights[i];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] += y[k] * f;
      }
    }
  }
  shares[tid] = v;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) total += __shfl_xor(total, d);
  if (lane == 0) sums[wave] = total;
  __syncthreads();
  if (group > 0 || e >= p.dim) return;
  total = 0.0f;
#pragma unroll
  for (int w = 0; w < kJoinWaves; ++w) total += sums[w];
  for (int g = 1; g < min(groups, parts); ++g) {
    const floatx4 x = shares[g * width + tid];
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
  const bool shares = p.log_rows != kLogWideRows && p.log_rows != kLogWideRows + 1;
  if (elem_bytes == 2) {
    if (shares) attend_join_kernel<uint16_t, true><<<grid, block, 0, stream>>>(p);
    else attend_join_kernel<uint16_t, false><<<grid, block, 0, stream>>>(p);
  } else {
    if (shares) attend_join_kernel<float, true><<<grid, block, 0, stream>>>(p);
    else attend_join_kernel<float, false><<<grid, block, 0, stream>>>(p);
  }
  return hipGetLastError();
}

}  // namespace sc
