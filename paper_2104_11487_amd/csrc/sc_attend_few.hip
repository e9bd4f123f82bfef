// Attention over the paged cache, few rows (sc_attend_few.h), and the join of the chunks that keys were split into.
#include "sc_attend_few.h"

#pragma clang fp contract(off)

namespace sc {

namespace {

constexpr int kJoinWaves = 4;  // waves of a workgroup that joins many rows
// Of one that joins a row: a thread for each of its parts, which are no more than the workgroups that share keys. 16 waves start later
// (one token over 262141, heads of 128: 61 instead of 62 us, but over 4000 16.4 instead of 15.1).
constexpr int kRowWaves = 8;
static_assert(64 * kRowWaves >= kMostShared, "a thread a part");

// Where a row's parts lie in the workspace.
struct Parts {
  int64_t slot0;
  int count, skip, in_tile;
  __device__ __forceinline__ int64_t at(int i, int log_rows) const { return ((slot0 + 2 * (int64_t)i + (i == 0 ? skip : 0)) << log_rows) + in_tile; }
};

// The parts of row (token, query head h), of which the sequence and its cut are known; count 0: the row was not split.
__device__ __forceinline__ Parts parts_of(const AttendParams& p, const Units& units, const Sequence& s, const Shape& o, int64_t first, int token, int h) {
  const int head = h / p.group, row = (token - s.start) * p.group + (h - head * p.group), tile = row >> p.log_rows;
  const int64_t unit = first + ((int64_t)head * o.tiles + (o.tiles - 1 - tile)) * o.parts;
  // workgroups w0 .. w1 held the item's units; each one's part is its first (slot 2 w), but where the share began before the item,
  // which only the first of them can, its last (2 w + 1)
  const Shares all = shares_of(units);
  const int w0 = all.holder(unit), w1 = all.holder(unit + o.parts - 1);
  Parts r = {2 * (int64_t)w0, w1 - w0 + 1, all.at(w0) < unit ? 1 : 0, row - (tile << p.log_rows)};
  if (r.count <= 1 || r.slot0 + 2 * (int64_t)r.count > p.slots) r.count = 0;
  return r;
}

template <typename T>
__device__ __forceinline__ void store_row(const AttendParams& p, int token, int h, int e, const floatx4& v, float top, float total) {
  const float inv = total == 0.0f ? 0.0f : 1.0f / total;
  char* to = p.out + ((int64_t)token * p.o_token + (int64_t)h * p.o_head) * (int64_t)sizeof(T);
  if constexpr (sizeof(T) == 2) *reinterpret_cast<u32x2*>(to + e * 2) = u32x2{pack2(v[0] * inv, v[1] * inv), pack2(v[2] * inv, v[3] * inv)};
  else *reinterpret_cast<floatx4*>(to + e * 4) = floatx4{v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv};
  if (p.lse && e == 0)
    p.lse[(int64_t)token * p.q_heads + h] = total == 0.0f ? kNegInf : (top + __builtin_amdgcn_logf(total)) * 0.69314718055994531f;
}

// Many rows: each takes `width` lanes (dim / 4, a power of two), which go through its parts in the order of their keys.
template <typename T>
__global__ void __launch_bounds__(64 * kJoinWaves) attend_join_rows_kernel(AttendParams p, int width) {
  const Units units(p);
  const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6), mine = lane / width, e = (lane - mine * width) * 4;
  const int rows = 64 / width, all = p.c.tokens * p.q_heads;
  const int row0 = ((int)blockIdx.x * kJoinWaves + wave) * rows;
  Parts parts = {0, 0, 0, 0};
  Sequence s;
  Shape o;
  int64_t first = 0;
  int b, known = -1;
  bool held = false;
  for (int i = 0; i < rows && row0 + i < all; ++i) {
    const int token = (row0 + i) / p.q_heads;
    if (token != known) held = units.find(token, true, &b, &s, &o, &first), known = token;
    if (!held || o.parts <= 1) continue;
    const Parts r = parts_of(p, units, s, o, first, token, row0 + i - token * p.q_heads);
    if (i == mine) parts = r;
  }
  if (parts.count == 0 || e >= p.dim) return;
  float top = kNegInf;
  for (int i = 0; i < parts.count; ++i) top = fmaxf(top, p.part_ml[parts.at(i, p.log_rows) * 2]);
  floatx4 v{0.0f, 0.0f, 0.0f, 0.0f};
  float total = 0.0f;
#pragma unroll 4
  for (int i = 0; i < parts.count; ++i) {
    const int64_t at = parts.at(i, p.log_rows);
    const floatx2 ml = *reinterpret_cast<const floatx2*>(p.part_ml + at * 2);
    const floatx4 x = *reinterpret_cast<const floatx4*>(p.part_o + at * p.dim + e);
    const float f = join_weight(ml.x, top);
    total += ml.y * f;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] += x[k] * f;
  }
  const int token = (row0 + mine) / p.q_heads;
  store_row<T>(p, token, row0 + mine - token * p.q_heads, e, v, top, total);
}

// Few rows, one a workgroup: its parts are dealt to groups of `width` lanes, which load their first ones before the weights are known.
// Their shares are added in a fixed order, within each wave and then over the waves.
template <typename T>
__global__ void __launch_bounds__(64 * kRowWaves) attend_join_kernel(AttendParams p, int width) {
  constexpr int kThreads = 64 * kRowWaves, kHeld = 8;
  __shared__ floatx4 shares[kThreads];
  __shared__ float weights[kThreads], tops[kRowWaves], sums[kRowWaves];
  const int token = (int)blockIdx.x / p.q_heads, h = (int)blockIdx.x - token * p.q_heads;
  int b;
  Sequence s;
  Shape o;
  int64_t first;
  const Units units(p);
  if (!units.find(token, true, &b, &s, &o, &first)) return;
  const Parts parts = parts_of(p, units, s, o, first, token, h);
  if (parts.count == 0) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int group = tid / width, groups = kThreads / width, e = (tid & (width - 1)) * 4;
  const auto part = [&](int i) {
    return i < parts.count && e < p.dim ? *reinterpret_cast<const floatx4*>(p.part_o + parts.at(i, p.log_rows) * p.dim + e) : floatx4{};
  };
  floatx4 held[kHeld];
#pragma unroll
  for (int j = 0; j < kHeld; ++j) held[j] = part(group + j * groups);
  floatx2 ml{kNegInf, 0.0f};
  if (tid < parts.count) ml = *reinterpret_cast<const floatx2*>(p.part_ml + parts.at(tid, p.log_rows) * 2);

  float top = ml.x;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  if (lane == 0) tops[wave] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kRowWaves; ++w) top = fmaxf(top, tops[w]);
  const float weight = tid < parts.count ? join_weight(ml.x, top) : 0.0f;
  float total = tid < parts.count ? ml.y * weight : 0.0f;
  weights[tid] = weight;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) total += __shfl_xor(total, d);
  if (lane == 0) sums[wave] = total;
  __syncthreads();

  floatx4 v{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int j = 0; j < kHeld; ++j) {
    if (group + j * groups >= parts.count) break;
    const float f = weights[group + j * groups];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] += held[j][k] * f;
  }
#pragma unroll 4
  for (int i = group + kHeld * groups; i < parts.count; i += groups) {
    const floatx4 y = part(i);
    const float f = weights[i];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] += y[k] * f;
  }
  for (int d = width; d < 64; d <<= 1)
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] += __shfl_xor(v[k], d);
  if (lane < width) shares[wave * width + lane] = v;
  __syncthreads();
  if (tid >= width || e >= p.dim) return;
  total = 0.0f, v = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int w = 0; w < kRowWaves; ++w) {
    const floatx4 x = shares[w * width + tid];
    total += sums[w];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] += x[k];
  }
  store_row<T>(p, token, h, e, v, top, total);
}

template <typename T>
void launch_join(const AttendParams& p, int few, hipStream_t stream) {
  const int rows = p.c.tokens * p.q_heads;
  int width = 8;
  while (width * 4 < p.dim) width *= 2;  // lanes of a row: 8..64
  // A workgroup a row while those do not fill the GPU (one token over 262141 keys, 8 rows of 241 parts); then lane groups, of
  // which many rows of few parts need no exchange.
  if (rows < few) {
    attend_join_kernel<T><<<dim3((unsigned)rows), dim3(64 * kRowWaves), 0, stream>>>(p, width);
  } else {
    const int each = kJoinWaves * (64 / width);
    attend_join_rows_kernel<T><<<dim3((unsigned)((rows + each - 1) / each)), dim3(64 * kJoinWaves), 0, stream>>>(p, width);
  }
}

}  // namespace

int few_waves_of(int elem_bytes, int dim) {
  const int tile = pow2_at_least(dim * elem_bytes < 64 ? 64 : dim * elem_bytes) * (elem_bytes == 2 ? 32 : 16);
  return tile * 4 * 8 <= 131072 ? 8 : 131072 / (tile * 4);
}

hipError_t launch_attend_few_bf16(const AttendParams& p, hipStream_t stream) { return launch_few_dim<uint16_t>(p, stream); }

hipError_t launch_attend_join(const AttendParams& p, int elem_bytes, int few, hipStream_t stream) {
  if (p.target > kMostShared) return hipErrorInvalidValue;
  if (elem_bytes == 2) launch_join<uint16_t>(p, few, stream);
  else launch_join<float>(p, few, stream);
  return hipGetLastError();
}

}  // namespace sc
