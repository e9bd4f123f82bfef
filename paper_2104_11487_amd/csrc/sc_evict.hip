// Eviction: of each sequence and key head the newest tokens and of the others those of the largest accumulated weight stay, in their order,
// and move to other pages.
//
// First launch, a workgroup a sequence and key head: the weight that divides kept from evicted is found digit by digit (11, 11 and 10 bits of
// the weights as ordered integers, a histogram in LDS each), then the kept positions are written in order by a scan. Of equal
// weights at the border the earlier tokens stay. Second launch: the kept rows' bytes move; source and destination pages are
// different ones, so rows move in any order.
#include "sc_packed_device.h"

#include <algorithm>

#pragma clang fp contract(off)

namespace sc {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64, kBins = 2048;
constexpr int kMoveThreads = 256;

// Integers in the order of the weights: NaN above all, -0 as +0. No weight maps to 0.
__device__ __forceinline__ uint32_t ordered(float w) {
  if (w != w) return 0xffffffffu;
  const uint32_t u = __float_as_uint(w + 0.0f);
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

struct Kept {
  int len, keep, late;  // tokens; kept ones; from `late` on all are kept
};
__device__ __forceinline__ Kept kept_of(const EvictParams& p, int b) {
  const int64_t room = (int64_t)p.c.width * p.c.page_size;
  const int len = (int)min((int64_t)max(p.c.kv_len[b], 0), min(room, (int64_t)kMostKeys));
  const int keep = min(len, p.keep);
  return {len, keep, len - min(keep, p.recent)};
}

__global__ void __launch_bounds__(kThreads) evict_select_kernel(EvictParams p) {
  __shared__ uint32_t bins[kBins];
  __shared__ int sums[2][kWaves];
  __shared__ uint32_t found[2];  // digit of the border, tokens above it
  const int b = (int)blockIdx.x / p.kv_heads, head = (int)blockIdx.x - b * p.kv_heads;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const Kept s = kept_of(p, b);
  if (head == 0 && tid == 0) p.lengths[b] = s.keep;
  int32_t* const out = p.kept + (int64_t)blockIdx.x * p.keep;
  for (int i = s.keep + tid; i < p.keep; i += kThreads) out[i] = -1;
  if (s.keep == s.len) {
    for (int i = tid; i < s.keep; i += kThreads) out[i] = i;
    return;
  }
  const auto key_at = [&](int l) {  // of a token that has no place in the cache: below all weights
    const int i = page_of(p.c, l), page = p.c.table[(int64_t)b * p.c.width + i];
    if (page < 0 || page >= p.c.pages) return 0u;
    return ordered(p.weights[((int64_t)page * p.kv_heads + head) * p.c.page_size + (l - i * p.c.page_size)]);
  };

  // The border: the key of the `want`-th largest of the tokens before `late`, and how many of those equal to it stay.
  int want = s.keep - (s.len - s.late);
  uint32_t border = 0xffffffffu, prefix = 0, known = 0;
  if (want > 0) {
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, width = pass == 2 ? 10 : 11;
      for (int i = tid; i < kBins; i += kThreads) bins[i] = 0;
      __syncthreads();
      for (int l = tid; l < s.late; l += kThreads) {
        const uint32_t key = key_at(l);
        if ((key & known) == prefix) atomicAdd(&bins[(key >> shift) & ((1u << width) - 1)], 1u);
      }
      __syncthreads();
      // from the largest digit on: lane and wave hold two bins each, in descending order
      const int top = kBins - 1 - 2 * tid;
      const int n0 = (int)bins[top], n1 = (int)bins[top - 1];
      int upto = scan32(n0 + n1);
      if (lane == 63) sums[0][wave] = upto;
      __syncthreads();
      for (int w = 0; w < wave; ++w) upto += sums[0][w];
      const int before = upto - n0 - n1;
      if (before < want && want <= before + n0) found[0] = (uint32_t)top, found[1] = (uint32_t)before;
      else if (before + n0 < want && want <= upto) found[0] = (uint32_t)top - 1, found[1] = (uint32_t)(before + n0);
      __syncthreads();
      prefix |= found[0] << shift, known |= ((1u << width) - 1) << shift;
      want -= (int)found[1];
      __syncthreads();
    }
    border = prefix;
  }
  // The kept ones in order: those above the border, the first `want` equal to it, and the late ones.
  int equals = 0, count = 0;
  for (int l0 = 0; l0 < s.len; l0 += kThreads) {
    const int l = l0 + tid;
    const bool old = l < s.late;
    const uint32_t key = old && want > 0 ? key_at(l) : 0u;
    const bool equal = old && want > 0 && key == border;
    const uint64_t before = (1ull << lane) - 1, equal_mask = __ballot(equal);
    if (lane == 0) sums[0][wave] = (int)__popcll(equal_mask);
    __syncthreads();
    int rank = equals + (int)__popcll(equal_mask & before);
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) rank += sums[0][w];
      equals += sums[0][w];
    }
    const bool stays = l < s.len && (!old || (want > 0 && (key > border || (equal && rank < want))));
    const uint64_t mask = __ballot(stays);
    if (lane == 0) sums[1][wave] = (int)__popcll(mask);
    __syncthreads();
    int place = count + (int)__popcll(mask & before);
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) place += sums[1][w];
      count += sums[1][w];
    }
    if (stays && place < s.keep) out[place] = l;
  }
}

__global__ void __launch_bounds__(kMoveThreads) evict_move_kernel(EvictParams p, int rows_per_wg, int blocks) {
  const int64_t item = (int64_t)blockIdx.x / blocks;
  const int b = (int)(item / p.kv_heads), head = (int)(item - (int64_t)b * p.kv_heads);
  const int first = (int)((int64_t)blockIdx.x - item * blocks) * rows_per_wg;
  const Kept s = kept_of(p, b);
  const int rows = min(rows_per_wg, s.keep - first);
  if (rows <= 0) return;
  const int32_t* const kept = p.kept + item * p.keep;
  // pieces of a row, part by part, and one for its weight
  int pieces = 1;
  for (int i = 0; i < p.parts; ++i) pieces += p.part[i].pieces;
  for (int i = threadIdx.x; i < rows * pieces; i += kMoveThreads) {
    const int r = i / pieces, to = first + r, from = kept[to];
    int piece = i - r * pieces;
    if (from < 0 || from >= s.len) continue;
    const int fi = page_of(p.c, from), ti = page_of(p.c, to);
    if (ti >= p.into_width) continue;
    const int64_t at = p.c.table[(int64_t)b * p.c.width + fi], into = p.into[(int64_t)b * p.into_width + ti];
    if (at < 0 || at >= p.c.pages || into < 0 || into >= p.c.pages) continue;
    const int from_slot = from - fi * p.c.page_size, to_slot = to - ti * p.c.page_size;
    int k = 0;
    while (k < p.parts && piece >= p.part[k].pieces) piece -= p.part[k].pieces, ++k;
    if (k == p.parts) {
      p.weights[(into * p.kv_heads + head) * p.c.page_size + to_slot] = p.weights[(at * p.kv_heads + head) * p.c.page_size + from_slot];
      continue;
    }
    const EvictPart& part = p.part[k];
    const char* const src = part.base + at * part.page + head * part.head + from_slot * part.slot + (int64_t)piece * part.piece_bytes;
    char* const dst = part.base + into * part.page + head * part.head + to_slot * part.slot + (int64_t)piece * part.piece_bytes;
    if (part.piece_bytes == 16) *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<const uint4*>(src);
    else *reinterpret_cast<uint32_t*>(dst) = *reinterpret_cast<const uint32_t*>(src);
  }
}

}  // namespace

hipError_t launch_evict(const EvictParams& p, hipStream_t stream) {
  const int items = p.c.batch * p.kv_heads;
  evict_select_kernel<<<dim3((unsigned)items), dim3(kThreads), 0, stream>>>(p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  constexpr int kRows = 64;
  const int most = (int)std::min<int64_t>(p.keep, (int64_t)p.c.width * p.c.page_size), blocks = (most + kRows - 1) / kRows;
  evict_move_kernel<<<dim3((unsigned)(items * blocks)), dim3(kMoveThreads), 0, stream>>>(p, kRows, blocks);
  return hipGetLastError();
}

}  // namespace sc
