// Eviction: of each sequence and key head the newest tokens and of the others those of the largest accumulated weight stay, in their order,
// and move to other pages.
//
// First launch, a workgroup a sequence and key head: the weights' keys (ordered integers) go to LDS, where 36864 fit (beyond, each pass reads
// the weights again); the key that divides kept from evicted is found digit by digit (11, 11 and 10 bits, a histogram in LDS each); then each
// wave counts what stays of its section of the tokens, and writes their positions behind those of the waves before. Of equal weights at the
// border the earlier tokens stay. Bound by latencies, of loads and of barriers: 16 waves, 16 loads of each in flight (16 sequences of up to 32768,
// 4 key heads: 54 us, one sequence of 1100: 9; histograms for every third wave took as long). Second launch: the kept rows'
// bytes move, in pieces of 16 bytes where the parts allow it; source and destination pages are different ones, so rows move in any order. Bound by
// memory: up to 8192 tokens of each of those, 152 MB read and written, in 54 us; kept rows of 64 and 16 bytes lie apart in lines of 128, of which
// the counters see 128 MB read.
#include "sc_packed_device.h"
#include "sc_stream.h"

#include <algorithm>

#pragma clang fp contract(off)

namespace sc {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64, kBins = 2048;
constexpr int kMoveThreads = 256, kMoveRows = 64;

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

constexpr int kHeldKeys = 36864;  // 144 KB of LDS
constexpr int kFewKeys = 4096;

template <int HELD>
__global__ void __launch_bounds__(kThreads) evict_select_kernel(EvictParams p) {
  __shared__ uint32_t held[HELD], bins[kBins];
  __shared__ int sums[2][kWaves];
  __shared__ uint32_t found[2];  // digit of the border, tokens above it
  const int b = (int)blockIdx.x / p.kv_heads, head = (int)blockIdx.x - b * p.kv_heads;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const Kept s = kept_of(p, b);
  if (head == 0 && tid == 0) p.lengths[b] = s.keep;
  int32_t* const out = p.kept + (int64_t)blockIdx.x * p.keep;
  for (int i = s.keep + tid; i < p.keep; i += kThreads) out[i] = -1;
  if (s.keep == s.len) {
    for (int i = tid; i < s.keep; i += kThreads) out[i] = i;
    return;
  }
  const int32_t* const table = p.c.table + (int64_t)b * p.c.width;
  const auto load_key = [&](int l) {  // of a token that has no place in the cache: below all weights
    const int i = page_of(p.c, l), page = table[i];
    const bool there = page >= 0 && page < p.c.pages;
    const float w = p.weights[((int64_t)(there ? page : 0) * p.kv_heads + head) * p.c.page_size + (l - i * p.c.page_size)];
    return there ? ordered(w) : 0u;
  };
  const bool kept_in_lds = s.late <= HELD;
  // f(token, key) over the tokens [from, to), step apart, whose loads are in flight eight at a time
  const auto each = [&](int from, int to, int step, auto f) {
    if (kept_in_lds) {
#pragma unroll 4
      for (int l = from; l < to; l += step) f(l, held[l]);
      return;
    }
    for (int l = from; l < to; l += 8 * step) {
      uint32_t key[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) key[i] = load_key(min(l + i * step, to - 1));
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (l + i * step < to) f(l + i * step, key[i]);
    }
  };

  // The border: the key of the `want`-th largest of the tokens before `late`, and how many of those equal to it stay.
  int want = s.keep - (s.len - s.late);
  uint32_t border = 0xffffffffu, prefix = 0, known = 0;
  if (want > 0) {
    if (kept_in_lds) {
      for (int l = tid; l < s.late; l += 16 * kThreads) {
        uint32_t key[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) key[i] = load_key(min(l + i * kThreads, s.late - 1));
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (l + i * kThreads < s.late) held[l + i * kThreads] = key[i];
      }
    }
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, width = pass == 2 ? 10 : 11;
      for (int i = tid; i < kBins; i += kThreads) bins[i] = 0;
      __syncthreads();
      each(tid, s.late, kThreads, [&](int, uint32_t key) {
        if ((key & known) == prefix) atomicAdd(&bins[(key >> shift) & ((1u << width) - 1)], 1u);
      });
      __syncthreads();
      // from the largest digit on: each thread holds two bins, in descending order
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
  // The kept ones in order: those above the border, the first `want` equal to it, and the late ones. A wave's section is whole 64s.
  const int section = ((s.late + kWaves - 1) / kWaves + 63) / 64 * 64;
  const int from = min(wave * section, s.late), to = min(from + section, s.late);
  const bool any = want > 0;
  int above = 0, equals = 0;
  if (any) {
    each(from + lane, to, 64, [&](int, uint32_t key) { above += key > border, equals += key == border; });
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) above += __shfl_xor(above, d), equals += __shfl_xor(equals, d);
  }
  if (lane == 0) sums[0][wave] = above, sums[1][wave] = equals;
  __syncthreads();
  int place = 0, rank = 0;
  for (int w = 0; w < wave; ++w) place += sums[0][w], rank += sums[1][w];
  place += min(rank, want);
  if (any) {
    const uint64_t before = (1ull << lane) - 1;
#pragma unroll 2
    for (int l0 = from; l0 < to; l0 += 64) {
      const int l = l0 + lane;
      const uint32_t key = l < to ? (kept_in_lds ? held[l] : load_key(l)) : 0u;
      const bool equal = l < to && key == border;
      const uint64_t equal_mask = __ballot(equal);
      const bool stays = l < to && (key > border || (equal && rank + (int)__popcll(equal_mask & before) < want));
      const uint64_t mask = __ballot(stays);
      if (stays) out[place + (int)__popcll(mask & before)] = l;
      rank += (int)__popcll(equal_mask), place += (int)__popcll(mask);
    }
  }
  const int late_from = s.keep - (s.len - s.late);
  for (int i = tid; i < s.len - s.late; i += kThreads) out[late_from + i] = s.late + i;
}

__global__ void __launch_bounds__(kMoveThreads) evict_move_kernel(EvictParams p, int rows_per_wg, int blocks) {
  __shared__ int from_page[kMoveRows], from_slot[kMoveRows], to_page[kMoveRows], to_slot[kMoveRows];
  const int item = (int)blockIdx.x / blocks;
  const int b = item / p.kv_heads, head = item - b * p.kv_heads;
  const int first = ((int)blockIdx.x - item * blocks) * rows_per_wg;
  const Kept s = kept_of(p, b);
  const int rows = min(rows_per_wg, s.keep - first);
  if (rows <= 0) return;
  if ((int)threadIdx.x < rows) {
    const int r = threadIdx.x, to = first + r, from = p.kept[(int64_t)item * p.keep + to];
    const int fi = page_of(p.c, from), ti = page_of(p.c, to);
    const int at = p.c.table[(int64_t)b * p.c.width + fi], into = ti < p.into_width ? p.into[(int64_t)b * p.into_width + ti] : -1;
    const bool there = at >= 0 && at < p.c.pages && into >= 0 && into < p.c.pages;
    from_page[r] = there ? at : -1, from_slot[r] = from - fi * p.c.page_size;
    to_page[r] = into, to_slot[r] = to - ti * p.c.page_size;
    if (there)
      p.weights[((int64_t)into * p.kv_heads + head) * p.c.page_size + to_slot[r]] = p.weights[((int64_t)at * p.kv_heads + head) * p.c.page_size + from_slot[r]];
  }
  __syncthreads();
#pragma unroll 1
  for (int k = 0; k < p.parts; ++k) {
    const EvictPart part = p.part[k];
    char* const base = part.base + head * part.head;
    const float inv = 1.0f / (float)part.pieces;
#pragma unroll 4
    for (int i = threadIdx.x; i < rows * part.pieces; i += kMoveThreads) {
      const int r = qdiv(i, inv), piece = i - r * part.pieces;
      if (from_page[r] < 0) continue;
      const char* const src = base + (int64_t)from_page[r] * part.page + (int64_t)from_slot[r] * part.slot + piece * part.piece_bytes;
      char* const dst = base + (int64_t)to_page[r] * part.page + (int64_t)to_slot[r] * part.slot + piece * part.piece_bytes;
      if (part.piece_bytes == 16) *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<const uint4*>(src);
      else *reinterpret_cast<uint32_t*>(dst) = *reinterpret_cast<const uint32_t*>(src);
    }
  }
}

}  // namespace

hipError_t launch_evict(const EvictParams& p, hipStream_t stream) {
  const int items = p.c.batch * p.kv_heads;
  const int64_t room = (int64_t)p.c.width * p.c.page_size;
  if (room <= kFewKeys) evict_select_kernel<kFewKeys><<<dim3((unsigned)items), dim3(kThreads), 0, stream>>>(p);
  else evict_select_kernel<kHeldKeys><<<dim3((unsigned)items), dim3(kThreads), 0, stream>>>(p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int most = (int)std::min<int64_t>(p.keep, room);
  // rows of a workgroup: fewer where they would leave the GPU idle
  int rows = kMoveRows;
  while (rows > 8 && (int64_t)items * ((most + rows - 1) / rows) < 1024) rows /= 2;
  const int blocks = (most + rows - 1) / rows;
  evict_move_kernel<<<dim3((unsigned)(items * blocks)), dim3(kMoveThreads), 0, stream>>>(p, rows, blocks);
  return hipGetLastError();
}

}  // namespace sc
