// The attention weight that each cached token received from a batch's new tokens, added to what it had:
//   w_l <- decay w_l + sum over the rows (new token, query head of the key head) that see l of exp(scale q . k_l - lse)
// (a new token's own: the sum alone). Scores as in the attention kernels, transposed: S' = K Q', keys held in registers, rows streamed.
//
// A unit of work is a tile of keys of one sequence and key head; workgroups take units in turn (lengths are on the device, so the launch does
// not know how many there are). Where rows are few the four waves take 32 keys each; where they are many the waves take
// the same 32 keys and every fourth block of 16 rows, and are added in LDS, in wave order: no atomics, equal calls give equal bits.
// Keys in 4 bits are fp16 numbers, which two bf16 parts hold exactly (8 + 3 bits), so bf16 queries enter the product as they are.
#include "sc_packed_device.h"

#include <algorithm>
#include <type_traits>

#pragma clang fp contract(off)

namespace sc {

namespace {

constexpr int kWaves = 4, kWaveKeys = 32;
constexpr float kLog2e = 1.4426950408889634f;

// Inclusive sum over the wave's lanes.
__device__ __forceinline__ int64_t scan64(int64_t v) {
  if (!__any(v >> 25)) return scan32((int)v);
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t t = __shfl_up(v, d);
    if (lane >= d) v += t;
  }
  return v;
}

// KIND of the keys: 0 fp32, 1 bf16, 2 packed with bf16 queries, 3 packed with fp32 queries. SPLIT: the waves share the rows.
template <int KIND, int NG, bool SPLIT>
__global__ void __launch_bounds__(64 * kWaves, 2) weigh_kernel(WeighParams p) {
  constexpr bool kHalf = KIND == 1 || KIND == 2, kPacked = KIND >= 2;
  constexpr int PARTS = KIND == 2 ? 2 : 1, KEYS = SPLIT ? kWaveKeys : kWaveKeys * kWaves;
  constexpr int kWords = kHalf ? 4 : 8;  // registers of eight elements
  using Q = std::conditional_t<kHalf, uint16_t, float>;
  __shared__ float shares[kWaves][kWaveKeys];
  const CodeBits bits = code_bits();
  const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6), col = lane & 15, quad = lane >> 4;

  // Sequences by 64s, one a lane, and where their units end.
  const auto units_of = [&](const Sequence& s) { return s.n > 0 ? (int64_t)((s.len + KEYS - 1) / KEYS) * p.kv_heads : 0; };
  const auto load = [&](int b) { return b < p.c.batch ? sequence_of(p.c, b) : Sequence{0, 0, 0}; };
  int b0 = 0;
  int64_t base = 0;
  Sequence mine = load(lane);
  int64_t upto = scan64(units_of(mine)), all = from_lane(upto, 63);
  for (int64_t unit = blockIdx.x;; unit += gridDim.x) {
    while (unit >= base + all) {
      base += all;
      b0 += 64;
      if (b0 >= p.c.batch) return;
      mine = load(b0 + lane);
      upto = scan64(units_of(mine)), all = from_lane(upto, 63);
    }
    const int src = (int)__ffsll((unsigned long long)__ballot(base + upto > unit)) - 1, b = b0 + src;
    const Sequence s = {__builtin_amdgcn_readlane(mine.start, src), __builtin_amdgcn_readlane(mine.n, src), __builtin_amdgcn_readlane(mine.len, src)};
    const int tiles = (s.len + KEYS - 1) / KEYS;
    const int64_t rel = unit - (base + from_lane(upto, src) - (int64_t)tiles * p.kv_heads);
    const int head = (int)divide(rel, tiles), key0 = (int)(rel - (int64_t)head * tiles) * KEYS + (SPLIT ? 0 : wave * kWaveKeys);

    // the keys, in the left operand's layout: lane (key of the block, quarter) holds elements 32 i + 8 quad ..
    uint32_t kf[2][PARTS][NG][kWords];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      int slot;
      const int64_t page = page_of_entry(p.c, entry_at(p.c, b, min(key0 + 16 * j + col, kMostKeys - 1), 1, &slot));
      const char* const row = p.c.k + page * p.c.k_page + (int64_t)head * p.c.k_head + slot * p.c.k_slot;
#pragma unroll
      for (int i = 0; i < NG; ++i) {
        const int d = 32 * i + 8 * quad;
        if constexpr (kPacked) {
          const bool there = i < p.groups;
          const char* const pairs = p.s.k + page * p.s.k_page + (int64_t)head * p.s.k_head + slot * p.s.k_slot;
          const uint32_t w = there ? reinterpret_cast<const uint32_t*>(row)[4 * i + quad] : 0u, pair = there ? reinterpret_cast<const uint32_t*>(pairs)[i] : 0u;
          const half8 v = values8(w, pair, bits);
          const float x[8] = {(float)v[0], (float)v[2], (float)v[4], (float)v[6], (float)v[1], (float)v[3], (float)v[5], (float)v[7]};
          if constexpr (kHalf) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t hi = pack2(x[2 * e], x[2 * e + 1]);
              kf[j][0][i][e] = hi;
              kf[j][PARTS - 1][i][e] = pack2(x[2 * e] - __uint_as_float(hi << 16), x[2 * e + 1] - __uint_as_float(hi & 0xffff0000u));
            }
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) kf[j][0][i][e] = __float_as_uint(x[e]);
          }
        } else {
          const uint4 none{0u, 0u, 0u, 0u};
#pragma unroll
          for (int part = 0; part < kWords / 4; ++part) {
            const uint4 w = d < p.dim ? reinterpret_cast<const uint4*>(row + (int64_t)d * (int)sizeof(Q))[part] : none;
            kf[j][0][i][4 * part] = w.x, kf[j][0][i][4 * part + 1] = w.y, kf[j][0][i][4 * part + 2] = w.z, kf[j][0][i][4 * part + 3] = w.w;
          }
        }
      }
    }

    // new tokens that see any of the keys: [i0, i1]
    const int p0 = s.len - s.n, key_end = min(key0 + kWaveKeys, s.len) - 1;
    int i0 = 0, i1 = s.n - 1;
    if (p.causal) {
      i0 = max(0, key0 - p0);
      if (p.window >= 0) i1 = (int)min((int64_t)i1, (int64_t)key_end - p0 + p.window);
    } else if (p.window >= 0 && (int64_t)key_end < (int64_t)p0 - p.window) {
      i1 = -1;
    }
    if (key0 >= s.len) i1 = -1;
    floatx4 got[2] = {floatx4{}, floatx4{}};
    const int rows_end = (i1 + 1) * p.group;
    for (int r0 = i0 * p.group + (SPLIT ? 16 * wave : 0); r0 < rows_end; r0 += SPLIT ? 16 * kWaves : 16) {
      const int row = min(r0 + col, rows_end - 1), t = row / p.group, h = head * p.group + (row - t * p.group);
      const Q* const q = reinterpret_cast<const Q*>(p.q) + (int64_t)(s.start + t) * p.q_token + (int64_t)h * p.q_head;
      const float l = p.lse[(int64_t)(s.start + t) * p.q_heads + h];
      const float less = l == kNegInf ? -kNegInf : l * kLog2e;  // a row that sees nothing gives nothing
      floatx4 score[2] = {floatx4{}, floatx4{}};
#pragma unroll
      for (int i = 0; i < NG; ++i) {
        const int d = 32 * i + 8 * quad;
        uint4 w[kWords / 4];
#pragma unroll
        for (int part = 0; part < kWords / 4; ++part) w[part] = d < p.dim ? reinterpret_cast<const uint4*>(q + d)[part] : uint4{0u, 0u, 0u, 0u};
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int part = 0; part < PARTS; ++part) {
            const uint32_t* const k = kf[j][part][i];
            if constexpr (kHalf) {
              score[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, uint4{k[0], k[1], k[2], k[3]}), __builtin_bit_cast(bf16x8, w[0]), score[j], 0, 0, 0);
            } else {
              const float x[8] = {__uint_as_float(w[0].x), __uint_as_float(w[0].y), __uint_as_float(w[0].z), __uint_as_float(w[0].w),
                                  __uint_as_float(w[kWords / 4 - 1].x), __uint_as_float(w[kWords / 4 - 1].y), __uint_as_float(w[kWords / 4 - 1].z), __uint_as_float(w[kWords / 4 - 1].w)};
#pragma unroll
              for (int e = 0; e < 8; ++e) score[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[e]), x[e], score[j], 0, 0, 0);
            }
          }
      }
      const int at = p0 + t;  // the row's position
      const int hi = p.causal ? min(at, s.len - 1) : s.len - 1, from = p.causal ? at : p0;
      const int lo = p.window >= 0 && from > p.window ? from - p.window : 0;
      const bool live = r0 + col < rows_end;
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int key = key0 + 16 * j + 4 * quad + r;
          const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(score[j][r], p.scale_log2, -less));
          got[j][r] += live && key >= lo && key <= hi ? e : 0.0f;
        }
    }
    // over the 16 rows of a block; lane r of a quarter then stores its key r's of the first block, lane 4 + r of the second
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int m = 1; m < 16; m <<= 1) got[j][r] += __shfl_xor(got[j][r], m);
    const int j = col >> 2 & 1;
    float sum = 0.0f;
#pragma unroll
    for (int r = 0; r < 4; ++r) sum = (col & 3) == r ? (j ? got[1][r] : got[0][r]) : sum;
    const int local = 16 * j + 4 * quad + (col & 3), key = key0 + local;
    if constexpr (SPLIT) {
      if (col < 8) shares[wave][local] = sum;
      __syncthreads();
      sum = 0.0f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) sum += shares[w][local];
      __syncthreads();  // read before the next unit writes
    }
    if (col < 8 && key < s.len && (!SPLIT || wave == 0)) {
      const int i = page_of(p.c, key);
      const int page = i < p.c.width ? p.c.table[(int64_t)b * p.c.width + i] : -1;
      if (page >= 0 && page < p.c.pages) {
        float* const to = p.weights + ((int64_t)page * p.kv_heads + head) * p.c.page_size + (key - i * p.c.page_size);
        *to = key >= p0 ? sum : p.decay * *to + sum;
      }
    }
  }
}

template <int KIND, int NG>
hipError_t launch(const WeighParams& p, bool split, hipStream_t stream) {
  const int64_t most = (int64_t)p.c.batch * p.kv_heads * p.tiles;
  const dim3 grid((unsigned)std::min<int64_t>(std::max<int64_t>(most, 1), 2048)), block(64 * kWaves);
  if (split) weigh_kernel<KIND, NG, true><<<grid, block, 0, stream>>>(p);
  else weigh_kernel<KIND, NG, false><<<grid, block, 0, stream>>>(p);
  return hipGetLastError();
}

template <int KIND>
hipError_t launch_kind(const WeighParams& p, bool split, hipStream_t stream) {
  if (p.dim <= 32) return launch<KIND, 1>(p, split, stream);
  if (p.dim <= 64) return launch<KIND, 2>(p, split, stream);
  if (p.dim <= 128) return launch<KIND, 4>(p, split, stream);
  return launch<KIND, 8>(p, split, stream);
}

}  // namespace

hipError_t launch_weigh(const WeighParams& p, int dtype, int split, hipStream_t stream) {
  if (p.packed) return dtype == 0 ? launch_kind<3>(p, split != 0, stream) : launch_kind<2>(p, split != 0, stream);
  return dtype == 0 ? launch_kind<0>(p, split != 0, stream) : launch_kind<1>(p, split != 0, stream);
}

}  // namespace sc
