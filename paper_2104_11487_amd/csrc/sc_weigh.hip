// The attention weight that each cached token received from a batch's new tokens, added to what it had:
//   w_l <- decay w_l + sum over the rows (new token, query head of the key head) that see l of exp(scale q . k_l - lse)
// (a new token's own: the sum alone). Scores as in the attention kernels, transposed: S' = K Q', keys held in registers, rows streamed.
//
// A unit of work is a tile of keys of one sequence and key head; a workgroup takes an equal share of them in a row (lengths are on the device, so
// the launch does not know how many there are). Where rows are few the four waves take keys of their own, and keep the rows' operand while the share
// stays with a key head; where they are many the waves take the same keys and every fourth block of 16 rows, and are added in LDS, in wave
// order: no atomics, equal calls give equal bits. Keys in 4 bits are fp16 numbers: few rows of bf16 come into fp16 by a power of two
// (exactly but for the smallest elements, as in sc_packed_attend.h); for many rows, that would cost more than it saves, and the keys become two bf16 parts (8 + 3 bits) instead.
//
// Few rows are bound by the vector unit's work on codes and sums and by a unit's chain of latencies (page number, keys, old weight), three waves a
// SIMD: one token of 32 sequences of up to 16384, 32 / 4 heads of 128 in 4 bits, 32 us, 2.9 TB/s. Many rows by the exponentials (a fused
// multiply-add, an exponential and a sum for each score of each row) and by waits, half of the waves' cycles: rows are fetched under branches (a row or an
// element that is not there is not loaded), so that the build cannot count the loads and each round of blocks begins by waiting for all in flight, the
// last block's too; a block's products, exponentials and sums follow one another. 512 tokens of 4 sequences over 12000, 8 / 2 heads of 64
// of bf16, 1504 units on 768 workgroups, 58 us, 424 TFLOP/s. Blocks of 32 rows and keys, whose sums take the registers of a wave, 67 us.
#include "sc_packed_device.h"

#include <algorithm>
#include <type_traits>

#pragma clang fp contract(off)

namespace sc {

namespace {

constexpr int kWaves = 4;
constexpr float kLog2e = 1.4426950408889634f;

// KIND of the keys: 0 fp32, 1 bf16, 2 packed with bf16 queries, 3 packed with fp32 queries. SPLIT: the waves share the rows.
template <int KIND, int NG, bool SPLIT>
struct Weigh {
  static constexpr bool kHalf = KIND == 1 || KIND == 2, kPacked = KIND >= 2;
  static constexpr bool kScaled = KIND == 2 && !SPLIT;  // products in fp16
  static constexpr int kParts = KIND == 2 && SPLIT ? 2 : 1;
  static constexpr int kWords = kHalf ? 4 : 8;          // registers of eight elements
  static constexpr int kRegs = NG * kParts * kWords;    // of an operand of 16 keys
  static constexpr int kPieces = NG == 8 ? 2 : 1;       // 16-byte pieces of codes, and pairs, of a lane
  static constexpr int kRaw = kPacked ? NG + kPieces : NG * kWords;  // of 16 keys as they lie in memory: codes and pairs, or elements
  // 16-key blocks of a wave: where rows are many it holds their operands; otherwise they are formed for each block of rows, from
  // what was loaded, all blocks' loads in flight together
  static constexpr int kBlocks = SPLIT ? (kRegs <= 16 ? 4 : kRegs <= 32 ? 2 : 1) : kRaw <= 16 ? 4 : kRaw <= 32 ? 2 : 1;
  static constexpr int kKeys = 16 * kBlocks * (SPLIT ? 1 : kWaves);  // of a unit
  static constexpr int kDepth = !SPLIT ? 1 : NG * kWords <= 16 ? 3 : 2;  // blocks of rows in registers
  static constexpr int kOperands = SPLIT ? kBlocks * kRegs + kDepth * NG * kWords : kBlocks * kRaw + kRegs + 2 * NG * kWords;
  static constexpr int kWavesPerSimd = kOperands <= 48 ? (SPLIT ? 3 : 4) : kOperands <= 80 ? 3 : 2;
  using Q = std::conditional_t<kHalf, uint16_t, float>;
};

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

// Sums of N values (16, 8 or 4) over each row of 16 lanes; lane c of a row has value c % N's. Lanes exchange halves of what they hold, with
// partners that differ by 8, 7, 2 and 1 (exclusive or): 15 exchanges for 16 values, where sums by themselves take 64.
template <int CONTROL>
__device__ __forceinline__ float from_partner(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CONTROL, 0xf, 0xf, true));
}
template <int N, int CONTROL>
__device__ __forceinline__ void exchange(float (&v)[16], bool upper) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float keep = upper ? v[i + N] : v[i], give = upper ? v[i] : v[i + N];
    v[i] = keep + from_partner<CONTROL>(give);
  }
}
template <int N>
__device__ __forceinline__ float sums16(float (&v)[16], int col) {
  if constexpr (N == 16) {
    exchange<8, 0x128>(v, col & 8);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += from_partner<0x128>(v[i]);
  }
  if constexpr (N >= 8) {
    exchange<4, 0x141>(v, col & 4);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += from_partner<0x141>(v[i]);
  }
  exchange<2, 0x4e>(v, col & 2);
  exchange<1, 0xb1>(v, col & 1);
  return v[0];
}

template <int KIND, int NG, bool SPLIT>
__global__ void __launch_bounds__(64 * kWaves, (Weigh<KIND, NG, SPLIT>::kWavesPerSimd)) weigh_kernel(WeighParams p) {
  using W = Weigh<KIND, NG, SPLIT>;
  using Q = typename W::Q;
  constexpr bool kHalf = W::kHalf;
  constexpr int PARTS = W::kParts, KEYS = W::kKeys, BLOCKS = W::kBlocks, kWords = W::kWords, DEPTH = W::kDepth;
  __shared__ float shares[SPLIT ? kWaves : 1][16 * BLOCKS];
  const CodeBits bits = code_bits();
  const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6), col = lane & 15, quad = lane >> 4;

  // Sequences by 64s, one a lane, and where their units end.
  const auto units_of = [&](const Sequence& s) { return s.n > 0 ? (int64_t)((s.len + KEYS - 1) / KEYS) * p.kv_heads : 0; };
  const auto load = [&](int b) { return b < p.c.batch ? sequence_of(p.c, b) : Sequence{0, 0, 0}; };
  Sequence mine = load(lane);
  int64_t upto = scan64(units_of(mine)), all = from_lane(upto, 63);
  int64_t total = all;
  for (int b = 64; b < p.c.batch; b += 64) total += from_lane(scan64(units_of(load(b + lane))), 63);
  const int64_t share = divide(total, gridDim.x), rest = total - share * gridDim.x;
  int64_t unit = blockIdx.x * share + min((int64_t)blockIdx.x, rest);
  const int64_t end = unit + share + ((int64_t)blockIdx.x < rest ? 1 : 0);

  int b0 = 0, b = 0, head = 0, tile = 0, tiles = 0;
  bool rows_held = false;  // few rows: they are in the operand
  int64_t base = 0, sequence_end = 0;
  Sequence s = {0, 0, 0};

  constexpr int kStep = SPLIT ? 16 * kWaves : 16;  // rows from a block of the wave to its next one
  const struct {
    int token, of_group;
    int64_t q, wrap, lse;
  } row_step = {kStep / p.group, kStep % p.group, kStep / p.group * p.q_token + kStep % p.group * p.q_head, p.q_token - p.group * p.q_head,
                (int64_t)(kStep / p.group) * p.q_heads + kStep % p.group};
  // Step i of a product takes of lane (row or key, quarter) eight elements from here on: where keys are codes a quarter's lie in a row, so
  // that one load brings a key's codes of all steps; otherwise the quarters' lie side by side, 64 or 128 bytes a load and key.
  const auto element = [&](int i) { return W::kPacked ? 8 * (NG * quad + i) : 32 * i + 8 * quad; };
  // a block of rows, in the right operand's layout
  uint32_t qf[NG][kWords];
  float less = 0.0f, factor = 0.0f;  // of the lane's row: lse in powers of two; of a score, to powers of two
  bool gives = false;                // whether it is a row, and not left out by an lse of minus infinity
  int seen_lo = 0, seen_hi = -1;

  for (; unit < end; ++unit) {
    if (unit >= sequence_end) {
      while (unit >= base + all) {
        base += all;
        b0 += 64;
        mine = load(b0 + lane);
        upto = scan64(units_of(mine)), all = from_lane(upto, 63);
      }
      const int src = (int)__ffsll((unsigned long long)__ballot(base + upto > unit)) - 1;
      b = b0 + src;
      s = {__builtin_amdgcn_readlane(mine.start, src), __builtin_amdgcn_readlane(mine.n, src), __builtin_amdgcn_readlane(mine.len, src)};
      tiles = (s.len + KEYS - 1) / KEYS;
      sequence_end = base + from_lane(upto, src);
      const int64_t rel = unit - (sequence_end - (int64_t)tiles * p.kv_heads);
      head = (int)divide(rel, tiles), tile = (int)(rel - (int64_t)head * tiles);
      rows_held = false;
    } else if (++tile == tiles) {
      tile = 0, ++head, rows_held = false;
    }
    const int key0 = tile * KEYS + (SPLIT ? 0 : wave * 16 * BLOCKS), p0 = s.len - s.n;

    // new tokens that see any of the wave's keys: [i0, i1]; those that see all of them: [all0, all1]
    const int key_end = min(key0 + 16 * BLOCKS, s.len) - 1;
    int i0 = 0, i1 = s.n - 1, all0 = 0, all1 = s.n - 1;
    if (p.causal) {
      i0 = max(0, key0 - p0), all0 = max(0, key_end - p0);
      if (p.window >= 0) i1 = (int)min((int64_t)i1, (int64_t)key_end - p0 + p.window), all1 = (int)min((int64_t)all1, (int64_t)key0 - p0 + p.window);
    } else if (p.window >= 0) {
      if ((int64_t)key_end < (int64_t)p0 - p.window) i1 = -1;
      if ((int64_t)key0 < (int64_t)p0 - p.window) all1 = -1;
    }
    if (key0 >= s.len) i1 = -1;
    const bool whole_keys = key0 + 16 * BLOCKS <= s.len;
    const int rows_end = (max(i1, -1) + 1) * p.group, row_begin = SPLIT ? i0 * p.group : 0;
    // (few rows: all of them, so that the operand holds for every unit)
    const int rows_all = SPLIT ? rows_end : s.n * p.group;

    // Blocks of rows that were fetched. Where rows are many, as many as the registers hold: products take them where they are, and the next
    // ones take their place.
    // What the head has no elements for, and what no row is there for, stays as it begins here.
    uint32_t raw[DEPTH][NG][kWords];
    float raw_lse[DEPTH];
    int raw_token[DEPTH];
    int token = 0, of_group = 0;  // of the lane's row that was fetched last
    const Q* row_q = nullptr;
    const float* row_lse = nullptr;
    const auto find_row = [&](int r0) {
      token = (r0 + col) / p.group, of_group = r0 + col - token * p.group;
      const int h = head * p.group + of_group;
      row_q = reinterpret_cast<const Q*>(p.q) + (int64_t)(s.start + token) * p.q_token + (int64_t)h * p.q_head;
      row_lse = p.lse + (int64_t)(s.start + token) * p.q_heads + h;
    };
    const auto next_row = [&](int r0) {  // of the next block that the wave takes, at r0
      if constexpr (!SPLIT) return find_row(r0);
      token += row_step.token, row_q += row_step.q, row_lse += row_step.lse;
      if (row_step.of_group > 0) {
        of_group += row_step.of_group;
        if (of_group >= p.group) of_group -= p.group, ++token, row_q += row_step.wrap, row_lse += p.q_heads - p.group;
      }
    };
    const auto fetch_rows = [&](int x) {
      raw_token[x] = token;
      if (token < s.n) {
#pragma unroll
        for (int i = 0; i < NG; ++i) {
          const int d = element(i);
          if (d < p.dim) {
#pragma unroll
            for (int part = 0; part < kWords / 4; ++part) {
              const uint4 w = reinterpret_cast<const uint4*>(row_q + d)[part];
              uint32_t* const to = &raw[x][i][4 * part];
              to[0] = w.x, to[1] = w.y, to[2] = w.z, to[3] = w.w;
            }
          }
        }
        raw_lse[x] = *row_lse;
      }
    };
    const auto take_rows = [&](int x, int r0) {  // what was fetched
      less = raw_lse[x] * kLog2e, gives = raw_lse[x] != kNegInf && r0 + col < rows_all;
      factor = p.scale_log2;
      if constexpr (W::kScaled) {
        float most = 0.0f;
#pragma unroll
        for (int i = 0; i < NG; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) most = fmaxf(most, fmaxf(fabsf(__uint_as_float(raw[x][i][e] << 16)), fabsf(__uint_as_float(raw[x][i][e] & 0xffff0000u))));
        most = max_across32(max_across16(most));
        const int lift = lift_of(most);
        factor = factor_of(p.scale_log2, lift);
#pragma unroll
        for (int i = 0; i < NG; ++i) {
          float y[8];
#pragma unroll
          for (int e = 0; e < 4; ++e) y[2 * e] = ldexpf(__uint_as_float(raw[x][i][e] << 16), lift), y[2 * e + 1] = ldexpf(__uint_as_float(raw[x][i][e] & 0xffff0000u), lift);
#pragma unroll
          for (int e = 0; e < 4; ++e) qf[i][e] = pack2h(y[e], y[e + 4]);  // in the order that the keys' codes come in
        }
      } else if constexpr (!SPLIT) {
#pragma unroll
        for (int i = 0; i < NG; ++i)
#pragma unroll
          for (int e = 0; e < kWords; ++e) qf[i][e] = raw[x][i][e];
      }
      const int at = p0 + min(raw_token[x], s.n - 1), from = p.causal ? at : p0;  // the row's position
      seen_hi = p.causal ? min(at, s.len - 1) : s.len - 1;
      seen_lo = p.window >= 0 && from > p.window ? from - p.window : 0;
    };

    const int first_row = row_begin + (SPLIT ? 16 * wave : 0);
    const int row_count = rows_end > 0 ? rows_all : 0;
    if (first_row < row_count && !rows_held) {
#pragma unroll
      for (int x = 0; x < DEPTH; ++x) {
        raw_lse[x] = kNegInf;
#pragma unroll
        for (int i = 0; i < NG; ++i)
#pragma unroll
          for (int e = 0; e < kWords; ++e) raw[x][i][e] = 0u;
      }
      find_row(first_row), fetch_rows(0);
#pragma unroll
      for (int x = 1; x < DEPTH; ++x)
        if (first_row + x * kStep < row_count) next_row(first_row + x * kStep), fetch_rows(x);
    }

    // what the lane will store: its key's place, and what that held
    const int local = 16 * (col >> 2) + 4 * quad + (col & 3), own_key = key0 + local;
    const bool stores = col < 4 * BLOCKS && own_key < s.len && (!SPLIT || wave == 0);
    int own_entry = -1;
    const int own_page = min(page_of(p.c, min(own_key, kMostKeys - 1)), p.c.width - 1);
    if (stores) own_entry = p.c.table[(int64_t)b * p.c.width + own_page];

    // the keys, in the left operand's layout
    uint32_t raw_keys[BLOCKS][W::kRaw];
    // Block j's, where the lane's key begins at `row`, its pairs at `pairs`.
    const auto bring = [&](int j, const char* row, const char* pairs) {
      if constexpr (W::kPacked) {
#pragma unroll
        for (int i = 0; i < W::kPieces; ++i) {
          const int g = min(NG >= 4 ? W::kPieces * quad + i : NG * quad / 4, p.groups - 1);  // groups past the head's: the queries are zero there
          if constexpr (NG >= 4) {
            const uint4 w = *reinterpret_cast<const uint4*>(row + 16 * g);
            uint32_t* const to = &raw_keys[j][4 * i];
            to[0] = w.x, to[1] = w.y, to[2] = w.z, to[3] = w.w;
          } else if constexpr (NG == 2) {
            const u32x2 w = *reinterpret_cast<const u32x2*>(row + 16 * g + 8 * (quad & 1));
            raw_keys[j][0] = w[0], raw_keys[j][1] = w[1];
          } else {
            raw_keys[j][0] = *reinterpret_cast<const uint32_t*>(row + 4 * quad);
          }
          raw_keys[j][NG + i] = *reinterpret_cast<const uint32_t*>(pairs + 4 * g);
        }
      } else {
#pragma unroll
        for (int i = 0; i < NG; ++i) {
          const int d = element(i);
#pragma unroll
          for (int e = 0; e < kWords; e += 4) {
            const uint4 w = d < p.dim ? reinterpret_cast<const uint4*>(row + d * (int)sizeof(Q))[e / 4] : uint4{0u, 0u, 0u, 0u};
            uint32_t* const to = &raw_keys[j][i * kWords + e];
            to[0] = w.x, to[1] = w.y, to[2] = w.z, to[3] = w.w;
          }
        }
      }
    };
    if (first_row < row_count) {
      const char* const k = p.c.k + (int64_t)head * p.c.k_head;
      const char* const ks = p.s.k + (int64_t)head * p.s.k_head;
      if (p.whole) {  // a block lies in one page, which the scalar unit looks up
        int entry[BLOCKS], slot[BLOCKS];
#pragma unroll
        for (int j = 0; j < BLOCKS; ++j) {
          const int at = min(uniform(key0) + 16 * j, kMostKeys - 16), i = min(page_of(p.c, at), p.c.width - 1);
          slot[j] = min(at - i * p.c.page_size, p.c.page_size - 16);
          entry[j] = ((const __attribute__((address_space(4))) int32_t*)(uintptr_t)(p.c.table + (int64_t)b * p.c.width))[i];
        }
        const uint32_t off = (uint32_t)col * (uint32_t)p.c.k_slot, pairs_off = (uint32_t)col * (uint32_t)p.s.k_slot;
#pragma unroll
        for (int j = 0; j < BLOCKS; ++j) {
          const uint64_t page = (uint32_t)page_of_entry(p.c, entry[j]), at = (uint32_t)slot[j];
          bring(j, k + (page * (uint32_t)p.c.k_page + at * (uint32_t)p.c.k_slot) + off, ks + (page * (uint32_t)p.s.k_page + at * (uint32_t)p.s.k_slot) + pairs_off);
        }
      } else {
        int entry[BLOCKS], slot[BLOCKS];
#pragma unroll
        for (int j = 0; j < BLOCKS; ++j) entry[j] = entry_at(p.c, b, min(key0 + 16 * j + col, kMostKeys - 1), 1, &slot[j]);
#pragma unroll
        for (int j = 0; j < BLOCKS; ++j) {
          const int64_t page = page_of_entry(p.c, entry[j]);
          bring(j, k + page * p.c.k_page + slot[j] * p.c.k_slot, ks + page * p.s.k_page + slot[j] * p.s.k_slot);
        }
      }
    }
    using Operand = uint32_t[PARTS][NG][kWords];
    const auto form = [&](int j, Operand& kf) {
#pragma unroll
      for (int i = 0; i < NG; ++i) {
        if constexpr (!W::kPacked) {
#pragma unroll
          for (int e = 0; e < kWords; ++e) kf[0][i][e] = raw_keys[j][i * kWords + e];
        } else {
          const half8 v = values8(raw_keys[j][i], raw_keys[j][NG + i / 4], bits);
          if constexpr (W::kScaled) {
            const uint4 w = __builtin_bit_cast(uint4, v);
            kf[0][i][0] = w.x, kf[0][i][1] = w.y, kf[0][i][2] = w.z, kf[0][i][3] = w.w;
          } else {
            const float x[8] = {(float)v[0], (float)v[2], (float)v[4], (float)v[6], (float)v[1], (float)v[3], (float)v[5], (float)v[7]};
            if constexpr (kHalf) {
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const uint32_t hi = pack2(x[2 * e], x[2 * e + 1]);
                kf[0][i][e] = hi;
                kf[PARTS - 1][i][e] = pack2(x[2 * e] - __uint_as_float(hi << 16), x[2 * e + 1] - __uint_as_float(hi & 0xffff0000u));
              }
            } else {
#pragma unroll
              for (int e = 0; e < 8; ++e) kf[0][i][e] = __float_as_uint(x[e]);
            }
          }
        }
      }
    };
    Operand held[SPLIT ? BLOCKS : 1];
    if constexpr (SPLIT) {
      if (first_row < row_count) {
#pragma unroll
        for (int j = 0; j < BLOCKS; ++j) form(j, held[j]);
      }
    }
    floatx4 got[BLOCKS];
#pragma unroll
    for (int j = 0; j < BLOCKS; ++j) got[j] = floatx4{};
    // The held rows' scores with the held keys, and what they give. kAll: 16 rows that give, and see every key; kRows: those that give see every key.
    constexpr int kAll = 0, kRows = 1, kSome = 2;
    const auto add = [&](const uint32_t (&rows)[NG][kWords], int which) {
#pragma unroll
      for (int j = 0; j < BLOCKS; ++j) {
        floatx4 score = floatx4{};
        if constexpr (!SPLIT) {  // here, not ahead of the loop over rows: no registers hold all blocks' operands
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int e = 0; e < W::kRaw; ++e) raw_keys[j][e] = here(raw_keys[j][e]);
          form(j, held[0]);
        }
        Operand& kf = held[SPLIT ? j : 0];
#pragma unroll
        for (int i = 0; i < NG; ++i)
#pragma unroll
          for (int part = 0; part < PARTS; ++part) {
            const uint32_t* const k = kf[part][i];
            if constexpr (W::kScaled) {
              score = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, uint4{k[0], k[1], k[2], k[3]}), __builtin_bit_cast(half8, uint4{rows[i][0], rows[i][1], rows[i][2], rows[i][3]}), score, 0, 0, 0);
            } else if constexpr (kHalf) {
              score = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, uint4{k[0], k[1], k[2], k[3]}), __builtin_bit_cast(bf16x8, uint4{rows[i][0], rows[i][1], rows[i][2], rows[i][3]}), score, 0, 0, 0);
            } else {
#pragma unroll
              for (int e = 0; e < 8; ++e) score = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[e]), __uint_as_float(rows[i][e % kWords]), score, 0, 0, 0);
            }
          }
        if (which == kAll) {
#pragma unroll
          for (int r = 0; r < 4; ++r) got[j][r] += __builtin_amdgcn_exp2f(__builtin_fmaf(score[r], factor, -less));
        } else if (which == kRows) {
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(score[r], factor, -less));
            got[j][r] += gives ? e : 0.0f;
          }
        } else {
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int key = key0 + 16 * j + 4 * quad + r;
            const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(score[r], factor, -less));
            got[j][r] += gives && key >= seen_lo && key <= seen_hi ? e : 0.0f;
          }
        }
      }
    };
    const int all_from = all0 * p.group, all_to = whole_keys ? (max(all1, -1) + 1) * p.group : 0;  // rows that see all of the wave's keys
    const auto which_of = [&](int r0) {  // of the 16 rows from r0 on, which were taken (uniform)
      return r0 < all_from || min(r0 + 16, rows_all) > all_to ? kSome : __all(gives) ? kAll : kRows;
    };

    if constexpr (SPLIT) {
      int r0 = first_row;
      while (r0 < row_count) {
#pragma unroll
        for (int x = 0; x < DEPTH; ++x) {
          if (r0 >= row_count) break;
          take_rows(x, r0);
          if (which_of(r0) == kAll) add(raw[x], kAll);
          else add(raw[x], kSome);
          if (r0 + DEPTH * kStep < row_count) next_row(r0 + DEPTH * kStep), fetch_rows(x);
          r0 += kStep;
        }
      }
    } else {
#pragma unroll 1
      for (int r0 = first_row; r0 < row_count; r0 += kStep) {
        if (!rows_held) take_rows(0, r0);
        if (r0 + kStep < row_count) next_row(r0 + kStep), fetch_rows(0);
        add(qf, which_of(r0));
      }
    }
    rows_held = rows_held || (!SPLIT && row_count > 0 && row_count <= 16);

    const bool there = stores && own_entry >= 0 && own_entry < p.c.pages && page_of(p.c, own_key) == own_page;
    float* const to = p.weights + ((int64_t)(there ? own_entry : 0) * p.kv_heads + head) * p.c.page_size + (there ? own_key - own_page * p.c.page_size : 0);
    const bool is_new = own_key >= p0;
    const float before = there && !is_new ? *to : 0.0f;

    // over the 16 rows of a block; lane r of a quarter then has its key r's of the first block, lane 4 + r of the second, ..
    float each[16];
#pragma unroll
    for (int i = 0; i < 4 * BLOCKS; ++i) each[i] = got[i / 4][i % 4];
    float sum = sums16<4 * BLOCKS>(each, col);
    if constexpr (SPLIT) {
      if (col < 4 * BLOCKS) shares[wave][local] = sum;
      __syncthreads();
      sum = 0.0f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) sum += shares[w][col < 4 * BLOCKS ? local : 0];
      __syncthreads();  // read before the next unit writes
    }
    if (there) *to = is_new ? sum : p.decay * before + sum;
  }
}

template <int KIND, int NG>
hipError_t launch(const WeighParams& p, bool split, hipStream_t stream) {
  const int64_t most = (int64_t)p.c.batch * p.kv_heads * p.tiles;
  // as many workgroups as the GPU holds: a wave of each on every SIMD
  const int holds = 256 * (split ? Weigh<KIND, NG, true>::kWavesPerSimd : Weigh<KIND, NG, false>::kWavesPerSimd);
  const dim3 grid((unsigned)std::min<int64_t>(std::max<int64_t>(most, 1), holds)), block(64 * kWaves);
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
