// Attention over a paged cache in 4 bits (sc_packed.h): few rows, and many rows of fp32.
//
//   o = sum_l exp(s_l - m) v_l / sum_l exp(s_l - m),   s_l = scale q . k_l,   over the keys l that the row sees
//
// Codes come into LDS by copies, each wave's own tiles into a ring of its own, two tiles ahead and without a barrier, and from there into registers
// in the layout of the matrix unit's operands, where they become fp16.
//   Scores, transposed: S' = K Q' on 16 x 16 x 32 products, K the left operand. Lane (c, g) = (lane & 15, lane >> 4) holds of key c the g-th
//   quarter of the row's bytes; which elements a step's k indexes stand for is free as long as the queries follow, so those are loaded in the
//   order in which a mask leaves the codes (0 4 1 5 2 6 3 7 of each eight).
//   Outputs: O' = V' P'. Lane (c, g) holds of the keys 4 g + r (r < 4) of each of the tile's two 16-key blocks the c-th 16th of the row's
//   bytes, two elements a byte: the two nibbles of a byte position over the 8 keys are the operands of two products, which stand for the
//   elements 2 NG c + j. A lane's scores are those of the same 8 keys, so the exponentials are the other operand as they are.
// Values are fp16 by the format. Queries: bf16 rows are scaled by a power of two into fp16 (the factor goes into the
// softmax's scale), exactly but for elements below 2^-31 of their row's largest, whose last bits pass fp16's least step (off by 2^-39 of the largest at
// most); fp32 rows are two fp16 parts (22 bits). Scores and sums are fp32. For bf16 the exponentials are rounded to fp16 (2^-11 of each)
// for the product with V, for fp32 they are two parts; they are formed 2^7 too large, so that those of up to 2^-21 of the
// reference's stay normal numbers.
//
// Few rows are bound by the stream of codes and, beside it, by the order of a wave's work: a tile of 32 keys is some 350 vector instructions (13 for
// eight codes) between its copies and its last product, of which two waves a SIMD hide half of each other's waits. One token of 64 sequences over
// 8192, 32 / 4 heads of 128: 83 us; without products 72, without copies 67, 8 of each the join. Two workgroups of four waves a compute unit rather than one
// of eight: a workgroup's waves join at an item's end, and the other's work goes on (sequences of up to 16384: 121 -> 104 us, 3.5 TB/s); three waves
// a SIMD have two stages of LDS each and lose more by waiting (139 us), a fourth stage changes nothing (111 us). One sequence over 262141, 8 / 2 heads of 128: 25 us and 7 for the join; over
// 777, 16 / 4 heads of 64: 12, a chain of latencies. fp32, up to 300 tokens of 9 sequences, window 700, heads of 80: 20 and 5.
#pragma once

#include <type_traits>

#include "sc_attend_tile.h"
#include "sc_packed_device.h"

#pragma clang fp contract(off)

namespace sc {

constexpr float kPackedSlack = 8.0f;  // powers of two that an exponential may exceed the reference's by
constexpr float kPackedLift = 7.0f;   // powers of two that exponentials are formed too large by: 2^15 at most

// Copies 4 bytes a lane from `base` + off into LDS at `to` + 4 lane, as copy16 does 16.
__device__ __forceinline__ void copy4(const char* base, uint32_t off, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tglobal_load_lds_dword %1, %2" ::"s"(uniform((int)to)), "v"(off), "s"(base) : "memory", "m0");
}

// A tile in LDS: 32 rows of keys and 32 of values, codes and then pairs. The 16-byte pieces of a row are permuted by an exclusive or, so that
// the lanes of a read, which go through 16 rows at one place or through four rows 4 apart, touch every bank.
template <int NG>
struct PackedRing {
  static constexpr int kRow = 16 * NG, kPairs = 64 * kRow, kStage = kPairs + 256 * NG;
  static constexpr int kOps = 2 * NG;   // copies of a tile
  static constexpr int kStages = 3;
  __device__ __forceinline__ static int swizzle(int row) { return NG == 8 ? (row >> 1) & 7 : NG == 4 ? (row >> 2) & 3 : NG == 2 ? (row >> 3) & 1 : 0; }
};

// NG: groups of a head, rounded up to a power of two. PARTS: fp16 parts of a query and an exponential. NW: waves of a workgroup.
// MANY: the waves take 16 rows each and all keys; otherwise they take the same 16 rows and every NW-th key tile. Rings take 127 KB of LDS at
// most: a compute unit holds eight waves, for heads above 128 four.
template <int NG, int PARTS, int NW, bool MANY, bool WHOLE>
__global__ void __launch_bounds__(64 * NW, NG == 8 ? 1 : 2) attend_packed_kernel(PackedAttendParams pp) {
  constexpr int WROWS = 16, ROWS = MANY ? NW * WROWS : WROWS;
  constexpr int KEYS = kPackedKeys, DP = 32 * NG, NJ = 2 * NG, PIECES = NG == 8 ? 2 : 1;
  constexpr int JP = DP + 4;  // joining: a row's stride in LDS, in floats
  using Ring = PackedRing<NG>;
  constexpr int kWaveBytes = Ring::kStages * Ring::kStage + (WHOLE ? 0 : 512);  // with two buffers of page numbers
  constexpr int kJoin = MANY ? 0 : NW * ROWS * (JP + 2) * 4;
  __shared__ alignas(16) char lds[NW * kWaveBytes > kJoin ? NW * kWaveBytes : kJoin];
  const AttendParams& p = pp.a;

  const Units batch(p);
  const Shares shares = shares_of(batch);
  if ((int)blockIdx.x >= shares.n) return;
  const int64_t first_unit = shares.at(blockIdx.x), end = shares.at(blockIdx.x + 1);
  Unit u;
  if (first_unit >= end || !unit_of(batch, first_unit, &u)) return;
  for (int64_t at = first_unit;;) {
    const int units = (int)min(end - at, (int64_t)(u.parts - u.part));  // of this item
    const bool whole = units == u.parts, begins = at == first_unit;
    at += units;
    u.hi = (int)min((int64_t)u.hi, u.lo + (int64_t)units * u.chunk);
    // derived anew for each item, so that no register holds from one item to the next what only its ends need
    int thread = (int)threadIdx.x;
    asm volatile("" : "+v"(thread));
    const int lane = thread & 63, wave = uniform(thread >> 6);
    const int col = lane & 15, quad = lane >> 4, last_group = pp.groups - 1;

    // LDS offsets in a stage: the lane's pieces of a key of the first block, of a value of its first row; of their pairs
    uint32_t k_at[PIECES], v_at[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      k_at[i] = col * Ring::kRow + (NG >= 4 ? ((quad * (NG / 4) + i) ^ Ring::swizzle(col)) << 4 : NG == 2 ? (((quad >> 1) ^ Ring::swizzle(col)) << 4) + (quad & 1) * 8 : quad * 4);
      const int row = 4 * quad + 2 * i;  // the permutation changes from rows 0, 1 to 2, 3 of the lane's four where a row has eight pieces
      v_at[i] = (32 + 4 * quad) * Ring::kRow + (((NG * col >> 4) ^ Ring::swizzle(row)) << 4) + (NG >= 4 ? (NG * col) & 15 : (NG * col & 15) & ~3);
    }
    const uint32_t kp_at = Ring::kPairs + col * (4 * NG) + (NG >= 4 ? quad * NG : NG * quad / 4 * 4);
    const uint32_t vp_at = Ring::kPairs + (32 + 4 * quad) * (4 * NG) + 4 * (NG * col >> 4);
    // of the copies: the lane's row of a copy of 64 pieces (pairs), and its piece
    const int copy_row = lane / NG, copy_piece = lane % NG;
    const CodeBits bits = code_bits();
    // page and slot strides of the keys' codes and pairs, the values' codes and pairs
    const uint32_t k_page = alone(p.c.k_page), k_slot = alone(p.c.k_slot), ks_page = alone(pp.s.k_page), ks_slot = alone(pp.s.k_slot);
    const uint32_t v_page = alone(p.c.v_page), v_slot = alone(p.c.v_slot), vs_page = alone(pp.s.v_page), vs_slot = alone(pp.s.v_slot);
    const bool alike = k_page == v_page && k_slot == v_slot && ks_page == vs_page && ks_slot == vs_slot;
    const uint32_t v_sel = NG >= 4 ? 0x0c040c00u : 0x0c040c00u + ((NG * col) & 3) * 0x00010001u;  // picks a byte of two words into 16-bit halves
    const int rows = u.n * p.group, row0 = u.row0 + (MANY ? wave * WROWS : 0);

    // keys that every row of the wave sees, that some row sees
    const Seen first = seen_by(p, u, row0), last = seen_by(p, u, row0 + WROWS - 1);
    const int all_lo = last.lo, all_hi = first.hi, any_lo = first.lo, any_hi = last.hi;

    floatx4 o[NJ];
    float ref = kNegInf, sum = 0.0f, raised = kNegInf;
#pragma unroll
    for (int j = 0; j < NJ; ++j) o[j] = floatx4{};

    const int inside_lo = uniform(all_lo), inside_hi = uniform(all_hi) - KEYS + 1;  // first keys of tiles that all rows see whole

    // the wave's tiles
    constexpr int kStep = MANY ? KEYS : KEYS * NW;
    int begin = u.lo + (MANY ? 0 : wave * KEYS), stop = u.hi;
    if constexpr (MANY) {
      begin = max(begin, any_lo & ~(KEYS - 1));
      stop = row0 < rows ? min(stop, any_hi + 1) : begin;
    }
    const int count = uniform(begin < stop ? (stop - begin + kStep - 1) / kStep : 0);

    const char* const kb = p.c.k + (int64_t)u.head * p.c.k_head;
    const char* const vb = p.c.v + (int64_t)u.head * p.c.v_head;
    const char* const ksb = pp.s.k + (int64_t)u.head * pp.s.k_head;
    const char* const vsb = pp.s.v + (int64_t)u.head * pp.s.v_head;

    char* const ring = lds + wave * kWaveBytes;
    const uint32_t ring_at = (uint32_t)(uintptr_t)SC_LDS(lds, char) + wave * kWaveBytes, entries_at = ring_at + Ring::kStages * Ring::kStage;
    // Where a tile's keys lie, looked up ahead: with whole pages of 16-key blocks a block's page and first slot, by the scalar unit; otherwise
    // its 32 keys' page numbers, by copies into LDS.
    int entry[2], slot[2];
    auto find = [&](int it) {
      const int key0 = begin + it * kStep;
      if constexpr (WHOLE) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int i = min(page_of(p.c, key0 + 16 * j), p.c.width - 1);
          slot[j] = min(key0 + 16 * j - i * p.c.page_size, p.c.page_size - 16);
          entry[j] = ((const __attribute__((address_space(4))) int32_t*)(uintptr_t)(p.c.table + (int64_t)u.b * p.c.width))[i];
        }
      } else {
        sc::copy4(p.c.table + (int64_t)u.b * p.c.width + min(page_of(p.c, key0 + (lane & 31)), p.c.width - 1), entries_at + (it & 1) * 256);
      }
    };
    auto copy = [&](int it, int stage) {  // the tile that was looked up
      const uint32_t to = ring_at + stage;
      if constexpr (WHOLE) {
        const char* base[4];  // keys of both blocks, values; their pairs
        const char* pairs[4];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint64_t page = (uint32_t)page_of_entry(p.c, entry[j]);
          const uint32_t at = (uint32_t)slot[j];
          const uint64_t k_off = page * k_page + at * k_slot, ks_off = page * ks_page + at * ks_slot;  // within a page 32 bits
          uint64_t v_off = k_off, vs_off = ks_off;
          if (!alike) v_off = page * v_page + at * v_slot, vs_off = page * vs_page + at * vs_slot;
          base[j] = kb + k_off, pairs[j] = ksb + ks_off, base[2 + j] = vb + v_off, pairs[2 + j] = vsb + vs_off;
        }
        if constexpr (NG >= 4) {  // a copy's rows are of one block
          constexpr int kRows = 64 / NG;
#pragma unroll
          for (int t = 0; t < NG; ++t) {
            const int from = t * kRows, row = from % 16 + copy_row;
            const bool val = from >= 32;
            const int g = min(copy_piece ^ Ring::swizzle(row), last_group);
            copy16(base[from / 16], here((uint32_t)row * (val ? v_slot : k_slot) + 16 * g), to + t * 1024);
            copy4(pairs[from / 16], here((uint32_t)row * (val ? vs_slot : ks_slot) + 4 * min(copy_piece, last_group)), to + Ring::kPairs + t * 256);
          }
        } else {
#pragma unroll
          for (int t = 0; t < NG; ++t) {
            const int row = t * (64 / NG) + copy_row, which = row / 16;
            const char* b = NG == 2 ? (t ? base[2] : base[0]) : base[0];
            const char* s = NG == 2 ? (t ? pairs[2] : pairs[0]) : pairs[0];
            if constexpr (NG == 2) {
              b = which & 1 ? (t ? base[3] : base[1]) : b, s = which & 1 ? (t ? pairs[3] : pairs[1]) : s;
            } else {
              b = which == 1 ? base[1] : which == 2 ? base[2] : which == 3 ? base[3] : b;
              s = which == 1 ? pairs[1] : which == 2 ? pairs[2] : which == 3 ? pairs[3] : s;
            }
            const bool val = which >= 2;
            copy16(b + (uint32_t)(row % 16) * (val ? v_slot : k_slot) + 16 * (copy_piece ^ Ring::swizzle(row)), to + t * 1024);
            sc::copy4(s + (uint32_t)(row % 16) * (val ? vs_slot : ks_slot) + 4 * copy_piece, to + Ring::kPairs + t * 256);
          }
        }
      } else {
        const char* from[NG];
        const char* pairs[NG];
#pragma unroll
        for (int t = 0; t < NG; ++t) {
          const int row = t * (64 / NG) + copy_row, key = begin + it * kStep + (row & 31);
          const bool val = row >= 32;
          const int64_t page = page_of_entry(p.c, *reinterpret_cast<const int*>(ring + Ring::kStages * Ring::kStage + (it & 1) * 256 + (row & 31) * 4));
          const int64_t at = min(key - min(page_of(p.c, key), p.c.width - 1) * p.c.page_size, p.c.page_size - 1);
          from[t] = (val ? vb + page * p.c.v_page + at * p.c.v_slot : kb + page * p.c.k_page + at * p.c.k_slot) + 16 * min(copy_piece ^ Ring::swizzle(row), last_group);
          pairs[t] = (val ? vsb + page * pp.s.v_page + at * pp.s.v_slot : ksb + page * pp.s.k_page + at * pp.s.k_slot) + 4 * min(copy_piece, last_group);
        }
#pragma unroll
        for (int t = 0; t < NG; ++t) {
          copy16(from[t], to + t * 1024);
          sc::copy4(pairs[t], to + Ring::kPairs + t * 256);
        }
      }
    };
    int stage = 0;  // of the tile in the products
    const auto after = [&](int at, int n) { return at + n * Ring::kStage >= Ring::kStages * Ring::kStage ? at + (n - Ring::kStages) * Ring::kStage : at + n * Ring::kStage; };
    // This tile's copies have landed (the next one's may be outstanding, and the page numbers two further on); those of the one after leave, into
    // the place of the tile before, whose reads have reached their products.
    auto advance = [&](int it) {
      wait_loads<Ring::kOps + (WHOLE ? 0 : 1)>();
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      copy(it + 2, after(stage, 2));
      if constexpr (!WHOLE) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the page numbers are read before others take their place
      find(WHOLE ? it + 3 : it + 4);
    };
    if (count > 0) {
      if constexpr (WHOLE) {
        find(0);
        copy(0, 0);
        find(1);
        copy(1, Ring::kStage);
        find(2);
      } else {
        find(0);
        find(1);
        wait_loads<0>();
#pragma unroll
        for (int it = 0; it < 2; ++it) {
          copy(it, it * Ring::kStage);
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          find(it + 2);
        }
      }
    }

    // the rows' queries, in the operand's layout: loaded while the first tiles' copies are in flight
    half8 qf[PARTS][NG];
    const int r = min(row0 + col, rows - 1), t = r / p.group, h = u.head * p.group + (r - t * p.group);
    const int64_t q_at = (int64_t)(u.start + t) * p.q_token + (int64_t)h * p.q_head;
    float x[NG][8];
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      const int d = 8 * (NG * quad + i);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[i][e] = 0.0f;
      if (d < p.dim) {
        if constexpr (PARTS == 1) Elem<uint16_t>::load8(reinterpret_cast<const uint16_t*>(p.q), q_at + d, x[i]);
        else Elem<float>::load8(reinterpret_cast<const float*>(p.q), q_at + d, x[i]);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(x[i][e]));
    }
    most = max_across32(max_across16(most));
    const int lift = lift_of(most);
    const float factor = factor_of(p.scale_log2, lift);  // of a score, to powers of two
#pragma unroll
    for (int i = 0; i < NG; ++i)
#pragma unroll
      for (int part = 0; part < PARTS; ++part) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float a = ldexpf(x[i][e], lift), b = ldexpf(x[i][e + 4], lift);
          w[e] = pack2h(a, b);
          if (part == 1) {
            const half2 hi = half2_of(w[e]);
            w[e] = pack2h(a - (float)hi[0], b - (float)hi[1]);
          }
        }
        qf[part][i] = __builtin_bit_cast(half8, uint4{w[0], w[1], w[2], w[3]});
      }
    const Seen seen = seen_by(p, u, row0 + col);

    // One tile's work. What is seldom needed ends it early, so that in the loop over tiles products alone touch the outputs' registers, which keep
    // their places:
    //   kRaise  a score passes the reference by more than the slack: nothing is done but to say by how much;
    //   kOdd    some row does not see a value that is not finite: all is done but to add those values.
    constexpr int kDone = 0, kRaise = 1, kOdd = 2;
    half8 pf[PARTS];  // exponentials
    auto load_values = [&](const char* tile_at, uint32_t (&vc)[8][PIECES], uint32_t (&vp)[8]) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const char* const at = tile_at + v_at[PIECES == 2 ? (e % 4) / 2 : 0] + ((e / 4) * 16 + e % 4) * Ring::kRow;
        if constexpr (PIECES == 2) {
          const u32x2 w = *reinterpret_cast<const u32x2*>(at);
          vc[e][0] = w[0], vc[e][1] = w[1];
        } else {
          vc[e][0] = *reinterpret_cast<const uint32_t*>(at);
        }
        vp[e] = *reinterpret_cast<const uint32_t*>(tile_at + vp_at + ((e / 4) * 16 + e % 4) * (4 * NG));
      }
    };
    // Whether a key's group holds values that are not finite: between minimum and largest value all are, or they show it.
    auto infinite = [&](uint32_t pair) {
      const half2 x = half2_of(pair);
      const uint32_t ends = bits_of(half2{x[1], (_Float16)__builtin_fmaf((float)x[0], 15.0f, (float)x[1])});
      return (ends & 0x7c00u) == 0x7c00u || (ends & 0x7c000000u) == 0x7c000000u;
    };
    auto tile = [&](int it) {
      const int key0 = begin + it * kStep;
      const bool edge = key0 < inside_lo || key0 > inside_hi;  // some row does not see some of the keys
      const char* const tile_at = ring + stage;
      floatx4 s[2];
      uint32_t codes[2][NG], k_pairs[2][PIECES];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        uint32_t (&kc)[NG] = codes[j];
        if constexpr (NG == 1) {
          kc[0] = *reinterpret_cast<const uint32_t*>(tile_at + k_at[0] + j * 16 * Ring::kRow);
        } else if constexpr (NG == 2) {
          const u32x2 w = *reinterpret_cast<const u32x2*>(tile_at + k_at[0] + j * 16 * Ring::kRow);
          kc[0] = w[0], kc[1] = w[1];
        } else {
#pragma unroll
          for (int i = 0; i < PIECES; ++i) {
            const uint4 w = *reinterpret_cast<const uint4*>(tile_at + k_at[i] + j * 16 * Ring::kRow);
            kc[4 * i] = w.x, kc[4 * i + 1] = w.y, kc[4 * i + 2] = w.z, kc[4 * i + 3] = w.w;
          }
        }
#pragma unroll
        for (int i = 0; i < PIECES; ++i) k_pairs[j][i] = *reinterpret_cast<const uint32_t*>(tile_at + kp_at + j * 64 * NG + 4 * i);
      }
      __builtin_amdgcn_sched_barrier(0);  // both blocks' reads before the first one's products
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        s[j] = floatx4{};
#pragma unroll
        for (int i = 0; i < NG; ++i) {
          const half8 kf = values8(codes[j][i], k_pairs[j][NG == 8 ? i / 4 : 0], bits);
#pragma unroll
          for (int part = 0; part < PARTS; ++part) s[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf, qf[part][i], s[j], 0, 0, 0);
        }
      }
      if (edge) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int key = key0 + 16 * j + 4 * quad + r;
            s[j][r] = key >= seen.lo && key <= seen.hi ? s[j][r] : kNegInf;
          }
      }
      float top = s[0][0];
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) top = fmaxf(top, s[j][r]);
      top = max_across32(max_across16(top)) * factor;
      if (__any(top > ref + kPackedSlack)) {
        if (it > 0) {
          raised = fmaxf(ref, top);
          return kRaise;
        }
        ref = fmaxf(ref, top);  // nothing to rescale yet
      }
      uint32_t vc[8][PIECES], pairs[8];
      load_values(tile_at, vc, pairs);  // ahead of the exponentials
      __builtin_amdgcn_sched_barrier(0);
      const float base = ref == kNegInf ? 0.0f : ref - kPackedLift;
      uint32_t w[PARTS][4];
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int r = 0; r < 4; r += 2) {
          const float a = __builtin_amdgcn_exp2f(__builtin_fmaf(s[j][r], factor, -base));
          const float b = __builtin_amdgcn_exp2f(__builtin_fmaf(s[j][r + 1], factor, -base));
          sum += a;
          sum += b;
          const uint32_t hi = pack2h(a, b);
          w[0][2 * j + r / 2] = hi;
          if constexpr (PARTS == 2) w[PARTS - 1][2 * j + r / 2] = pack2h(a - (float)half2_of(hi)[0], b - (float)half2_of(hi)[1]);
        }
#pragma unroll
      for (int part = 0; part < PARTS; ++part) pf[part] = __builtin_bit_cast(half8, uint4{w[part][0], w[part][1], w[part][2], w[part][3]});
      // Where some row does not see some key, that key's exponential is zero, but zero times an infinity or a NaN is not: pairs of keys that
      // no row sees become zero, and so do those whose smallest or largest value is not finite, which are added by themselves.
      bool odd = false;
      if (edge) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int key = key0 + 16 * (e / 4) + 4 * quad + e % 4;
          const bool seen_by_some = key >= any_lo && key <= any_hi, bad = infinite(pairs[e]);
          pairs[e] = seen_by_some && !bad ? pairs[e] : 0u;
          odd = odd || (seen_by_some && bad);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      half2 scale[4], low[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) scale[e] = scales2(pairs[2 * e], pairs[2 * e + 1]), low[e] = lows2(pairs[2 * e], pairs[2 * e + 1]);  // pairs of keys
#pragma unroll
      for (int b = 0; b < NG; ++b) {
        uint32_t even[4], odds[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t w = __builtin_amdgcn_perm(vc[2 * e + 1][b / 4], vc[2 * e][b / 4], v_sel + (b % 4) * 0x00010001u);
          even[e] = values2(codes_low(w, bits), scale[e], low[e]);
          odds[e] = values2(codes_high(w, bits), scale[e], low[e]);
        }
        const half8 v0 = __builtin_bit_cast(half8, uint4{even[0], even[1], even[2], even[3]});
        const half8 v1 = __builtin_bit_cast(half8, uint4{odds[0], odds[1], odds[2], odds[3]});
#pragma unroll
        for (int part = 0; part < PARTS; ++part) {
          o[2 * b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, pf[part], o[2 * b], 0, 0, 0);
          o[2 * b + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, pf[part], o[2 * b + 1], 0, 0, 0);
        }
      }
      return edge && __any(odd) ? kOdd : kDone;
    };
    // A key at a time: the product of its bad groups' values alone, added for the rows that see the key.
    auto add_odd = [&](int it) {
      const int key0 = begin + it * kStep;
      uint32_t vc[8][PIECES], vp[8];
      load_values(ring + stage, vc, vp);
      const int from = max(key0, any_lo), to = min(key0 + KEYS - 1, any_hi);
#pragma unroll 1
      for (int key = from; key <= to; ++key) {
#pragma unroll
        for (int b = 0; b < NG; ++b) {
          uint32_t x[2][4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int first_key = key0 + 16 * (e / 2) + 4 * quad + 2 * (e & 1);
            const uint32_t only = (first_key == key && infinite(vp[2 * e]) ? 0xffffu : 0u) | (first_key + 1 == key && infinite(vp[2 * e + 1]) ? 0xffff0000u : 0u);
            const uint32_t w = __builtin_amdgcn_perm(vc[2 * e + 1][b / 4], vc[2 * e][b / 4], v_sel + (b % 4) * 0x00010001u);
            const half2 scale = scales2(vp[2 * e], vp[2 * e + 1]), low = lows2(vp[2 * e], vp[2 * e + 1]);
            x[0][e] = values2(codes_low(w, bits), scale, low) & only;
            x[1][e] = values2(codes_high(w, bits), scale, low) & only;
          }
#pragma unroll
          for (int k = 0; k < 2; ++k) {
#pragma unroll
            for (int part = 0; part < PARTS; ++part) {
              const floatx4 got = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, uint4{x[k][0], x[k][1], x[k][2], x[k][3]}), pf[part], floatx4{}, 0, 0, 0);
#pragma unroll
              for (int r = 0; r < 4; ++r)
                if (key >= seen.lo && key <= seen.hi) o[2 * b + k][r] += got[r];
            }
          }
        }
      }
    };
    auto raise = [&]() {
      const float keep = raised == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(ref - raised);
      ref = raised;
      sum *= keep;
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) o[j][r] *= keep;
    };

    bool again = false;  // the tile was gone through as far as its scores
    for (int it = 0; it < count;) {
      int end = kDone;
#pragma unroll 1
      for (; it < count; ++it, stage = after(stage, 1)) {
        if (!again) advance(it);
        again = false;
        end = tile(it);
        if (end != kDone) break;
      }
      if (end == kRaise) {
        raise();
        again = true;
      } else if (end == kOdd) {
        add_odd(it);
        ++it, stage = after(stage, 1);
      }
    }
    wait_loads<0>();  // copies of tiles past the last one too: their place is used otherwise

    // A row's statistics: the reference that its exponentials and their sum are relative to.
    sum = sum_across32(sum_across16(sum));
    ref = ref == kNegInf ? kNegInf : ref - kPackedLift;
    auto store_out = [&](int row, int e, const float* v, int n, float inv) {  // n elements of a row, from e on
      const int t = row / p.group, h = u.head * p.group + (row - t * p.group);
      const int64_t to = (int64_t)(u.start + t) * p.o_token + (int64_t)h * p.o_head + e;
      for (int i = 0; i < n; i += 2) {
        if constexpr (PARTS == 1) reinterpret_cast<uint32_t*>(p.out)[(to + i) / 2] = pack2(v[i] * inv, v[i + 1] * inv);
        else reinterpret_cast<floatx2*>(p.out)[(to + i) / 2] = floatx2{v[i] * inv, v[i + 1] * inv};
      }
    };
    auto store_lse = [&](int row, float top, float total) {
      const int t = row / p.group, h = u.head * p.group + (row - t * p.group);
      p.lse[(int64_t)(u.start + t) * p.q_heads + h] = total == 0.0f ? kNegInf : (top + __builtin_amdgcn_logf(total)) * 0.69314718055994531f;
    };
    if constexpr (MANY) {
      const int row = row0 + col;
      if (row < rows) {
        const int64_t part = (2 * (int64_t)blockIdx.x + (begins ? 0 : 1)) * ROWS + (row - u.row0);
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int e = NJ * (4 * quad + r);
          float v[NJ];
#pragma unroll
          for (int j = 0; j < NJ; ++j) v[j] = o[j][r];
          constexpr int kRun = NJ < 8 ? NJ : 8;  // heads are multiples of 8
#pragma unroll
          for (int i = 0; i < NJ; i += kRun) {
            if (e + i >= p.dim) continue;
            if (whole) {
              store_out(row, e + i, v + i, kRun, inv);
            } else {
#pragma unroll
              for (int k = 0; k < kRun; k += 2) *reinterpret_cast<floatx2*>(p.part_o + part * p.dim + e + i + k) = floatx2{v[i + k], v[i + k + 1]};
            }
          }
        }
        if (quad == 0) {
          if (!whole) *reinterpret_cast<floatx2*>(p.part_ml + part * 2) = floatx2{ref, sum};
          else if (p.lse) store_lse(row, ref, sum);
        }
      }
    } else {
      __syncthreads();
      float* const joined = reinterpret_cast<float*>(lds);                    // [wave][row][JP]
      float* const stats = joined + NW * ROWS * JP;  // [wave][row][2]
      const int r = wave * ROWS + col;
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int j = 0; j < NJ; j += 2) *reinterpret_cast<floatx2*>(joined + r * JP + NJ * (4 * quad + k) + j) = floatx2{o[j][k], o[j + 1][k]};
      if (quad == 0) stats[r * 2] = ref, stats[r * 2 + 1] = sum;
      __syncthreads();
      constexpr int kQuads = DP / 4;
      for (int i = thread; i < ROWS * kQuads; i += 64 * NW) {
        const int r = i / kQuads, e = (i % kQuads) * 4, row = u.row0 + r;
        if (row >= rows || e >= p.dim) continue;
        float top = kNegInf;
#pragma unroll
        for (int w = 0; w < NW; ++w) top = fmaxf(top, stats[(w * ROWS + r) * 2]);
        floatx4 v{0.0f, 0.0f, 0.0f, 0.0f};
        float total = 0.0f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
          const float f = join_weight(stats[(w * ROWS + r) * 2], top);
          const floatx4 x = *reinterpret_cast<const floatx4*>(joined + (w * ROWS + r) * JP + e);
          total += stats[(w * ROWS + r) * 2 + 1] * f;
#pragma unroll
          for (int k = 0; k < 4; ++k) v[k] += x[k] * f;
        }
        if (!whole) {  // a workgroup's first item and its last one may be shared: two parts
          const int64_t part = (2 * (int64_t)blockIdx.x + (begins ? 0 : 1)) * ROWS + r;
          *reinterpret_cast<floatx4*>(p.part_o + part * p.dim + e) = v;
          if (e == 0) *reinterpret_cast<floatx2*>(p.part_ml + part * 2) = floatx2{top, total};
        } else {
          const float y[4] = {v[0], v[1], v[2], v[3]};
          store_out(row, e, y, 4, total == 0.0f ? 0.0f : 1.0f / total);
          if (p.lse && e == 0) store_lse(row, top, total);
        }
      }
    }
    if (at >= end || !next_item(batch, at, &u)) break;
    if constexpr (!MANY) __syncthreads();  // the join's reads come before the next item's writes
  }
}

template <int NG, int PARTS, int NW, bool MANY>
hipError_t launch_packed(const PackedAttendParams& p, int whole_pages, hipStream_t stream) {
  const dim3 grid((unsigned)p.a.units), block(64 * NW);
  if (p.a.keys != kPackedKeys || (1 << p.a.log_rows) != 16 * (MANY ? NW : 1)) return hipErrorInvalidValue;
  if (whole_pages) attend_packed_kernel<NG, PARTS, NW, MANY, true><<<grid, block, 0, stream>>>(p);
  else attend_packed_kernel<NG, PARTS, NW, MANY, false><<<grid, block, 0, stream>>>(p);
  return hipGetLastError();
}

// NW: waves of a workgroup for heads of up to 128.
template <int PARTS, int NW, bool MANY>
hipError_t launch_packed_dim(const PackedAttendParams& p, int whole_pages, hipStream_t stream) {
  if (p.a.dim <= 32) return launch_packed<1, PARTS, NW, MANY>(p, whole_pages, stream);
  if (p.a.dim <= 64) return launch_packed<2, PARTS, NW, MANY>(p, whole_pages, stream);
  if (p.a.dim <= 128) return launch_packed<4, PARTS, NW, MANY>(p, whole_pages, stream);
  return launch_packed<8, PARTS, 4, MANY>(p, whole_pages, stream);
}

}  // namespace sc
