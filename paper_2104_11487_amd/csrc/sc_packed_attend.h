// Attention over a paged cache in 4 bits (sc_packed.h), every row count.
//
//   o = sum_l exp(s_l - m) v_l / sum_l exp(s_l - m),   s_l = scale q . k_l,   over the keys l that the row sees
//
// Codes go from memory into registers in the layout of the matrix unit's operands and become fp16 there: nothing passes through LDS.
//   Scores, transposed: S' = K Q' on 16 x 16 x 32 products, K the left operand. Lane (c, g) = (lane & 15, lane >> 4) holds of key c the g-th
//   quarter of the row's bytes; which elements a step's k indexes stand for is free as long as the queries follow, so those are loaded in the
//   order in which a mask leaves the codes (0 4 1 5 2 6 3 7 of each eight).
//   Outputs: O' = V' P'. Lane (c, g) holds of the keys 4 g + r (r < 4) of each of the tile's two 16-key blocks the c-th 16th of the row's
//   bytes, two elements a byte: the two nibbles of a byte position over the 8 keys are the operands of two products, which stand for the
//   elements 2 NG c + j. A lane's scores are those of the same 8 keys, so the exponentials are the other operand as they are.
// Values are fp16 by the format, and queries exact: bf16 rows are scaled by a power of two into fp16 (the factor goes into the
// softmax's scale), fp32 rows are two fp16 parts (22 bits). Scores and sums are fp32. For bf16 the exponentials are rounded to fp16 (2^-11 of each)
// for the product with V, for fp32 they are two parts; they are formed 2^7 too large, so that those of up to 2^-21 of the
// reference's stay normal numbers.
#pragma once

#include <type_traits>

#include "sc_packed_device.h"

#pragma clang fp contract(off)

namespace sc {

constexpr float kPackedSlack = 8.0f;  // powers of two that an exponential may exceed the reference's by
constexpr float kPackedLift = 7.0f;   // powers of two that exponentials are formed too large by: 2^15 at most

// Where a tile's keys lie, looked up ahead: with whole pages of 16-key blocks a block's page and first slot, alike in all lanes; otherwise the
// lane's key's (lane & 31).
template <bool WHOLE>
struct PackedPlace {
  int entry[WHOLE ? 2 : 1], slot[WHOLE ? 2 : 1];
};

// NG: groups of a head, rounded up to a power of two. NB: 16-row blocks of a wave. PARTS: fp16 parts of a query and an exponential.
// MANY: the waves take rows of their own and all keys; otherwise they take the same rows and every NW-th key tile.
template <int NG, int NB, int PARTS, bool MANY, bool WHOLE>
__global__ void __launch_bounds__(64 * (MANY ? kPackedManyWaves : kPackedFewWaves), MANY ? 2 : 1) attend_packed_kernel(PackedAttendParams pp) {
  constexpr int NW = MANY ? kPackedManyWaves : kPackedFewWaves, WROWS = 16 * NB, ROWS = MANY ? NW * WROWS : WROWS;
  constexpr int KEYS = kPackedKeys, DP = 32 * NG, NJ = 2 * NG, PIECES = NG == 8 ? 2 : 1;
  constexpr int JP = DP + 4;  // joining: a row's stride in LDS, in floats
  __shared__ alignas(16) float lds[MANY ? 4 : NW * ROWS * (JP + 2)];
  const AttendParams& p = pp.a;

  const Units batch(p);
  const Shares shares = shares_of(batch);
  if ((int)blockIdx.x >= shares.n) return;
  const int64_t first_unit = shares.at(blockIdx.x), end = shares.at(blockIdx.x + 1);
  Unit u;
  if (first_unit >= end || !unit_of(batch, first_unit, &u)) return;
  const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6);
  const int col = lane & 15, quad = lane >> 4, last_group = pp.groups - 1;

  // Byte offsets in a row: the lane's pieces of a key, of a value; of their pairs. Groups past the head's are led to the last one (the queries
  // are zero there, and the outputs are not stored). With whole pages the lane's row of a block is in them.
  uint32_t k_at[PIECES], kp_at[PIECES], v_at[WHOLE ? 4 : 1], vp_at[WHOLE ? 4 : 1];
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    const int g = NG >= 4 ? min(quad * (NG / 4) + i, last_group) : NG * quad / 4;
    k_at[i] = (NG >= 4 ? 16 * g : 4 * NG * quad) + (WHOLE ? (uint32_t)(col * (int)p.c.k_slot) : 0u);
    kp_at[i] = 4 * g + (WHOLE ? (uint32_t)(col * (int)pp.s.k_slot) : 0u);
  }
  const int v_group = min(NG * col / 16, last_group);
  const uint32_t v_byte = NG >= 4 ? 16 * v_group + (NG * col) % 16 : (NG * col) & ~3;
#pragma unroll
  for (int r = 0; r < (WHOLE ? 4 : 1); ++r) {
    v_at[r] = v_byte + (WHOLE ? (uint32_t)((4 * quad + r) * (int)p.c.v_slot) : 0u);
    vp_at[r] = 4 * v_group + (WHOLE ? (uint32_t)((4 * quad + r) * (int)pp.s.v_slot) : 0u);
  }
  const CodeBits bits = code_bits();
  // page and slot strides of the keys' codes and pairs, the values' codes and pairs
  const uint32_t k_page = alone(p.c.k_page), k_slot = alone(p.c.k_slot), ks_page = alone(pp.s.k_page), ks_slot = alone(pp.s.k_slot);
  const uint32_t v_page = alone(p.c.v_page), v_slot = alone(p.c.v_slot), vs_page = alone(pp.s.v_page), vs_slot = alone(pp.s.v_slot);
  const uint32_t v_sel = NG >= 4 ? 0x0c040c00u : 0x0c040c00u + ((NG * col) & 3) * 0x00010001u;  // picks a byte of two words into 16-bit halves

  for (int64_t at = first_unit;;) {
    const int units = (int)min(end - at, (int64_t)(u.parts - u.part));  // of this item
    const bool whole = units == u.parts, begins = at == first_unit;
    at += units;
    u.hi = (int)min((int64_t)u.hi, u.lo + (int64_t)units * u.chunk);
    const int rows = u.n * p.group, row0 = u.row0 + (MANY ? wave * WROWS : 0);

    // the rows' queries, in the operand's layout
    half8 qf[NB][PARTS][NG];
    Seen seen[NB];
    float factor[NB];  // of a score, to powers of two
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const int r = min(row0 + 16 * n + col, rows - 1), t = r / p.group, h = u.head * p.group + (r - t * p.group);
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
      const int lift = 141 - (int)((__float_as_uint(most) >> 23) & 255u);  // the largest element comes into [2^14, 2^15)
      factor[n] = ldexpf(p.scale_log2, -lift);
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
          qf[n][part][i] = __builtin_bit_cast(half8, uint4{w[0], w[1], w[2], w[3]});
        }
      seen[n] = seen_by(p, u, row0 + 16 * n + col);
    }
    // keys that every row of the wave sees, that some row sees
    const Seen first = seen_by(p, u, row0), last = seen_by(p, u, row0 + WROWS - 1);
    const int all_lo = last.lo, all_hi = first.hi, any_lo = first.lo, any_hi = last.hi;

    floatx4 o[NB][NJ];
    float ref[NB], sum[NB], raised[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      ref[n] = raised[n] = kNegInf, sum[n] = 0.0f;
#pragma unroll
      for (int j = 0; j < NJ; ++j) o[n][j] = floatx4{};
    }

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

    // A tile in the lane's registers: codes and pairs of keys and of values.
    uint32_t kc[2][NG], kp[2][PIECES], vc[8][PIECES], vp[8];
    PackedPlace<WHOLE> place;
    const char* v_rows[2];  // whole pages: a block's first value, its pairs
    const char* v_pairs[2];
    int page_l = 0, slot_l = 0;  // otherwise: the lane's key's

    auto find = [&](int key0) {
      if constexpr (WHOLE) {
#pragma unroll
        for (int j = 0; j < 2; ++j) place.entry[j] = entry_at(p.c, u.b, key0 + 16 * j, 16, &place.slot[j]);
      } else {
        place.entry[0] = entry_at(p.c, u.b, key0 + (lane & 31), 1, &place.slot[0]);
      }
    };
    auto load_key = [&](const char* row, const char* pairs, uint32_t* codes, uint32_t* pair) {
      if constexpr (NG == 1) {
        codes[0] = *reinterpret_cast<const uint32_t*>(row + here(k_at[0]));
      } else if constexpr (NG == 2) {
        const u32x2 w = *reinterpret_cast<const u32x2*>(row + here(k_at[0]));
        codes[0] = w[0], codes[1] = w[1];
      } else {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
          const uint4 w = *reinterpret_cast<const uint4*>(row + here(k_at[i]));
          codes[4 * i] = w.x, codes[4 * i + 1] = w.y, codes[4 * i + 2] = w.z, codes[4 * i + 3] = w.w;
        }
      }
#pragma unroll
      for (int i = 0; i < PIECES; ++i) pair[i] = *reinterpret_cast<const uint32_t*>(pairs + here(kp_at[i]));
    };
    auto load_value = [&](const char* row, const char* pairs, int r, uint32_t* codes, uint32_t* pair) {
      if constexpr (PIECES == 2) {
        const u32x2 w = *reinterpret_cast<const u32x2*>(row + here(v_at[r]));
        codes[0] = w[0], codes[1] = w[1];
      } else {
        codes[0] = *reinterpret_cast<const uint32_t*>(row + here(v_at[r]));
      }
      *pair = *reinterpret_cast<const uint32_t*>(pairs + here(vp_at[r]));
    };
    auto fetch_keys = [&]() {  // of the tile at `place`, which then is free
      if constexpr (WHOLE) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint64_t page = (uint32_t)page_of_entry(p.c, uniform(place.entry[j])), slot = (uint32_t)uniform(place.slot[j]);
          load_key(kb + (page * k_page + slot * k_slot), ksb + (page * ks_page + slot * ks_slot), kc[j], kp[j]);
          v_rows[j] = vb + (page * v_page + slot * v_slot);
          v_pairs[j] = vsb + (page * vs_page + slot * vs_slot);
        }
      } else {
        page_l = page_of_entry(p.c, place.entry[0]), slot_l = place.slot[0];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int64_t page = __shfl(page_l, 16 * j + col), slot = __shfl(slot_l, 16 * j + col);
          load_key(kb + page * p.c.k_page + slot * p.c.k_slot, ksb + page * pp.s.k_page + slot * pp.s.k_slot, kc[j], kp[j]);
        }
      }
    };
    auto fetch_values = [&]() {  // of the tile whose keys were fetched last
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if constexpr (WHOLE) {
          load_value(v_rows[e / 4], v_pairs[e / 4], e % 4, vc[e], &vp[e]);
        } else {
          const int64_t page = __shfl(page_l, 16 * (e / 4) + 4 * quad + e % 4), slot = __shfl(slot_l, 16 * (e / 4) + 4 * quad + e % 4);
          load_value(vb + page * p.c.v_page + slot * p.c.v_slot, vsb + page * pp.s.v_page + slot * pp.s.v_slot, 0, vc[e], &vp[e]);
        }
      }
    };

    // One tile's work, and the loads of the next one, whose keys take the place of this one's as soon as these are in the product, and values
    // likewise. edge: some row does not see some of its keys. Where a score passes the reference by more than the slack nothing is done but to
    // raise it, and the tile is to be gone through again: so the outputs' registers are touched by products alone in the loop, and keep their places.
    auto tile = [&](auto edge_, int it) {
      constexpr bool edge = edge_;
      const int key0 = begin + it * kStep;
      floatx4 s[NB][2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
#pragma unroll
        for (int n = 0; n < NB; ++n) s[n][j] = floatx4{};
#pragma unroll
        for (int i = 0; i < NG; ++i) {
          const half8 kf = values8(kc[j][i], kp[j][NG == 8 ? i / 4 : 0], bits);
#pragma unroll
          for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int part = 0; part < PARTS; ++part) s[n][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf, qf[n][part][i], s[n][j], 0, 0, 0);
        }
      }
      bool past = false;
      float top[NB];
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        if constexpr (edge) {
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int key = key0 + 16 * j + 4 * quad + r;
              s[n][j][r] = key >= seen[n].lo && key <= seen[n].hi ? s[n][j][r] : kNegInf;
            }
        }
        top[n] = s[n][0][0];
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) top[n] = fmaxf(top[n], s[n][j][r]);
        top[n] = max_across32(max_across16(top[n])) * factor[n];
        past = past || top[n] > ref[n] + kPackedSlack;
      }
      if (__any(past)) {
#pragma unroll
        for (int n = 0; n < NB; ++n) raised[n] = fmaxf(ref[n], top[n]);
        return false;
      }
      __builtin_amdgcn_sched_barrier(0);
      fetch_keys();
      find(key0 + 2 * kStep);
      __builtin_amdgcn_sched_barrier(0);
      half8 pf[NB][PARTS];
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        const float base = ref[n] == kNegInf ? 0.0f : ref[n] - kPackedLift;
        uint32_t w[PARTS][4];
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int r = 0; r < 4; r += 2) {
            const float a = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n][j][r], factor[n], -base));
            const float b = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n][j][r + 1], factor[n], -base));
            sum[n] += a;
            sum[n] += b;
            const uint32_t hi = pack2h(a, b);
            w[0][2 * j + r / 2] = hi;
            if constexpr (PARTS == 2) w[PARTS - 1][2 * j + r / 2] = pack2h(a - (float)half2_of(hi)[0], b - (float)half2_of(hi)[1]);
          }
#pragma unroll
        for (int part = 0; part < PARTS; ++part) pf[n][part] = __builtin_bit_cast(half8, uint4{w[part][0], w[part][1], w[part][2], w[part][3]});
      }
      // Values. Where some row does not see some key, a masked key's exponential is zero, but zero times an infinity or a
      // NaN is not: values of keys that no row sees are cleared, and those that are not finite leave the product and
      // are added to the rows that see their key.
      __builtin_amdgcn_sched_barrier(0);
      int odd = 0;
      half2 scale[4], low[4];
      uint32_t mask[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {  // pairs of keys
        scale[e] = scales2(vp[2 * e], vp[2 * e + 1]), low[e] = lows2(vp[2 * e], vp[2 * e + 1]);
        if constexpr (edge) {
          const int key = key0 + 16 * (e / 2) + 4 * quad + 2 * (e & 1);
          mask[e] = (key >= any_lo && key <= any_hi ? 0xffffu : 0u) | (key + 1 >= any_lo && key + 1 <= any_hi ? 0xffff0000u : 0u);
        }
      }
#pragma unroll
      for (int b = 0; b < NG; ++b) {
        uint32_t even[4], odds[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t w = __builtin_amdgcn_perm(vc[2 * e + 1][b / 4], vc[2 * e][b / 4], v_sel + (b % 4) * 0x00010001u);
          even[e] = values2(codes_low(w, bits), scale[e], low[e]);
          odds[e] = values2(codes_high(w, bits), scale[e], low[e]);
          if constexpr (edge) even[e] = finite2h(even[e], mask[e], &odd), odds[e] = finite2h(odds[e], mask[e], &odd);
        }
        const half8 v0 = __builtin_bit_cast(half8, uint4{even[0], even[1], even[2], even[3]});
        const half8 v1 = __builtin_bit_cast(half8, uint4{odds[0], odds[1], odds[2], odds[3]});
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int part = 0; part < PARTS; ++part) {
            o[n][2 * b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, pf[n][part], o[n][2 * b], 0, 0, 0);
            o[n][2 * b + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, pf[n][part], o[n][2 * b + 1], 0, 0, 0);
          }
      }
      if (edge && __any(odd)) {
        // A key at a time: its values alone in the left operand, ones in the other, give every row its values; those that are not finite
        // are added where the row sees the key.
        const uint32_t one2 = bits_of(half2{1.0f16, 1.0f16});
        const half8 ones = __builtin_bit_cast(half8, uint4{one2, one2, one2, one2});
        const int from = max(key0, any_lo), to = min(key0 + KEYS - 1, any_hi);
#pragma unroll 1
        for (int key = from; key <= to; ++key) {
#pragma unroll
          for (int b = 0; b < NG; ++b) {
            uint32_t x[2][4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int first_key = key0 + 16 * (e / 2) + 4 * quad + 2 * (e & 1);
              const uint32_t only = first_key == key ? 0xffffu : first_key + 1 == key ? 0xffff0000u : 0u;
              const uint32_t w = __builtin_amdgcn_perm(vc[2 * e + 1][b / 4], vc[2 * e][b / 4], v_sel + (b % 4) * 0x00010001u);
              x[0][e] = values2(codes_low(w, bits), scale[e], low[e]) & only;
              x[1][e] = values2(codes_high(w, bits), scale[e], low[e]) & only;
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const floatx4 got = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, uint4{x[k][0], x[k][1], x[k][2], x[k][3]}), ones, floatx4{}, 0, 0, 0);
#pragma unroll
              for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                  if ((__float_as_uint(got[r]) & 0x7f800000u) == 0x7f800000u && key >= seen[n].lo && key <= seen[n].hi) o[n][2 * b + k][r] += got[r];
            }
          }
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      fetch_values();
      return true;
    };
    auto raise = [&]() {
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        const float keep = raised[n] == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(ref[n] - raised[n]);
        ref[n] = raised[n];
        sum[n] *= keep;
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) o[n][j][r] *= keep;
      }
    };

    if (count > 0) {
      find(begin);
      fetch_keys();
      fetch_values();
      find(begin + kStep);
    }
    // Tiles that all rows see whole have a loop of their own. The last tile's loads are of tiles past it, which no product takes.
    const int inside_lo = uniform(all_lo), inside_hi = uniform(all_hi) - KEYS + 1;
    for (int it = 0; it < count;) {
#pragma unroll 1
      for (; it < count && begin + it * kStep >= inside_lo && begin + it * kStep <= inside_hi && tile(std::false_type{}, it); ++it) {}
      if (it >= count) break;
      if (begin + it * kStep >= inside_lo && begin + it * kStep <= inside_hi) raise();
      else if (tile(std::true_type{}, it)) ++it;
      else raise();
    }

    // A row's statistics: the reference that its exponentials and their sum are relative to.
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      sum[n] = sum_across32(sum_across16(sum[n]));
      ref[n] = ref[n] == kNegInf ? kNegInf : ref[n] - kPackedLift;
    }
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
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        const int row = row0 + 16 * n + col;
        if (row >= rows) continue;
        const int64_t part = (2 * (int64_t)blockIdx.x + (begins ? 0 : 1)) * ROWS + (row - u.row0);
        const float inv = sum[n] == 0.0f ? 0.0f : 1.0f / sum[n];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int e = NJ * (4 * quad + r);
          float v[NJ];
#pragma unroll
          for (int j = 0; j < NJ; ++j) v[j] = o[n][j][r];
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
          if (!whole) *reinterpret_cast<floatx2*>(p.part_ml + part * 2) = floatx2{ref[n], sum[n]};
          else if (p.lse) store_lse(row, ref[n], sum[n]);
        }
      }
    } else {
      __syncthreads();
      float* const joined = lds;                    // [wave][row][JP]
      float* const stats = joined + NW * ROWS * JP;  // [wave][row][2]
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        const int r = wave * ROWS + 16 * n + col;
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int j = 0; j < NJ; j += 2) *reinterpret_cast<floatx2*>(joined + r * JP + NJ * (4 * quad + k) + j) = floatx2{o[n][j][k], o[n][j + 1][k]};
        if (quad == 0) stats[r * 2] = ref[n], stats[r * 2 + 1] = sum[n];
      }
      __syncthreads();
      constexpr int kQuads = DP / 4;
      for (int i = threadIdx.x; i < ROWS * kQuads; i += 64 * NW) {
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

template <int NG, int NB, int PARTS, bool MANY>
hipError_t launch_packed(const PackedAttendParams& p, int whole_pages, hipStream_t stream) {
  const dim3 grid((unsigned)p.a.units), block(64 * (MANY ? kPackedManyWaves : kPackedFewWaves));
  if (p.a.keys != kPackedKeys || (1 << p.a.log_rows) != 16 * NB * (MANY ? kPackedManyWaves : 1)) return hipErrorInvalidValue;
  if (whole_pages) attend_packed_kernel<NG, NB, PARTS, MANY, true><<<grid, block, 0, stream>>>(p);
  else attend_packed_kernel<NG, NB, PARTS, MANY, false><<<grid, block, 0, stream>>>(p);
  return hipGetLastError();
}

// NARROW, WIDE: row blocks for heads of up to 128, above.
template <int NARROW, int WIDE, int PARTS, bool MANY>
hipError_t launch_packed_dim(const PackedAttendParams& p, int whole_pages, hipStream_t stream) {
  if (p.a.dim <= 32) return launch_packed<1, NARROW, PARTS, MANY>(p, whole_pages, stream);
  if (p.a.dim <= 64) return launch_packed<2, NARROW, PARTS, MANY>(p, whole_pages, stream);
  if (p.a.dim <= 128) return launch_packed<4, NARROW, PARTS, MANY>(p, whole_pages, stream);
  return launch_packed<8, WIDE, PARTS, MANY>(p, whole_pages, stream);
}

}  // namespace sc
