// Attention over the paged cache for many rows at once (new tokens x query heads of a key head).
//
//   o = sum_l exp(s_l - m) v_l / sum_l exp(s_l - m),   s_l = scale q . k_l,   over the keys l that the row sees
//
// in one pass over the keys with a running reference m and sum. A workgroup of 4 waves takes 128 rows (256 where two row blocks a
// wave fit the registers of two waves a SIMD: bf16 heads of up to 64), and walks the keys in tiles that all waves share, the next
// tile's copies into LDS in flight during this one's products. Where a launch has fewer items (128 rows and a key head) than workgroups
// fit the GPU, they share its key tiles (sc_attend_device.h), and a second launch joins the parts.
// With many rows the matrix and vector units bound it (8192 tokens over 24576, heads of 128: 1.55 to 1.69 ms by card, 0.95 to 1.04 PFLOP/s, matrix
// units busy half of the time, the exponentials' vector work beside them as long); with a row of each of many sequences the
// cache's bytes do (64 sequences of up to 16384, heads of 128: 220 us, 5.2 TB/s).
// Heads above 128 (fp32: above 96) leave one wave a SIMD (bf16 heads of 256, 4096 tokens of 4 streams over 12288: 2.1 ms, 64 % of the product's rate). Builds that
// do not hold everything in registers: fp32 above 192, 114 to 147 in scratch memory (256 tokens of 4 sequences over
// 1500, 4 heads of 256: 210 us, of 192: 82); fp32 96 (7 to 23, not where nothing is shared and pages are whole), bf16 64 with two row blocks where keys are
// shared (12 to 23), bf16 96 and 128 where they are (1), bf16 256 (3 in one build).
// Products are formed transposed: scores S' = K Q' have a row's scores in two lanes (l and l + 32), so softmax needs one
// lane exchange a block of 32 keys, and O' = V' P' takes the exponentials from the registers that the scores left them in: the key
// that a k index of the product stands for is free, as long as V's fragment follows, so no lane exchange and no LDS is needed for P.
// Scores, exponentials' sums and outputs are fp32. For bf16 caches the exponentials are rounded to bf16 for the
// product with V (the matrix unit's operand type: up to 2^-8 of each, averaged over the keys); their sum takes them unrounded.
// The reference m is the largest score seen only up to 2^8: a row's output and sum are rescaled when a score passes it by
// more, which after the first tiles is seldom.
//
// Every 32 x 32 x 16 product reads a fragment of 1 KB from LDS, which at 128 bytes a cycle and 32 cycles a product on each of four SIMDs
// is all that LDS gives; two row blocks a wave halve that (4096 tokens over 12288, heads of 64: 517 -> 441 us), but with heads of 128
// they leave one wave a SIMD, whose vector work no longer runs beside its products (8192 tokens over 24576: 1522 -> 1987 us).
#pragma once

#include <type_traits>
#include <utility>

#include "sc_attend_tile.h"

#pragma clang fp contract(off)

namespace sc {

constexpr int kWideWaves = 4;
constexpr float kSlack = 8.0f;  // powers of two that an exponential may exceed one by

typedef uint32_t u32x4_lds __attribute__((ext_vector_type(4)));

// f(0), f(1), ... f(N - 1), each with its index as a constant.
template <int... I, typename F>
__device__ __forceinline__ void unrolled_(std::integer_sequence<int, I...>, F f) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void unrolled(F f) {
  unrolled_(std::make_integer_sequence<int, N>{}, f);
}

// Order of a block's fragments (each a slot of products): NQ of the next block's scores (0 ..), and for each half of its 32 keys ND of
// its values (NQ + k * ND ..). A value product needs its keys' exponentials, the largest score needs all score products: three
// quarters of the scores come first, the rest between the halves.
template <int NQ, int ND>
struct SlotPlan {
  static constexpr int kSlots = NQ + 2 * ND;
  struct Order {
    int at[kSlots];
    int last_score;
  };
  static constexpr Order order() {
    Order o = {};
    int n = 0, q = 0;
    for (; q < (NQ * 3 + 3) / 4; ++q) o.at[n++] = q;
    for (int d = 0; d < ND; ++d) o.at[n++] = NQ + d;
    for (; q < NQ; ++q) o.at[n++] = q;
    for (int m = 0; m < n; ++m)
      if (o.at[m] < NQ) o.last_score = m;
    for (int d = 0; d < ND; ++d) o.at[n++] = NQ + ND + d;
    return o;
  }
  static constexpr Order kOrder = order();
  // Exponentials, of `all`, formed by the end of slot n (-1: before the first): evenly until the last score product, but in time for
  // the first value product of each half.
  static constexpr int exps_by(int n, int all) {
    int e = ((n + 2) * all / (kOrder.last_score + 2) + 1) / 2 * 2;
    if (e > all) e = all;
    for (int m = 0; m <= n + 1 && m < kSlots; ++m)
      if (kOrder.at[m] >= NQ && e < ((kOrder.at[m] - NQ) / ND + 1) * (all / 2)) e = ((kOrder.at[m] - NQ) / ND + 1) * (all / 2);
    return e;
  }
  // Scores of the next block whose largest is known by the end of slot n: in the slots behind the last score product.
  static constexpr int tops_by(int n, int all) {
    const int from = kOrder.last_score + 2;
    if (n >= kSlots - 1) return all;
    if (n < from) return 0;
    return (n - from + 1) * all / (kSlots - from) / 2 * 2;
  }
};

// SHARED: workgroups may take keys of several items (a launch without them is spared what finds and ends a share, 0.4 us a workgroup).
template <typename T, int DP, int NR, bool UNI, bool SHARED>
__global__ void __launch_bounds__(64 * kWideWaves, wide_groups_of(sizeof(T), DP)) attend_wide_kernel(AttendParams p) {
  constexpr bool kHalf = sizeof(T) == 2;
  constexpr int NW = kWideWaves, WROWS = 32 * NR, ROWS = WROWS * NW, KEYS = wide_keys_of((int)sizeof(T), DP, NR);
  constexpr int NB = KEYS / 32, ND = DP / 32;  // blocks of 32 keys of a tile; of 32 dimensions
  using TL = Tile<T, DP, KEYS, NW, true>;
  constexpr int QF = kHalf ? DP / 16 : DP / 8;  // 16-byte pieces of a row that a lane holds
  __shared__ alignas(16) char lds[4 * TL::kBytes];  // keys, values; two buffers

  const Units batch(p);
  int64_t first_unit = blockIdx.x, end = first_unit + 1;
  if constexpr (SHARED) {
    const Shares shares = shares_of(batch);
    if ((int)blockIdx.x >= shares.n) return;
    first_unit = shares.at(blockIdx.x), end = shares.at(blockIdx.x + 1);
  }
  Unit u;
  if (first_unit >= end || !unit_of(batch, first_unit, &u)) return;
  const int chunks = p.dim / TL::kElems;
  // chunks that no copy fills: those past the head's dimension
  if (chunks < TL::kChunks) {
    for (int i = threadIdx.x; i < 4 * TL::kBytes / 16; i += 64 * NW) reinterpret_cast<uint4*>(lds)[i] = uint4{0u, 0u, 0u, 0u};
    __syncthreads();
  }
  for (int64_t at = first_unit;;) {
    const int units = (int)min(end - at, (int64_t)(u.parts - u.part));  // of this item
    const bool whole = !SHARED || units == u.parts, begins = at == first_unit;
    at += units;
    u.hi = (int)min((int64_t)u.hi, u.lo + (int64_t)units * u.chunk);
    // derived anew for each item, so that no register holds from one item to the next what only its ends need
    int thread = (int)threadIdx.x;
    asm volatile("" : "+v"(thread));
    const int lane = thread & 63, wave = uniform(thread >> 6), col = lane & 31, half = lane >> 5;
    // LDS addresses of the fragments. Keys: row (key) col of a 32-key block, 16-byte piece 2 i + half.
    // Values: see read_column4; e picks the upper four of eight keys.
    const uint32_t lds0 = (uint32_t)(uintptr_t)SC_LDS(lds, char);
    const int vr = 4 * half + ((lane & 15) >> 2), vc = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    uint32_t kat[QF], vat[kHalf ? 2 : 1][ND];
  #pragma unroll
    for (int i = 0; i < QF; ++i) kat[i] = lds0 + col * TL::kRowBytes + (((2 * i + half) ^ (TL::swizzle(col) & (TL::kChunks - 1))) << 4);
  #pragma unroll
    for (int e = 0; e < (kHalf ? 2 : 1); ++e)
  #pragma unroll
      for (int d = 0; d < ND; ++d)
        vat[e][d] = lds0 + 2 * TL::kBytes + (8 * e + vr) * TL::kRowBytes + (((4 * d + vc) ^ (TL::swizzle(8 * e + vr) & (TL::kChunks - 1))) << 4) + (lane & 1) * 8;

    const int rows = u.n * p.group;
    const int row0 = u.row0 + WROWS * wave;

    // the rows' queries: lane `half` holds the dimensions that its k indexes of the products stand for
    uint4 qf[NR][QF];
    Seen seen[NR];
  #pragma unroll
    for (int n = 0; n < NR; ++n) {
      const int r = min(row0 + 32 * n + col, rows - 1), t = r / p.group, h = u.head * p.group + (r - t * p.group);
      const char* q = p.q + ((int64_t)(u.start + t) * p.q_token + (int64_t)h * p.q_head) * (int64_t)sizeof(T);
  #pragma unroll
      for (int i = 0; i < QF; ++i) {
        const int c = 2 * i + half;
        qf[n][i] = c < chunks ? *reinterpret_cast<const uint4*>(q + c * 16) : uint4{0u, 0u, 0u, 0u};
      }
      seen[n] = seen_by(p, u, row0 + 32 * n + col);
    }
    // keys that every row of the unit sees: [all_lo, all_hi]
    const int all_lo = seen_by(p, u, u.row0 + ROWS - 1).lo, all_hi = min(seen_by(p, u, u.row0).hi, u.hi - 1);

    floatx16 o[NR][ND];
    float ref[NR], base[NR], sum[NR];  // base: what exponents are taken relative to, the reference or 0 before there is one
  #pragma unroll
    for (int n = 0; n < NR; ++n) {
      ref[n] = kNegInf, base[n] = 0.0f, sum[n] = 0.0f;
  #pragma unroll
      for (int d = 0; d < ND; ++d) o[n][d] = floatx16{};
    }

    // `at`: byte offset of a block's rows in the keys' (values') two buffers
    auto key_piece = [&](int i, int at) {  // 16 bytes of a key's row: the score products' operand
      return *(__attribute__((address_space(3))) const u32x4_lds*)(kat[i] + at);
    };
    auto value_piece = [&](int k, int d, int at) {  // 8 keys' values of a dimension: the value products' operand
      // rows 16 keys on keep the permutation, which repeats every 16 rows
      const u32x2 a = read_column4(vat[0][d] + at + 16 * k * TL::kRowBytes), b = read_column4(vat[kHalf ? 1 : 0][d] + at + 16 * k * TL::kRowBytes);
      return u32x4_lds{a[0], a[1], b[0], b[1]};
    };
    auto value1 = [&](int key, int d, int at) {
      const int e = 32 * d + col, c = (e >> 2) ^ (TL::swizzle(key) & (TL::kChunks - 1));
      return *reinterpret_cast<const float*>(lds + 2 * TL::kBytes + at + key * TL::kRowBytes + c * 16 + (e & 3) * 4);
    };

    using Scores = floatx16[NR];
    auto score_block = [&](int at, Scores& s) {  // the scores of the 32 keys at `at`
  #pragma unroll
      for (int n = 0; n < NR; ++n) s[n] = floatx16{};
  #pragma unroll
      for (int i = 0; i < QF; ++i) {
        const u32x4_lds kf = key_piece(i, at);
  #pragma unroll
        for (int n = 0; n < NR; ++n) {
          if constexpr (kHalf) {
            s[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf), __builtin_bit_cast(bf16x8, qf[n][i]), s[n], 0, 0, 0);
          } else {
            const floatx4 a = __builtin_bit_cast(floatx4, kf), b = __builtin_bit_cast(floatx4, qf[n][i]);
  #pragma unroll
            for (int e = 0; e < 4; ++e) s[n] = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], s[n], 0, 0, 0);
          }
        }
      }
    };
    struct Tops {
      float at[NR];
    };
    auto largest = [](const Scores& s) {
      Tops top;
  #pragma unroll
      for (int n = 0; n < NR; ++n) {
        top.at[n] = s[n][0];
  #pragma unroll
        for (int r = 1; r < 16; ++r) top.at[n] = fmaxf(top.at[n], s[n][r]);
      }
      return top;
    };
    auto key_of = [&](int r) { return 8 * (r >> 2) + 4 * half + (r & 3); };  // of a block, that score r of a lane belongs to
    auto hide = [&](Scores& s, int key0) {
  #pragma unroll
      for (int n = 0; n < NR; ++n)
  #pragma unroll
        for (int r = 0; r < 16; ++r) s[n][r] = key0 + key_of(r) >= seen[n].lo && key0 + key_of(r) <= seen[n].hi ? s[n][r] : kNegInf;
    };
    auto refer = [&](Tops top) {  // takes the largest score of the next block into the reference
      bool past = false;
  #pragma unroll
      for (int n = 0; n < NR; ++n) {
        top.at[n] = max_across32(top.at[n]) * p.scale_log2;
        past = past || top.at[n] > ref[n] + kSlack;
      }
      if (__any(past)) {
  #pragma unroll
        for (int n = 0; n < NR; ++n) {
          const float next = fmaxf(ref[n], top.at[n]);
          const float keep = ref[n] == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(ref[n] - next);  // 1: nothing to rescale yet
          ref[n] = next;
          base[n] = next == kNegInf ? 0.0f : next;
          sum[n] *= keep;
  #pragma unroll
          for (int d = 0; d < ND; ++d)
  #pragma unroll
            for (int r = 0; r < 16; ++r) o[n][d][r] *= keep;
        }
      }
    };
    auto exponent = [&](float x, int n) { return __builtin_amdgcn_exp2f(__builtin_fmaf(x, p.scale_log2, -base[n])); };

    // A block's exponentials and values, and the scores of the next one (keys at `kt`, values at `vt`).
    auto run_block = [&](int kt, int vt, Scores& s, Scores& next) {
      if constexpr (kHalf) {
        // Laid out by hand: each slot is one fragment's products, with the LDS reads of the one PRE slots later and a share of the
        // vector unit's work (this block's exponentials, then the next one's largest score) to run beside it.
        using PL = SlotPlan<QF, ND>;
        constexpr int PRE = 3, kAll = NR * 16;
        u32x4_lds frag[PL::kSlots];
        uint32_t packed[NR][8];
        auto read = [&](auto slot) {
          constexpr int m = slot;
          if constexpr (m < PL::kSlots) {
            constexpr int x = PL::kOrder.at[m];
            if constexpr (x < QF) frag[m] = key_piece(x, kt);
            else frag[m] = value_piece((x - QF) / ND, (x - QF) % ND, vt);
          }
        };
        auto form = [&](auto from, auto to) {  // exponentials [from, to) of the lane, in pairs: a half's keys, row block by row block
          constexpr int f = from, t = to;
  #pragma unroll
          for (int e = f; e < t; e += 2) {
            const int n = e / 8 % NR, r = e / (8 * NR) * 8 + e % 8;
            const float a = exponent(s[n][r], n), b = exponent(s[n][r + 1], n);
            sum[n] += a;
            sum[n] += b;
            packed[n][r / 2] = pack2(a, b);
          }
        };
        Tops top;
  #pragma unroll
        for (int n = 0; n < NR; ++n) top.at[n] = kNegInf, next[n] = floatx16{};
        unrolled<PRE>([&](auto m) { read(m); });
        form(std::integral_constant<int, 0>{}, std::integral_constant<int, PL::exps_by(-1, kAll)>{});
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);  // ahead of the other workgroup's wave, which is then in its copies, waits and reference
        unrolled<PL::kSlots>([&](auto slot) {
          constexpr int m = slot, x = PL::kOrder.at[m];
          read(std::integral_constant<int, m + PRE>{});
  #pragma unroll
          for (int n = 0; n < NR; ++n) {
            if constexpr (x < QF) {
              next[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, frag[m]), __builtin_bit_cast(bf16x8, qf[n][x]), next[n], 0, 0, 0);
            } else {
              constexpr int k = (x - QF) / ND, d = (x - QF) % ND;
              const uint4 w{packed[n][4 * k], packed[n][4 * k + 1], packed[n][4 * k + 2], packed[n][4 * k + 3]};
              o[n][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, frag[m]), __builtin_bit_cast(bf16x8, w), o[n][d], 0, 0, 0);
            }
          }
          form(std::integral_constant<int, PL::exps_by(m - 1, kAll)>{}, std::integral_constant<int, PL::exps_by(m, kAll)>{});
          constexpr int f = PL::tops_by(m - 1, kAll), t = PL::tops_by(m, kAll);
  #pragma unroll
          for (int e = f; e < t; e += 2) top.at[e / 16] = fmaxf(fmaxf(next[e / 16][e % 16], next[e / 16][e % 16 + 1]), top.at[e / 16]);
          __builtin_amdgcn_sched_barrier(0);
        });
        __builtin_amdgcn_s_setprio(0);
        return top;
      } else {
        score_block(kt, next);
  #pragma unroll
        for (int r = 0; r < 16; ++r) {
  #pragma unroll
          for (int n = 0; n < NR; ++n) {
            s[n][r] = exponent(s[n][r], n);
            sum[n] += s[n][r];
          }
  #pragma unroll
          for (int d = 0; d < ND; ++d) {
            const float v = value1(key_of(r), d, vt);
  #pragma unroll
            for (int n = 0; n < NR; ++n) o[n][d] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[n][r], o[n][d], 0, 0, 0);
          }
        }
        return largest(next);
      }
    };

    // Keys run one block ahead of values: with the values of tile i (keys i * KEYS ..) come the keys 32 further on, both in buffer i & 1.
    constexpr int kBlock = 32 * TL::kRowBytes;
    char* const values = lds + 2 * TL::kBytes;
    Stager<T, TL, NW, UNI, 32> stager(p, u, wave, lane, chunks);
    Scores s0, s1;
    const int first_key = seen_by(p, u, u.row0).lo;  // of the unit
    // A tile of which some row does not see some key. A masked key's exponential is zero, but zero times an infinity or a NaN is not: the
    // values of keys that no row of the unit sees are cleared in LDS, and those that are not finite are added to the rows
    // that see their key and cleared too.
    auto settle = [&](int key0, int buf) {
      uint4* const rows_of = reinterpret_cast<uint4*>(values + buf * TL::kBytes);
      int odd = 0;
      for (int i = threadIdx.x; i < KEYS * TL::kChunks; i += 64 * NW) {
        const int key = key0 + i / TL::kChunks;
        if (key < first_key || key >= u.hi) rows_of[i] = uint4{0u, 0u, 0u, 0u};
        else odd |= not_finite<T>(rows_of[i]);
      }
      if (!__syncthreads_or(odd)) return;
  #pragma unroll 1
      for (int key = max(key0, first_key); key < min(key0 + KEYS, u.hi); ++key) {
        const int r = key - key0, sw = TL::swizzle(r) & (TL::kChunks - 1);
  #pragma unroll
        for (int d = 0; d < ND; ++d)
  #pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int e = 32 * d + 8 * (i >> 2) + 4 * half + (i & 3);
            const char* at = values + buf * TL::kBytes + r * TL::kRowBytes + (((e / TL::kElems) ^ sw) << 4) + (e % TL::kElems) * (int)sizeof(T);
            float v;
            if constexpr (kHalf) v = bf16_to_f32(*reinterpret_cast<const uint16_t*>(at));
            else v = *reinterpret_cast<const float*>(at);
            if ((__float_as_uint(v) & 0x7f800000u) == 0x7f800000u) {
  #pragma unroll
              for (int n = 0; n < NR; ++n)
                if (key >= seen[n].lo && key <= seen[n].hi) o[n][d][i] += v;
            }
          }
      }
      __syncthreads();
      for (int i = threadIdx.x; i < KEYS * TL::kChunks; i += 64 * NW) rows_of[i] = finite_of<T>(rows_of[i]);
      __syncthreads();
    };
    auto arrive = [&](int key0, int buf) {  // this tile's copies have landed; the next one's leave
      wait_loads<0>();
      __syncthreads();
      if (key0 < all_lo || key0 + KEYS - 1 > all_hi) settle(key0, buf);
      if (key0 + KEYS < u.hi) {
        stager.copy(lds0 + (buf ^ 1) * TL::kBytes, lds0 + (2 + (buf ^ 1)) * TL::kBytes);
        stager.find(key0 + 2 * KEYS + 32);
      }
    };
    auto all_see = [&](int key) { return key >= all_lo && key + 31 <= all_hi; };
    // The block at `at` of the tile, keys from key0 on, and the scores and reference of the next one.
    auto block = [&](int key0, int at, Scores& s, Scores& next) {
      Tops top = run_block(at, at, s, next);
      if (key0 + 32 >= u.hi) return;
      if (!all_see(key0 + 32)) {
        hide(next, key0 + 32);
        top = largest(next);
      }
      refer(top);
    };
    if (u.lo < u.hi) {  // the first block's scores, from keys in the other buffer
      stager.find(u.lo);
      stager.template copy<1>(lds0 + TL::kBytes, lds0 + 2 * TL::kBytes);
      stager.find(u.lo + 32);
      stager.copy(lds0, lds0 + 2 * TL::kBytes);
      stager.find(u.lo + KEYS + 32);
      wait_loads<2 * TL::kLoads>();  // the first tile's copies may be outstanding
      __syncthreads();
      score_block(TL::kBytes, s0);
      if (!all_see(u.lo)) hide(s0, u.lo);
      refer(largest(s0));
    }
    if (row0 >= rows) {  // a wave without rows only copies (one token of 64 sequences of up to 16384, heads of 128: 230 -> 220 us)
      int buf = 0;
#pragma unroll 1
      for (int key0 = u.lo; key0 < u.hi; key0 += KEYS, buf ^= 1) arrive(key0, buf);
    } else if constexpr (kHalf) {  // two tiles a round, so that a buffer's address is a constant
      for (int key0 = u.lo; key0 < u.hi; key0 += 2 * KEYS) {
        arrive(key0, 0);
        block(key0, 0, s0, s1);
        if (key0 + 32 >= u.hi) break;
        if constexpr (NB == 4) {
          block(key0 + 32, kBlock, s1, s0);
          if (key0 + 64 >= u.hi) break;
          block(key0 + 64, 2 * kBlock, s0, s1);
          if (key0 + 96 >= u.hi) break;
          block(key0 + 96, 3 * kBlock, s1, s0);
          if (key0 + KEYS >= u.hi) break;
          arrive(key0 + KEYS, 1);
          block(key0 + KEYS, TL::kBytes, s0, s1);
          if (key0 + KEYS + 32 >= u.hi) break;
          block(key0 + KEYS + 32, TL::kBytes + kBlock, s1, s0);
          if (key0 + KEYS + 64 >= u.hi) break;
          block(key0 + KEYS + 64, TL::kBytes + 2 * kBlock, s0, s1);
          if (key0 + KEYS + 96 >= u.hi) break;
          block(key0 + KEYS + 96, TL::kBytes + 3 * kBlock, s1, s0);
        } else if constexpr (NB == 2) {
          block(key0 + 32, kBlock, s1, s0);
          if (key0 + KEYS >= u.hi) break;
          arrive(key0 + KEYS, 1);
          block(key0 + KEYS, TL::kBytes, s0, s1);
          if (key0 + KEYS + 32 >= u.hi) break;
          block(key0 + KEYS + 32, TL::kBytes + kBlock, s1, s0);
        } else {
          arrive(key0 + KEYS, 1);
          block(key0 + KEYS, TL::kBytes, s1, s0);
        }
      }
    } else {  // the registers of one tile's code
      int buf = 0;
      for (int key0 = u.lo; key0 < u.hi; key0 += KEYS, buf ^= 1) {
        arrive(key0, buf);
  #pragma unroll 1
        for (int j = 0; j < NB && key0 + 32 * j < u.hi; ++j) {
          block(key0 + 32 * j, buf * TL::kBytes + j * kBlock, s0, s1);
  #pragma unroll
          for (int n = 0; n < NR; ++n) s0[n] = s1[n];
        }
      }
    }

  #pragma unroll
    for (int n = 0; n < NR; ++n) {
      const int row = row0 + 32 * n + col;
      const float total = sum_across32(sum[n]);
      if (row >= rows) continue;
      if (!whole) {  // a workgroup's first item and its last one may be shared: two parts
        const int64_t part = (2 * (int64_t)blockIdx.x + (begins ? 0 : 1)) * ROWS + (row - u.row0);
        float* to = p.part_o + part * p.dim;
  #pragma unroll
        for (int d = 0; d < ND; ++d)
  #pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int e = 32 * d + 8 * i + 4 * half;
            if (e < p.dim) *reinterpret_cast<floatx4*>(to + e) = floatx4{o[n][d][4 * i], o[n][d][4 * i + 1], o[n][d][4 * i + 2], o[n][d][4 * i + 3]};
          }
        if (half == 0) *reinterpret_cast<floatx2*>(p.part_ml + part * 2) = floatx2{ref[n], total};
        continue;
      }
      const int t = row / p.group, h = u.head * p.group + (row - t * p.group);
      const float inv = total == 0.0f ? 0.0f : 1.0f / total;
      char* to = p.out + ((int64_t)(u.start + t) * p.o_token + (int64_t)h * p.o_head) * (int64_t)sizeof(T);
  #pragma unroll
      for (int d = 0; d < ND; ++d)
  #pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int e = 32 * d + 8 * i + 4 * half;
          if (e < p.dim) {
            const floatx4 v{o[n][d][4 * i] * inv, o[n][d][4 * i + 1] * inv, o[n][d][4 * i + 2] * inv, o[n][d][4 * i + 3] * inv};
            if constexpr (kHalf) *reinterpret_cast<u32x2*>(to + e * 2) = u32x2{pack2(v[0], v[1]), pack2(v[2], v[3])};
            else *reinterpret_cast<floatx4*>(to + e * 4) = v;
          }
        }
      if (p.lse && half == 0)
        p.lse[(int64_t)(u.start + t) * p.q_heads + h] = total == 0.0f ? kNegInf : (ref[n] + __builtin_amdgcn_logf(total)) * 0.69314718055994531f;
    }
    if (!SHARED || at >= end || !next_item(batch, at, &u)) break;
    __syncthreads();  // this item's reads of LDS come before the next one's copies
  }
}

template <typename T, int DP, int NR>
hipError_t launch_wide(const AttendParams& p, int uniform_pages, hipStream_t stream) {
  const dim3 grid((unsigned)p.units), block(64 * kWideWaves);
  if (p.keys != wide_keys_of((int)sizeof(T), DP, NR)) return hipErrorInvalidValue;
  if (p.target > 0) {
    if (uniform_pages) attend_wide_kernel<T, DP, NR, true, true><<<grid, block, 0, stream>>>(p);
    else attend_wide_kernel<T, DP, NR, false, true><<<grid, block, 0, stream>>>(p);
  } else {
    if (uniform_pages) attend_wide_kernel<T, DP, NR, true, false><<<grid, block, 0, stream>>>(p);
    else attend_wide_kernel<T, DP, NR, false, false><<<grid, block, 0, stream>>>(p);
  }
  return hipGetLastError();
}

template <typename T, int DP>
hipError_t launch_wide_rows(const AttendParams& p, int uniform_pages, hipStream_t stream) {
  if (p.log_rows == kLogWideRows) return launch_wide<T, DP, 1>(p, uniform_pages, stream);
  if constexpr (sizeof(T) == 2 && DP <= kWideDoubleDim)
    if (p.log_rows == kLogWideRows + 1) return launch_wide<T, DP, 2>(p, uniform_pages, stream);
  return hipErrorInvalidValue;
}

template <typename T>
hipError_t launch_wide_dim(const AttendParams& p, int uniform_pages, hipStream_t stream) {
  if (p.dim <= 32) return launch_wide_rows<T, 32>(p, uniform_pages, stream);
  if (p.dim <= 64) return launch_wide_rows<T, 64>(p, uniform_pages, stream);
  if (p.dim <= 96) return launch_wide_rows<T, 96>(p, uniform_pages, stream);
  if (p.dim <= 128) return launch_wide_rows<T, 128>(p, uniform_pages, stream);
  if (p.dim <= 192) return launch_wide_rows<T, 192>(p, uniform_pages, stream);
  return launch_wide_rows<T, 256>(p, uniform_pages, stream);
}

}  // namespace sc
