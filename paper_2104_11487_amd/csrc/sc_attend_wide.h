// Attention over the paged cache for many rows at once (new tokens x query heads of a key head).
//
//   o = sum_l exp(s_l - m) v_l / sum_l exp(s_l - m),   s_l = scale q . k_l,   over the keys l that the row sees
//
// in one pass over the keys with a running reference m and sum. A workgroup of 4 waves takes 128 rows, 32 of them a wave,
// and walks the keys in tiles that all waves share, the next tile's copies into LDS in flight during this one's products.
// Products are formed transposed: scores S' = K Q' have a row's scores in two lanes (l and l + 32), so softmax needs one
// lane exchange a tile, and O' = V' P' takes the exponentials from the registers that the scores left them in: the key that
// a k index of the product stands for is free, as long as V's fragment follows, so no lane exchange and no LDS is needed for P.
// Scores, exponentials' sums and outputs are fp32. For bf16 caches the exponentials are rounded to bf16 for the
// product with V (the matrix unit's operand type: up to 2^-8 of each, averaged over the keys); their sum takes them unrounded.
// The reference m is the largest score seen only up to 2^8: a row's output and sum are rescaled when a score passes it by
// more, which after the first tiles is seldom.
#pragma once

#include <type_traits>
#include <utility>

#include "sc_attend_tile.h"

#pragma clang fp contract(off)

namespace sc {

// Keys of a tile: two buffers of keys and values take 64 KB where the head allows 32 rows or more of it.
template <typename T, int DP>
constexpr int wide_keys() {
  return pow2_at_least(DP * (int)sizeof(T)) >= 512 ? 32 : 64;
}

constexpr int kWideWaves = 4;
constexpr float kSlack = 8.0f;  // powers of two that an exponential may exceed one by

// f(0), f(1), ... f(N - 1), each with its index as a constant.
template <int... I, typename F>
__device__ __forceinline__ void unrolled_(std::integer_sequence<int, I...>, F f) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void unrolled(F f) {
  unrolled_(std::make_integer_sequence<int, N>{}, f);
}

// Order of a tile's products: NQ of the next tile's scores (0 ..), and for each 16 of its NK * 16 keys ND of its values
// (NQ + k * ND ..). A value product needs its keys' exponentials, the largest score needs all score products: half of the scores
// (three quarters where there are but two key groups) come first, the rest between the value products.
template <int NQ, int ND, int NK>
struct SlotPlan {
  static constexpr int kSlots = NQ + NK * ND;
  struct Order {
    int at[kSlots];
    int last_score;
  };
  static constexpr Order order() {
    Order o = {};
    int n = 0, q = 0, upto = NK > 2 ? NQ / 2 : NQ * 3 / 4;
    for (int k = 0; k <= NK; ++k) {
      if (k == NK - 1) upto = NQ;
      while (q < upto) o.last_score = n, o.at[n++] = q++;
      if (k < NK)
        for (int d = 0; d < ND; ++d) o.at[n++] = NQ + k * ND + d;
      upto += (NQ - NQ / 2) / (NK > 2 ? NK - 2 : 1);
      if (upto > NQ) upto = NQ;
    }
    return o;
  }
  static constexpr Order kOrder = order();
  // Exponentials formed by the end of slot n (even; -1: before the first): evenly until the last score product, but in time
  // for the first value product of each key group.
  static constexpr int exps_by(int n, int all) {
    const int until = kOrder.last_score + 1;
    int e = (n + 2) * all / (until + 1);
    e = (e + 1) / 2 * 2;
    if (e > all) e = all;
    for (int m = 0; m <= n + 1 && m < kSlots; ++m)
      if (kOrder.at[m] >= NQ && e < ((kOrder.at[m] - NQ) / ND + 1) * (all / NK)) e = ((kOrder.at[m] - NQ) / ND + 1) * (all / NK);
    return e;
  }
  // Scores of the next tile whose largest is known by the end of slot n: those after the last score product, in the slots behind it.
  static constexpr int tops_by(int n, int all) {
    const int from = kOrder.last_score + 2;
    if (n >= kSlots - 1) return all;
    if (n < from) return 0;
    return (n - from + 1) * all / (kSlots - from) / 2 * 2;
  }
};

template <typename T, int DP, bool UNI>
__global__ void __launch_bounds__(64 * kWideWaves, (DP * (int)sizeof(T) <= 256 ? 2 : 1)) attend_wide_kernel(AttendParams p) {
  constexpr bool kHalf = sizeof(T) == 2;
  constexpr int NW = kWideWaves, ROWS = 32 * NW, KEYS = wide_keys<T, DP>();
  constexpr int NS = KEYS / 32, ND = DP / 32;
  using TL = Tile<T, DP, KEYS, NW, true>;
  constexpr int QF = kHalf ? DP / 16 : DP / 8;  // 16-byte pieces of a row that a lane holds
  __shared__ char lds[4 * TL::kBytes];          // keys, values; two buffers

  Unit u;
  if (!unit_of(p, (int)blockIdx.x, &u)) return;
  const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int rows = u.n * p.group;
  const int row0 = u.row0 + 32 * wave, row = row0 + col;
  const int chunks = p.dim / TL::kElems;

  // the row's queries: lane `half` holds the dimensions that its k indexes of the products stand for
  uint4 qf[QF];
  {
    const int r = min(row, rows - 1), t = r / p.group, h = u.head * p.group + (r - t * p.group);
    const char* q = p.q + ((int64_t)(u.start + t) * p.q_token + (int64_t)h * p.q_head) * (int64_t)sizeof(T);
#pragma unroll
    for (int i = 0; i < QF; ++i) {
      const int c = 2 * i + half;
      qf[i] = c < chunks ? *reinterpret_cast<const uint4*>(q + c * 16) : uint4{0u, 0u, 0u, 0u};
    }
  }
  // chunks that no copy fills: those past the head's dimension
  if (chunks < TL::kChunks) {
    for (int i = threadIdx.x; i < 4 * TL::kBytes / 16; i += 64 * NW) reinterpret_cast<uint4*>(lds)[i] = uint4{0u, 0u, 0u, 0u};
    __syncthreads();
  }

  const Seen seen = seen_by(p, u, row);
  // keys that every row of the unit sees are [all_lo, all_hi]; that a row of the wave sees, [any_lo, any_hi]
  const int all_lo = seen_by(p, u, u.row0 + ROWS - 1).lo, all_hi = seen_by(p, u, u.row0).hi;
  const int any_lo = seen_by(p, u, row0).lo, any_hi = row0 < rows ? seen_by(p, u, row0 + 31).hi : -1;

  floatx16 o[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) o[d] = floatx16{};
  float ref = kNegInf, sum = 0.0f;

  // scores: row (key) col of a 32-key block, 16-byte piece 2 i + half; values: see read_column4
  const int krow = TL::swizzle(col) & (TL::kChunks - 1);
  const int vr = 4 * half + ((lane & 15) >> 2), vc = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
  const char* kbase = lds + col * TL::kRowBytes;
  const char* vbase = lds + 2 * TL::kBytes + vr * TL::kRowBytes + (lane & 1) * 8;

  auto score_step = [&](int i, int buf, floatx16(&s)[NS]) {  // 16 (fp32: 8) dimensions of the scores of the keys in `buf`
#pragma unroll
    for (int j = 0; j < NS; ++j) {
      const uint4 kf = *reinterpret_cast<const uint4*>(kbase + (((2 * i + half) ^ krow) << 4) + buf * TL::kBytes + j * 32 * TL::kRowBytes);
      if constexpr (kHalf) {
        s[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf), __builtin_bit_cast(bf16x8, qf[i]), s[j], 0, 0, 0);
      } else {
        const floatx4 a = __builtin_bit_cast(floatx4, kf), b = __builtin_bit_cast(floatx4, qf[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[j] = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], s[j], 0, 0, 0);
      }
    }
  };
  auto clear = [](floatx16(&s)[NS]) {
#pragma unroll
    for (int j = 0; j < NS; ++j) s[j] = floatx16{};
  };
  auto largest = [](const floatx16(&s)[NS]) {
    float top = s[0][0];
#pragma unroll
    for (int j = 0; j < NS; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, s[j][r]);
    return top;
  };
  auto hide = [&](floatx16(&s)[NS], int key0) {
#pragma unroll
    for (int j = 0; j < NS; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int key = key0 + 32 * j + 8 * (r >> 2) + 4 * half + (r & 3);
        s[j][r] = key >= seen.lo && key <= seen.hi ? s[j][r] : kNegInf;
      }
  };
  float base = 0.0f;  // what exponents are taken relative to: the reference, or 0 before there is one
  auto refer = [&](float top) {  // takes the largest score of the next tile into the reference
    top = max_across32(top) * p.scale_log2;
    if (__any(top > ref + kSlack)) {
      const float next = fmaxf(ref, top);
      const float keep = next == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(ref - next);
      ref = next;
      base = ref == kNegInf ? 0.0f : ref;
      sum *= keep;
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= keep;
    }
  };
  auto exponent = [&](floatx16& x, int from, int n) {  // scores to exponentials
#pragma unroll
    for (int r = from; r < from + n; ++r) {
      x[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r], p.scale_log2, -base));
      sum += x[r];
    }
  };
  auto exponentials = [](const floatx16& x, int r) {  // eight of them as the product's operand
    const uint4 w{pack2(x[r], x[r + 1]), pack2(x[r + 2], x[r + 3]), pack2(x[r + 4], x[r + 5]), pack2(x[r + 6], x[r + 7])};
    return __builtin_bit_cast(bf16x8, w);
  };
  auto column4 = [&](int buf, int k, int e, int d) {
    const int c = (4 * d + vc) ^ (TL::swizzle(8 * e + vr + 16 * k) & (TL::kChunks - 1));
    return read_column4(vbase + c * 16 + buf * TL::kBytes + (16 * k + 8 * e) * TL::kRowBytes);
  };
  auto value1 = [&](int buf, int key, int d) {
    const int e = 32 * d + col, c = (e >> 2) ^ (TL::swizzle(key) & (TL::kChunks - 1));
    return *reinterpret_cast<const float*>(lds + (2 + buf) * TL::kBytes + key * TL::kRowBytes + c * 16 + (e & 3) * 4);
  };

  auto value_step = [&](int k, int buf, const floatx16(&s)[NS]) {  // the values of 16 keys
    if constexpr (kHalf) {
      const bf16x8 pf = exponentials(s[k >> 1], 8 * (k & 1));
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        const u32x2 a = column4(buf, k, 0, d), b = column4(buf, k, 1, d);
        const uint4 w{a[0], a[1], b[0], b[1]};
        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w), pf, o[d], 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int r = 8 * (k & 1) + i, key = 32 * (k >> 1) + 8 * (r >> 2) + 4 * half + (r & 3);
#pragma unroll
        for (int d = 0; d < ND; ++d) o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(value1(buf, key, d), s[k >> 1][r], o[d], 0, 0, 0);
      }
    }
  };

  // A tile whose keys every row sees, and the scores of the next one, laid out by hand: each slot is one product, with the LDS
  // reads of the one PRE slots later and a share of the vector unit's work (this tile's exponentials, then the next
  // tile's largest score) to run beside it.
  auto whole_tile_half = [&](int buf, floatx16(&s)[NS], floatx16(&next)[NS]) {
    using PL = SlotPlan<QF * NS, ND, KEYS / 16>;
    constexpr int PRE = 3, kExps = 16 * NS;
    uint4 frag[PL::kSlots];
    uint32_t packed[kExps / 2];
    auto read = [&](auto slot) {
      constexpr int n = slot;
      if constexpr (n < PL::kSlots) {
        constexpr int x = PL::kOrder.at[n];
        if constexpr (x < QF * NS) {
          constexpr int i = x / NS, j = x % NS;
          frag[n] = *reinterpret_cast<const uint4*>(kbase + (((2 * i + half) ^ krow) << 4) + (buf ^ 1) * TL::kBytes + j * 32 * TL::kRowBytes);
        } else {
          constexpr int k = (x - QF * NS) / ND, d = (x - QF * NS) % ND;
          const u32x2 a = column4(buf, k, 0, d), b = column4(buf, k, 1, d);
          frag[n] = uint4{a[0], a[1], b[0], b[1]};
        }
      }
    };
    auto form = [&](auto from, auto to) {  // exponentials [from, to) of the lane, in pairs
      constexpr int f = from, t = to;
#pragma unroll
      for (int e = f; e < t; e += 2) {
        floatx16& x = s[e / 16];
        const float u0 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e % 16], p.scale_log2, -base));
        const float u1 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e % 16 + 1], p.scale_log2, -base));
        sum += u0;
        sum += u1;
        packed[e / 2] = pack2(u0, u1);
      }
    };
    float top = kNegInf;
    clear(next);
    unrolled<PRE>([&](auto n) { read(n); });
    form(std::integral_constant<int, 0>{}, std::integral_constant<int, PL::exps_by(-1, kExps)>{});
    __builtin_amdgcn_sched_barrier(0);
    unrolled<PL::kSlots>([&](auto slot) {
      constexpr int n = slot, x = PL::kOrder.at[n];
      read(std::integral_constant<int, n + PRE>{});
      if constexpr (x < QF * NS) {
        constexpr int i = x / NS, j = x % NS;
        next[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, frag[n]), __builtin_bit_cast(bf16x8, qf[i]), next[j], 0, 0, 0);
      } else {
        constexpr int k = (x - QF * NS) / ND, d = (x - QF * NS) % ND;
        const uint4 w{packed[4 * k], packed[4 * k + 1], packed[4 * k + 2], packed[4 * k + 3]};
        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, frag[n]), __builtin_bit_cast(bf16x8, w), o[d], 0, 0, 0);
      }
      form(std::integral_constant<int, PL::exps_by(n - 1, kExps)>{}, std::integral_constant<int, PL::exps_by(n, kExps)>{});
      constexpr int f = PL::tops_by(n - 1, kExps), t = PL::tops_by(n, kExps);
#pragma unroll
      for (int e = f; e < t; e += 2) top = fmaxf(fmaxf(next[e / 16][e % 16], next[e / 16][e % 16 + 1]), top);
      __builtin_amdgcn_sched_barrier(0);
    });
    return top;
  };

  auto whole_tile_single = [&](int buf, floatx16(&s)[NS], floatx16(&next)[NS]) {
    clear(next);
#pragma unroll
    for (int k = 0; k < KEYS / 16; ++k) {
      exponent(s[k >> 1], 8 * (k & 1), 8);
#pragma unroll
      for (int i = 0; i < QF; ++i)
        if (i * (KEYS / 16) / QF == k) score_step(i, buf ^ 1, next);
      if (k > 0) value_step(k - 1, buf, s);
    }
    value_step(KEYS / 16 - 1, buf, s);
    return largest(next);
  };
  auto whole_tile = [&](int buf, floatx16(&s)[NS], floatx16(&next)[NS]) {
    if constexpr (kHalf) return whole_tile_half(buf, s, next);
    else return whole_tile_single(buf, s, next);
  };

  // A tile of which some row does not see some key. A masked key's exponential is zero, but zero times an infinity or a
  // NaN is not: values of keys that no row of the wave sees are cleared, and those that are not finite leave the product
  // and are added to the rows that see their key.
  auto edge_tile = [&](int key0, int buf, floatx16(&s)[NS]) {
#pragma unroll
    for (int j = 0; j < NS; ++j) exponent(s[j], 0, 16);
    int odd = 0;
    if constexpr (kHalf) {
#pragma unroll
      for (int k = 0; k < KEYS / 16; ++k) {
        const bf16x8 pf = exponentials(s[k >> 1], 8 * (k & 1));
        uint32_t mask[2][2];
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int key = key0 + 16 * k + 8 * e + 4 * half + 2 * i;
            mask[e][i] = (key >= any_lo && key <= any_hi ? 0xffffu : 0u) | (key + 1 >= any_lo && key + 1 <= any_hi ? 0xffff0000u : 0u);
          }
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          u32x2 a = column4(buf, k, 0, d), b = column4(buf, k, 1, d);
          const uint4 w{finite2(a[0], mask[0][0], &odd), finite2(a[1], mask[0][1], &odd), finite2(b[0], mask[1][0], &odd),
                        finite2(b[1], mask[1][1], &odd)};
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w), pf, o[d], 0, 0, 0);
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < NS; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int key = 32 * j + 8 * (r >> 2) + 4 * half + (r & 3);
          const bool keep = key0 + key >= any_lo && key0 + key <= any_hi;
#pragma unroll
          for (int d = 0; d < ND; ++d)
            o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(finite1(value1(buf, key, d), keep, &odd), s[j][r], o[d], 0, 0, 0);
        }
    }
    if (__any(odd)) {
      const int from = max(key0, any_lo), to = min(key0 + KEYS - 1, any_hi);
      for (int key = from; key <= to; ++key) {
        const bool sees = key >= seen.lo && key <= seen.hi;
        const int r = key - key0, sw = TL::swizzle(r) & (TL::kChunks - 1);
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int e = 32 * d + 8 * (i >> 2) + 4 * half + (i & 3);
            const char* at = lds + (2 + buf) * TL::kBytes + r * TL::kRowBytes + (((e / TL::kElems) ^ sw) << 4) + (e % TL::kElems) * (int)sizeof(T);
            float v;
            if constexpr (kHalf) v = bf16_to_f32(*reinterpret_cast<const uint16_t*>(at));
            else v = *reinterpret_cast<const float*>(at);
            if (sees && (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u) o[d][i] += v;
          }
      }
    }
  };

  // Copies: the keys of tile i are in buffer i & 1 while tile i - 1 is worked on, its values while it is worked on itself.
  char* const keys = lds;
  char* const values = lds + 2 * TL::kBytes;
  Stager<T, TL, NW, UNI, KEYS> stager(p, u, wave, lane, chunks);
  floatx16 s0[NS], s1[NS];
  auto whole = [&](int key0) { return key0 >= all_lo && key0 + KEYS - 1 <= all_hi && key0 + KEYS <= u.hi; };
  auto arrive = [&](int key0, int buf) {  // the values of this tile and the keys of the next have landed; the copies after them leave
    wait_loads<0>();
    __syncthreads();
    if (key0 + KEYS < u.hi) {
      stager.copy(keys + buf * TL::kBytes, values + (buf ^ 1) * TL::kBytes);
      stager.find(key0 + 3 * KEYS);
    }
  };
  if (u.lo < u.hi) {
    stager.find(u.lo);
    stager.template copy<1>(keys, values);
    stager.find(u.lo + KEYS);
    stager.copy(keys + TL::kBytes, values);
    stager.find(u.lo + 2 * KEYS);
    wait_loads<2 * TL::kLoads>();  // the copies of the second tile's keys may be outstanding
    __syncthreads();
    clear(s0);
#pragma unroll
    for (int i = 0; i < QF; ++i) score_step(i, 0, s0);
    if (!whole(u.lo)) hide(s0, u.lo);
    refer(largest(s0));
  }
  int key0 = u.lo, buf = 0;
  while (key0 < u.hi) {
    // two a round, so that a buffer's address is a constant
    while (buf == 0 && whole(key0) && whole(key0 + KEYS) && key0 + 2 * KEYS < u.hi) {
      arrive(key0, 0);
      refer(whole_tile(0, s0, s1));
      arrive(key0 + KEYS, 1);
      float top = whole_tile(1, s1, s0);
      key0 += 2 * KEYS;
      if (!whole(key0)) {
        hide(s0, key0);
        top = largest(s0);
      }
      refer(top);
    }
    arrive(key0, buf);
    const bool more = key0 + KEYS < u.hi;
    clear(s1);
    if (more) {
#pragma unroll
      for (int i = 0; i < QF; ++i) score_step(i, buf ^ 1, s1);
    }
    if (key0 <= any_hi && key0 + KEYS > any_lo) edge_tile(key0, buf, s0);
    key0 += KEYS;
    buf ^= 1;
    if (more) {
      if (!whole(key0)) hide(s1, key0);
      refer(largest(s1));
#pragma unroll
      for (int j = 0; j < NS; ++j) s0[j] = s1[j];
    }
  }

  sum = sum_across32(sum);
  if (row >= rows) return;
  if (u.splits > 1) {
    const int64_t at = (int64_t)blockIdx.x * ROWS + (row - u.row0);
    float* to = p.part_o + at * p.dim;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int e = 32 * d + 8 * i + 4 * half;
        if (e < p.dim) *reinterpret_cast<floatx4*>(to + e) = floatx4{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
      }
    if (half == 0) *reinterpret_cast<floatx2*>(p.part_ml + at * 2) = floatx2{ref, sum};
    return;
  }
  const int t = row / p.group, h = u.head * p.group + (row - t * p.group);
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  char* to = p.out + ((int64_t)(u.start + t) * p.o_token + (int64_t)h * p.o_head) * (int64_t)sizeof(T);
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = 32 * d + 8 * i + 4 * half;
      if (e < p.dim) {
        const floatx4 v{o[d][4 * i] * inv, o[d][4 * i + 1] * inv, o[d][4 * i + 2] * inv, o[d][4 * i + 3] * inv};
        if constexpr (kHalf) *reinterpret_cast<u32x2*>(to + e * 2) = u32x2{pack2(v[0], v[1]), pack2(v[2], v[3])};
        else *reinterpret_cast<floatx4*>(to + e * 4) = v;
      }
    }
  if (p.lse && half == 0)
    p.lse[(int64_t)(u.start + t) * p.q_heads + h] = sum == 0.0f ? kNegInf : (ref + __builtin_amdgcn_logf(sum)) * 0.69314718055994531f;
}

template <typename T, int DP>
hipError_t launch_wide(const AttendParams& p, int uniform_pages, hipStream_t stream) {
  if (p.keys != wide_keys<T, DP>() || p.log_rows != kLogWideRows) return hipErrorInvalidValue;
  const dim3 grid((unsigned)p.units), block(64 * kWideWaves);
  if (uniform_pages) attend_wide_kernel<T, DP, true><<<grid, block, 0, stream>>>(p);
  else attend_wide_kernel<T, DP, false><<<grid, block, 0, stream>>>(p);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_wide_dim(const AttendParams& p, int uniform_pages, hipStream_t stream) {
  if (p.dim <= 32) return launch_wide<T, 32>(p, uniform_pages, stream);
  if (p.dim <= 64) return launch_wide<T, 64>(p, uniform_pages, stream);
  if (p.dim <= 96) return launch_wide<T, 96>(p, uniform_pages, stream);
  if (p.dim <= 128) return launch_wide<T, 128>(p, uniform_pages, stream);
  if (p.dim <= 192) return launch_wide<T, 192>(p, uniform_pages, stream);
  return launch_wide<T, 256>(p, uniform_pages, stream);
}

}  // namespace sc
