// Attention over a paged cache in 4 bits (sc_packed.h) for many rows at once, bf16.
//
// The products, the cut and the order of work are those of the float cache's kernel for many rows (sc_attend_wide.h): a workgroup's rows share key
// tiles in LDS, scores and outputs are formed transposed, keys run one block of 32 ahead of values. What differs: a tile's codes come through
// registers, become fp16 values (13 vector operations for 8) and are written to LDS by all waves, each value once for all of the workgroup's
// rows; so workgroups are of eight waves, one a compute unit, and the tile after next is in flight as codes, a quarter of the
// bytes. Queries and exponentials are fp16 as in sc_packed_attend.h. Heads above 128 leave a SIMD one wave. What is small is made to be inlined: the
// program is long enough for the compiler to call it otherwise, with operands in scratch memory.
//
// Bound by the vector unit beside the matrix unit, as there, with the codes' share on top, a tenth: 8192 tokens of two sequences over up to 24576, 16 / 4 heads
// of 128, 1720 to 1840 us by card (the float cache's kernel: 1570), 875 to 936 TFLOP/s; 4096 tokens of 4 sequences over 12288, 8 / 4 heads of 64, 446 to 478 us (409).
#pragma once

#include "sc_attend_wide.h"
#include "sc_packed_attend.h"

#pragma clang fp contract(off)

namespace sc {

// Whether 16 bytes of fp16 values hold one that is not finite; those with it zero.
__device__ __forceinline__ int not_finite_h(uint4 v) {
  const uint32_t mask = 0x7c007c00u, one = 0x04000400u;
  return ((((v.x & mask) + one) | ((v.y & mask) + one) | ((v.z & mask) + one) | ((v.w & mask) + one)) & 0x80008000u) != 0;
}
__device__ __forceinline__ uint4 finite_of_h(uint4 v) {
  int odd;
  return uint4{finite2h(v.x, 0xffffffffu, &odd), finite2h(v.y, 0xffffffffu, &odd), finite2h(v.z, 0xffffffffu, &odd), finite2h(v.w, 0xffffffffu, &odd)};
}

// A thread's share of a tile: groups of rows, keys first (32 keys ahead), then values; their codes and pairs in registers between load() and place().
template <typename TL, int KEYS, int NG, int THREADS>
struct PackedStager {
  static constexpr int kItems = (2 * KEYS * NG + THREADS - 1) / THREADS;
  const PackedAttendParams& p;
  const int b, head, groups, first_key, hi;
  const uint32_t lds0;
  int row[kItems], group[kItems];  // row < 0: none
  bool value[kItems];
  uint4 codes[kItems];
  uint32_t pair[kItems];
  int entry[kItems], slot[kItems];  // of the tile to be loaded next
  const CodeBits bits = code_bits();

  __device__ __forceinline__ PackedStager(const PackedAttendParams& q, const Unit& u, int thread, int g, uint32_t at, int first)
      : p(q), b(u.b), head(u.head), groups(g), first_key(first), hi(u.hi), lds0(at) {
#pragma unroll
    for (int t = 0; t < kItems; ++t) {
      const int i = t * THREADS + thread, r = i / groups;
      value[t] = r >= KEYS;
      row[t] = r < 2 * KEYS ? spread(r & (KEYS - 1)) : -1;
      group[t] = i - r * groups;
    }
  }
  // Rows whose pieces a wave writes together: of each 16 in the order in which the permutation of a row's pieces puts those of one place
  // into other banks (in their own order four rows' met in one, 15 % of a prompt's cycles).
  __device__ __forceinline__ static int spread(int r) {
    if constexpr (TL::kChunks >= 16) return (r & ~15) | ((r & 3) << 2) | ((r >> 2) & 3);
    else if constexpr (TL::kChunks == 8) return (r & ~15) | (r & 1) | ((r & 6) << 1) | ((r & 8) >> 2);
    else return r;
  }
  __device__ __forceinline__ void load_row(int t, uint4* c, uint32_t* s) const {
    const CacheView& v = p.a.c;
    const bool val = value[t];
    const int64_t page = page_of_entry(v, entry[t]), at = slot[t];
    const char* const from = val ? v.v + page * v.v_page + (int64_t)head * v.v_head + at * v.v_slot : v.k + page * v.k_page + (int64_t)head * v.k_head + at * v.k_slot;
    const char* const pairs = val ? p.s.v + page * p.s.v_page + (int64_t)head * p.s.v_head + at * p.s.v_slot
                                  : p.s.k + page * p.s.k_page + (int64_t)head * p.s.k_head + at * p.s.k_slot;
    *c = reinterpret_cast<const uint4*>(from)[group[t]];
    *s = reinterpret_cast<const uint32_t*>(pairs)[group[t]];
  }
  // Looks up the pages of the tile whose values begin at key0 and whose keys `lag` further on.
  __device__ __forceinline__ void find(int key0, int lag = 32) {
#pragma unroll
    for (int t = 0; t < kItems; ++t)
      if (row[t] >= 0) entry[t] = entry_at(p.a.c, b, key0 + row[t] + (value[t] ? 0 : lag), 1, &slot[t]);
  }
  __device__ __forceinline__ void load() {  // the tile that was looked up
#pragma unroll
    for (int t = 0; t < kItems; ++t)
      if (row[t] >= 0) load_row(t, &codes[t], &pair[t]);
  }
  __device__ __forceinline__ void write_row(int r, uint32_t region, int g, const uint4& c, uint32_t s, bool clear) const {
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
    const uint32_t at = lds0 + region + r * TL::kRowBytes, sw = TL::swizzle(r) & (TL::kChunks - 1);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const u32x4_lds v = clear ? u32x4_lds{0u, 0u, 0u, 0u} : __builtin_bit_cast(u32x4_lds, values8(w[i], s, bits));
      *(__attribute__((address_space(3))) u32x4_lds*)(at + (((4 * g + i) ^ sw) << 4)) = v;
    }
  }
  // The tile that was loaded, keys from key0 (+ 32) on, into buffer `buf`. Values of keys that no row sees are zero.
  __device__ __forceinline__ void place(int key0, int buf) const {
#pragma unroll
    for (int t = 0; t < kItems; ++t)
      if (row[t] >= 0) {
        const int key = key0 + row[t];
        write_row(row[t], (value[t] ? 2 + buf : buf) * TL::kBytes, group[t], codes[t], pair[t], value[t] && (key < first_key || key >= hi));
      }
  }
  // The first block's keys, looked up without a lag, into the second buffer.
  __device__ __forceinline__ void first() {
#pragma unroll
    for (int t = 0; t < kItems; ++t)
      if (row[t] >= 0 && row[t] < 32 && !value[t]) {
        uint4 c;
        uint32_t s;
        load_row(t, &c, &s);
        write_row(row[t], TL::kBytes, group[t], c, s, false);
      }
  }
};

// Waves of a workgroup: heads above 128 leave one a SIMD.
constexpr int packed_wide_waves(int dp) { return dp <= 128 ? 8 : 4; }


template <int DP, int NR, bool SHARED>
__global__ void __launch_bounds__(64 * packed_wide_waves(DP), packed_wide_waves(DP) / 4) attend_packed_wide_kernel(PackedAttendParams pp) {
  constexpr int NW = packed_wide_waves(DP), WROWS = 32 * NR, ROWS = WROWS * NW, KEYS = packed_wide_keys(DP);
  constexpr int NB = KEYS / 32, ND = DP / 32;  // blocks of 32 keys of a tile; of 32 dimensions
  using TL = Tile<uint16_t, DP, KEYS, NW, true>;
  constexpr int QF = DP / 16;  // 16-byte pieces of a row that a lane holds
  __shared__ alignas(512) char lds[4 * TL::kBytes];  // keys, values; two buffers
  const AttendParams& p = pp.a;

  const Units batch(p);
  int64_t first_unit = blockIdx.x, end = first_unit + 1;
  if constexpr (SHARED) {
    const Shares shares = shares_of(batch);
    if ((int)blockIdx.x >= shares.n) return;
    first_unit = shares.at(blockIdx.x), end = shares.at(blockIdx.x + 1);
  }
  Unit u;
  if (first_unit >= end || !unit_of(batch, first_unit, &u)) return;
  const int groups = pp.groups;
  if (4 * groups < TL::kChunks) {  // pieces that no group fills: the queries are zero there
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
    // Where registers are short, a fragment's address is formed from one of three: a row is aligned to its length, so that a piece is bits of it
    // (heads of 256, 8192 tokens of two sequences: 2765 -> 1618 us; heads of 64, two blocks of rows: 645 -> 634; of 128 it would cost 2 %).
    constexpr bool kForm = DP > 128 || NR == 2;
    static_assert((TL::kRowBytes & (TL::kRowBytes - 1)) == 0 && TL::kRowBytes <= 512, "the tile's alignment");
    uint32_t kat[kForm ? 1 : QF], vat[2][kForm ? 1 : ND];
#pragma unroll
    for (int i = 0; i < (kForm ? 1 : QF); ++i) kat[i] = lds0 + col * TL::kRowBytes + (((2 * i + half) ^ (TL::swizzle(col) & (TL::kChunks - 1))) << 4);
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int d = 0; d < (kForm ? 1 : ND); ++d)
        vat[e][d] = lds0 + 2 * TL::kBytes + (8 * e + vr) * TL::kRowBytes + (((4 * d + vc) ^ (TL::swizzle(8 * e + vr) & (TL::kChunks - 1))) << 4) + (lane & 1) * 8;

    const int rows = u.n * p.group;
    const int row0 = u.row0 + WROWS * wave;

    // the rows' queries, scaled by a power of two into fp16 and in the keys' order of elements: lane `half` holds the eights that its k indexes
    // of the products stand for
    half8 qf[NR][QF];
    Seen seen[NR];
    float factor[NR];  // of a score, to powers of two
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      const int r = min(row0 + 32 * n + col, rows - 1), t = r / p.group, h = u.head * p.group + (r - t * p.group);
      const char* q = p.q + ((int64_t)(u.start + t) * p.q_token + (int64_t)h * p.q_head) * 2;
      uint4 raw[QF];
      float most = 0.0f;
#pragma unroll
      for (int i = 0; i < QF; ++i) {
        const int c = 2 * i + half;
        raw[i] = c * 8 < p.dim ? *reinterpret_cast<const uint4*>(q + c * 16) : uint4{0u, 0u, 0u, 0u};
        const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) most = fmaxf(most, fmaxf(fabsf(__uint_as_float(w[e] << 16)), fabsf(__uint_as_float(w[e] & 0xffff0000u))));
      }
      most = max_across32(most);
      const int lift = lift_of(most);
      factor[n] = factor_of(p.scale_log2, lift);
#pragma unroll
      for (int i = 0; i < QF; ++i) {
        const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
        float x[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[2 * e] = ldexpf(__uint_as_float(w[e] << 16), lift), x[2 * e + 1] = ldexpf(__uint_as_float(w[e] & 0xffff0000u), lift);
        qf[n][i] = __builtin_bit_cast(half8, uint4{pack2h(x[0], x[4]), pack2h(x[1], x[5]), pack2h(x[2], x[6]), pack2h(x[3], x[7])});
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
    auto key_piece = [&](int i, int at) __attribute__((always_inline)) {  // 16 bytes of a key's row: the score products' operand
      const uint32_t from = kForm ? kat[0] ^ (uint32_t)(i << 5) : kat[kForm ? 0 : i];
      return *(__attribute__((address_space(3))) const u32x4_lds*)(from + at);
    };
    auto value_piece = [&](int k, int d, int at) __attribute__((always_inline)) {  // 8 keys' values of a dimension: the value products' operand
      // rows 16 keys on keep the permutation, which repeats every 16 rows
      const uint32_t piece = kForm ? (uint32_t)(d << 6) : 0u;
      const u32x2 a = read_column4((vat[0][kForm ? 0 : d] ^ piece) + at + 16 * k * TL::kRowBytes), b = read_column4((vat[1][kForm ? 0 : d] ^ piece) + at + 16 * k * TL::kRowBytes);
      return u32x4_lds{a[0], a[1], b[0], b[1]};
    };
    using Scores = floatx16[NR];
    auto score_block = [&](int at, Scores& s) __attribute__((always_inline)) {  // the scores of the 32 keys at `at`
#pragma unroll
      for (int n = 0; n < NR; ++n) s[n] = floatx16{};
#pragma unroll
      for (int i = 0; i < QF; ++i) {
        const u32x4_lds kf = key_piece(i, at);
#pragma unroll
        for (int n = 0; n < NR; ++n) {
          s[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, kf), qf[n][i], s[n], 0, 0, 0);
        }
      }
    };
    struct Tops {
      float at[NR];
    };
    auto largest = [](const Scores& s) __attribute__((always_inline)) {
      Tops top;
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        top.at[n] = s[n][0];
#pragma unroll
        for (int r = 1; r < 16; ++r) top.at[n] = fmaxf(top.at[n], s[n][r]);
      }
      return top;
    };
    auto key_of = [&](int r) __attribute__((always_inline)) { return 8 * (r >> 2) + 4 * half + (r & 3); };  // of a block, that score r of a lane belongs to
    auto hide = [&](Scores& s, int key0) __attribute__((always_inline)) {
#pragma unroll
      for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[n][r] = key0 + key_of(r) >= seen[n].lo && key0 + key_of(r) <= seen[n].hi ? s[n][r] : kNegInf;
    };
    auto refer = [&](Tops top) __attribute__((always_inline)) {  // takes the largest score of the next block into the reference
      bool past = false;
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        top.at[n] = max_across32(top.at[n]) * factor[n];
        past = past || top.at[n] > ref[n] + kSlack;
      }
      if (__any(past)) {
#pragma unroll
        for (int n = 0; n < NR; ++n) {
          const float next = fmaxf(ref[n], top.at[n]);
          const float keep = ref[n] == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(ref[n] - next);  // 1: nothing to rescale yet
          ref[n] = next;
          base[n] = next == kNegInf ? 0.0f : next - kPackedLift;
          sum[n] *= keep;
#pragma unroll
          for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[n][d][r] *= keep;
        }
      }
    };
    auto exponent = [&](float x, int n) __attribute__((always_inline)) { return __builtin_amdgcn_exp2f(__builtin_fmaf(x, factor[n], -base[n])); };

    // A block's exponentials and values, and the scores of the next one (keys at `kt`, values at `vt`).
    auto run_block = [&](int kt, int vt, Scores& s, Scores& next) __attribute__((always_inline)) {
      {
        if constexpr (kForm) kat[0] = here(kat[0]), vat[0][0] = here(vat[0][0]), vat[1][0] = here(vat[1][0]);  // no addresses from one block to the next
        // Laid out by hand: each slot is one fragment's products, with the LDS reads of the one PRE slots later and a share of the
        // vector unit's work (this block's exponentials, then the next one's largest score) to run beside it.
        using PL = SlotPlan<QF, ND>;
        constexpr int PRE = 3, kAll = NR * 16;
        u32x4_lds frag[PL::kSlots];
        uint32_t packed[NR][8];
        auto read = [&](auto slot) __attribute__((always_inline)) {
          constexpr int m = slot;
          if constexpr (m < PL::kSlots) {
            constexpr int x = PL::kOrder.at[m];
            if constexpr (x < QF) frag[m] = key_piece(x, kt);
            else frag[m] = value_piece((x - QF) / ND, (x - QF) % ND, vt);
          }
        };
        auto form = [&](auto from, auto to) __attribute__((always_inline)) {  // exponentials [from, to) of the lane, in pairs: a half's keys, row block by row block
          constexpr int f = from, t = to;
#pragma unroll
          for (int e = f; e < t; e += 2) {
            const int n = e / 8 % NR, r = e / (8 * NR) * 8 + e % 8;
            const float a = exponent(s[n][r], n), b = exponent(s[n][r + 1], n);
            sum[n] += a;
            sum[n] += b;
            packed[n][r / 2] = pack2h(a, b);
          }
        };
        Tops top;
#pragma unroll
        for (int n = 0; n < NR; ++n) top.at[n] = kNegInf, next[n] = floatx16{};
        unrolled<PRE>([&](auto m) __attribute__((always_inline)) { read(m); });
        form(std::integral_constant<int, 0>{}, std::integral_constant<int, PL::exps_by(-1, kAll)>{});
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);  // ahead of the other workgroup's wave, which is then in its copies, waits and reference
        unrolled<PL::kSlots>([&](auto slot) __attribute__((always_inline)) {
          constexpr int m = slot, x = PL::kOrder.at[m];
          read(std::integral_constant<int, m + PRE>{});
#pragma unroll
          for (int n = 0; n < NR; ++n) {
            if constexpr (x < QF) {
              next[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, frag[m]), qf[n][x], next[n], 0, 0, 0);
            } else {
              constexpr int k = (x - QF) / ND, d = (x - QF) % ND;
              const uint4 w{packed[n][4 * k], packed[n][4 * k + 1], packed[n][4 * k + 2], packed[n][4 * k + 3]};
              o[n][d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, frag[m]), __builtin_bit_cast(half8, w), o[n][d], 0, 0, 0);
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
      }
    };

    // Keys run one block ahead of values: with the values of tile i (keys i * KEYS ..) come the keys 32 further on, both in buffer i & 1.
    constexpr int kBlock = 32 * TL::kRowBytes;
    char* const values = lds + 2 * TL::kBytes;
    const int first_key = seen_by(p, u, u.row0).lo;  // of the unit
    PackedStager<TL, KEYS, DP / 32, 64 * NW> stager(pp, u, thread, groups, lds0, first_key);
    Scores s0, s1;
    // A tile of which some row does not see some key. A masked key's exponential is zero, but zero times an infinity or a NaN is not: the
    // values of keys that no row of the unit sees are zero in LDS already, and those that are not finite are added to the rows
    // that see their key and cleared too.
    auto settle = [&](int key0, int buf) __attribute__((always_inline)) {
      uint4* const rows_of = reinterpret_cast<uint4*>(values + buf * TL::kBytes);
      int odd = 0;
      for (int i = threadIdx.x; i < KEYS * TL::kChunks; i += 64 * NW) odd |= not_finite_h(rows_of[i]);
      if (!__syncthreads_or(odd)) return;
#pragma unroll 1
      for (int key = max(key0, first_key); key < min(key0 + KEYS, u.hi); ++key) {
        const int r = key - key0, sw = TL::swizzle(r) & (TL::kChunks - 1);
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int e = 32 * d + 8 * (i >> 2) + 4 * half + (i & 3);
            const char* at = values + buf * TL::kBytes + r * TL::kRowBytes + (((e / 8) ^ sw) << 4) + (e % 8) * 2;
            const float v = (float)*reinterpret_cast<const _Float16*>(at);
            if ((__float_as_uint(v) & 0x7f800000u) == 0x7f800000u) {
#pragma unroll
              for (int n = 0; n < NR; ++n)
                if (key >= seen[n].lo && key <= seen[n].hi) o[n][d][i] += v;
            }
          }
      }
      __syncthreads();
      for (int i = threadIdx.x; i < KEYS * TL::kChunks; i += 64 * NW) rows_of[i] = finite_of_h(rows_of[i]);
      __syncthreads();
    };
    auto arrive = [&](int key0, int buf) __attribute__((always_inline)) {  // this tile is in LDS; the other buffers are free
      __syncthreads();
      if (key0 < all_lo || key0 + KEYS - 1 > all_hi) settle(key0, buf);
    };
    // The next tile's codes become values in LDS, and those of the one after it leave memory. Half of the waves do so at a tile's begin, the others
    // in its middle, so that a SIMD's matrix unit has one wave's products meanwhile.
    const bool early = wave < NW / 2;
    auto stage = [&](int key0, int buf) __attribute__((always_inline)) {
      if (key0 + KEYS >= u.hi) return;
      stager.place(key0 + KEYS, buf ^ 1);
      if (key0 + 2 * KEYS >= u.hi) return;
      stager.load();
      stager.find(key0 + 3 * KEYS);
    };
    auto all_see = [&](int key) __attribute__((always_inline)) { return key >= all_lo && key + 31 <= all_hi; };
    // The block at `at` of the tile, keys from key0 on, and the scores and reference of the next one.
    auto block = [&](int key0, int at, Scores& s, Scores& next) __attribute__((always_inline)) {
      Tops top = run_block(at, at, s, next);
      if (key0 + 32 >= u.hi) return;
      if (!all_see(key0 + 32)) {
        hide(next, key0 + 32);
        top = largest(next);
      }
      refer(top);
    };
    if (u.lo < u.hi) {  // the first block's scores, from keys in the other buffer
      stager.find(u.lo, 0);
      stager.first();
      stager.find(u.lo);
      stager.load();
      stager.find(u.lo + KEYS);
      stager.place(u.lo, 0);
      stager.load();
      stager.find(u.lo + 2 * KEYS);
      __syncthreads();
      if (row0 < rows) {
        score_block(TL::kBytes, s0);
        if (!all_see(u.lo)) hide(s0, u.lo);
        refer(largest(s0));
      }
    }
    if (row0 >= rows) {  // a wave without rows only stages
      int buf = 0;
#pragma unroll 1
      for (int key0 = u.lo; key0 < u.hi; key0 += KEYS, buf ^= 1) {
        arrive(key0, buf);
        stage(key0, buf);
      }
    } else {  // two tiles a round, so that a buffer's address is a constant
      for (int key0 = u.lo; key0 < u.hi; key0 += 2 * KEYS) {
        arrive(key0, 0);
        if (early) stage(key0, 0);
        block(key0, 0, s0, s1);
        if constexpr (NB == 4) {
          if (key0 + 32 < u.hi) block(key0 + 32, kBlock, s1, s0);
          if (!early) stage(key0, 0);
          if (key0 + 64 < u.hi) block(key0 + 64, 2 * kBlock, s0, s1);
          if (key0 + 96 < u.hi) block(key0 + 96, 3 * kBlock, s1, s0);
          if (key0 + KEYS >= u.hi) break;
          arrive(key0 + KEYS, 1);
          if (early) stage(key0 + KEYS, 1);
          block(key0 + KEYS, TL::kBytes, s0, s1);
          if (key0 + KEYS + 32 < u.hi) block(key0 + KEYS + 32, TL::kBytes + kBlock, s1, s0);
          if (!early) stage(key0 + KEYS, 1);
          if (key0 + KEYS + 64 < u.hi) block(key0 + KEYS + 64, TL::kBytes + 2 * kBlock, s0, s1);
          if (key0 + KEYS + 96 < u.hi) block(key0 + KEYS + 96, TL::kBytes + 3 * kBlock, s1, s0);
        } else {
          if (!early) stage(key0, 0);
          if (key0 + 32 < u.hi) block(key0 + 32, kBlock, s1, s0);
          if (key0 + KEYS >= u.hi) break;
          arrive(key0 + KEYS, 1);
          if (early) stage(key0 + KEYS, 1);
          block(key0 + KEYS, TL::kBytes, s0, s1);
          if (!early) stage(key0 + KEYS, 1);
          if (key0 + KEYS + 32 < u.hi) block(key0 + KEYS + 32, TL::kBytes + kBlock, s1, s0);
        }
      }
    }

#pragma unroll
    for (int n = 0; n < NR; ++n) {
      const int row = row0 + 32 * n + col;
      const float total = sum_across32(sum[n]), top = ref[n] == kNegInf ? kNegInf : ref[n] - kPackedLift;
      // from the order 0 4 1 5 | 2 6 3 7 of eight elements in a row's two lanes to 0 1 2 3 | 4 5 6 7
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(o[n][d][4 * i]), __float_as_uint(o[n][d][4 * i + 1]), false, false);
          const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(o[n][d][4 * i + 2]), __float_as_uint(o[n][d][4 * i + 3]), false, false);
          o[n][d][4 * i] = __uint_as_float(a[0]), o[n][d][4 * i + 1] = __uint_as_float(b[0]);
          o[n][d][4 * i + 2] = __uint_as_float(a[1]), o[n][d][4 * i + 3] = __uint_as_float(b[1]);
        }
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
        if (half == 0) *reinterpret_cast<floatx2*>(p.part_ml + part * 2) = floatx2{top, total};
        continue;
      }
      const int t = row / p.group, h = u.head * p.group + (row - t * p.group);
      const float inv = total == 0.0f ? 0.0f : 1.0f / total;
      char* to = p.out + ((int64_t)(u.start + t) * p.o_token + (int64_t)h * p.o_head) * 2;
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int e = 32 * d + 8 * i + 4 * half;
          if (e < p.dim) {
            const floatx4 v{o[n][d][4 * i] * inv, o[n][d][4 * i + 1] * inv, o[n][d][4 * i + 2] * inv, o[n][d][4 * i + 3] * inv};
            *reinterpret_cast<u32x2*>(to + e * 2) = u32x2{pack2(v[0], v[1]), pack2(v[2], v[3])};
          }
        }
      if (p.lse && half == 0)
        p.lse[(int64_t)(u.start + t) * p.q_heads + h] = total == 0.0f ? kNegInf : (top + __builtin_amdgcn_logf(total)) * 0.69314718055994531f;
    }
    if (!SHARED || at >= end || !next_item(batch, at, &u)) break;
    __syncthreads();  // this item's reads of LDS come before the next one's copies
  }
}

template <int DP, int NR>
hipError_t launch_packed_wide(const PackedAttendParams& p, hipStream_t stream) {
  const dim3 grid((unsigned)p.a.units), block(64 * packed_wide_waves(DP));
  if (p.a.keys != packed_wide_keys(DP) || (1 << p.a.log_rows) != 32 * NR * packed_wide_waves(DP)) return hipErrorInvalidValue;
  if constexpr (NR == 1) {
    if (p.a.target > 0) {
      attend_packed_wide_kernel<DP, NR, true><<<grid, block, 0, stream>>>(p);
      return hipGetLastError();
    }
  }
  if (p.a.target > 0) return hipErrorInvalidValue;  // two blocks of rows are taken where they fill the GPU: nothing is shared
  attend_packed_wide_kernel<DP, NR, false><<<grid, block, 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace sc
