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

  // Scores of the tile in buffer `buf`, the running reference, and the exponentials in s.
  auto scores = [&](auto masked, int key0, int buf, floatx16(&s)[NS]) {
#pragma unroll
    for (int j = 0; j < NS; ++j) s[j] = floatx16{};
#pragma unroll
    for (int i = 0; i < QF; ++i) {
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
    }
    if constexpr (masked) {
#pragma unroll
      for (int j = 0; j < NS; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int key = key0 + 32 * j + 8 * (r >> 2) + 4 * half + (r & 3);
          s[j][r] = key >= seen.lo && key <= seen.hi ? s[j][r] : kNegInf;
        }
    }
    float top = s[0][0];
#pragma unroll
    for (int j = 0; j < NS; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, s[j][r]);
    top = max_across32(top) * p.scale_log2;
    if (__any(top > ref + kSlack)) {
      const float next = fmaxf(ref, top);
      const float keep = next == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(ref - next);
      ref = next;
      sum *= keep;
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= keep;
    }
    const float base = masked && ref == kNegInf ? 0.0f : ref;
#pragma unroll
    for (int j = 0; j < NS; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[j][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[j][r], p.scale_log2, -base));
        sum += s[j][r];
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

  // A tile whose keys every row sees.
  auto whole_tile = [&](int key0, int buf) {
    floatx16 s[NS];
    scores(std::false_type{}, key0, buf, s);
    if constexpr (kHalf) {
#pragma unroll
      for (int k = 0; k < KEYS / 16; ++k) {
        const bf16x8 pf = exponentials(s[k >> 1], 8 * (k & 1));
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          const u32x2 a = column4(buf, k, 0, d), b = column4(buf, k, 1, d);
          const uint4 w{a[0], a[1], b[0], b[1]};
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w), pf, o[d], 0, 0, 0);
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < NS; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int key = 32 * j + 8 * (r >> 2) + 4 * half + (r & 3);
#pragma unroll
          for (int d = 0; d < ND; ++d) o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(value1(buf, key, d), s[j][r], o[d], 0, 0, 0);
        }
    }
  };

  // A tile of which some row does not see some key. A masked key's exponential is zero, but zero times an infinity or a
  // NaN is not: values of keys that no row of the wave sees are cleared, and those that are not finite leave the product
  // and are added to the rows that see their key.
  auto edge_tile = [&](int key0, int buf) {
    floatx16 s[NS];
    scores(std::true_type{}, key0, buf, s);
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

  Stager<T, TL, NW, UNI> stager(p, u, wave, lane, chunks);
  if (u.lo < u.hi) {
    stager.find(u.lo);
    stager.copy(lds, lds + 2 * TL::kBytes);
    stager.find(u.lo + KEYS);
  }
  auto arrive = [&](int key0, int buf) {  // the tile in `buf` has landed; the next one's copies leave
    wait_loads<0>();
    __syncthreads();
    if (key0 + KEYS < u.hi) {
      stager.copy(lds + (buf ^ 1) * TL::kBytes, lds + (2 + (buf ^ 1)) * TL::kBytes);
      stager.find(key0 + 2 * KEYS);
    }
  };
  auto whole = [&](int key0) { return key0 >= all_lo && key0 + KEYS - 1 <= all_hi && key0 + KEYS <= u.hi; };
  int key0 = u.lo, buf = 0;
  while (key0 < u.hi) {
    // the tiles that all rows see, two a round so that a buffer's address is a constant
    while (buf == 0 && whole(key0) && whole(key0 + KEYS)) {
      arrive(key0, 0);
      whole_tile(key0, 0);
      arrive(key0 + KEYS, 1);
      whole_tile(key0 + KEYS, 1);
      key0 += 2 * KEYS;
    }
    if (key0 >= u.hi) break;
    arrive(key0, buf);
    if (key0 <= any_hi && key0 + KEYS > any_lo) edge_tile(key0, buf);
    key0 += KEYS;
    buf ^= 1;
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
