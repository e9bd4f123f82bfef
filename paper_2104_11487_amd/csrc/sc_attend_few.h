// Attention over the paged cache for few rows of a key head (the next token of each sequence, or a few of them) or brief keys:
// the cache's bytes bound it where those are many, the launch and the loads' latency where they are not. Measured: fp32 heads of 32,
// one token of 103 sequences over 7959: 92 us, 4.6 TB/s; bf16 heads of 64, one token over 777 keys: 9.8 us.
//
// One workgroup a compute unit. Where no item has keys for more than four tiles a wave it takes one item; otherwise each takes an
// equal share of all the key tiles of the launch, from wherever in an item its share begins to wherever in a later one it ends, so that
// sequences of all lengths end together. For the keys of one item, each wave
// walks key tiles of its own (every n-th) with its own buffers in LDS and its own running reference and sum, so the loop has no barrier:
// while a tile is in the products the next one's copies are in flight, and the copies after that leave as soon as its buffer is
// free. At the item's end the waves' outputs are joined in LDS, in wave order; an item that several workgroups shared is joined by a
// second launch, in the order of its keys.
// Products as in the wide kernel (sc_attend_wide.h), transposed, on 16 x 16 tiles: 16 rows a unit. A second row block in the same wave
// (NB) reads keys once for 32 rows but doubles the registers and the vector work behind each tile; two units side by side find the
// second reading in the caches (bf16 heads of 64, 4 tokens of 8 rows over 12000: 33 us with two blocks, 25 with one), so it is
// left to fp32 heads of up to 96 over brief keys, where it saves rounds of workgroups. The build for fp32 heads above 192 keeps 66 registers in scratch
// memory (one token of 16 sequences over 4000, 4 heads of 256: 274 us, of 128: 86).
#pragma once

#include <type_traits>

#include "sc_attend_tile.h"

#pragma clang fp contract(off)

namespace sc {

constexpr float kFewSlack = 8.0f;  // powers of two that an exponential may exceed one by

// Waves of a workgroup: their buffers take 128 KB of LDS.
template <typename T, int DP>
constexpr int few_waves() {
  constexpr int row = pow2_at_least(DP * (int)sizeof(T)), tile = row * (sizeof(T) == 2 ? 32 : 16);
  return tile * 4 * 8 <= 131072 ? 8 : 131072 / (tile * 4);
}

template <typename T, int DP, int NB>
__global__ void __launch_bounds__((64 * few_waves<T, DP>())) attend_few_kernel(AttendParams p) {
  constexpr bool kHalf = sizeof(T) == 2;
  constexpr int NW = few_waves<T, DP>(), KEYS = kHalf ? 32 : 16, ROWS = 16 * NB;
  constexpr int NS = KEYS / 16, ND = DP / 16;
  using TL = Tile<T, DP, KEYS, 1, false>;
  constexpr int QF = TL::kElems * 4 > DP ? 1 : DP / (4 * TL::kElems);  // 16-byte pieces of a row that a lane holds
  constexpr int JP = DP + 4;                                           // joining: a row's stride in LDS, in floats
  constexpr int kWaveBytes = 4 * TL::kBytes + 512;                     // two buffers of keys and values, of page numbers
  constexpr int kBuffers = NW * kWaveBytes, kJoin = NW * ROWS * (JP + 2) * 4;
  __shared__ alignas(16) char lds[kBuffers > kJoin ? kBuffers : kJoin];

  const Units batch(p);
  const Shares shares = shares_of(batch);
  if ((int)blockIdx.x >= shares.n) return;
  const int64_t end = shares.at(blockIdx.x + 1);
  const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6);
  const int col = lane & 15, quad = lane >> 4, chunks = p.dim / TL::kElems;
  char* mine = lds + wave * kWaveBytes;
  const uint32_t mine_at = (uint32_t)(uintptr_t)SC_LDS(lds, char) + wave * kWaveBytes;

  const int64_t first_unit = shares.at(blockIdx.x);
  Unit u;
  if (first_unit >= end || !unit_of(batch, first_unit, &u)) return;
  for (int64_t at = first_unit;;) {
    const int units = (int)min(end - at, (int64_t)(u.parts - u.part));  // of this item
    const bool whole = units == u.parts, begins = at == first_unit;
    at += units;
    u.hi = (int)min((int64_t)u.hi, u.lo + (int64_t)units * u.chunk);
    const int rows = u.n * p.group;

    if (chunks < TL::kChunks) {  // chunks that no copy fills: those past the head's dimension
      for (int i = lane; i < 4 * TL::kBytes / 16; i += 64) reinterpret_cast<uint4*>(mine)[i] = uint4{0u, 0u, 0u, 0u};
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }

    constexpr int kStep = KEYS * NW;
    const int begin = u.lo + wave * KEYS;
    const int count = begin < u.hi ? (u.hi - begin + kStep - 1) / kStep : 0;  // tiles of this wave
    // Page numbers are looked up three tiles ahead, copies run two tiles ahead.
    const LoneStager<T, TL, KEYS> stager(p, u, lane, chunks);
    const char* const entries = mine + 4 * TL::kBytes;
    const uint32_t entries_at = mine_at + 4 * TL::kBytes;
    if (count > 0) {
      stager.find(begin, entries_at);
      if (count > 1) stager.find(begin + kStep, entries_at + 256);
      wait_loads<0>();
      stager.copy(begin, entries, mine_at, mine_at + TL::kBytes);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (count > 2) stager.find(begin + 2 * kStep, entries_at);
      if (count > 1) stager.copy(begin + kStep, entries + 256, mine_at + 2 * TL::kBytes, mine_at + 3 * TL::kBytes);
    }

    // the rows' queries, in the operand's layout
    uint4 qf[NB][QF];
    Seen seen[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const int r = min(u.row0 + 16 * n + col, rows - 1), t = r / p.group, h = u.head * p.group + (r - t * p.group);
      const char* q = p.q + ((int64_t)(u.start + t) * p.q_token + (int64_t)h * p.q_head) * (int64_t)sizeof(T);
#pragma unroll
      for (int i = 0; i < QF; ++i) {
        const int c = 4 * i + quad;
        qf[n][i] = c < chunks ? *reinterpret_cast<const uint4*>(q + c * 16) : uint4{0u, 0u, 0u, 0u};
      }
      seen[n] = seen_by(p, u, u.row0 + 16 * n + col);
    }
    const Seen first = seen_by(p, u, u.row0), last = seen_by(p, u, u.row0 + ROWS - 1);
    const int all_lo = last.lo, all_hi = first.hi, any_lo = first.lo, any_hi = last.hi;

    floatx4 o[NB][ND];
    float ref[NB], sum[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      ref[n] = kNegInf, sum[n] = 0.0f;
#pragma unroll
      for (int d = 0; d < ND; ++d) o[n][d] = floatx4{};
    }

    const int krow = TL::swizzle(col) & (TL::kChunks - 1);
    const int vr = 4 * quad + (col >> 2), vc = (col & 3) >> 1;

    // One tile's work. edge: some row does not see some of its keys.
    auto tile = [&](auto edge_, int key0, const char* kt, const char* vt) {
      constexpr bool edge = edge_;
      floatx4 s[NB][NS];
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int j = 0; j < NS; ++j) s[n][j] = floatx4{};
#pragma unroll
      for (int i = 0; i < QF; ++i)
#pragma unroll
        for (int j = 0; j < NS; ++j) {
          const uint4 kf = *reinterpret_cast<const uint4*>(kt + (16 * j + col) * TL::kRowBytes + (((4 * i + quad) ^ krow) << 4));
#pragma unroll
          for (int n = 0; n < NB; ++n) {
            if constexpr (kHalf) {
              s[n][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf), __builtin_bit_cast(bf16x8, qf[n][i]), s[n][j], 0, 0, 0);
            } else {
              const floatx4 a = __builtin_bit_cast(floatx4, kf), b = __builtin_bit_cast(floatx4, qf[n][i]);
#pragma unroll
              for (int e = 0; e < 4; ++e) s[n][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], s[n][j], 0, 0, 0);
            }
          }
        }
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        if constexpr (edge) {
#pragma unroll
          for (int j = 0; j < NS; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int key = key0 + 16 * j + 4 * quad + r;
              s[n][j][r] = key >= seen[n].lo && key <= seen[n].hi ? s[n][j][r] : kNegInf;
            }
        }
        float top = s[n][0][0];
#pragma unroll
        for (int j = 0; j < NS; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) top = fmaxf(top, s[n][j][r]);
        top = max_across32(max_across16(top)) * p.scale_log2;
        if (__any(top > ref[n] + kFewSlack)) {
          const float to = fmaxf(ref[n], top);
          const float keep = to == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(ref[n] - to);
          ref[n] = to;
          sum[n] *= keep;
#pragma unroll
          for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int r = 0; r < 4; ++r) o[n][d][r] *= keep;
        }
        const float base = ref[n] == kNegInf ? 0.0f : ref[n];
#pragma unroll
        for (int j = 0; j < NS; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            s[n][j][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n][j][r], p.scale_log2, -base));
            sum[n] += s[n][j][r];
          }
      }
      // Values. Where some row does not see some key, a masked key's exponential is zero, but zero times an infinity or a
      // NaN is not: values of keys that no row sees are cleared, and those that are not finite leave the product and
      // are added to the rows that see their key.
      int odd = 0;
      if constexpr (kHalf) {
        bf16x8 pf[NB];
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          const uint4 w{pack2(s[n][0][0], s[n][0][1]), pack2(s[n][0][2], s[n][0][3]), pack2(s[n][NS - 1][0], s[n][NS - 1][1]),
                        pack2(s[n][NS - 1][2], s[n][NS - 1][3])};
          pf[n] = __builtin_bit_cast(bf16x8, w);
        }
        uint32_t mask[2][2];
        if constexpr (edge) {
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int key = key0 + 16 * e + 4 * quad + 2 * i;
              mask[e][i] = (key >= any_lo && key <= any_hi ? 0xffffu : 0u) | (key + 1 >= any_lo && key + 1 <= any_hi ? 0xffff0000u : 0u);
            }
        }
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          u32x2 q[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int r = 16 * e + vr, c = (2 * d + vc) ^ (TL::swizzle(r) & (TL::kChunks - 1));
            q[e] = read_column4(vt + r * TL::kRowBytes + c * 16 + (lane & 1) * 8);
            if constexpr (edge) {
              q[e][0] = finite2(q[e][0], mask[e][0], &odd);
              q[e][1] = finite2(q[e][1], mask[e][1], &odd);
            }
          }
          const uint4 a{q[0][0], q[0][1], q[1][0], q[1][1]};
#pragma unroll
          for (int n = 0; n < NB; ++n) o[n][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), pf[n], o[n][d], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int key = 4 * quad + r;
          const bool keep = key0 + key >= any_lo && key0 + key <= any_hi;
#pragma unroll
          for (int d = 0; d < ND; ++d) {
            const int e = 16 * d + col, c = (e >> 2) ^ (TL::swizzle(key) & (TL::kChunks - 1));
            float a = *reinterpret_cast<const float*>(vt + key * TL::kRowBytes + c * 16 + (e & 3) * 4);
            if constexpr (edge) a = finite1(a, keep, &odd);
#pragma unroll
            for (int n = 0; n < NB; ++n) o[n][d] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, s[n][0][r], o[n][d], 0, 0, 0);
          }
        }
      }
      if (edge && __any(odd)) {
        const int from = max(key0, any_lo), to = min(key0 + KEYS - 1, any_hi);
        for (int key = from; key <= to; ++key) {
          const int r = key - key0, sw = TL::swizzle(r) & (TL::kChunks - 1);
#pragma unroll
          for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int e = 16 * d + 4 * quad + i;
              const char* at = vt + r * TL::kRowBytes + (((e / TL::kElems) ^ sw) << 4) + (e % TL::kElems) * (int)sizeof(T);
              float v;
              if constexpr (kHalf) v = bf16_to_f32(*reinterpret_cast<const uint16_t*>(at));
              else v = *reinterpret_cast<const float*>(at);
              if ((__float_as_uint(v) & 0x7f800000u) == 0x7f800000u) {
#pragma unroll
                for (int n = 0; n < NB; ++n)
                  if (key >= seen[n].lo && key <= seen[n].hi) o[n][d][i] += v;
              }
            }
        }
      }
    };

    for (int it = 0; it < count; ++it) {
      const int key0 = begin + it * kStep;
      const int tile_at = (it & 1) * 2 * TL::kBytes;
      const char* const kt = mine + tile_at;
      const char* const vt = kt + TL::kBytes;
      if (it + 1 < count) wait_loads<LoneStager<T, TL, KEYS>::kOps>();  // the younger tile's copies stay in flight
      else wait_loads<0>();
      if (key0 >= all_lo && key0 + KEYS - 1 <= all_hi) tile(std::false_type{}, key0, kt, vt);
      else tile(std::true_type{}, key0, kt, vt);
      // this tile's buffers are free: the fragments read from them have reached their products
      if (it + 2 < count) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (it + 3 < count) stager.find(key0 + 3 * kStep, entries_at + ((it + 1) & 1) * 256);
        stager.copy(key0 + 2 * kStep, entries + (it & 1) * 256, mine_at + tile_at, mine_at + tile_at + TL::kBytes);
      }
    }

    // Join the waves (every copy has landed: the last tile waited for all of them).
    __syncthreads();
    float* joined = reinterpret_cast<float*>(lds);           // [wave][row][JP]
    float* stats = joined + NW * ROWS * JP;                  // [wave][row][2]
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      sum[n] = sum_across32(sum_across16(sum[n]));
      const int r = wave * ROWS + 16 * n + col;
#pragma unroll
      for (int d = 0; d < ND; ++d) *reinterpret_cast<floatx4*>(joined + r * JP + 16 * d + 4 * quad) = o[n][d];
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
        const int t = row / p.group, h = u.head * p.group + (row - t * p.group);
        const float inv = total == 0.0f ? 0.0f : 1.0f / total;
        char* to = p.out + ((int64_t)(u.start + t) * p.o_token + (int64_t)h * p.o_head) * (int64_t)sizeof(T);
        if constexpr (kHalf) *reinterpret_cast<u32x2*>(to + e * 2) = u32x2{pack2(v[0] * inv, v[1] * inv), pack2(v[2] * inv, v[3] * inv)};
        else *reinterpret_cast<floatx4*>(to + e * 4) = floatx4{v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv};
        if (p.lse && e == 0)
          p.lse[(int64_t)(u.start + t) * p.q_heads + h] = total == 0.0f ? kNegInf : (top + __builtin_amdgcn_logf(total)) * 0.69314718055994531f;
      }
    }
    if (at >= end || !next_item(batch, at, &u)) break;
    __syncthreads();  // the join's reads come before the next item's copies
  }
}

template <typename T, int DP>
hipError_t launch_few(const AttendParams& p, hipStream_t stream) {
  const dim3 grid((unsigned)p.units), block(64 * few_waves<T, DP>());
  if (p.keys != few_keys_of((int)sizeof(T))) return hipErrorInvalidValue;
  if (p.log_rows == kLogFewRows) {
    attend_few_kernel<T, DP, 1><<<grid, block, 0, stream>>>(p);
    return hipGetLastError();
  }
  if constexpr (sizeof(T) == 4 && DP <= kFewDoubleDim) {
    if (p.log_rows == kLogFewRows + 1) {
      attend_few_kernel<T, DP, 2><<<grid, block, 0, stream>>>(p);
      return hipGetLastError();
    }
  }
  return hipErrorInvalidValue;
}

template <typename T>
hipError_t launch_few_dim(const AttendParams& p, hipStream_t stream) {
  if (p.dim <= 32) return launch_few<T, 32>(p, stream);
  if (p.dim <= 64) return launch_few<T, 64>(p, stream);
  if constexpr (sizeof(T) == 4) {
    if (p.dim <= 96) return launch_few<T, 96>(p, stream);
    if (p.dim <= 128) return launch_few<T, 128>(p, stream);
    if (p.dim <= 192) return launch_few<T, 192>(p, stream);
    return launch_few<T, 256>(p, stream);
  }
  return hipErrorInvalidValue;
}

}  // namespace sc
