// Appending to the cache in 4 bits, with the rotation on the way, and reading its values back.
//
// Per token, key head and group of 32 elements, on the elements x in fp32 (keys: turned in 64 bits and rounded once):
//   y = clamp(x, +-32768), low = fl16(min y), scale = fl16(max(0, (max y - low) / 15)), code = clamp(rint((y - low) / scale), 0, 15)
// (scale 0: code 0). A group with an element that is not finite has scale and minimum NaN, so that it reads as NaN. All operations round to
// nearest, ties to even. The turn is formed in 64 bits because a code changes where (y - low) / scale passes a half: so a code depends on the
// inputs alone, not on how the call was cut. Queries turn as skipconv_rotate's.
//
// Four lanes hold a group, a word of eight codes each; a workgroup takes up to eight tokens, whose sines and cosines all heads share. Many
// tokens: 4 x 4096 of 8 + 4 + 4 heads of 64 28 us, 2 TB/s, bound neither by memory nor by the vector unit (two 64-bit products and sums an element, a
// division where a quotient is near a half), which is busy for 47 % of the time: waves wait for half of theirs, for the loads of the first round and the
// sines and cosines, and at each round's barrier, which queries that turn in place need. 32 tokens 8 us, a chain of latencies. Reading back is bound by memory: 16 x 8192 tokens of 4 heads of 128, 352 MB, in 82 us, 4.3 TB/s.
#include "sc_packed_device.h"
#include "sc_stream.h"

#include <algorithm>
#include <type_traits>

#pragma clang fp contract(off)

namespace sc {

namespace {

constexpr int kThreads = 256;
constexpr int kMostTokens = 8;  // of a workgroup

// Eight elements of a head as they lie in memory, those past `dim` zero. WIDE: 16-byte loads.
template <typename T>
struct Chunk {
  static constexpr int kWords = 2 * (int)sizeof(T);
  uint32_t w[kWords];
  __device__ __forceinline__ void widen(float* x) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (sizeof(T) == 4) x[i] = __uint_as_float(w[i]);
      else x[i] = __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    }
  }
  __device__ __forceinline__ void set(int i, T v) {
    if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(v);
    else w[i / 2] = i & 1 ? w[i / 2] | (uint32_t)v << 16 : (uint32_t)v;
  }
};
template <typename T, bool WIDE>
__device__ __forceinline__ Chunk<T> load_chunk(const T* head, int d, int dim) {
  Chunk<T> c = {};
  if (d < dim) {
    if constexpr (WIDE) {
#pragma unroll
      for (int i = 0; i < Chunk<T>::kWords; i += 4) {
        const uint4 v = *reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(head + d) + 4 * i);
        c.w[i] = v.x, c.w[i + 1] = v.y, c.w[i + 2] = v.z, c.w[i + 3] = v.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) c.set(i, head[d + i]);
    }
  }
  return c;
}

// Cosine and sine of an angle, in 64 bits for keys and rounded to 32 for queries.
struct Turn {
  double c, s;
  floatx2 rounded;
};

// The code of x >= low: rint((x - low) / scale) within 0..15. The quotient by a reciprocal is off by less than 2^-17 (up to 23 steps, reciprocal
// within one unit, product and difference rounded); only where that could take it over a half is the division made.
struct Codes {
  float low, scale, inverse;
  __device__ __forceinline__ uint32_t of(const float* x) const {
    float q[8];
    bool near = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      q[i] = (x[i] - low) * inverse;
      near = near || fabsf(fabsf(q[i] - rintf(q[i])) - 0.5f) < 1.0f / 65536.0f;
    }
    if (__any(near)) {
#pragma unroll 1
      for (int i = 0; i < 8; ++i) {
        float v = x[0];
#pragma unroll
        for (int k = 1; k < 8; ++k) v = i == k ? x[k] : v;
        const float exact = __fdiv_rn(v - low, scale);
#pragma unroll
        for (int k = 0; k < 8; ++k) q[k] = i == k ? exact : q[k];
      }
    }
    // four codes side by side are a number below 2^16, which fp32 holds exactly
    float half[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      half[k] = 0.0f;
#pragma unroll
      for (int i = 3; i >= 0; --i) half[k] = __builtin_fmaf(half[k], 16.0f, __builtin_amdgcn_fmed3f(rintf(q[4 * k + i]), 0.0f, 15.0f));
    }
    return (uint32_t)half[0] | (uint32_t)half[1] << 16;
  }
};

// Where a token's rows of keys, values and their pairs begin, from the first head's on.
struct Rows {
  int64_t k, v, ks, vs;
};

// MODE: the turn: 0 pairs of halves, whole chunks of them; 1 neighbours, likewise; 2 any.
template <typename T, bool WIDE, int MODE>
__global__ void __launch_bounds__(kThreads) pack_kernel(PackParams pp) {
  const RotateParams& p = pp.r;
  extern __shared__ char lds[];
  Turn* turn = reinterpret_cast<Turn*>(lds);  // [token][pair]
  __shared__ int where[kMostTokens];          // [token]: 0 a row of no sequence, 1 one without a place, 2 one in the cache
  __shared__ Rows rows[kMostTokens];
  const int t0 = (int)blockIdx.x * pp.tok_per_wg, nt = min(pp.tok_per_wg, p.tokens - t0);
  const int lane = threadIdx.x & 63;
  const int words = (p.dim + kPackGroup - 1) / kPackGroup * 4;  // of a head
  const int heads = p.heads[0] + 2 * p.heads[1], each = kThreads / words, all = nt * heads;
  const int mine = qdiv((int)threadIdx.x, __builtin_amdgcn_rcpf((float)words)), word = (int)threadIdx.x - mine * words, d = word * 8;
  const float inv_heads = __builtin_amdgcn_rcpf((float)heads);

  // Whole heads at a time: all of one is loaded before any of it is stored. A round's loads go out a round ahead, the first ones before all else.
  struct Item {
    Chunk<T> own, other;  // the lane's eight elements, and their partners
    int tk, h, which;
    bool live;
  };
  const auto load = [&](int h0) {
    Item m;
    const int at = h0 + mine;
    m.live = mine < each && at < all;
    m.tk = m.live ? qdiv(at, inv_heads) : 0, m.h = at - m.tk * heads, m.which = 0;
    if (m.h >= p.heads[0]) m.h -= p.heads[0], m.which = 1;
    if (m.which == 1 && m.h >= p.heads[1]) m.h -= p.heads[1], m.which = 2;
    if (m.live) {
      const T* const src = reinterpret_cast<const T*>(p.src[m.which]) + (int64_t)(t0 + m.tk) * p.src_token[m.which] + (int64_t)m.h * p.src_head[m.which];
      m.own = load_chunk<T, WIDE>(src, d, p.dim);
      if (MODE != 1 && p.freq && m.which < 2 && !p.adjacent && d < 2 * p.pairs) {
        if constexpr (MODE == 0) {
          m.other = load_chunk<T, WIDE>(src, d < p.pairs ? d + p.pairs : d - p.pairs, p.dim);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int e = min(d + i, 2 * p.pairs - 1);
            m.other.set(i, src[e < p.pairs ? e + p.pairs : e - p.pairs]);
          }
        }
      }
    }
    return m;
  };
  Item next = load(0);

  for (int t = uniform((int)threadIdx.x >> 6); t < nt; t += kThreads / 64) {
    const int s = owner_of(p.cache.row_start, p.cache.batch, t0 + t);
    int page = -1, slot = 0, found = 0;
    if (s < p.cache.batch) {
      const Sequence q = sequence_of(p.cache, s);
      const int at = p.cache.kv_len[s] - q.n + (t0 + t - q.start);
      found = 1;
      if (t0 + t >= q.start && at >= 0 && page_of(p.cache, at) < p.cache.width) {
        const int i = page_of(p.cache, at), got = p.cache.table[(int64_t)s * p.cache.width + i];
        slot = at - i * p.cache.page_size;
        if (got >= 0 && got < p.cache.pages) page = got, found = 2;
      }
    }
    if (lane == 0) {
      where[t] = found;
      rows[t] = Rows{page * p.cache.k_page + slot * p.cache.k_slot, page * p.cache.v_page + slot * p.cache.v_slot,
                     page * pp.s.k_page + slot * pp.s.k_slot, page * pp.s.v_page + slot * pp.s.v_slot};
    }
  }
  if (p.freq) {
    const float inv_pairs = __builtin_amdgcn_rcpf((float)p.pairs);
    for (int i = threadIdx.x; i < nt * p.pairs; i += kThreads) {
      const int t = qdiv(i, inv_pairs), j = i - t * p.pairs;
      double angle = 0.0;
      for (int a = 0; a < p.axes; ++a) angle += (double)p.pos[(int64_t)(t0 + t) * p.axes + a] * (double)p.freq[a * p.pairs + j];
      double turns = angle * 0.15915494309189533577;  // 1 / (2 pi)
      turns -= rint(turns);
      double c, s;
      sincospi(2.0 * turns, &s, &c);
      s = p.sign < 0.0f ? -s : s;
      turn[i] = Turn{c, s, floatx2{(float)c, (float)s}};
    }
  }
  __syncthreads();

  const auto turn_chunk = [&](float* x, const float* y, int tk, auto wide_) {
    using F = std::conditional_t<decltype(wide_)::value, double, float>;
    const Turn* const tt = turn + tk * p.pairs;
    const auto get = [&](int pair, F* c, F* s) {
      if constexpr (decltype(wide_)::value) *c = tt[pair].c, *s = tt[pair].s;
      else *c = tt[pair].rounded.x, *s = tt[pair].rounded.y;
    };
    if (MODE == 1 || (MODE == 2 && p.adjacent)) {
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        F c, s;
        get(MODE == 2 ? min((d + i) >> 1, p.pairs - 1) : (d + i) >> 1, &c, &s);
        const F u = x[i], w = x[i + 1];
        const float a = (float)(u * c - w * s), b = (float)(w * c + u * s);
        if (MODE != 2 || d + i < 2 * p.pairs) x[i] = a, x[i + 1] = b;
      }
    } else if constexpr (MODE == 0) {
      const bool second = d >= p.pairs;
      const Turn* const from = tt + (second ? d - p.pairs : d);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const Turn& t = from[i];
        const F c = decltype(wide_)::value ? (F)t.c : (F)t.rounded.x, s = decltype(wide_)::value ? (F)t.s : (F)t.rounded.y;
        x[i] = (float)((F)x[i] * c + (F)y[i] * (second ? s : -s));
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int e = d + i;
        F c, s;
        get(min(e >= p.pairs ? e - p.pairs : e, p.pairs - 1), &c, &s);
        const float a = (float)((F)x[i] * c + (F)y[i] * (e >= p.pairs ? s : -s));
        if (e < 2 * p.pairs) x[i] = a;
      }
    }
  };

  for (int h0 = 0; h0 < all; h0 += each) {
    const Item now = next;
    if (h0 + each < all) next = load(h0 + each);
    const int tk = now.tk, h = now.h, which = now.which;
    const bool live = now.live && where[tk] >= (which == 0 ? 1 : 2);
    float x[8], y[8];
    now.own.widen(x);
    if (live && p.freq && which < 2 && d < 2 * p.pairs) {
      now.other.widen(y);
      if (which == 0) turn_chunk(x, y, tk, std::false_type{});
      else turn_chunk(x, y, tk, std::true_type{});
    }
    __syncthreads();  // queries may turn in place
    if (live && which == 0) {
      if (d >= p.dim) continue;
      T* dst = reinterpret_cast<T*>(p.dst) + (int64_t)(t0 + tk) * p.dst_token + (int64_t)h * p.dst_head + d;
      if constexpr (WIDE) {
        if constexpr (sizeof(T) == 2) {
          *reinterpret_cast<uint4*>(dst) = uint4{pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7])};
        } else {
          reinterpret_cast<floatx4*>(dst)[0] = floatx4{x[0], x[1], x[2], x[3]};
          reinterpret_cast<floatx4*>(dst)[1] = floatx4{x[4], x[5], x[6], x[7]};
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if constexpr (sizeof(T) == 2) dst[i] = (uint16_t)(pack2(x[i], x[i]) & 0xffffu);
          else dst[i] = x[i];
      }
    } else if (live) {
      // of the lane's elements (all eight are of the head, or none: heads are multiples of 8), then of the group's four lanes
      float low = -kNegInf, high = kNegInf;
      int odd = 0;
      const bool some = d < p.dim;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        odd |= (__float_as_uint(x[i]) & 0x7f800000u) == 0x7f800000u;
        x[i] = __builtin_amdgcn_fmed3f(x[i], -kPackMost, kPackMost);
        low = fminf(low, x[i]), high = fmaxf(high, x[i]);
      }
      low = some ? low : -kNegInf, high = some ? high : kNegInf;
#pragma unroll
      for (int m = 1; m < 4; m <<= 1) {
        low = fminf(low, __shfl_xor(low, m)), high = fmaxf(high, __shfl_xor(high, m));
        odd |= __shfl_xor(odd, m);
      }
      const _Float16 low16 = (_Float16)low;
      const float base = (float)low16;
      const _Float16 scale16 = (_Float16)fmaxf(__fdiv_rn(high - base, 15.0f), 0.0f);
      const float scale = (float)scale16;
      uint32_t codes = Codes{base, scale, __builtin_amdgcn_rcpf(scale)}.of(x);
      if (odd || !some || scale == 0.0f) codes = 0;
      char* const row = which == 1 ? p.cache.k + rows[tk].k + h * p.cache.k_head : p.cache.v + rows[tk].v + h * p.cache.v_head;
      reinterpret_cast<uint32_t*>(row)[word] = codes;
      if ((word & 3) == 0) {
        char* const pairs = which == 1 ? pp.s.k + rows[tk].ks + h * pp.s.k_head : pp.s.v + rows[tk].vs + h * pp.s.v_head;
        reinterpret_cast<uint32_t*>(pairs)[word >> 2] = odd ? 0x7e007e00u : bits_of(half2{scale16, low16});
      }
    }
  }
}

template <typename T>
hipError_t launch_pack_type(PackParams p, bool wide, hipStream_t stream) {
  // Tokens of a workgroup: as many as leave it four rounds or fewer, but fewer while the launch has under 1024 workgroups.
  const int words = pack_groups(p.r.dim) * 4, heads = p.r.heads[0] + 2 * p.r.heads[1];
  const int round = kThreads / words;
  p.tok_per_wg = std::max(1, std::min(kMostTokens, 4 * round / heads));
  while (p.tok_per_wg > 1 && (p.r.tokens + p.tok_per_wg - 1) / p.tok_per_wg < 1024) --p.tok_per_wg;
  const unsigned grid = (unsigned)((p.r.tokens + p.tok_per_wg - 1) / p.tok_per_wg);
  const size_t lds = p.r.freq ? (size_t)p.tok_per_wg * p.r.pairs * sizeof(Turn) : 0;
  const int mode = !p.r.freq ? 0 : p.r.adjacent ? (p.r.pairs % 4 == 0 ? 1 : 2) : p.r.pairs % 8 == 0 ? 0 : 2;
  const dim3 block(kThreads);
  if (!wide) pack_kernel<T, false, 2><<<dim3(grid), block, lds, stream>>>(p);
  else if (mode == 0) pack_kernel<T, true, 0><<<dim3(grid), block, lds, stream>>>(p);
  else if (mode == 1) pack_kernel<T, true, 1><<<dim3(grid), block, lds, stream>>>(p);
  else pack_kernel<T, true, 2><<<dim3(grid), block, lds, stream>>>(p);
  return hipGetLastError();
}

// A thread makes eight values of a row: out[which][entry][head][slot][8 word ..].
__global__ void __launch_bounds__(kThreads) unpack_kernel(UnpackParams p, int words, int64_t items) {
  const int64_t rows = (int64_t)p.kv_heads * p.c.page_size;
  const CodeBits bits = code_bits();
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < items; i += (int64_t)gridDim.x * kThreads) {
    const int64_t row = i / words, entry = row / rows;
    const int64_t rest = row - entry * rows;  // heads and slots of a page together may pass 2^31
    const int word = (int)(i - row * words), h = (int)divide(rest, p.c.page_size), slot = (int)(rest - (int64_t)h * p.c.page_size);
    const int page = p.list[entry];
    const bool there = page >= 0 && page < p.c.pages;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      uint4 out{0u, 0u, 0u, 0u};
      if (there) {
        const char* codes = which ? p.c.v + page * p.c.v_page + h * p.c.v_head + slot * p.c.v_slot : p.c.k + page * p.c.k_page + h * p.c.k_head + slot * p.c.k_slot;
        const char* pairs = which ? p.s.v + page * p.s.v_page + h * p.s.v_head + slot * p.s.v_slot : p.s.k + page * p.s.k_page + h * p.s.k_head + slot * p.s.k_slot;
        const uint4 v = __builtin_bit_cast(uint4, values8(reinterpret_cast<const uint32_t*>(codes)[word], reinterpret_cast<const uint32_t*>(pairs)[word >> 2], bits));
        out = uint4{__builtin_amdgcn_perm(v.y, v.x, 0x05040100u), __builtin_amdgcn_perm(v.w, v.z, 0x05040100u),
                    __builtin_amdgcn_perm(v.y, v.x, 0x07060302u), __builtin_amdgcn_perm(v.w, v.z, 0x07060302u)};
      }
      *reinterpret_cast<uint4*>(p.out[which] + (row * p.dim + 8 * word) * 2) = out;
    }
  }
}

}  // namespace

hipError_t launch_pack(const PackParams& p, int dtype, int wide, hipStream_t stream) {
  return dtype == 0 ? launch_pack_type<float>(p, wide != 0, stream) : launch_pack_type<uint16_t>(p, wide != 0, stream);
}

hipError_t launch_unpack(const UnpackParams& p, hipStream_t stream) {
  const int words = p.dim / 8;
  const int64_t items = p.count * p.kv_heads * p.c.page_size * words;
  const unsigned grid = (unsigned)std::min<int64_t>((items + kThreads - 1) / kThreads, 1 << 20);
  unpack_kernel<<<dim3(grid), dim3(kThreads), 0, stream>>>(p, words, items);
  return hipGetLastError();
}

}  // namespace sc
