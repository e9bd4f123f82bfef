// Appending to the cache in 4 bits, with the rotation on the way, and reading its values back.
//
// Per token, key head and group of 32 elements, on the elements x in fp32 (keys: turned in 64 bits and rounded once):
//   y = clamp(x, +-32768), low = fl16(min y), scale = fl16(max(0, (max y - low) / 15)), code = clamp(rint((y - low) / scale), 0, 15)
// (scale 0: code 0). A group with an element that is not finite has scale and minimum NaN, so that it reads as NaN. All operations round to
// nearest, ties to even. The turn is formed in 64 bits because a code changes where (y - low) / scale passes a half: so a code depends on the
// inputs alone, not on how the call was cut. Queries turn as skipconv_rotate's.
//
// Four lanes hold a group, a word of eight codes each. Bound by memory, and a few tokens by the launch.
#include "sc_packed_device.h"
#include "sc_stream.h"

#include <algorithm>

#pragma clang fp contract(off)

namespace sc {

namespace {

constexpr int kThreads = 256;
constexpr int kMostTokens = 8;  // of a workgroup

// Eight elements from element d of a head on, as fp32, those past `dim` zero. WIDE: 16-byte loads.
template <typename T, bool WIDE>
__device__ __forceinline__ void load_chunk(const T* head, int d, int dim, float* x) {
  if (WIDE && d + 8 <= dim) {
    Elem<T>::load8(head, d, x);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = d + i < dim ? Elem<T>::load1(head, d + i) : 0.0f;
  }
}

struct Turn {
  double c, s;
};

template <typename T, bool WIDE>
__global__ void __launch_bounds__(kThreads) pack_kernel(PackParams pp) {
  const RotateParams& p = pp.r;
  extern __shared__ char lds[];
  Turn* turn = reinterpret_cast<Turn*>(lds);  // [token][pair]
  __shared__ int where[kMostTokens][2];       // [token]: page (-1: no sequence's, -2: no place), slot
  const int t0 = (int)blockIdx.x * pp.tok_per_wg, nt = min(pp.tok_per_wg, p.tokens - t0);
  const int lane = threadIdx.x & 63;
  for (int tk = uniform((int)threadIdx.x >> 6); tk < nt; tk += kThreads / 64) {
    const int s = owner_of(p.cache.row_start, p.cache.batch, t0 + tk);
    int page = -1, slot = 0;
    if (s < p.cache.batch) {
      const Sequence q = sequence_of(p.cache, s);
      const int at = p.cache.kv_len[s] - q.n + (t0 + tk - q.start);
      page = -2;
      if (t0 + tk >= q.start && at >= 0 && page_of(p.cache, at) < p.cache.width) {
        const int i = page_of(p.cache, at), got = p.cache.table[(int64_t)s * p.cache.width + i];
        slot = at - i * p.cache.page_size;
        if (got >= 0 && got < p.cache.pages) page = got;
      }
    }
    if (lane == 0) where[tk][0] = page, where[tk][1] = slot;
  }
  if (p.freq) {
    for (int i = threadIdx.x; i < nt * p.pairs; i += kThreads) {
      const int tk = i / p.pairs, j = i - tk * p.pairs;
      double angle = 0.0;
      for (int x = 0; x < p.axes; ++x) angle += (double)p.pos[(int64_t)(t0 + tk) * p.axes + x] * (double)p.freq[x * p.pairs + j];
      double turns = angle * 0.15915494309189533577;  // 1 / (2 pi)
      turns -= rint(turns);
      sincospi(2.0 * turns, &turn[i].s, &turn[i].c);
    }
  }
  __syncthreads();

  const int words = (p.dim + kPackGroup - 1) / kPackGroup * 4;  // of a head
  const int heads = p.heads[0] + 2 * p.heads[1], each = kThreads / words;
  const int mine = (int)threadIdx.x / words, word = (int)threadIdx.x - mine * words, d = word * 8;
  for (int h0 = 0; h0 < nt * heads; h0 += each) {  // whole heads at a time: all of one is loaded before any of it is stored
    const int at = h0 + mine;
    bool live = mine < each && at < nt * heads;
    int tk = 0, h = 0, which = 0;
    const T* src = nullptr;
    if (live) {
      tk = at / heads, h = at - tk * heads;
      if (h >= p.heads[0]) h -= p.heads[0], which = 1;
      if (which == 1 && h >= p.heads[1]) h -= p.heads[1], which = 2;
      live = where[tk][0] >= (which == 0 ? -2 : 0) && where[tk][0] != -1;
      src = reinterpret_cast<const T*>(p.src[which]) + (int64_t)(t0 + tk) * p.src_token[which] + (int64_t)h * p.src_head[which];
    }
    float x[8];
    if (live) {
      load_chunk<T, WIDE>(src, d, p.dim, x);
      if (p.freq && which < 2 && d < 2 * p.pairs) {
        const Turn* tt = turn + tk * p.pairs;
        if (p.adjacent) {
#pragma unroll
          for (int i = 0; i < 8; i += 2) {
            if (d + i >= 2 * p.pairs) break;
            const Turn c = tt[(d + i) >> 1];
            const float u = x[i], w = x[i + 1];
            if (which == 1) {
              x[i] = (float)((double)u * c.c - (double)w * c.s);
              x[i + 1] = (float)((double)w * c.c + (double)u * c.s);
            } else {
              x[i] = u * (float)c.c - w * (float)c.s;
              x[i + 1] = w * (float)c.c + u * (float)c.s;
            }
          }
        } else {
          float y[8];
          if (p.pairs % 8 == 0) {
            load_chunk<T, WIDE>(src, d < p.pairs ? d + p.pairs : d - p.pairs, p.dim, y);
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const int e = d + i;
              y[i] = e < 2 * p.pairs ? Elem<T>::load1(src, e < p.pairs ? e + p.pairs : e - p.pairs) : 0.0f;
            }
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int e = d + i;
            if (e >= 2 * p.pairs) break;
            const bool second = e >= p.pairs;
            const Turn c = tt[second ? e - p.pairs : e];
            if (which == 1) {
              const double b = (double)y[i] * c.s, a = (double)x[i] * c.c;
              x[i] = (float)(second ? a + b : a - b);
            } else {
              const float b = y[i] * (float)c.s, a = x[i] * (float)c.c;
              x[i] = second ? a + b : a - b;
            }
          }
        }
      }
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
      float low = -kNegInf, high = kNegInf;
      int odd = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (d + i >= p.dim) break;
        odd |= (__float_as_uint(x[i]) & 0x7f800000u) == 0x7f800000u;
        x[i] = fminf(fmaxf(x[i], -kPackMost), kPackMost);
        low = fminf(low, x[i]), high = fmaxf(high, x[i]);
      }
#pragma unroll
      for (int m = 1; m < 4; m <<= 1) {
        low = fminf(low, __shfl_xor(low, m)), high = fmaxf(high, __shfl_xor(high, m));
        odd |= __shfl_xor(odd, m);
      }
      const _Float16 low16 = (_Float16)low;
      const float base = (float)low16;
      const _Float16 scale16 = (_Float16)fmaxf(__fdiv_rn(high - base, 15.0f), 0.0f);
      const float scale = (float)scale16;
      uint32_t codes = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (d + i < p.dim && scale > 0.0f && !odd) codes |= (uint32_t)fminf(fmaxf(rintf(__fdiv_rn(x[i] - base, scale)), 0.0f), 15.0f) << (4 * i);
      const int64_t page = where[tk][0], slot = where[tk][1];
      char* row = which == 1 ? p.cache.k + page * p.cache.k_page + h * p.cache.k_head + slot * p.cache.k_slot
                             : p.cache.v + page * p.cache.v_page + h * p.cache.v_head + slot * p.cache.v_slot;
      reinterpret_cast<uint32_t*>(row)[word] = codes;
      if ((word & 3) == 0) {
        char* pairs = which == 1 ? pp.s.k + page * pp.s.k_page + h * pp.s.k_head + slot * pp.s.k_slot
                                 : pp.s.v + page * pp.s.v_page + h * pp.s.v_head + slot * pp.s.v_slot;
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
  if (wide) pack_kernel<T, true><<<dim3(grid), dim3(kThreads), lds, stream>>>(p);
  else pack_kernel<T, false><<<dim3(grid), dim3(kThreads), lds, stream>>>(p);
  return hipGetLastError();
}

// A thread makes eight values of a row: out[which][entry][head][slot][8 word ..].
__global__ void __launch_bounds__(kThreads) unpack_kernel(UnpackParams p, int words, int64_t items) {
  const int64_t rows = (int64_t)p.kv_heads * p.c.page_size;
  const CodeBits bits = code_bits();
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < items; i += (int64_t)gridDim.x * kThreads) {
    const int64_t row = i / words, entry = row / rows;
    const int word = (int)(i - row * words), rest = (int)(row - entry * rows), h = rest / p.c.page_size, slot = rest - h * p.c.page_size;
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
