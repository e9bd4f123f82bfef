// Key and value tiles of the paged cache in LDS, and what the attention kernels do with them: staging with
// direct global-to-LDS loads, operand fragments, masks (gfx950 only).
//
// A tile holds KEYS keys (or values) of one key head. A row is CH 16-byte chunks (the least power of two that holds the
// head), its chunks permuted by an exclusive or with a function of the row, so that both the fragments that walk along
// rows (scores) and those that walk down columns (values, read transposed) touch every LDS bank evenly. The copies into
// LDS place lane l's 16 bytes at a wave-uniform base + 16 l, so the permutation is applied to the address that is read.
#pragma once

#include "sc_attend_device.h"

#pragma clang fp contract(off)

namespace sc {

constexpr int pow2_at_least(int v) {
  int p = 1;
  while (p < v) p *= 2;
  return p;
}

#define SC_LDS(ptr, type) ((__attribute__((address_space(3))) type*)(ptr))
typedef short shortx4 __attribute__((ext_vector_type(4)));

// Geometry of a tile: T element type, DP head dimension rounded up to 32, KEYS rows, NW waves that stage it.
template <typename T, int DP, int KEYS, int NW, bool TALL>
struct Tile {
  static constexpr int kElems = 16 / (int)sizeof(T);         // of a chunk
  static constexpr int kChunks = pow2_at_least(DP / kElems);  // of a row (CH)
  static constexpr int kRowBytes = kChunks * 16;
  static constexpr int kBytes = KEYS * kRowBytes;
  static constexpr int kGroup = 64 / kChunks;                // rows of one wave's load
  static constexpr int kLoads = KEYS * kChunks / 64 / NW;    // of a wave
  static_assert(kChunks <= 64 && kLoads * NW * 64 == KEYS * kChunks, "whole loads");

  // The permutation. Lanes of one LDS pass read one chunk of 16 rows (scores): with rows of 256 bytes or more all 16 rows
  // need another chunk; with shorter rows those that lie in the same bank. TALL: four rows x 64 bytes a pass (values of
  // 32-wide products); otherwise eight rows x 32 bytes.
  __device__ __forceinline__ static int swizzle(int row) {
    if constexpr (kChunks >= 16) {
      return TALL ? ((row & 3) << 2) | ((row >> 2) & 3) : ((row & 7) << 1) | ((row >> 3) & 1);
    } else if constexpr (kChunks == 8) {
      return TALL ? ((row & 2) << 1) | ((row >> 2) & 3) : (((row >> 1) & 3) << 1) | ((row >> 3) & 1);
    } else {
      return TALL ? (row >> 2) & 3 : ((row & 4) >> 1) | ((row >> 3) & 1);
    }
  }
};

// A wave's share of the copies of one tile of keys and one of values, in two steps, so that page numbers are looked up a
// tile before the copies that need them.
//
// UNI: the rows of each load lie in one page (page sizes that are a multiple of kGroup). Then lane i finds the address of
// load i's first row (keys, then values), all loads in one go, and the copies take it as their scalar base: their
// lanes' offsets to it never change. Otherwise each lane finds its own row's.
template <typename T, typename TL, int NW, bool UNI>
struct Stager {
  const AttendParams& p;
  const int b, lane, wave, chunks;
  const char* kb;
  const char* vb;
  int page[UNI ? 1 : TL::kLoads], slot[UNI ? 1 : TL::kLoads];

  __device__ __forceinline__ Stager(const AttendParams& q, const Unit& u, int w, int l, int c)
      : p(q), b(u.b), lane(l), wave(w), chunks(c), kb(q.c.k + (int64_t)u.head * q.c.k_head * (int64_t)sizeof(T)),
        vb(q.c.v + (int64_t)u.head * q.c.v_head * (int64_t)sizeof(T)) {}

  __device__ __forceinline__ void find(int key0) {
    if constexpr (UNI) {
      page[0] = page_at(p.c, b, key0 + ((lane % TL::kLoads) * NW + wave) * TL::kGroup, TL::kGroup, &slot[0]);
    } else {
#pragma unroll
      for (int t = 0; t < TL::kLoads; ++t) page[t] = page_at(p.c, b, key0 + (t * NW + wave) * TL::kGroup + lane / TL::kChunks, 1, &slot[t]);
    }
  }

  __device__ __forceinline__ void take(const Stager& other) {
#pragma unroll
    for (int t = 0; t < (UNI ? 1 : TL::kLoads); ++t) page[t] = other.page[t], slot[t] = other.slot[t];
  }

  __device__ __forceinline__ int chunk_of(int t) const {  // that this lane's 16 bytes of load t come from
    return (lane % TL::kChunks) ^ (TL::swizzle((t * NW + wave) * TL::kGroup + lane / TL::kChunks) & (TL::kChunks - 1));
  }

  __device__ __forceinline__ void copy(char* keys, char* values) const {
    if constexpr (UNI) {
      const bool val = (lane / TL::kLoads) & 1;
      const uint64_t row0 = (uint64_t)(val ? vb : kb) + (uint64_t)(uint32_t)page[0] * (uint32_t)((val ? p.c.v_page : p.c.k_page) * sizeof(T)) +
                            (uint64_t)(uint32_t)slot[0] * (uint32_t)((val ? p.c.v_slot : p.c.k_slot) * sizeof(T));
      const int lo = (int)(uint32_t)row0, hi = (int)(uint32_t)(row0 >> 32);
#pragma unroll
      for (int i = 0; i < 2 * TL::kLoads; ++i) {
        const int t = i % TL::kLoads;
        const char* from = reinterpret_cast<const char*>(((uint64_t)(uint32_t)__builtin_amdgcn_readlane(hi, i) << 32) | (uint32_t)__builtin_amdgcn_readlane(lo, i));
        const int stride = (int)((i < TL::kLoads ? p.c.k_slot : p.c.v_slot) * (int)sizeof(T));
        const uint32_t off = (uint32_t)((lane / TL::kChunks) * stride + chunk_of(t) * 16);
        char* to = (i < TL::kLoads ? keys : values) + (t * NW + wave) * 1024;
        if (chunk_of(t) < chunks) __builtin_amdgcn_global_load_lds(from + off, SC_LDS(to, void), 16, 0, 0);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 2 * TL::kLoads; ++i) {
        const int t = i % TL::kLoads;
        const bool val = i >= TL::kLoads;
        const char* from = (val ? vb : kb) + ((int64_t)page[t] * (val ? p.c.v_page : p.c.k_page) + (int64_t)slot[t] * (val ? p.c.v_slot : p.c.k_slot)) * (int64_t)sizeof(T) + chunk_of(t) * 16;
        char* to = (val ? values : keys) + (t * NW + wave) * 1024;
        if (chunk_of(t) < chunks) __builtin_amdgcn_global_load_lds(from, SC_LDS(to, void), 16, 0, 0);
      }
    }
  }
};

// Four bf16 of one column, from four consecutive rows: lane l of each 16 lanes gives the address of row l / 4,
// columns 4 (l % 4).., and receives column l.
__device__ __forceinline__ u32x2 read_column4(const char* at) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(SC_LDS(const_cast<char*>(at), shortx4)));
}

// Of two packed bf16 values: those outside the mask become zero, and those that are infinite or NaN too, which sets *odd.
__device__ __forceinline__ uint32_t finite2(uint32_t v, uint32_t mask, int* odd) {
  v &= mask;
  if ((v & 0x7f80u) == 0x7f80u) v &= 0xffff0000u, *odd = 1;
  if ((v & 0x7f800000u) == 0x7f800000u) v &= 0x0000ffffu, *odd = 1;
  return v;
}
__device__ __forceinline__ float finite1(float v, bool keep, int* odd) {
  if (!keep) return 0.0f;
  if ((__float_as_uint(v) & 0x7f800000u) != 0x7f800000u) return v;
  *odd = 1;
  return 0.0f;
}

}  // namespace sc
