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

// Where a wave's loads of one tile come from. UNI: the rows of a load lie in one page (page sizes that are a multiple of
// kGroup), so the page is looked up once a load, by the scalar unit; otherwise each lane looks up its row.
template <typename TL, bool UNI>
struct Source {
  int page[TL::kLoads], slot[TL::kLoads];
};

template <typename TL, int NW, bool UNI>
__device__ __forceinline__ void find_pages(const CacheView& c, int b, int key0, int wave, int lane, Source<TL, UNI>* s) {
#pragma unroll
  for (int t = 0; t < TL::kLoads; ++t) {
    const int row = (t * NW + wave) * TL::kGroup + (UNI ? 0 : lane / TL::kChunks);
    s->page[t] = page_at(c, b, key0 + row, UNI ? TL::kGroup : 1, &s->slot[t]);
  }
}

// Copies the tile's rows of one head (keys or values) into LDS at `to`.
template <typename T, typename TL, int NW, bool UNI>
__device__ __forceinline__ void stage(const char* base, int64_t page_stride, int64_t slot_stride, const Source<TL, UNI>& s, int chunks,
                                      int wave, int lane, char* to) {
  const int in = lane / TL::kChunks, at = lane % TL::kChunks;
#pragma unroll
  for (int t = 0; t < TL::kLoads; ++t) {
    const int g = t * NW + wave;
    const int chunk = at ^ (TL::swizzle(g * TL::kGroup + in) & (TL::kChunks - 1));
    const char* from;
    if constexpr (UNI) {
      const char* row0 = base + ((int64_t)s.page[t] * page_stride + (int64_t)s.slot[t] * slot_stride) * (int64_t)sizeof(T);
      from = row0 + (uint32_t)(in * (int)slot_stride * (int)sizeof(T) + chunk * 16);
    } else {
      from = base + ((int64_t)s.page[t] * page_stride + (int64_t)s.slot[t] * slot_stride) * (int64_t)sizeof(T) + chunk * 16;
    }
    if (chunk < chunks) __builtin_amdgcn_global_load_lds(from, SC_LDS(to + g * 1024, void), 16, 0, 0);
  }
}

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
