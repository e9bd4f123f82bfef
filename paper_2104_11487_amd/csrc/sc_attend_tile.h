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

// The LDS address of what a pointer to a __shared__ array names.
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

// Copies 16 bytes a lane from `base` + off (base alike in all lanes; or from each lane's own address) into LDS at `to` + 16 lane (`to` alike
// in all lanes), without a wait: wait_loads and a barrier (or the wave's own use) come before the data is read. Written as assembly because the compiler
// takes every later LDS read for a reader of such a copy and would wait for all that are in flight. No register but M0, the destination's base, is
// written, and the addresses are read when the instruction issues. The wait states that the compiler would put between instructions are the
// statement's own matter, as it knows nothing of what comes before: one between M0 and the load that reads it, and five between a vector instruction
// that writes a scalar register (the base comes from v_readlane) and the load that reads that: the move and four idle ones. The base added into each
// lane's own address instead needs none of these, but costs more (8192 tokens over 24576, heads of 128: 1622 -> 1652 us).
__device__ __forceinline__ void copy16(const char* base, uint32_t off, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %1, %2"
               ::"s"(uniform((int)to)), "v"(off), "s"(base)
               : "memory", "m0");
}
__device__ __forceinline__ void copy16(const char* from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(uniform((int)to)), "v"(from) : "memory", "m0");
}

// The same, 4 bytes a lane from each lane's own address.
__device__ __forceinline__ void copy4(const void* from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(uniform((int)to)), "v"(from) : "memory", "m0");
}

// A wave's share of the copies of one tile of keys and one of values (of the keys `lag` before), in two steps, so that page
// numbers are looked up a tile before the copies that need them.
//
// UNI: the rows of each load lie in one page (page sizes that are a multiple of kGroup). Then lane i finds the address of
// load i's first row (keys, then values), all loads in one go, and the copies take it as their scalar base: their
// lanes' offsets to it never change. Otherwise each lane finds its own row's.
template <typename T, typename TL, int NW, bool UNI, int LAG>
struct Stager {
  const CacheView& c;
  const int b, lane, wave, chunks;
  const char* kb;                     // the head's first page
  const char* vb;
  const char* base;                   // UNI: those of this lane's load
  uint32_t page_bytes, slot_bytes;
  static constexpr int kFound = UNI ? 1 : 2 * TL::kLoads;  // rows that a lane looks up
  int entry[kFound], slot[kFound];

  __device__ __forceinline__ Stager(const AttendParams& p, const Unit& u, int w, int l, int n)
      : c(p.c), b(u.b), lane(l), wave(w), chunks(n), kb(c.k + (int64_t)u.head * c.k_head * (int64_t)sizeof(T)),
        vb(c.v + (int64_t)u.head * c.v_head * (int64_t)sizeof(T)) {
    if constexpr (UNI) {
      const bool val = ((lane / TL::kLoads) & 1) != 0;
      const int64_t kp = c.k_page, vp = c.v_page, ks = c.k_slot, vs = c.v_slot;
      base = val ? vb : kb;
      page_bytes = (uint32_t)((val ? vp : kp) * (int64_t)sizeof(T));
      slot_bytes = (uint32_t)((val ? vs : ks) * (int64_t)sizeof(T));
    }
  }

  __device__ __forceinline__ void find(int key0) {
    if constexpr (UNI) {
      const int lag = ((lane / TL::kLoads) & 1) ? LAG : 0;
      entry[0] = entry_at(c, b, max(key0 - lag, 0) + ((lane % TL::kLoads) * NW + wave) * TL::kGroup, TL::kGroup, &slot[0]);
    } else {
#pragma unroll
      for (int i = 0; i < kFound; ++i)
        entry[i] = entry_at(c, b, max(key0 - (i < TL::kLoads ? 0 : LAG), 0) + (i % TL::kLoads * NW + wave) * TL::kGroup + lane / TL::kChunks, 1, &slot[i]);
    }
  }

  __device__ __forceinline__ int chunk_of(int t) const {  // that this lane's 16 bytes of load t come from
    return (lane % TL::kChunks) ^ (TL::swizzle((t * NW + wave) * TL::kGroup + lane / TL::kChunks) & (TL::kChunks - 1));
  }

  // FULL: the head fills its chunks, so every lane copies. PARTS: 1 keys, 2 values, 3 both.
  template <bool FULL, int PARTS>
  __device__ __forceinline__ void copy_rows(uint32_t keys, uint32_t values) const {
    uint64_t row0 = 0;
    if constexpr (UNI) row0 = (uint64_t)base + (uint64_t)(uint32_t)page_of_entry(c, entry[0]) * page_bytes + (uint64_t)(uint32_t)slot[0] * slot_bytes;
    const int lo = (int)(uint32_t)row0, hi = (int)(uint32_t)(row0 >> 32);
#pragma unroll
    for (int i = 0; i < 2 * TL::kLoads; ++i) {
      const int t = i % TL::kLoads;
      const bool val = i >= TL::kLoads;
      if (!(PARTS & (val ? 2 : 1))) continue;
      const int64_t slot_stride = val ? c.v_slot : c.k_slot, page_stride = val ? c.v_page : c.k_page;
      const uint32_t to = (val ? values : keys) + (t * NW + wave) * 1024;
      if constexpr (UNI) {
        const uint64_t first = ((uint64_t)(uint32_t)__builtin_amdgcn_readlane(hi, i) << 32) | (uint32_t)__builtin_amdgcn_readlane(lo, i);
        const uint32_t off = (uint32_t)((lane / TL::kChunks) * (int)slot_stride * (int)sizeof(T) + chunk_of(t) * 16);
        if (FULL || chunk_of(t) < chunks) copy16(reinterpret_cast<const char*>(first), off, to);
      } else {
        const char* from = (val ? vb : kb) + ((int64_t)page_of_entry(c, entry[i]) * page_stride + (int64_t)slot[i] * slot_stride) * (int64_t)sizeof(T) + chunk_of(t) * 16;
        if (FULL || chunk_of(t) < chunks) copy16(from, to);
      }
    }
  }
  template <int PARTS = 3>
  __device__ __forceinline__ void copy(uint32_t keys, uint32_t values) const {
    if (chunks == TL::kChunks) copy_rows<true, PARTS>(keys, values);
    else copy_rows<false, PARTS>(keys, values);
  }
};

// The copies of one wave that has tiles of its own. Page numbers too arrive by copies into LDS, `entries` (64 of them a tile), so that
// no wait of the compiler's for a loaded register lets the copies in flight run dry.
template <typename T, typename TL, int KEYS>
struct LoneStager {
  const CacheView& c;
  const int b, lane, chunks;
  const char* kb;
  const char* vb;
  static constexpr int kOps = 2 * TL::kLoads;  // loads of copy()

  __device__ __forceinline__ LoneStager(const AttendParams& p, const Unit& u, int l, int n)
      : c(p.c), b(u.b), lane(l), chunks(n), kb(c.k + (int64_t)u.head * c.k_head * (int64_t)sizeof(T)),
        vb(c.v + (int64_t)u.head * c.v_head * (int64_t)sizeof(T)) {}

  __device__ __forceinline__ void find(int key0, uint32_t entries) const {
    copy4(c.table + (int64_t)b * c.width + min(page_of(c, key0 + (lane & (KEYS - 1))), c.width - 1), entries);
  }
  __device__ __forceinline__ void copy(int key0, const char* entries, uint32_t keys, uint32_t values) const {
    const char* from[2 * TL::kLoads];
#pragma unroll
    for (int t = 0; t < TL::kLoads; ++t) {
      const int row = t * TL::kGroup + lane / TL::kChunks, at = key0 + row;
      const int page = page_of_entry(c, *reinterpret_cast<const int*>(entries + row * 4));
      const int slot = min(at - min(page_of(c, at), c.width - 1) * c.page_size, c.page_size - 1);
      const int chunk = (lane % TL::kChunks) ^ (TL::swizzle(row) & (TL::kChunks - 1));
      from[t] = kb + ((int64_t)page * c.k_page + (int64_t)slot * c.k_slot) * (int64_t)sizeof(T) + chunk * 16;
      from[TL::kLoads + t] = vb + ((int64_t)page * c.v_page + (int64_t)slot * c.v_slot) * (int64_t)sizeof(T) + chunk * 16;
    }
#pragma unroll
    for (int i = 0; i < 2 * TL::kLoads; ++i) {
      const int t = i % TL::kLoads;
      const int chunk = (lane % TL::kChunks) ^ (TL::swizzle(t * TL::kGroup + lane / TL::kChunks) & (TL::kChunks - 1));
      if (chunk < chunks) copy16(from[i], (i < TL::kLoads ? keys : values) + t * 1024);
    }
  }
};

// Four bf16 of one column, from four consecutive rows: lane l of each 16 lanes gives the address of row l / 4,
// columns 4 (l % 4).., and receives column l.
__device__ __forceinline__ u32x2 read_column4(uint32_t lds_at) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) shortx4*)(lds_at)));
}
__device__ __forceinline__ u32x2 read_column4(const char* at) { return read_column4((uint32_t)(uintptr_t)SC_LDS(at, const char)); }

// Of two packed bf16 values those that are infinite or NaN become zero.
__device__ __forceinline__ uint32_t finite2(uint32_t v) {
  if ((v & 0x7f80u) == 0x7f80u) v &= 0xffff0000u;
  if ((v & 0x7f800000u) == 0x7f800000u) v &= 0x0000ffffu;
  return v;
}
__device__ __forceinline__ float finite1(float v) { return (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u ? 0.0f : v; }

// Of 16 bytes of values: whether one is infinite or NaN (its exponent is all ones, which a carry shows); with those zero.
template <typename T>
__device__ __forceinline__ int not_finite(uint4 v) {
  const uint32_t mask = sizeof(T) == 2 ? 0x7f807f80u : 0x7f800000u, one = sizeof(T) == 2 ? 0x00800080u : 0x00800000u;
  const uint32_t x = ((v.x & mask) + one) | ((v.y & mask) + one) | ((v.z & mask) + one) | ((v.w & mask) + one);
  return (x & (sizeof(T) == 2 ? 0x80008000u : 0x80000000u)) != 0;
}
template <typename T>
__device__ __forceinline__ uint4 finite_of(uint4 v) {
  if constexpr (sizeof(T) == 2) return uint4{finite2(v.x), finite2(v.y), finite2(v.z), finite2(v.w)};
  else return uint4{__float_as_uint(finite1(__uint_as_float(v.x))), __float_as_uint(finite1(__uint_as_float(v.y))),
                    __float_as_uint(finite1(__uint_as_float(v.z))), __float_as_uint(finite1(__uint_as_float(v.w)))};
}

// Of two bf16 values (a float): those outside the mask become zero too, and one inside it that is not finite sets *odd.
__device__ __forceinline__ uint32_t finite2(uint32_t v, uint32_t mask, int* odd) {
  v &= mask;
  const uint32_t f = finite2(v);
  if (f != v) *odd = 1;
  return f;
}
__device__ __forceinline__ float finite1(float v, bool keep, int* odd) {
  if (!keep) return 0.0f;
  if ((__float_as_uint(v) & 0x7f800000u) == 0x7f800000u) *odd = 1;
  return finite1(v);
}

}  // namespace sc
