// Device-side helpers shared by the streaming attention kernels (gfx950 only): which sequence a
// row belongs to, which units of work a batch makes, lane exchanges, bf16 packing.
#pragma once

#include "sc_attend.h"
#include "sc_device.h"

#pragma clang fp contract(off)

namespace sc {

typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr float kNegInf = -__builtin_huge_valf();

// bf16 round-to-nearest-even of two floats, packed (v_cvt_pk_bf16_f32).
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(floatx2{a, b}, bf16x2));
}

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Wait until at most N of the wave's vector memory loads are outstanding (older ones have landed,
// copies into LDS among them); LDS reads that follow stay behind it.
template <int N>
__device__ __forceinline__ void wait_loads() {
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x0f70);
  asm volatile("" ::: "memory");
}

// Value of the lane 32 (16) away joined with the lane's own.
__device__ __forceinline__ float max_across32(float v) {
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float sum_across32(float v) {
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}
__device__ __forceinline__ float max_across16(float v) {
  const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float sum_across16(float v) {
  const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

// The sequence that row t belongs to: how many of row_start[1..batch] are <= t (`batch`: none).
// All lanes of a wave probe together, 64 places a step.
__device__ __forceinline__ int owner_of(const int32_t* row_start, int batch, int t) {
  const int lane = threadIdx.x & 63;
  int lo = 0, len = batch;
  while (len > 0) {
    const int step = (len + 63) >> 6;
    const int at = (lane + 1) * step - 1;
    const bool below = at < len && row_start[lo + at + 1] <= t;
    const int n = (int)__popcll(__ballot(below));
    lo += n * step;
    len = min(step - 1, len - n * step);
  }
  return uniform(lo);
}

// One sequence as the batch describes it, kept within the tensors whatever the arrays hold.
struct Sequence {
  int start, n, len;  // first row, rows, tokens in the cache with them
};
__device__ __forceinline__ Sequence sequence_of(const CacheView& c, int b) {
  Sequence s;
  s.start = min(max(c.row_start[b], 0), c.tokens);
  s.n = min(max(c.row_start[b + 1], s.start), c.tokens) - s.start;
  const int64_t room = (int64_t)c.width * c.page_size;
  s.len = (int)min((int64_t)max(c.kv_len[b], 0), min(room, (int64_t)kMostKeys));
  return s;
}

// ---- units of work ----
//
// Rows of one key head: a sequence's n new tokens x `group` query heads, the token slowest. They
// are cut into tiles of 2^log_rows; the keys that a tile may see are cut into `splits` chunks where
// a launch's tiles alone would leave compute units idle. Every workgroup derives the same cut from
// the lengths on the device (no host copy of them exists), by a scan over the sequences.
// Unit index: sequences in order; within one: key head, tile (the last one, which sees most keys
// under a causal mask, first), chunk.
struct Shape {
  int tiles, splits, chunk, span;
};

__device__ __forceinline__ Shape shape_of(const AttendParams& p, const Sequence& s) {
  Shape o;
  const int rows = 1 << p.log_rows;
  o.tiles = (s.n * p.group + rows - 1) >> p.log_rows;
  const int reach = p.causal ? min(s.n, (rows - 1) / p.group + 2) : s.n;  // tokens that a tile spans
  o.span = p.window < 0 ? s.len : (int)min((int64_t)s.len, (int64_t)p.window + reach);
  o.splits = o.tiles > 0 ? 1 : 0;
  o.chunk = kMostKeys;
  return o;
}

// Keys that a chunk should have; 0: nothing is split.
__device__ __forceinline__ int chunk_goal(const AttendParams& p) {
  if (p.target <= 0) return 0;
  const int lane = threadIdx.x & 63;
  int64_t total = 0;
  for (int b0 = 0; b0 < p.c.batch; b0 += 64) {
    if (b0 + lane < p.c.batch) {
      const Shape o = shape_of(p, sequence_of(p.c, b0 + lane));
      total += (int64_t)o.tiles * o.span;
    }
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) total += __shfl_xor(total, d);
  return max(p.min_chunk, (int)min(ceil((double)total / (double)p.target), (double)kMostKeys));
}

__device__ __forceinline__ Shape cut_of(const AttendParams& p, const Sequence& s, int goal) {
  Shape o = shape_of(p, s);
  if (goal > 0 && o.tiles > 0 && o.span > goal) {
    o.splits = (int)((uint32_t)(o.span + goal - 1) / (uint32_t)goal);
    const uint32_t each = (uint32_t)(o.span + p.keys - 1 + o.splits - 1) / (uint32_t)o.splits;  // the first key is rounded down to a tile
    o.chunk = (int)((each + p.keys - 1) & ~(uint32_t)(p.keys - 1));
  }
  return o;
}

struct Unit {
  int b, start, n, len;  // sequence
  int head;              // key head
  int row0;              // first row of the tile
  int lo, hi;            // keys [lo, hi) of this chunk, lo a multiple of the key tile
  int splits;            // chunks of the tile
};

// Finds the sequence whose units hold index `at` (`by` 0), or whose rows hold row `at` (`by` 1): its number, extents, cut and
// the index of its first unit. False where there is none. Called by whole waves.
__device__ __forceinline__ bool find_units(const AttendParams& p, int at, int by, int* b, Sequence* seq, Shape* cut, int* first) {
  const int lane = threadIdx.x & 63;
  const int goal = chunk_goal(p);
  int64_t base = 0;
  for (int b0 = 0; b0 < p.c.batch; b0 += 64) {
    Sequence s = {0, 0, 0};
    Shape o = {0, 0, 0, 0};
    if (b0 + lane < p.c.batch) {
      s = sequence_of(p.c, b0 + lane);
      o = cut_of(p, s, goal);
    }
    const int64_t mine = (int64_t)o.tiles * o.splits * p.kv_heads;
    int64_t upto = mine;  // inclusive scan
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int64_t t = __shfl_up(upto, d);
      if (lane >= d) upto += t;
    }
    const uint64_t past = __ballot(by ? at >= s.start && at < s.start + s.n : base + upto > at);
    if (past) {
      const int src = (int)__ffsll((unsigned long long)past) - 1;
      *b = b0 + src;
      seq->start = uniform(__shfl(s.start, src));
      seq->n = uniform(__shfl(s.n, src));
      seq->len = uniform(__shfl(s.len, src));
      cut->tiles = uniform(__shfl(o.tiles, src));
      cut->splits = uniform(__shfl(o.splits, src));
      cut->chunk = uniform(__shfl(o.chunk, src));
      *first = uniform((int)min(base + __shfl(upto - mine, src), (int64_t)0x7fffffff));
      return true;
    }
    base += __shfl(upto, 63);
  }
  return false;
}

__device__ __forceinline__ bool unit_of(const AttendParams& p, int at, Unit* u) {
  Sequence s;
  Shape o;
  int first;
  if (!find_units(p, at, 0, &u->b, &s, &o, &first)) return false;
  u->start = s.start, u->n = s.n, u->len = s.len;
  const int rel = at - first, per = o.tiles * o.splits;
  u->head = rel / per;
  const int r = rel - u->head * per, t = r / o.splits, split = r - t * o.splits;
  u->row0 = (o.tiles - 1 - t) << p.log_rows;
  u->splits = o.splits;
  // keys that the tile's rows see: up to the last row's end, from the first row's begin
  const int t0 = u->row0 / p.group, t1 = min(u->row0 + (1 << p.log_rows) - 1, u->n * p.group - 1) / p.group;
  const int p0 = u->len - u->n;
  const int hi = p.causal ? min(p0 + t1, u->len - 1) + 1 : u->len;
  const int lo = p.window < 0 ? 0 : max(0, p0 + (p.causal ? t0 : 0) - p.window);
  const int64_t from = (int64_t)(lo & ~(p.keys - 1)) + (int64_t)split * o.chunk;
  u->lo = (int)min(from, (int64_t)kMostKeys);
  u->hi = (int)min((int64_t)hi, from + o.chunk);
  return true;
}

// Keys [lo, hi] that row r of the tile's rows sees (lo > hi: none). Rows past the last one follow it.
struct Seen {
  int lo, hi;
};
__device__ __forceinline__ Seen seen_by(const AttendParams& p, const Unit& u, int row) {
  const int t = min(row, u.n * p.group - 1) / p.group, p0 = u.len - u.n;
  Seen s;
  s.hi = p.causal ? min(p0 + t, u.len - 1) : u.len - 1;
  s.lo = p.window < 0 ? 0 : max(0, p0 + (p.causal ? t : 0) - p.window);
  return s;
}

// What a share with reference `ref` counts in a join whose largest reference is `top`. Shares without a key (reference -inf) hold
// zeros, or NaN where all their scores are: they count by 0, or by 1 where no share has a key, so that a NaN stays one.
__device__ __forceinline__ float join_weight(float ref, float top) { return ref == top ? 1.0f : __builtin_amdgcn_exp2f(ref - top); }

// Where key position `at` lies: the slot, which `rows` slots of its page begin at, and the page table's entry. Positions past the
// table and entries outside the cache are led to slots that exist (no row sees their keys). The entry is loaded by a
// relaxed atomic so that the load stays where it is written: ahead of copies that it would otherwise wait for.
__device__ __forceinline__ int entry_at(const CacheView& c, int b, int at, int rows, int* slot) {
  const int i = min(page_of(c, at), c.width - 1);
  *slot = min(at - i * c.page_size, c.page_size - rows);
  return __hip_atomic_load(c.table + (int64_t)b * c.width + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT);
}
__device__ __forceinline__ int page_of_entry(const CacheView& c, int entry) { return min(max(entry, 0), c.pages - 1); }

}  // namespace sc
