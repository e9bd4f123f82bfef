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
// Rows of one key head: a sequence's n new tokens x `group` query heads, the token slowest. They are cut into tiles of 2^log_rows;
// an item is one tile with one key head and all the keys that its rows may see. Every workgroup derives the same cut of the items'
// keys from the lengths on the device (no host copy of them exists), by a scan over the sequences. An item is
//   one unit, where the launch does not share keys;
//   else as many units as it has key tiles, of which each workgroup takes an equal share in a row, wherever that begins and ends;
//   or units of some key tiles, one a workgroup, where that loses little to equal shares: a workgroup whose share ends inside one item
//   and begins inside another pays twice for an item's begin and end.
// Unit index: sequences in order; within one: key head, tile (the last one, which sees most keys under a causal mask, first), keys.
struct Shape {
  int tiles, parts, chunk, span;  // row tiles; units of an item; keys of a unit; keys that an item may have
};

__device__ __forceinline__ Shape shape_of(const AttendParams& p, const Sequence& s) {
  Shape o;
  const int rows = 1 << p.log_rows;
  o.tiles = (s.n * p.group + rows - 1) >> p.log_rows;
  const int reach = p.causal ? min(s.n, (rows - 1) / p.group + 2) : s.n;  // tokens that a tile spans
  o.span = p.window < 0 ? s.len : (int)min((int64_t)s.len, (int64_t)p.window + reach);
  o.parts = o.tiles > 0 ? 1 : 0;
  o.chunk = kMostKeys;
  return o;
}

// The quotient; by the short division where both sides allow it (64-bit divisions are long programs).
__device__ __forceinline__ int64_t divide(int64_t a, int64_t b) {
  return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}

// The cut of a sequence: into key tiles where keys are shared. A span begins anywhere, the first tile at a whole one.
__device__ __forceinline__ Shape cut_of(const AttendParams& p, const Sequence& s) {
  Shape o = shape_of(p, s);
  if (p.target > 0 && o.tiles > 0) {
    o.parts = max(1, (int)(((uint32_t)o.span + 2 * (uint32_t)p.keys - 2) / (uint32_t)p.keys));
    o.chunk = p.keys;
  }
  return o;
}

__device__ __forceinline__ int64_t from_lane(int64_t v, int lane) {
  return ((int64_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}

// Inclusive sum over the wave's lanes by data-parallel moves (within rows of 16 lanes, then the rows' last lanes onwards).
__device__ __forceinline__ int scan32(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);  // row_shr 1, 2, 4, 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // row_bcast 15 into rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // row_bcast 31 into rows 2 and 3
  return v;
}

// A wave's view of the batch's units: lane i holds sequence i, and where its units end; sequences from the 65th on are gone through by 64s.
struct Units {
  const AttendParams& p;
  Sequence s;
  Shape o;
  int64_t upto, all;  // units of the sequences up to the lane's; of the batch
  bool single;        // a workgroup takes one unit

  __device__ __forceinline__ explicit Units(const AttendParams& q) : p(q), single(q.target == 0) {
    s = load(0);
    o = cut_of(p, s);
    upto = scan(o);
    all = from_lane(upto, 63);
    for (int b0 = 64; b0 < p.c.batch; b0 += 64) all += from_lane(scan(cut_of(p, load(b0))), 63);
    if (p.slack > 0 && p.c.batch <= 64 && all < (1 << 24)) whole_units();
  }
  // Looks for the least number of key tiles a unit at which the units are no more than the workgroups, from equal shares' up to `slack` more.
  __device__ __forceinline__ void whole_units() {
    const int items = o.tiles * p.kv_heads, least = max(p.min_chunk, (int)(((uint32_t)all + p.target - 1) / (uint32_t)p.target));
    int each = least;
#pragma unroll 1
    for (int i = 0; i < 3 && each <= least + p.slack; ++i) {
      const int parts = (int)(((uint32_t)o.parts + each - 1) / (uint32_t)each);
      const int sum = scan32(items * parts), n = __builtin_amdgcn_readlane(sum, 63);
      if (n <= p.target) {
        o.parts = parts, o.chunk = (int)min((int64_t)each * p.keys, (int64_t)kMostKeys);
        upto = sum, all = n, single = true;
        return;
      }
      each = max(each + 1, (int)(((uint32_t)each * (uint32_t)n + p.target - 1) / (uint32_t)p.target));
    }
  }
  __device__ __forceinline__ Sequence load(int b0) const {
    const int b = b0 + (threadIdx.x & 63);
    return b < p.c.batch ? sequence_of(p.c, b) : Sequence{0, 0, 0};
  }
  __device__ __forceinline__ int64_t scan(const Shape& x) const {  // inclusive, over the wave
    int64_t v = (int64_t)x.tiles * x.parts * p.kv_heads;
    if (!__any(v >> 25)) return scan32((int)v);
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int64_t t = __shfl_up(v, d);
      if (lane >= d) v += t;
    }
    return v;
  }
  // The sequence whose units hold index `at` (by_row false), or whose rows hold row `at`: its number, extents, cut and the index of its
  // first unit. False where there is none.
  __device__ __forceinline__ bool find(int64_t at, bool by_row, int* b, Sequence* seq, Shape* cut, int64_t* first) const {
    int64_t base = 0;
    for (int b0 = 0; b0 < p.c.batch; b0 += 64) {
      const Sequence x = b0 ? load(b0) : s;
      const Shape y = b0 ? cut_of(p, x) : o;
      const int64_t end = b0 ? scan(y) : upto;
      const uint64_t past = __ballot(by_row ? at >= x.start && at < x.start + x.n : base + end > at);
      if (past) {
        const int src = (int)__ffsll((unsigned long long)past) - 1;
        *b = b0 + src;
        seq->start = __builtin_amdgcn_readlane(x.start, src);
        seq->n = __builtin_amdgcn_readlane(x.n, src);
        seq->len = __builtin_amdgcn_readlane(x.len, src);
        cut->tiles = __builtin_amdgcn_readlane(y.tiles, src);
        cut->parts = __builtin_amdgcn_readlane(y.parts, src);
        cut->chunk = __builtin_amdgcn_readlane(y.chunk, src);
        *first = base + from_lane(end, src) - (int64_t)cut->tiles * cut->parts * p.kv_heads;
        return true;
      }
      base += from_lane(end, 63);
    }
    return false;
  }
};

// Workgroup w of n takes the units [at(w), at(w + 1)) of `all`, the first `rest` workgroups one more than the others; one each where a
// workgroup takes one.
struct Shares {
  int64_t all, each;
  int n, rest;
  bool single;
  __device__ __forceinline__ int64_t at(int w) const { return single ? w : w * each + min(w, rest); }
  __device__ __forceinline__ int holder(int64_t unit) const {
    if (__builtin_expect(single, 1)) return (int)unit;
    const int64_t larger = rest * (each + 1);
    return unit < larger ? (int)divide(unit, each + 1) : rest + (int)divide(unit - larger, each);
  }
};
__device__ __forceinline__ Shares shares_of(const Units& units) {
  Shares s = {units.all, 1, (int)min(units.all, (int64_t)units.p.units), 0, units.single};
  if (__builtin_expect(!units.single, 0)) {
    s.n = (int)max((int64_t)1, min((int64_t)units.p.target, divide(s.all, max(1, units.p.min_chunk))));
    s.each = divide(s.all, s.n);
    s.rest = (int)(s.all - s.each * s.n);
  }
  return s;
}

struct Unit {
  int b, start, n, len;  // sequence
  int head;              // key head
  int tile;              // row tile, counted from the last one
  int tiles, part, parts, chunk;  // of the sequence and head; of the item; keys of a unit
  int row0;              // first row of the tile
  int lo, hi;            // keys [lo, hi) from this unit on (hi: the item's end), lo a multiple of the key tile
};

// The first key that a row at position `at` may see (it may lie before the sequence's begin: no difference is formed that the window
// could take past 32 bits).
__device__ __forceinline__ int first_seen(const AttendParams& p, int at) { return p.window >= 0 && at > p.window ? at - p.window : 0; }

// Fills in the rows and keys of an item's unit `part`.
__device__ __forceinline__ void enter_item(const AttendParams& p, Unit* u) {
  u->row0 = (u->tiles - 1 - u->tile) << p.log_rows;
  // keys that the tile's rows see: up to the last row's end, from the first row's begin
  const int t0 = u->row0 / p.group, t1 = min(u->row0 + (1 << p.log_rows) - 1, u->n * p.group - 1) / p.group;
  const int p0 = u->len - u->n;
  const int lo = first_seen(p, p0 + (p.causal ? t0 : 0));
  const int64_t from = (int64_t)(lo & ~(p.keys - 1)) + (int64_t)u->part * u->chunk;
  u->hi = p.causal ? min(p0 + t1, u->len - 1) + 1 : u->len;
  u->lo = (int)min(from, (int64_t)kMostKeys);
}

__device__ __forceinline__ bool unit_of(const Units& units, int64_t at, Unit* u) {
  const AttendParams& p = units.p;
  Sequence s;
  Shape o;
  int64_t first;
  if (!units.find(at, false, &u->b, &s, &o, &first)) return false;
  u->start = s.start, u->n = s.n, u->len = s.len;
  const int64_t rel = at - first, item = divide(rel, o.parts);
  u->part = (int)(rel - item * o.parts);
  u->tiles = o.tiles, u->parts = o.parts, u->chunk = o.chunk;
  u->head = (int)divide(item, o.tiles);
  u->tile = (int)(item - (int64_t)u->head * o.tiles);
  enter_item(p, u);
  return true;
}

// The item after u's, at index `at`: another tile or head of the sequence, or another sequence's first.
__device__ __forceinline__ bool next_item(const Units& units, int64_t at, Unit* u) {
  if (++u->tile == u->tiles) u->tile = 0, ++u->head;
  if (u->head == units.p.kv_heads) return unit_of(units, at, u);
  u->part = 0;
  enter_item(units.p, u);
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
  s.lo = first_seen(p, p0 + (p.causal ? t : 0));
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
