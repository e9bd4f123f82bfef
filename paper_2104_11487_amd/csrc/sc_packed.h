// The cache in 4 bits: its format, parameter blocks and launchers of what works on it (host + device).
//
// A head's elements lie in groups of 32 (the last may be shorter). A token's key (value) of one key head is a row of `groups` x 16
// bytes, element e in the lower (e even) or upper half of byte e / 2, and `groups` pairs (scale, minimum) of fp16. Code c stands for
//   value = fl16(minimum + c * scale),
// an fp16 number by definition: the matrix unit takes it exactly, and every kernel that reads the cache reads the same value.
#pragma once

#include "sc_attend.h"

namespace sc {

constexpr int kPackGroup = 32;          // elements with a scale and a minimum
constexpr float kPackMost = 32768.0f;   // elements are held up to it: minimum + 15 scale stays within fp16

inline int pack_groups(int dim) { return (dim + kPackGroup - 1) / kPackGroup; }

// Scales and minima beside a CacheView whose strides count bytes. Strides in bytes.
struct ScaleView {
  char* k;
  char* v;
  int64_t k_page, k_head, k_slot, v_page, v_head, v_slot;
};

// Appending: a RotateParams whose keys and values go to codes.
struct PackParams {
  RotateParams r;
  ScaleView s;
  int tok_per_wg;  // set by the launcher
};
hipError_t launch_pack(const PackParams& p, int dtype, int wide, hipStream_t stream);

// The values of listed pages, as fp16: count x kv_heads x page_size x dim.
struct UnpackParams {
  CacheView c;
  ScaleView s;
  const int32_t* list;
  int64_t count;
  int kv_heads, dim;
  char* out[2];
};
hipError_t launch_unpack(const UnpackParams& p, hipStream_t stream);

struct PackedAttendParams {
  AttendParams a;
  ScaleView s;
  int groups;
};
constexpr int kPackedKeys = 32;      // of a key tile
constexpr int kPackedManyWaves = 4;  // of a workgroup whose waves take 16 rows each
// Few rows: a unit is 16 rows, whose keys the workgroup's waves share.
hipError_t launch_packed_few_bf16(const PackedAttendParams& p, int waves, int whole_pages, hipStream_t stream);
hipError_t launch_packed_few_f32(const PackedAttendParams& p, int waves, int whole_pages, hipStream_t stream);
hipError_t launch_packed_many_f32(const PackedAttendParams& p, int whole_pages, hipStream_t stream);
// Many rows of bf16 sharing key tiles in LDS: rows of a unit, of which heads of up to kWideDoubleDim also take twice as many; keys of a tile.
inline int log_packed_wide_rows(int dim) { return dim <= 128 ? 8 : 7; }
constexpr int packed_wide_keys(int dim) { return dim <= 64 ? 128 : 64; }
hipError_t launch_packed_wide_bf16(const PackedAttendParams& p, hipStream_t stream);

// Accumulated attention weight. The cache's keys are codes where `packed`, else of the dtype.
struct WeighParams {
  CacheView c;
  ScaleView s;
  const char* q;
  const float* lse;   // tokens x q_heads
  float* weights;     // pages x kv_heads x page_size
  int64_t q_token, q_head;
  int q_heads, kv_heads, group, dim, groups;
  int causal, window, packed, whole;  // whole: 16-key blocks lie in one page each
  float scale_log2, decay;
  int64_t tiles;      // units of a sequence and key head, at most
};
hipError_t launch_weigh(const WeighParams& p, int dtype, int split, hipStream_t stream);

// Eviction: what a token's row is made of, up to four parts of 16- or 4-byte pieces.
struct EvictPart {
  char* base;
  int64_t page, head, slot;  // bytes
  int pieces, piece_bytes;   // of a row
};
struct EvictParams {
  CacheView c;
  EvictPart part[4];
  int parts;
  float* weights;
  const int32_t* into;
  int32_t* lengths;
  int32_t* kept;             // batch x kv_heads x keep
  int kv_heads, into_width, keep, recent;
};
hipError_t launch_evict(const EvictParams& p, hipStream_t stream);

}  // namespace sc
