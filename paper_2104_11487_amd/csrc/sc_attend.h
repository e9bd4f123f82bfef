// Parameter blocks and launchers of the streaming attention operators (host + device):
// rotary positions, appending to a paged cache, attention over it.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sc {

// The paged cache and what says where a batch's tokens lie in it. Strides in elements.
struct CacheView {
  char* k;
  char* v;
  int64_t k_page, k_head, k_slot, v_page, v_head, v_slot;
  const int32_t* table;      // batch x width page numbers
  const int32_t* row_start;  // batch + 1
  const int32_t* kv_len;     // batch
  int batch, width, page_size, pages;
  uint32_t magic;            // position / page_size = umulhi(2 * position, magic) >> shift
  int shift;
  int tokens;                // rows of the new tokens' tensors
};

// position / page_size for 0 <= position < 2^31. magic = ceil(2^(31 + shift) / d) with
// 2^shift the least power of two >= d: the product's excess is below 2^31 * 2^shift / 2^(31 + shift)
// parts of 1 / d, so truncation gives the quotient.
__host__ __device__ __forceinline__ int page_of(const CacheView& c, int position) {
  return (int)((((uint64_t)(2u * (uint32_t)position) * c.magic) >> 32) >> c.shift);
}

// Heads of up to three tensors turned (or copied) in one launch: queries into a tensor, keys and values into the cache.
struct RotateParams {
  const char* src[3];
  int64_t src_token[3], src_head[3];
  char* dst;                  // of the queries
  int64_t dst_token, dst_head;
  int heads[3];
  CacheView cache;            // used where `paged`
  const int32_t* pos;         // tokens x axes
  const float* freq;          // axes x pairs; NULL = nothing turns
  int tokens, dim, axes, pairs;
  int adjacent;
  float sign;                 // -1 turns back
  int paged;                  // 1: keys and values go to the cache, and rows of no sequence are left alone
  int tok_per_wg, heads_per_wg, head_groups;  // set by the launcher
};

// dtype: SKIPCONV_*; mode: what a thread turns at a time (see sc_rotary.hip).
hipError_t launch_rotate(const RotateParams& p, int dtype, int mode, hipStream_t stream);

struct AttendParams {
  CacheView c;
  const char* q;
  char* out;
  float* lse;        // tokens x q_heads or NULL
  float* part_o;     // per unit: rows x dim
  float* part_ml;    // per unit: rows x {reference, sum}
  int64_t q_token, q_head, o_token, o_head;
  int q_heads, kv_heads, group, dim;
  int causal, window;
  float scale_log2;  // scale * log2(e)
  int log_rows;      // a unit's rows (new tokens x query heads of one key head): 2^log_rows
  int keys;          // rows of a key tile: chunks are whole tiles
  int target;        // workgroups that share all key tiles; 0: one an item
  int min_chunk;     // fewest key tiles of a share
  int slack;         // key tiles that a workgroup may have more than its equal share for the sake of taking them from one item
  int units;         // workgroups of the launch
  int slots;         // parts in the workspace, of 2^log_rows rows
};

constexpr int kMostKeys = 1 << 30;  // positions of a sequence stay below it
constexpr int kLogWideRows = 7;     // rows of a unit of the wide kernel; bf16 heads of up to kWideDoubleDim also take twice as many
constexpr int kWideDoubleDim = 64;
constexpr int kLogFewRows = 4;      // rows of a unit of the few-rows kernel; fp32 heads of up to kFewDoubleDim also take twice as many
constexpr int kMostShared = 512;    // workgroups that share a launch's keys, at most
constexpr int kFewDoubleDim = 96;
constexpr int kFewHalfDim = 64;     // largest bf16 head of the few-rows kernel

// Rows of a key tile. The wide kernel's: two buffers of keys and values take 64 KB of a workgroup's half of LDS, or more where the head
// allows no fewer than 32 rows; units of 128 rows get 64 at most. For those of 256 rows, which have long to go, a tile of 64 keys would
// wait for copies twice as often (4096 tokens over 12288 of a window, heads of 64: 441 instead of 434 us); for the others the longer
// first wait shows (12 tokens over 1500, heads of 64: 14.8 -> 16.3 us).
constexpr int wide_keys_of(int elem_bytes, int dim, int blocks) { return dim * elem_bytes > 256 ? 32 : blocks == 2 ? 128 : 64; }
// Workgroups of the wide kernel that a compute unit holds (registers, then LDS).
constexpr int wide_groups_of(int elem_bytes, int dim) { return (dim + 31) / 32 * 32 * elem_bytes <= (elem_bytes == 2 ? 256 : 384) ? 2 : 1; }
inline int few_keys_of(int elem_bytes) { return elem_bytes == 2 ? 32 : 16; }
int few_waves_of(int elem_bytes, int dim);  // waves of a workgroup of the few-rows kernel

hipError_t launch_attend_wide_bf16(const AttendParams& p, int uniform_pages, hipStream_t stream);
hipError_t launch_attend_wide_f32(const AttendParams& p, int uniform_pages, hipStream_t stream);
hipError_t launch_attend_few_bf16(const AttendParams& p, hipStream_t stream);
hipError_t launch_attend_few_f32(const AttendParams& p, hipStream_t stream);
hipError_t launch_attend_join(const AttendParams& p, int elem_bytes, int few, hipStream_t stream);  // fewer rows than `few`: a workgroup each

}  // namespace sc
