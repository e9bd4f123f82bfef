// Checks of the streaming attention operators' descriptions, and what the kernels take from them (host only).
#pragma once

#include <algorithm>
#include <cmath>
#include <cstdio>

#include "sc_attend.h"
#include "sc_kernels.h"
#include "skipconv.h"

namespace sc {

inline int fail(int code, const char* msg) {
  snprintf(thread_error(), 256, "%s", msg);
  return code;
}
inline int invalid(const char* msg) { return fail(SKIPCONV_E_INVALID_ARG, msg); }

inline int hip_result(hipError_t e, const char* what) {
  if (e == hipSuccess) return SKIPCONV_OK;
  snprintf(thread_error(), 256, "%s: %s", what, hipGetErrorString(e));
  return SKIPCONV_E_HIP;
}

constexpr int64_t kMostRows = 0x7fffffff;

inline bool on16(const void* p) { return ((uintptr_t)p & 15) == 0; }
inline bool whole16(int64_t stride, int elem) { return (stride * elem) % 16 == 0; }
// The stride of a dimension of n: nothing is reached by that of one place, which a view may leave at any value.
inline int64_t stride_of(int64_t n, int64_t stride) { return n > 1 ? stride : 0; }

inline int check_rotary(const skipconv_rotary* r, int64_t tokens, int head_dim) {
  if (r->axes < 1 || r->axes > 8) return invalid("rotary: axes must be 1..8");
  if (r->pairs < 1 || r->pairs > head_dim / 2) return invalid("rotary: pairs must be 1..head_dim / 2");
  if (r->pairing != SKIPCONV_PAIR_HALVES && r->pairing != SKIPCONV_PAIR_ADJACENT)
    return invalid("rotary: pairing must be a SKIPCONV_PAIR_* value");
  if (r->inverse != 0 && r->inverse != 1) return invalid("rotary: inverse must be 0 or 1");
  if (!r->freq || (tokens > 0 && !r->pos)) return invalid("rotary: pos or freq is NULL");
  return SKIPCONV_OK;
}

// 16-byte accesses where every tensor allows them, and among those the pairing's form (see sc_rotary.hip).
inline int rotate_mode(bool wide, const skipconv_rotary* r, int elem, int head_dim) {
  const int v = 16 / elem;
  if (!wide || head_dim % v != 0) return 3;
  if (!r) return 0;
  if (r->pairing == SKIPCONV_PAIR_ADJACENT) return 1;
  return r->pairs % v == 0 ? 0 : 2;
}

inline void fill_rotary(RotateParams* p, const skipconv_rotary* r) {
  p->pos = r ? r->pos : nullptr;
  p->freq = r ? r->freq : nullptr;
  p->axes = r ? r->axes : 0;
  p->pairs = r ? r->pairs : 0;
  p->adjacent = r && r->pairing == SKIPCONV_PAIR_ADJACENT;
  p->sign = r && r->inverse ? -1.0f : 1.0f;
}

// `e`: bytes of what strides count, elements or (codes of 4 bits) bytes.
inline int check_cache(const skipconv_cache* c, bool pointers, int e) {
  if (c->dtype != SKIPCONV_F32 && c->dtype != SKIPCONV_BF16) return invalid("cache: unknown dtype");
  if (c->tokens < 0 || c->batch < 0) return invalid("cache: tokens and batch must be >= 0");
  if (c->kv_heads < 1 || c->pages < 1 || c->page_size < 1 || c->table_width < 1)
    return invalid("cache: kv_heads, pages, page_size and table_width must be >= 1");
  if (c->head_dim < 8 || c->head_dim > 256 || c->head_dim % 8 != 0)
    return fail(SKIPCONV_E_UNSUPPORTED, "cache: head_dim must be a multiple of 8, 8..256");
  if (c->tokens > kMostRows / std::max(1, c->kv_heads)) return fail(SKIPCONV_E_UNSUPPORTED, "cache: too many rows");
  if ((int64_t)c->table_width * c->page_size > kMostKeys)
    return fail(SKIPCONV_E_UNSUPPORTED, "cache: table_width * page_size must be at most 2^30");
  for (int64_t s : {stride_of(c->pages, c->k_page), stride_of(c->kv_heads, c->k_head), stride_of(c->page_size, c->k_slot),
                    stride_of(c->pages, c->v_page), stride_of(c->kv_heads, c->v_head), stride_of(c->page_size, c->v_slot)})
    if (s < 0 || !whole16(s, e)) return invalid("cache: strides must be >= 0 and multiples of 16 bytes");
  if (!pointers) return SKIPCONV_OK;
  if (!c->k_pages || !c->v_pages) return invalid("cache: NULL pointer");
  if (c->batch > 0 && (!c->page_table || !c->row_start || !c->kv_len)) return invalid("cache: NULL pointer");  // arrays of no element have none
  if (!on16(c->k_pages) || !on16(c->v_pages)) return invalid("cache: the pages must be 16-byte aligned");
  return SKIPCONV_OK;
}

inline void fill_cache(CacheView* v, const skipconv_cache* c) {
  v->k = static_cast<char*>(c->k_pages);
  v->v = static_cast<char*>(c->v_pages);
  v->k_page = stride_of(c->pages, c->k_page), v->k_head = stride_of(c->kv_heads, c->k_head), v->k_slot = stride_of(c->page_size, c->k_slot);
  v->v_page = stride_of(c->pages, c->v_page), v->v_head = stride_of(c->kv_heads, c->v_head), v->v_slot = stride_of(c->page_size, c->v_slot);
  v->table = c->page_table;
  v->row_start = c->row_start;
  v->kv_len = c->kv_len;
  v->batch = c->batch;
  v->width = c->table_width;
  v->page_size = c->page_size;
  v->pages = c->pages;
  v->tokens = (int)c->tokens;
  v->shift = 0;
  while ((1ll << v->shift) < c->page_size) ++v->shift;
  v->magic = (uint32_t)(((1ull << (31 + v->shift)) + c->page_size - 1) / c->page_size);
}

// The factor of a score as the exponent of a power of two.
inline float scale_log2_of(float scale) { return (float)((double)scale * 1.4426950408889634); }
inline bool scale_ok(float scale) { return scale > 0.0f && std::isfinite(scale_log2_of(scale)); }  // infinite, it would make a score of zero NaN

inline int check_attend(const skipconv_cache* c, const skipconv_attend* a) {
  if (a->q_heads < 1 || a->q_heads % c->kv_heads != 0) return invalid("attend: q_heads must be a multiple of kv_heads");
  if (c->tokens > kMostRows / a->q_heads) return fail(SKIPCONV_E_UNSUPPORTED, "attend: too many rows");
  if (a->causal != 0 && a->causal != 1) return invalid("attend: causal must be 0 or 1");
  if (!scale_ok(a->scale)) return invalid("attend: scale must be positive and at most 2.3e38");
  if (a->max_new < 0) return invalid("attend: max_new must be >= 0");
  return SKIPCONV_OK;
}

inline int elem_of(const skipconv_cache* c) { return c->dtype == SKIPCONV_BF16 ? 2 : 4; }

// Checks an append's tensors (after the cache's) and takes them up; p->tokens stays 0 where there is nothing to do. *wide: 16-byte accesses
// reach every row.
inline int take_append(const skipconv_cache* c, const skipconv_append* a, RotateParams* p, bool* wide) {
  const int heads = a->q ? a->q_heads : 0;
  if (a->q && (a->q_heads < 1 || !a->q_out)) return invalid("append: queries need q_heads >= 1 and q_out");
  if (a->q && !a->rotary) return invalid("append: queries without a rotation");
  if (c->tokens > kMostRows / (heads + 2ll * c->kv_heads)) return fail(SKIPCONV_E_UNSUPPORTED, "append: too many rows");
  if (a->rotary)
    if (int e = check_rotary(a->rotary, c->tokens, c->head_dim)) return e;
  if (c->tokens == 0 || c->batch == 0) return SKIPCONV_OK;
  if (!a->k || !a->v) return invalid("append: k or v is NULL");
  if (a->q && a->q == a->q_out && ((c->tokens > 1 && a->q_token != a->q_out_token) || (heads > 1 && a->q_head != a->q_out_head)))
    return invalid("append: in place, q and q_out must have the same strides");
  if (a->q && ((c->tokens > 1 && a->q_out_token == 0) || (heads > 1 && a->q_out_head == 0))) return invalid("append: rows of q_out overlap");
  const int elem = elem_of(c);
  if (((uintptr_t)a->k | (uintptr_t)a->v | (uintptr_t)a->q | (uintptr_t)a->q_out) % elem != 0)
    return invalid("append: a tensor is not aligned to its elements");
  const void* src[3] = {a->q, a->k, a->v};
  const int64_t token[3] = {stride_of(c->tokens, a->q_token), stride_of(c->tokens, a->k_token), stride_of(c->tokens, a->v_token)};
  const int64_t head[3] = {stride_of(heads, a->q_head), stride_of(c->kv_heads, a->k_head), stride_of(c->kv_heads, a->v_head)};
  *wide = true;
  for (int i = a->q ? 0 : 1; i < 3; ++i) {
    p->src[i] = static_cast<const char*>(src[i]), p->src_token[i] = token[i], p->src_head[i] = head[i];
    *wide = *wide && on16(src[i]) && whole16(token[i], elem) && whole16(head[i], elem);
  }
  if (a->q) {
    p->dst = static_cast<char*>(a->q_out), p->dst_token = stride_of(c->tokens, a->q_out_token), p->dst_head = stride_of(heads, a->q_out_head);
    *wide = *wide && on16(a->q_out) && whole16(p->dst_token, elem) && whole16(p->dst_head, elem);
  }
  p->heads[0] = heads, p->heads[1] = p->heads[2] = c->kv_heads;
  p->tokens = (int)c->tokens, p->dim = c->head_dim;
  fill_cache(&p->cache, c);
  p->paged = 1;
  fill_rotary(p, a->rotary);
  return SKIPCONV_OK;
}

// Checks an attention's tensors (after its description) and takes them up.
inline int take_attend(const skipconv_cache* c, const skipconv_attend* a, AttendParams* p) {
  if (!a->q || !a->out) return invalid("attend: q or out is NULL");
  const int elem = elem_of(c);
  const int64_t q_token = stride_of(c->tokens, a->q_token), q_head = stride_of(a->q_heads, a->q_head);
  const int64_t o_token = stride_of(c->tokens, a->out_token), o_head = stride_of(a->q_heads, a->out_head);
  if (!on16(a->q) || !on16(a->out) || !whole16(q_token, elem) || !whole16(q_head, elem) || !whole16(o_token, elem) || !whole16(o_head, elem))
    return invalid("attend: q and out must be 16-byte aligned with strides of whole 16 bytes");
  if ((c->tokens > 1 && a->out_token == 0) || (a->q_heads > 1 && a->out_head == 0)) return invalid("attend: rows of out overlap");
  if ((uintptr_t)a->lse % 4 != 0) return invalid("attend: lse is not aligned to its elements");
  fill_cache(&p->c, c);
  p->q = static_cast<const char*>(a->q), p->q_token = q_token, p->q_head = q_head;
  p->out = static_cast<char*>(a->out), p->o_token = o_token, p->o_head = o_head;
  p->lse = a->lse;
  p->q_heads = a->q_heads, p->kv_heads = c->kv_heads, p->group = a->q_heads / c->kv_heads, p->dim = c->head_dim;
  p->causal = a->causal;
  p->window = a->window < 0 ? -1 : a->window;
  p->scale_log2 = scale_log2_of(a->scale);
  return SKIPCONV_OK;
}

}  // namespace sc
