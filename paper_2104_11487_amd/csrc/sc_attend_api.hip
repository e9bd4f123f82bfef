// Entry points of the streaming attention operators: checks of the descriptions, the choice of kernels, workspaces.
#include <algorithm>
#include <cmath>
#include <cstdio>

#include "sc_attend.h"
#include "sc_kernels.h"
#include "skipconv.h"

namespace {

int fail(int code, const char* msg) {
  snprintf(sc::thread_error(), 256, "%s", msg);
  return code;
}
int invalid(const char* msg) { return fail(SKIPCONV_E_INVALID_ARG, msg); }

int hip_result(hipError_t e, const char* what) {
  if (e == hipSuccess) return SKIPCONV_OK;
  snprintf(sc::thread_error(), 256, "%s: %s", what, hipGetErrorString(e));
  return SKIPCONV_E_HIP;
}

constexpr int64_t kMostRows = 0x7fffffff;
// Workgroups that keep the GPU's 256 compute units busy: each holds two of the wide kernel's, one of the few-rows kernel's.
constexpr int kWantWide = 512;
constexpr int kWantFew = 256;

bool on16(const void* p) { return ((uintptr_t)p & 15) == 0; }
bool whole16(int64_t stride, int elem) { return (stride * elem) % 16 == 0; }
// The stride of a dimension of n: nothing is reached by that of one place, which a view may leave at any value.
int64_t stride_of(int64_t n, int64_t stride) { return n > 1 ? stride : 0; }

int check_rotary(const skipconv_rotary* r, int64_t tokens, int head_dim) {
  if (r->axes < 1 || r->axes > 8) return invalid("rotary: axes must be 1..8");
  if (r->pairs < 1 || r->pairs > head_dim / 2) return invalid("rotary: pairs must be 1..head_dim / 2");
  if (r->pairing != SKIPCONV_PAIR_HALVES && r->pairing != SKIPCONV_PAIR_ADJACENT)
    return invalid("rotary: pairing must be a SKIPCONV_PAIR_* value");
  if (r->inverse != 0 && r->inverse != 1) return invalid("rotary: inverse must be 0 or 1");
  if (!r->freq || (tokens > 0 && !r->pos)) return invalid("rotary: pos or freq is NULL");
  return SKIPCONV_OK;
}

// 16-byte accesses where every tensor allows them, and among those the pairing's form (see sc_rotary.hip).
int rotate_mode(bool wide, const skipconv_rotary* r, int elem, int head_dim) {
  const int v = 16 / elem;
  if (!wide || head_dim % v != 0) return 3;
  if (!r) return 0;
  if (r->pairing == SKIPCONV_PAIR_ADJACENT) return 1;
  return r->pairs % v == 0 ? 0 : 2;
}

void fill_rotary(sc::RotateParams* p, const skipconv_rotary* r) {
  p->pos = r ? r->pos : nullptr;
  p->freq = r ? r->freq : nullptr;
  p->axes = r ? r->axes : 0;
  p->pairs = r ? r->pairs : 0;
  p->adjacent = r && r->pairing == SKIPCONV_PAIR_ADJACENT;
  p->sign = r && r->inverse ? -1.0f : 1.0f;
}

int check_cache(const skipconv_cache* c, bool pointers) {
  if (c->dtype != SKIPCONV_F32 && c->dtype != SKIPCONV_BF16) return invalid("cache: unknown dtype");
  if (c->tokens < 0 || c->batch < 0) return invalid("cache: tokens and batch must be >= 0");
  if (c->kv_heads < 1 || c->pages < 1 || c->page_size < 1 || c->table_width < 1)
    return invalid("cache: kv_heads, pages, page_size and table_width must be >= 1");
  if (c->head_dim < 8 || c->head_dim > 256 || c->head_dim % 8 != 0)
    return fail(SKIPCONV_E_UNSUPPORTED, "cache: head_dim must be a multiple of 8, 8..256");
  if (c->tokens > kMostRows / std::max(1, c->kv_heads)) return fail(SKIPCONV_E_UNSUPPORTED, "cache: too many rows");
  if ((int64_t)c->table_width * c->page_size > sc::kMostKeys)
    return fail(SKIPCONV_E_UNSUPPORTED, "cache: table_width * page_size must be at most 2^30");
  const int e = c->dtype == SKIPCONV_BF16 ? 2 : 4;
  for (int64_t s : {stride_of(c->pages, c->k_page), stride_of(c->kv_heads, c->k_head), stride_of(c->page_size, c->k_slot),
                    stride_of(c->pages, c->v_page), stride_of(c->kv_heads, c->v_head), stride_of(c->page_size, c->v_slot)})
    if (s < 0 || !whole16(s, e)) return invalid("cache: strides must be >= 0 and multiples of 16 bytes");
  if (!pointers) return SKIPCONV_OK;
  if (!c->k_pages || !c->v_pages) return invalid("cache: NULL pointer");
  if (c->batch > 0 && (!c->page_table || !c->row_start || !c->kv_len)) return invalid("cache: NULL pointer");  // arrays of no element have none
  if (!on16(c->k_pages) || !on16(c->v_pages)) return invalid("cache: the pages must be 16-byte aligned");
  return SKIPCONV_OK;
}

void fill_cache(sc::CacheView* v, const skipconv_cache* c) {
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

int check_attend(const skipconv_cache* c, const skipconv_attend* a) {
  if (a->q_heads < 1 || a->q_heads % c->kv_heads != 0) return invalid("attend: q_heads must be a multiple of kv_heads");
  if (c->tokens > kMostRows / a->q_heads) return fail(SKIPCONV_E_UNSUPPORTED, "attend: too many rows");
  if (a->causal != 0 && a->causal != 1) return invalid("attend: causal must be 0 or 1");
  if (!(a->scale > 0.0f) || !std::isfinite(a->scale)) return invalid("attend: scale must be positive and finite");
  if (a->max_new < 0) return invalid("attend: max_new must be >= 0");
  return SKIPCONV_OK;
}

// The kernel and the cut of a launch, from the shapes alone (the lengths are on the device).
struct Plan {
  bool few;
  int log_rows, keys, target, min_chunk, slack, units, slots;
  size_t part_o, part_ml;
};

int plan_attend(const skipconv_cache* c, const skipconv_attend* a, Plan* p) {
  const int elem = c->dtype == SKIPCONV_BF16 ? 2 : 4, group = a->q_heads / c->kv_heads;
  const int64_t rows = c->tokens * group;  // of one key head
  const int64_t most = a->max_new > 0 ? std::min<int64_t>(a->max_new, c->tokens) : c->tokens;
  const int64_t room = (int64_t)c->table_width * c->page_size;
  const int64_t reach = std::min(room, a->window < 0 ? room : (int64_t)a->window + most);  // keys that an item may have
  const int few_waves = sc::few_waves_of(elem, c->head_dim);
  // Where no item has keys for more than four tiles a wave of the few-rows kernel, a workgroup takes one item: a join's launch would
  // cost more than shares save.
  const bool brief = reach <= 4ll * sc::few_keys_of(elem) * few_waves;
  // Items of a launch with 2^log_rows rows a tile, at most.
  const auto items = [&](int log_rows) { return ((rows >> log_rows) + std::min<int64_t>(c->batch, c->tokens)) * c->kv_heads; };
  // The few-rows kernel. bf16 heads of more than 64 leave it four waves, and the wide kernel's two workgroups a compute unit stream
  // faster (one token of 64 sequences of up to 16384, heads of 128: 226 -> 220 us) and start sooner (over 3000: 69 -> 52 us). Up to 64,
  // and fp32, which has less to gain from many rows: up to 32 rows a sequence and key head (fp32, heads of 64, one token of 19 sequences
  // over 4016: 41 -> 23 us); where keys are brief, any number of rows that a workgroup a compute unit holds (bf16, heads of 64, 24 tokens
  // over 300: 10.2 -> 8.2 us; fp32: 14 -> 11 us), and for fp32 heads of up to 96 with two row blocks a wave some more (172 tokens of 5
  // sequences over 384, heads of 64: 35 -> 17 us).
  // But bf16 items that take a second round of workgroups for a few tiles each fit the wide kernel's compute units at once (one token of
  // 39 sequences of up to 218, 8 heads of 64: 13.7 -> 9.5 us).
  const bool second_round = elem == 2 && reach <= 256 && items(sc::kLogFewRows) > kWantFew;
  const bool blocks2 = elem == 4 && c->head_dim <= sc::kFewDoubleDim && brief && items(sc::kLogFewRows) > kWantFew && most * group > 16;
  p->few = (elem == 4 || c->head_dim <= sc::kFewHalfDim) &&
           ((most * group <= 32 && !second_round) || (brief && c->head_dim <= 128 && items(sc::kLogFewRows) <= kWantFew) || (blocks2 && items(sc::kLogFewRows + 1) <= 2048));
  // 256 rows a unit read LDS less than 128, but only where they are enough to fill the GPU
  const bool twice = elem == 2 && c->head_dim <= sc::kWideDoubleDim && most * group > 128 && (rows >> (sc::kLogWideRows + 1)) * c->kv_heads >= kWantWide / 2;
  p->log_rows = p->few ? sc::kLogFewRows + blocks2 : sc::kLogWideRows + twice;
  p->keys = p->few ? sc::few_keys_of(elem) : sc::wide_keys_of(elem, c->head_dim, 1 + twice);
  int64_t units = items(p->log_rows);
  // Workgroups that share keys: `want`, or as many as all items' keys are least shares.
  const auto shares = [&](int want) {
    const int64_t tiles = (reach + 2 * p->keys - 2) / p->keys;
    return (int)std::min<int64_t>(want, units * ((tiles + p->min_chunk - 1) / p->min_chunk));
  };
  if (p->few) {
    p->min_chunk = 2 * few_waves;
    p->target = brief ? 0 : shares(kWantFew);
    p->slack = 0;
    p->slots = 2 * p->target;
  } else {
    // Keys are shared where the items leave compute units idle and a share still outweighs the join (about 7 us): a block of 32 keys
    // takes a workgroup some 0.6 us for bf16, 4 us for fp32 heads of 128. Ending one item and beginning another takes one about 4 us,
    // the slack that whole units are worth (4 sequences of 12 tokens over 8000, heads of 64: 32 -> 29 us).
    const int least = elem == 2 ? 256 : std::max(p->keys, 32 * std::max(1, 3 * 96 / c->head_dim));
    const bool shared = units < kWantWide && reach > 3 * least;
    p->min_chunk = least / p->keys;
    p->target = shared ? shares(256 * sc::wide_groups_of(elem, c->head_dim)) : 0;
    p->slack = shared ? (elem == 2 ? 256 : 64) / p->keys : 0;
    p->slots = 2 * p->target;
  }
  if (p->target) units = p->target;
  if (units > kMostRows) return fail(SKIPCONV_E_UNSUPPORTED, "attend: too many rows");
  p->units = (int)units;
  const size_t parts = (size_t)p->slots << p->log_rows;
  p->part_o = parts * c->head_dim * 4;
  p->part_ml = parts * 2 * 4;
  return SKIPCONV_OK;
}

}  // namespace

extern "C" {

int skipconv_rotate(const skipconv_rotary* r, int64_t tokens, int32_t heads, int32_t head_dim, int32_t dtype, const void* x,
                    int64_t x_token, int64_t x_head, void* y, int64_t y_token, int64_t y_head, void* stream) {
  if (!r) return invalid("rotate: rotary is NULL");
  if (dtype != SKIPCONV_F32 && dtype != SKIPCONV_BF16) return invalid("rotate: unknown dtype");
  if (tokens < 0 || heads < 0) return invalid("rotate: tokens and heads must be >= 0");
  if (head_dim < 2 || head_dim > 1024) return fail(SKIPCONV_E_UNSUPPORTED, "rotate: head_dim must be 2..1024");
  if (tokens > kMostRows / std::max(1, heads)) return fail(SKIPCONV_E_UNSUPPORTED, "rotate: too many rows");
  if (int e = check_rotary(r, tokens, head_dim)) return e;
  if (tokens == 0 || heads == 0) return SKIPCONV_OK;
  if (!x || !y) return invalid("rotate: x or y is NULL");
  if (x == y && ((tokens > 1 && x_token != y_token) || (heads > 1 && x_head != y_head)))
    return invalid("rotate: in place, x and y must have the same strides");
  if ((tokens > 1 && y_token == 0) || (heads > 1 && y_head == 0)) return invalid("rotate: rows of y overlap");
  const int elem = dtype == SKIPCONV_BF16 ? 2 : 4;
  if (((uintptr_t)x | (uintptr_t)y) % elem != 0) return invalid("rotate: x or y is not aligned to its elements");
  x_token = stride_of(tokens, x_token), x_head = stride_of(heads, x_head);
  y_token = stride_of(tokens, y_token), y_head = stride_of(heads, y_head);
  sc::RotateParams p = {};
  p.src[0] = static_cast<const char*>(x), p.src_token[0] = x_token, p.src_head[0] = x_head;
  p.dst = static_cast<char*>(y), p.dst_token = y_token, p.dst_head = y_head;
  p.heads[0] = heads;
  p.tokens = (int)tokens, p.dim = head_dim;
  fill_rotary(&p, r);
  const bool wide = on16(x) && on16(y) && whole16(x_token, elem) && whole16(x_head, elem) && whole16(y_token, elem) && whole16(y_head, elem);
  return hip_result(sc::launch_rotate(p, dtype, rotate_mode(wide, r, elem, head_dim), static_cast<hipStream_t>(stream)), "rotate launch");
}

int skipconv_cache_append(const skipconv_cache* c, const skipconv_append* a, void* stream) {
  if (!c || !a) return invalid("append: NULL description");
  if (int e = check_cache(c, true)) return e;
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
  const int elem = c->dtype == SKIPCONV_BF16 ? 2 : 4;
  if (((uintptr_t)a->k | (uintptr_t)a->v | (uintptr_t)a->q | (uintptr_t)a->q_out) % elem != 0)
    return invalid("append: a tensor is not aligned to its elements");
  sc::RotateParams p = {};
  const void* src[3] = {a->q, a->k, a->v};
  const int64_t token[3] = {stride_of(c->tokens, a->q_token), stride_of(c->tokens, a->k_token), stride_of(c->tokens, a->v_token)};
  const int64_t head[3] = {stride_of(heads, a->q_head), stride_of(c->kv_heads, a->k_head), stride_of(c->kv_heads, a->v_head)};
  bool wide = true;
  for (int i = a->q ? 0 : 1; i < 3; ++i) {
    p.src[i] = static_cast<const char*>(src[i]), p.src_token[i] = token[i], p.src_head[i] = head[i];
    wide = wide && on16(src[i]) && whole16(token[i], elem) && whole16(head[i], elem);
  }
  if (a->q) {
    p.dst = static_cast<char*>(a->q_out), p.dst_token = stride_of(c->tokens, a->q_out_token), p.dst_head = stride_of(heads, a->q_out_head);
    wide = wide && on16(a->q_out) && whole16(p.dst_token, elem) && whole16(p.dst_head, elem);
  }
  p.heads[0] = heads, p.heads[1] = p.heads[2] = c->kv_heads;
  p.tokens = (int)c->tokens, p.dim = c->head_dim;
  fill_cache(&p.cache, c);
  p.paged = 1;
  fill_rotary(&p, a->rotary);
  return hip_result(sc::launch_rotate(p, c->dtype, rotate_mode(wide, a->rotary, elem, c->head_dim), static_cast<hipStream_t>(stream)),
                    "append launch");
}

int skipconv_attend_workspace(const skipconv_cache* c, const skipconv_attend* a, size_t* bytes) {
  if (!c || !a || !bytes) return invalid("attend: NULL argument");
  if (int e = check_cache(c, false)) return e;
  if (int e = check_attend(c, a)) return e;
  Plan p;
  if (int e = plan_attend(c, a, &p)) return e;
  *bytes = c->tokens == 0 || c->batch == 0 ? 0 : p.part_o + p.part_ml;
  return SKIPCONV_OK;
}

int skipconv_cache_attend(const skipconv_cache* c, const skipconv_attend* a, void* workspace, size_t workspace_bytes, void* stream) {
  if (!c || !a) return invalid("attend: NULL description");
  if (int e = check_cache(c, true)) return e;
  if (int e = check_attend(c, a)) return e;
  if (c->tokens == 0 || c->batch == 0) return SKIPCONV_OK;
  if (!a->q || !a->out) return invalid("attend: q or out is NULL");
  const int elem = c->dtype == SKIPCONV_BF16 ? 2 : 4, group = a->q_heads / c->kv_heads;
  const int64_t q_token = stride_of(c->tokens, a->q_token), q_head = stride_of(a->q_heads, a->q_head);
  const int64_t o_token = stride_of(c->tokens, a->out_token), o_head = stride_of(a->q_heads, a->out_head);
  if (!on16(a->q) || !on16(a->out) || !whole16(q_token, elem) || !whole16(q_head, elem) || !whole16(o_token, elem) || !whole16(o_head, elem))
    return invalid("attend: q and out must be 16-byte aligned with strides of whole 16 bytes");
  if ((c->tokens > 1 && a->out_token == 0) || (a->q_heads > 1 && a->out_head == 0)) return invalid("attend: rows of out overlap");
  if ((uintptr_t)a->lse % 4 != 0) return invalid("attend: lse is not aligned to its elements");
  Plan plan;
  if (int e = plan_attend(c, a, &plan)) return e;
  if (plan.part_o + plan.part_ml > workspace_bytes)
    return fail(SKIPCONV_E_SMALL_BUFFER, "attend: workspace smaller than skipconv_attend_workspace");
  if (plan.part_o && (!workspace || !on16(workspace))) return invalid("attend: workspace must be a 16-byte aligned pointer");

  sc::AttendParams p = {};
  fill_cache(&p.c, c);
  p.q = static_cast<const char*>(a->q), p.q_token = q_token, p.q_head = q_head;
  p.out = static_cast<char*>(a->out), p.o_token = o_token, p.o_head = o_head;
  p.lse = a->lse;
  p.part_o = static_cast<float*>(workspace);
  p.part_ml = plan.part_o ? p.part_o + plan.part_o / 4 : nullptr;
  p.q_heads = a->q_heads, p.kv_heads = c->kv_heads, p.group = group, p.dim = c->head_dim;
  p.causal = a->causal;
  p.window = a->window < 0 ? -1 : a->window;
  p.scale_log2 = (float)((double)a->scale * 1.4426950408889634);
  p.log_rows = plan.log_rows, p.keys = plan.keys, p.target = plan.target, p.min_chunk = plan.min_chunk, p.slack = plan.slack, p.units = plan.units;
  p.slots = plan.slots;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t e;
  if (plan.few) {
    e = elem == 2 ? sc::launch_attend_few_bf16(p, s) : sc::launch_attend_few_f32(p, s);
  } else {
    // rows of one load of a wave: their page is looked up once where pages hold whole such groups
    int chunks = 4;
    while (chunks * 16 < ((c->head_dim + 31) / 32 * 32) * elem) chunks *= 2;
    const int rows = 64 / chunks;
    const int64_t reach = (int64_t)rows * std::max(p.c.k_slot, p.c.v_slot) * elem;
    const int64_t page_bytes = std::max(p.c.k_page, p.c.v_page) * elem;
    const int uniform = c->page_size % rows == 0 && reach < (1ll << 31) && page_bytes < (1ll << 32);
    e = elem == 2 ? sc::launch_attend_wide_bf16(p, uniform, s) : sc::launch_attend_wide_f32(p, uniform, s);
  }
  if (e == hipSuccess && plan.slots) e = sc::launch_attend_join(p, elem, s);
  return hip_result(e, "attend launch");
}

}  // extern "C"
