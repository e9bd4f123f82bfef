// Entry points of the cache in 4 bits, of accumulated attention weight and of eviction: checks of the descriptions, the choice of kernels.
#include "sc_attend_checks.h"
#include "sc_packed.h"

using namespace sc;

namespace {

constexpr int64_t kMostGroups = (1 << 22) - 1;  // workgroups of a launch: 1024 threads each stay under 2^32

int check_packing(const skipconv_cache* c, const skipconv_packing* s, bool pointers) {
  for (int64_t x : {stride_of(c->pages, s->ks_page), stride_of(c->kv_heads, s->ks_head), stride_of(c->page_size, s->ks_slot),
                    stride_of(c->pages, s->vs_page), stride_of(c->kv_heads, s->vs_head), stride_of(c->page_size, s->vs_slot)})
    if (x < 0 || x % 2 != 0) return invalid("packing: strides must be >= 0 and even");
  if (!pointers) return SKIPCONV_OK;
  if (!s->k_scales || !s->v_scales) return invalid("packing: NULL pointer");
  if (((uintptr_t)s->k_scales | (uintptr_t)s->v_scales) % 4 != 0) return invalid("packing: the scales must be 4-byte aligned");
  return SKIPCONV_OK;
}

void fill_packing(ScaleView* v, const skipconv_cache* c, const skipconv_packing* s) {
  v->k = static_cast<char*>(s->k_scales);
  v->v = static_cast<char*>(s->v_scales);
  v->k_page = 2 * stride_of(c->pages, s->ks_page), v->k_head = 2 * stride_of(c->kv_heads, s->ks_head), v->k_slot = 2 * stride_of(c->page_size, s->ks_slot);
  v->v_page = 2 * stride_of(c->pages, s->vs_page), v->v_head = 2 * stride_of(c->kv_heads, s->vs_head), v->v_slot = 2 * stride_of(c->page_size, s->vs_slot);
}

// The kernel and the cut of a launch, from the shapes alone (the lengths are on the device).
struct PackedPlan {
  bool few, wide;
  int waves, log_rows, keys, target, min_chunk, slack, units, slots;
  size_t part_o, part_ml;
};

int plan_packed(const skipconv_cache* c, const skipconv_attend* a, PackedPlan* p) {
  const int group = a->q_heads / c->kv_heads;
  const int64_t rows = c->tokens * group;  // of one key head
  const int64_t most = a->max_new > 0 ? std::min<int64_t>(a->max_new, c->tokens) : c->tokens;
  const int64_t room = (int64_t)c->table_width * c->page_size;
  const int64_t reach = std::min(room, a->window < 0 ? room : (int64_t)a->window + most);  // keys that an item may have
  const auto items = [&](int log_rows) { return ((rows >> log_rows) + std::min<int64_t>(c->batch, c->tokens)) * c->kv_heads; };
  // Few rows: 16 a workgroup, whose waves share the keys, while a second block of rows costs less than rows that share keys in LDS or with
  // waves of their own. 16 sequences over 4000, heads of 64: 8 rows of bf16 21 us, by the other kernel 25, 32 rows 30 and 26, but over 300 keys
  // 10 and 12, and 64 sequences over 4000 40 and 47 (64 rows: 61 and 49); of fp32, 64 rows 34 and 33, over 300 keys 10 and 18, 128 rows 40 and 41,
  // of 64 sequences 112 and 105. Larger heads, 64 sequences over 4000: of 192, bf16, 64 rows 157 and 141, over 4096 of 16 sequences 60 both, 128 rows
  // 297 and 232; of 256, 64 rows 155 and 240, 128 rows 297 and 371, of one sequence 35 and 52; of fp32, 128 rows 335 and 320, of 16 sequences 94 and 113.
  const bool half = c->dtype == SKIPCONV_BF16, large = c->head_dim > 128;
  p->few = most * group <= (half ? (c->head_dim > 192 ? 128 : large ? 64 : 32) : large ? 128 : 64);
  p->wide = !p->few && half;
  // 512 rows a unit read LDS less than 256, where they are enough to fill the GPU: 4096 rows, 8 heads of 64 over 8192 269 and 323 us, 2048 rows over
  // 4096 123 and 91.
  const bool twice = p->wide && c->head_dim <= kWideDoubleDim && most * group > 256 && items(9) >= 256;
  p->log_rows = p->few ? 4 : p->wide ? log_packed_wide_rows(c->head_dim) + twice : 6;
  p->keys = p->wide ? packed_wide_keys(c->head_dim) : kPackedKeys;
  int64_t units = items(p->log_rows);
  // Workgroups that share keys: `want`, or as many as all items' keys are least shares.
  const auto shares = [&](int want) {
    const int64_t tiles = (reach + 2 * p->keys - 2) / p->keys;
    return (int)std::min<int64_t>(want, units * ((tiles + p->min_chunk - 1) / p->min_chunk));
  };
  if (p->few) {
    // A second launch, which joins shares of keys, costs some 7 us: short items are not shared, longer ones neither where they fill the GPU. Heads of 64,
    // one token of 1 sequence over 1536: 15.2 us, shared 16.9, over 2048 17.6 and 16.8; of 128 sequences over 2048 25 and 36. Where each compute unit
    // has one item or none its workgroup is of eight waves (1024 keys: 12.6 us, of four 13.6; 256 keys: 8.7 and 7.9).
    const bool alone = reach <= (units >= 256 ? 2048 : large ? 1024 : 1536);
    p->waves = !large && alone && reach > 512 && units <= 256 ? 8 : 4;
    p->min_chunk = 8;  // 256 keys, of 4096 17.6 us, 512 19.4
    p->target = alone ? 0 : shares(large ? 256 : 512);  // workgroups that the GPU holds
    p->slack = 0;
  } else {
    // 64 rows of 8 sequences over 700, heads of 128: shared 29 us, else 33; 64 rows over 500, heads of 64, 21 and 19.
    const int want = p->wide || large ? 256 : 512;
    p->min_chunk = 256 / p->keys;
    p->target = units < want && reach > 512 ? shares(want) : 0;
    p->slack = p->target ? 256 / p->keys : 0;
  }
  p->slots = 2 * p->target;
  if (p->target) units = p->target;
  if (units > kMostGroups) return fail(SKIPCONV_E_UNSUPPORTED, "attend: too many rows");
  p->units = (int)units;
  const size_t parts = (size_t)p->slots << p->log_rows;
  p->part_o = parts * c->head_dim * 4;
  p->part_ml = parts * 2 * 4;
  return SKIPCONV_OK;
}

// Every lane's row of a 16-key block lies in the block's page, at an offset of 30 bits, and a page's stride and its slots' offsets have 32.
bool whole_pages(const CacheView& c, const ScaleView& s) {
  const int64_t slot = std::max(std::max(c.k_slot, c.v_slot), std::max(s.k_slot, s.v_slot));
  const int64_t page = std::max(std::max(c.k_page, c.v_page), std::max(s.k_page, s.v_page));
  return c.page_size % 16 == 0 && 16 * slot < (1ll << 30) && page < (1ll << 32) && c.page_size * slot < (1ll << 32);
}

int check_weigh(const skipconv_cache* c, const skipconv_weigh* w) {
  if (w->q_heads < 1 || w->q_heads % c->kv_heads != 0) return invalid("weigh: q_heads must be a multiple of kv_heads");
  if (c->tokens > (kMostRows - 1024) / w->q_heads) return fail(SKIPCONV_E_UNSUPPORTED, "weigh: too many rows");  // rows are counted ahead
  if (w->causal != 0 && w->causal != 1) return invalid("weigh: causal must be 0 or 1");
  if (!scale_ok(w->scale)) return invalid("weigh: scale must be positive and at most 2.3e38");
  if (!std::isfinite(w->decay)) return invalid("weigh: decay must be finite");
  if (w->max_new < 0) return invalid("weigh: max_new must be >= 0");
  return SKIPCONV_OK;
}

// Whether arrays of n and m 32-bit numbers share any.
bool overlap(const void* a, int64_t n, const void* b, int64_t m) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x < y + 4 * (uintptr_t)m && y < x + 4 * (uintptr_t)n;
}

int check_any_cache(const skipconv_cache* c, const skipconv_packing* s) {
  if (int e = check_cache(c, true, s ? 1 : elem_of(c))) return e;
  return s ? check_packing(c, s, true) : SKIPCONV_OK;
}

}  // namespace

extern "C" {

int skipconv_packed_append(const skipconv_cache* c, const skipconv_packing* s, const skipconv_append* a, void* stream) {
  if (!c || !s || !a) return invalid("append: NULL description");
  if (int e = check_any_cache(c, s)) return e;
  PackParams p = {};
  bool wide;
  if (int e = take_append(c, a, &p.r, &wide)) return e;
  if (p.r.tokens == 0) return SKIPCONV_OK;
  if (c->tokens > 4 * kMostGroups || p.r.heads[0] + 2ll * c->kv_heads > 1 << 16) return fail(SKIPCONV_E_UNSUPPORTED, "append: too many rows");
  fill_packing(&p.s, c, s);
  return hip_result(launch_pack(p, c->dtype, wide, static_cast<hipStream_t>(stream)), "append launch");
}

int skipconv_packed_attend_workspace(const skipconv_cache* c, const skipconv_attend* a, size_t* bytes) {
  if (!c || !a || !bytes) return invalid("attend: NULL argument");
  if (int e = check_cache(c, false, 1)) return e;
  if (int e = check_attend(c, a)) return e;
  PackedPlan p;
  if (int e = plan_packed(c, a, &p)) return e;
  *bytes = c->tokens == 0 || c->batch == 0 ? 0 : p.part_o + p.part_ml;
  return SKIPCONV_OK;
}

int skipconv_packed_attend(const skipconv_cache* c, const skipconv_packing* s, const skipconv_attend* a, void* workspace, size_t workspace_bytes, void* stream) {
  if (!c || !s || !a) return invalid("attend: NULL description");
  if (int e = check_any_cache(c, s)) return e;
  if (int e = check_attend(c, a)) return e;
  if (c->tokens == 0 || c->batch == 0) return SKIPCONV_OK;
  PackedAttendParams p = {};
  if (int e = take_attend(c, a, &p.a)) return e;
  PackedPlan plan;
  if (int e = plan_packed(c, a, &plan)) return e;
  if (plan.part_o + plan.part_ml > workspace_bytes)
    return fail(SKIPCONV_E_SMALL_BUFFER, "attend: workspace smaller than skipconv_packed_attend_workspace");
  if (plan.part_o && (!workspace || !on16(workspace))) return invalid("attend: workspace must be a 16-byte aligned pointer");
  p.a.part_o = static_cast<float*>(workspace);
  p.a.part_ml = plan.part_o ? p.a.part_o + plan.part_o / 4 : nullptr;
  p.a.log_rows = plan.log_rows, p.a.keys = plan.keys, p.a.target = plan.target, p.a.min_chunk = plan.min_chunk, p.a.slack = plan.slack;
  p.a.units = plan.units, p.a.slots = plan.slots;
  fill_packing(&p.s, c, s);
  p.groups = pack_groups(c->head_dim);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const int whole = whole_pages(p.a.c, p.s);
  const bool half = c->dtype == SKIPCONV_BF16;
  hipError_t e = plan.few    ? (half ? launch_packed_few_bf16(p, plan.waves, whole, st) : launch_packed_few_f32(p, plan.waves, whole, st))
                 : plan.wide ? launch_packed_wide_bf16(p, st) : launch_packed_many_f32(p, whole, st);
  // (512 rows of 16 sequences over 4000: a workgroup a row 22 us, lane groups 28; 2048 rows of 64 sequences over 8192 74 and 67)
  if (e == hipSuccess && plan.slots) e = launch_attend_join(p.a, elem_of(c), 1024, st);
  return hip_result(e, "attend launch");
}

int skipconv_packed_unpack(const skipconv_cache* c, const skipconv_packing* s, const int32_t* list, int64_t count, void* k, void* v, void* stream) {
  if (!c || !s) return invalid("unpack: NULL description");
  skipconv_cache pages_only = *c;  // the batch is not looked at
  pages_only.tokens = 0, pages_only.batch = 0, pages_only.table_width = 1;
  if (int e = check_any_cache(&pages_only, s)) return e;
  if (count < 0) return invalid("unpack: count must be >= 0");
  if (count > (1ll << 40) / ((int64_t)c->kv_heads * c->page_size)) return fail(SKIPCONV_E_UNSUPPORTED, "unpack: too many rows");
  if (count == 0) return SKIPCONV_OK;
  if (!list || !k || !v) return invalid("unpack: NULL pointer");
  if ((uintptr_t)list % 4 != 0 || !on16(k) || !on16(v)) return invalid("unpack: list must be 4-byte, k and v 16-byte aligned");
  UnpackParams p = {};
  fill_cache(&p.c, &pages_only);
  fill_packing(&p.s, c, s);
  p.list = list, p.count = count, p.kv_heads = c->kv_heads, p.dim = c->head_dim;
  p.out[0] = static_cast<char*>(k), p.out[1] = static_cast<char*>(v);
  return hip_result(launch_unpack(p, static_cast<hipStream_t>(stream)), "unpack launch");
}

int skipconv_cache_weigh(const skipconv_cache* c, const skipconv_packing* s, const skipconv_weigh* w, void* stream) {
  if (!c || !w) return invalid("weigh: NULL description");
  if (int e = check_any_cache(c, s)) return e;
  if (int e = check_weigh(c, w)) return e;
  if (c->tokens == 0 || c->batch == 0) return SKIPCONV_OK;
  if (!w->q || !w->lse || !w->weights) return invalid("weigh: NULL pointer");
  const int elem = elem_of(c);
  WeighParams p = {};
  p.q_token = stride_of(c->tokens, w->q_token), p.q_head = stride_of(w->q_heads, w->q_head);
  if (!on16(w->q) || !whole16(p.q_token, elem) || !whole16(p.q_head, elem)) return invalid("weigh: q must be 16-byte aligned with strides of whole 16 bytes");
  if (((uintptr_t)w->lse | (uintptr_t)w->weights) % 4 != 0) return invalid("weigh: lse or weights is not aligned to its elements");
  fill_cache(&p.c, c);
  if (s) {
    fill_packing(&p.s, c, s);
  } else {
    p.c.k_page *= elem, p.c.k_head *= elem, p.c.k_slot *= elem;
  }
  p.q = static_cast<const char*>(w->q), p.lse = w->lse, p.weights = w->weights;
  p.q_heads = w->q_heads, p.kv_heads = c->kv_heads, p.group = w->q_heads / c->kv_heads, p.dim = c->head_dim, p.groups = pack_groups(c->head_dim);
  p.causal = w->causal, p.window = w->window < 0 ? -1 : w->window, p.packed = s != nullptr;
  p.whole = c->page_size % 16 == 0 && 16 * std::max(p.c.k_slot, p.s.k_slot) < (1ll << 30) && std::max(p.c.k_page, p.s.k_page) < (1ll << 32);
  p.scale_log2 = scale_log2_of(w->scale), p.decay = w->decay;
  p.tiles = ((int64_t)c->table_width * c->page_size + 31) / 32;
  const int64_t most = w->max_new > 0 ? std::min<int64_t>(w->max_new, c->tokens) : c->tokens;
  // The waves of a workgroup share a key tile's rows where these are many, else its keys. Over 8192 keys, heads of 64 of bf16 (of 128 in 4 bits),
  // keys shared and rows shared: 128 rows of 16 sequences 24 and 30 us (40 and 75), of 4 sequences 13 and 11 (19 and 21); 512 rows of 16
  // sequences 69 and 54 (142 and 150), of 4 sequences 39 and 18 (61 and 39).
  return hip_result(launch_weigh(p, c->dtype, most * p.group > 128, static_cast<hipStream_t>(stream)), "weigh launch");
}

int skipconv_cache_evict(const skipconv_cache* c, const skipconv_packing* s, const skipconv_evict* e, void* stream) {
  if (!c || !e) return invalid("evict: NULL description");
  skipconv_cache no_rows = *c;  // the new tokens are not looked at
  no_rows.tokens = 0;
  if (!no_rows.row_start) no_rows.row_start = c->kv_len;
  if (int x = check_any_cache(&no_rows, s)) return x;
  if (e->keep < 1) return invalid("evict: keep must be >= 1");
  if (e->recent < 0 || e->recent > e->keep) return invalid("evict: recent must be 0..keep");
  if (e->into_width < 1) return invalid("evict: into_width must be >= 1");
  const int64_t room = (int64_t)c->table_width * c->page_size;
  if ((int64_t)e->into_width * c->page_size < std::min<int64_t>(e->keep, room)) return invalid("evict: into has no room for the kept tokens");
  if (c->batch == 0) return SKIPCONV_OK;
  if (!e->weights || !e->into || !e->lengths || !e->kept) return invalid("evict: NULL pointer");
  if (((uintptr_t)e->weights | (uintptr_t)e->into | (uintptr_t)e->lengths | (uintptr_t)e->kept) % 4 != 0) return invalid("evict: a tensor is not aligned to its elements");
  if ((int64_t)c->batch * c->kv_heads > kMostGroups / (std::min<int64_t>(e->keep, room) / 8 + 1)) return fail(SKIPCONV_E_UNSUPPORTED, "evict: too many rows");
  // Both launches read the lengths and tables in many workgroups: what is written must lie elsewhere.
  const int64_t places = (int64_t)c->batch * c->kv_heads * e->keep;
  const struct {
    const void* at;
    int64_t n;
  } read[] = {{c->kv_len, c->batch}, {c->page_table, (int64_t)c->batch * c->table_width}, {e->into, (int64_t)c->batch * e->into_width}};
  for (const auto& r : read)
    if (overlap(e->lengths, c->batch, r.at, r.n) || overlap(e->kept, places, r.at, r.n))
      return invalid("evict: lengths and kept must not overlap kv_len, page_table or into");
  if (overlap(e->lengths, c->batch, e->kept, places)) return invalid("evict: lengths and kept must not overlap");
  EvictParams p = {};
  fill_cache(&p.c, &no_rows);
  const int64_t unit = s ? 1 : elem_of(c);
  const int row = s ? pack_groups(c->head_dim) * 16 : c->head_dim * elem_of(c);
  const auto add = [&](char* base, int64_t page, int64_t head, int64_t slot, int bytes) {
    const bool wide = ((uintptr_t)base | (uint64_t)page | (uint64_t)head | (uint64_t)slot | (uint64_t)bytes) % 16 == 0;
    p.part[p.parts++] = {base, page, head, slot, bytes / (wide ? 16 : 4), wide ? 16 : 4};
  };
  add(p.c.k, p.c.k_page * unit, p.c.k_head * unit, p.c.k_slot * unit, row);
  add(p.c.v, p.c.v_page * unit, p.c.v_head * unit, p.c.v_slot * unit, row);
  if (s) {
    ScaleView v;
    fill_packing(&v, c, s);
    add(v.k, v.k_page, v.k_head, v.k_slot, 4 * pack_groups(c->head_dim));
    add(v.v, v.v_page, v.v_head, v.v_slot, 4 * pack_groups(c->head_dim));
  }
  p.weights = e->weights, p.into = e->into, p.lengths = e->lengths, p.kept = e->kept;
  p.kv_heads = c->kv_heads, p.into_width = e->into_width, p.keep = e->keep, p.recent = e->recent;
  return hip_result(launch_evict(p, static_cast<hipStream_t>(stream)), "evict launch");
}

}  // extern "C"
