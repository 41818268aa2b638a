// Host side of the paged KV cache: argument validation, workspace sizes and
// launches. Tables, lengths and plans stay on the GPU; every call enqueues
// kernels only.
#include "paged.h"

#include <cmath>
#include <cstring>

#include "../../include/augtree.h"
#include "host_checks.h"
#include "internal.h"
#include "kernels.h"

using namespace augtree;

namespace {

static_assert((int)CACHE_BF16 == (int)AUGTREE_CACHE_BF16 && (int)CACHE_E4M3 == (int)AUGTREE_CACHE_E4M3, "cache types");
static_assert((int)PAGES_SHORT == (int)AUGTREE_PAGES_SHORT && (int)PAGES_PAGE == (int)AUGTREE_PAGES_PAGE, "status bits");

constexpr int64_t kMaxSlots = (int64_t)1 << 30;  // of a pool; tokens of a table; (row, head) pairs of a plan

// The shape of a plan, checked.
int shape_of(const augtree_pages* p, int32_t rows, int32_t hq, int32_t hkv, PagedShape* s) {
  if (!p) return fail(AUGTREE_ERR_INVALID_ARGUMENT, "null descriptor");
  if (p->num_seqs < 1 || p->max_pages < 1 || p->num_pages < 1 || rows < 0)
    return fail(AUGTREE_ERR_INVALID_ARGUMENT, "num_seqs=%d, max_pages=%d, num_pages=%d must be >= 1, rows=%d >= 0",
                p->num_seqs, p->max_pages, p->num_pages, rows);
  if (p->page_size < 16 || p->page_size > 256 || (p->page_size & (p->page_size - 1)))
    return fail(AUGTREE_ERR_UNSUPPORTED, "page_size %d not in {16,32,64,128,256}", p->page_size);
  if ((int64_t)p->max_pages * p->page_size > kMaxSlots || (int64_t)p->num_pages * p->page_size > kMaxSlots)
    return fail(AUGTREE_ERR_UNSUPPORTED, "max_pages=%d or num_pages=%d of %d tokens pass 2^30 tokens", p->max_pages,
                p->num_pages, p->page_size);
  if (p->num_seqs > 1 << 20) return fail(AUGTREE_ERR_UNSUPPORTED, "num_seqs %d > 2^20", p->num_seqs);
  if (hq < 1 || hkv < 1) return fail(AUGTREE_ERR_INVALID_ARGUMENT, "head counts must be >= 1");
  if (hq % hkv) return fail(AUGTREE_ERR_UNSUPPORTED, "num_q_heads %d not a multiple of num_kv_heads %d", hq, hkv);
  if (hq > 65536 || (int64_t)rows * hq > kMaxSlots)
    return fail(AUGTREE_ERR_UNSUPPORTED, "%d rows of %d query heads (at most 65536, and 2^30 together)", rows, hq);
  *s = PagedShape{p->num_seqs, rows, hq, hkv, p->page_size, p->max_pages, p->num_pages};
  return AUGTREE_OK;
}

int check_tables(const augtree_pages* p, bool all) {
  int st = check_ptr(p->table, "table", true);
  if (st || !all) return st;
  if ((st = check_ptr(p->length, "length", true)) || (st = check_ptr(p->parent, "parent", false)) ||
      (st = check_ptr(p->free_pages, "free_pages", true)) || (st = check_ptr(p->free_state, "free_state", true)))
    return st;
  return AUGTREE_OK;
}

size_t plan_bytes(const PagedShape& s) { return align_up((size_t)plan_layout(s).words * 4); }

// K and V caches of a call: types, strides and places
struct Caches {
  size_t page;          // bytes of a page
  size_t k_all, v_all;  // bytes from a cache's first page to the end of its last
};

int check_caches(const PagedShape& s, int d, int type, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                 const float* k_scale, const float* v_scale, Caches* c) {
  if (d != 64 && d != 128) return fail(AUGTREE_ERR_UNSUPPORTED, "head_dim %d not in {64,128}", d);
  if (type != AUGTREE_CACHE_BF16 && type != AUGTREE_CACHE_E4M3)
    return fail(AUGTREE_ERR_INVALID_ARGUMENT, "unknown cache type %d", type);
  const Named need[] = {{k, "k_cache"}, {v, "v_cache"}};
  int st = check_all(need, 2, true);
  if (st) return st;
  if ((st = check_ptr(k_scale, "k_scale", type == AUGTREE_CACHE_E4M3, 4)) ||
      (st = check_ptr(v_scale, "v_scale", type == AUGTREE_CACHE_E4M3, 4)))
    return st;
  const int64_t page = (int64_t)s.hkv * s.page * d * (type == AUGTREE_CACHE_E4M3 ? 1 : 2);
  if (page > INT32_MAX) return fail(AUGTREE_ERR_UNSUPPORTED, "a page of %lld bytes", (long long)page);
  const int64_t strides[] = {k_stride, v_stride};
  for (int64_t b : strides) {
    if (b < page || b > (int64_t)1 << 40)
      return fail(AUGTREE_ERR_INVALID_ARGUMENT, "pages %lld bytes apart, a page has %lld", (long long)b, (long long)page);
    if (b % 16) return fail(AUGTREE_ERR_MISALIGNED, "pages %lld bytes apart, not a multiple of 16", (long long)b);
  }
  c->page = (size_t)page;
  c->k_all = (size_t)k_stride * (s.num_pages - 1) + page;
  c->v_all = (size_t)v_stride * (s.num_pages - 1) + page;
  // apart, or pages of one stride that lie between one another (views of one tensor)
  if (overlap(k, c->k_all, v, c->v_all)) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(k), b = reinterpret_cast<uintptr_t>(v);
    const int64_t off = (int64_t)((a < b ? b - a : a - b) % (uint64_t)k_stride);
    if (k_stride != v_stride || off < page || off > k_stride - page)
      return fail(AUGTREE_ERR_INVALID_ARGUMENT, "k_cache overlaps v_cache");
  }
  return AUGTREE_OK;
}

}  // namespace

extern "C" {

size_t augtree_page_plan_size(const augtree_pages* pages, int32_t rows, int32_t num_q_heads, int32_t num_kv_heads) {
  PagedShape s;
  if (shape_of(pages, rows, num_q_heads, num_kv_heads, &s)) return 0;
  fail_status(AUGTREE_OK, "");
  return plan_bytes(s);
}

int64_t augtree_page_plan_offset(const augtree_pages* pages, int32_t rows, int32_t num_q_heads, int32_t num_kv_heads,
                                 int field) {
  PagedShape s;
  if (shape_of(pages, rows, num_q_heads, num_kv_heads, &s)) return -1;
  const PlanLayout L = plan_layout(s);
  int64_t at = -1;
  switch (field) {
    case AUGTREE_PLAN_STATUS: at = PH_STATUS; break;
    case AUGTREE_PLAN_CU_ROWS: at = L.cu; break;
    case AUGTREE_PLAN_SLOTS: at = L.slots; break;
    case AUGTREE_PLAN_POSITIONS: at = L.positions; break;
    default: fail(AUGTREE_ERR_INVALID_ARGUMENT, "unknown field %d", field); return -1;
  }
  fail_status(AUGTREE_OK, "");
  return at;
}

int augtree_page_plan(const augtree_pages* pages, const int32_t* new_rows, int32_t rows, int32_t num_q_heads,
                      int32_t num_kv_heads, int32_t* length_out, int32_t* free_state_out, void* plan, size_t plan_size,
                      void* stream) {
  PagedShape s;
  int st = shape_of(pages, rows, num_q_heads, num_kv_heads, &s);
  if (st || (st = check_tables(pages, true))) return st;
  const Named need[] = {{new_rows, "new_rows"}, {length_out, "length_out"}, {free_state_out, "free_state_out"}};
  if ((st = check_all(need, 3, true))) return st;
  if (!plan || plan_size < plan_bytes(s))
    return fail(AUGTREE_ERR_WORKSPACE, "plan of %zu bytes, %zu needed", plan ? plan_size : (size_t)0, plan_bytes(s));
  if ((st = check_ptr(plan, "plan", true))) return st;
  const size_t seqs = 4 * (size_t)s.seqs;
  const Span ins[] = {{pages->length, seqs, "length", true}, {pages->parent, seqs, "parent"},
                      {pages->free_state, 8, "free_state", true}, {new_rows, seqs, "new_rows"}};
  const Span outs[] = {{pages->table, seqs * s.max_pages, "table"}, {pages->free_pages, 4 * (size_t)s.num_pages, "free_pages"},
                       {length_out, seqs, "length_out", true}, {free_state_out, 8, "free_state_out", true},
                       {plan, plan_bytes(s), "plan"}};
  if ((st = check_apart(ins, 4, outs, 5))) return st;
  // each may be the array that it follows from, not the other one's
  if (overlap(length_out, seqs, pages->free_state, 8) || overlap(free_state_out, 8, pages->length, seqs))
    return fail(AUGTREE_ERR_INVALID_ARGUMENT, "length_out overlaps free_state, or free_state_out overlaps length");
  if ((st = augtree_check_device())) return st;
  PlanParams p;
  std::memset(&p, 0, sizeof(p));
  p.s = s;
  p.L = plan_layout(s);
  p.group = num_q_heads / num_kv_heads;
  p.shift = paged_shift(s.page);
  p.table = pages->table;
  p.length = pages->length;
  p.parent = pages->parent;
  p.free_pages = pages->free_pages;
  p.state = pages->free_state;
  p.fresh = new_rows;
  p.length_out = length_out;
  p.state_out = free_state_out;
  p.plan = static_cast<int32_t*>(plan);
  // little to write: by the one workgroup that scans, else by a second launch (captured, us: 1500 rows of two sequences
  // 16.3, in two launches 18.7; 600 of 512 sequences 17.8 and 24.0, 2048 18.7 and 20.6; 4096 of two 20.6 and 18.9, of 512
  // 20.3 and 21.2)
  const bool apart = rows > 2048 || s.seqs > kFillSeqs;
  const hipStream_t str = static_cast<hipStream_t>(stream);
  Hook h("page_plan", str);
  if ((st = hip_ok(launch_page_plan(p, apart, str), "page plan launch"))) return st;
  return fail_status(AUGTREE_OK, "");
}

int augtree_cache_write(const augtree_pages* pages, const void* plan, int32_t rows, int32_t num_q_heads,
                        int32_t num_kv_heads, int32_t head_dim, const uint16_t* k, const uint16_t* v, int cache_type,
                        void* k_cache, int64_t k_page_stride, void* v_cache, int64_t v_page_stride,
                        const float* k_scale, const float* v_scale, void* stream) {
  PagedShape s;
  Caches c;
  int st = shape_of(pages, rows, num_q_heads, num_kv_heads, &s);
  if (st || (st = check_caches(s, head_dim, cache_type, k_cache, k_page_stride, v_cache, v_page_stride, k_scale, v_scale, &c)))
    return st;
  if ((st = check_ptr(plan, "plan", true))) return st;
  if ((int64_t)rows * num_kv_heads * (head_dim / 8) + 255 > UINT32_MAX)
    return fail(AUGTREE_ERR_UNSUPPORTED, "%d rows of %d KV heads exceed a launch", rows, num_kv_heads);
  if (rows == 0) return fail_status(AUGTREE_OK, "");
  const Named need[] = {{k, "k"}, {v, "v"}};
  if ((st = check_all(need, 2, true))) return st;
  const size_t kv = 2 * (size_t)rows * num_kv_heads * head_dim, heads = 4 * (size_t)num_kv_heads;
  const bool e4m3 = cache_type == AUGTREE_CACHE_E4M3;
  const Span ins[] = {{k, kv, "k"}, {v, kv, "v"}, {plan, plan_bytes(s), "plan"}, {e4m3 ? k_scale : nullptr, heads, "k_scale"},
                      {e4m3 ? v_scale : nullptr, heads, "v_scale"}};
  const Span kc[] = {{k_cache, c.k_all, "k_cache"}}, vc[] = {{v_cache, c.v_all, "v_cache"}};
  if ((st = check_apart(ins, 5, kc, 1)) || (st = check_apart(ins, 5, vc, 1)) || (st = augtree_check_device())) return st;
  CacheWriteParams p;
  std::memset(&p, 0, sizeof(p));
  p.s = s;
  p.plan = static_cast<const int32_t*>(plan);
  p.k = k;
  p.v = v;
  p.k_cache = k_cache;
  p.v_cache = v_cache;
  p.k_stride = k_page_stride;
  p.v_stride = v_page_stride;
  p.k_scale = k_scale;
  p.v_scale = v_scale;
  p.d = head_dim;
  p.type = cache_type;
  const hipStream_t str = static_cast<hipStream_t>(stream);
  Hook h("cache_write", str);
  if ((st = hip_ok(launch_cache_write(p, str), "cache write launch"))) return st;
  return fail_status(AUGTREE_OK, "");
}

size_t augtree_paged_workspace_size(const augtree_pages* pages, int32_t rows, int32_t num_q_heads, int32_t num_kv_heads,
                                    int32_t head_dim) {
  PagedShape s;
  if (shape_of(pages, rows, num_q_heads, num_kv_heads, &s)) return 0;
  if (head_dim != 64 && head_dim != 128) {
    fail(AUGTREE_ERR_UNSUPPORTED, "head_dim %d not in {64,128}", head_dim);
    return 0;
  }
  fail_status(AUGTREE_OK, "");
  const size_t pairs = (size_t)plan_layout(s).max_slots * num_kv_heads * kSlotPairs;
  return align_up(pairs * head_dim * 4) + align_up(pairs * 4);
}

int augtree_paged_fwd(const augtree_pages* pages, const void* plan, int32_t rows, int32_t num_q_heads,
                      int32_t num_kv_heads, int32_t head_dim, float softmax_scale, const uint16_t* q, int cache_type,
                      const void* k_cache, int64_t k_page_stride, const void* v_cache, int64_t v_page_stride,
                      const float* k_scale, const float* v_scale, uint16_t* o, float* lse, void* ws, size_t ws_bytes,
                      void* stream) {
  PagedShape s;
  Caches c;
  int st = shape_of(pages, rows, num_q_heads, num_kv_heads, &s);
  if (st || (st = check_tables(pages, false))) return st;
  if ((st = check_caches(s, head_dim, cache_type, k_cache, k_page_stride, v_cache, v_page_stride, k_scale, v_scale, &c)))
    return st;
  if ((st = check_ptr(plan, "plan", true))) return st;
  if (!(softmax_scale > 0.f) || !std::isfinite(softmax_scale))
    return fail(AUGTREE_ERR_INVALID_ARGUMENT, "softmax_scale must be finite and > 0");
  const PlanLayout L = plan_layout(s);
  if ((int64_t)L.max_items * s.hkv * 256 > UINT32_MAX)
    return fail(AUGTREE_ERR_UNSUPPORTED, "%d rows of %d KV heads exceed a launch", rows, num_kv_heads);
  if (rows == 0) return fail_status(AUGTREE_OK, "");
  const Named need[] = {{q, "q"}, {o, "o"}};
  const size_t want = augtree_paged_workspace_size(pages, rows, num_q_heads, num_kv_heads, head_dim);
  if ((st = check_all(need, 2, true)) || (st = check_ptr(lse, "lse", false)) || (st = check_ws(ws, ws_bytes, want))) return st;
  const size_t qb = 2 * (size_t)rows * num_q_heads * head_dim, heads = 4 * (size_t)num_kv_heads;
  const bool e4m3 = cache_type == AUGTREE_CACHE_E4M3;
  const Span ins[] = {{q, qb, "q"}, {plan, plan_bytes(s), "plan"}, {pages->table, 4 * (size_t)s.seqs * s.max_pages, "table"},
                      {k_cache, c.k_all, "k_cache"}, {v_cache, c.v_all, "v_cache"},
                      {e4m3 ? k_scale : nullptr, heads, "k_scale"}, {e4m3 ? v_scale : nullptr, heads, "v_scale"}};
  const Span outs[] = {{o, qb, "o"}, {lse, 4 * (size_t)rows * num_q_heads, "lse"}, {ws, want, "ws"}};
  if ((st = check_apart(ins, 7, outs, 3)) || (st = augtree_check_device())) return st;
  const size_t pairs = (size_t)L.max_slots * num_kv_heads * kSlotPairs;
  PagedFwdParams p;
  std::memset(&p, 0, sizeof(p));
  p.s = s;
  p.plan = static_cast<const int32_t*>(plan);
  p.table = pages->table;
  p.q = q;
  p.k_cache = k_cache;
  p.v_cache = v_cache;
  p.k_stride = k_page_stride;
  p.v_stride = v_page_stride;
  p.k_scale = k_scale;
  p.v_scale = v_scale;
  p.o = o;
  p.lse = lse;
  p.part_o = static_cast<float*>(ws);
  p.part_lse = reinterpret_cast<float*>(static_cast<char*>(ws) + align_up(pairs * head_dim * 4));
  p.scale_log2 = softmax_scale * kLog2e;
  p.d = head_dim;
  p.type = cache_type;
  p.group = num_q_heads / num_kv_heads;
  p.max_items = L.max_items;
  p.max_slots = L.max_slots;
  p.group_magic = div_magic(p.group);
  p.hkv_magic = div_magic(num_kv_heads);
  p.items_at = L.items;
  const hipStream_t str = static_cast<hipStream_t>(stream);
  {
    Hook h("paged_fwd", str);
    if ((st = hip_ok(launch_paged_fwd(p, str), "paged attention launch"))) return st;
  }
  Hook h("paged_merge", str);
  if ((st = hip_ok(launch_paged_merge(p, str), "paged merge launch"))) return st;
  return fail_status(AUGTREE_OK, "");
}

}  // extern "C"
