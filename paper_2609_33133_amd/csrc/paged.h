// Shared declarations of the paged KV cache: the plan of a step, its
// construction (one source for the kernel and for the host's tests), the
// kernels' parameters and launchers.
//
// A plan is an array of int32 that page_plan fills on the GPU from the tables
// and the numbers of new tokens. It names the new tokens' slots and cuts their
// attention into items, so that neither the tables nor the lengths are needed
// on the host.
//
// Attention units. A sequence's new rows against its own tokens (causal) are
// one unit; where it has a parent and many rows, or no sibling beside it, the
// unit begins with the parent's tokens. Neighbouring sequences of one parent
// with few rows each (kSmallPairs) form a run: their rows together are one
// more unit against the parent's tokens, which are then read once for all of
// them. A unit's (row, head) pairs of one KV head are cut into tiles of
// kTilePairs, its keys (in blocks of kPagedBlock) into parts of C blocks, and
// an item is one part of one tile. Rows of units with several parts, and of
// runs, leave partial results that a merge kernel joins.
#pragma once

#include <hip/hip_runtime_api.h>
#include <stdint.h>

#if !defined(__host__)  // plain C++ (the host library)
#define __host__
#define __device__
#endif

namespace augtree {

constexpr int kPagedBlock = 64;     // keys per block
constexpr int kTilePairs = 128;     // (row, head) pairs of a tile
constexpr int kSlotPairs = 32;      // pairs of a slot of partial results
// A sequence of a run has at most so many pairs: a tile's worth, from which on
// its tiles are full and reading the parent's keys once for several sequences
// saves no matrix work.
constexpr int kSmallPairs = 128;
constexpr int kChipSlots = 512;     // workgroups that the chip runs at once (two on each of 256 CUs)
constexpr int kItemInts = 16;
constexpr int kPlanHeader = 32;

// Status bits of a plan (augtree_page_status).
enum : int32_t {
  PAGES_SHORT = 1,    // the pool has fewer free pages than the step needs
  PAGES_LONG = 2,     // a sequence outgrows its table
  PAGES_ROWS = 4,     // more new tokens than the plan has rows for
  PAGES_LENGTH = 8,   // a cached length is negative or longer than the table, or the free list's state is out of range
  PAGES_PARENT = 16,  // a parent that is no sequence, is the sequence itself, has a parent or ends in this step
  PAGES_PAGE = 32,    // a page outside the pool
};

// Header words.
enum {
  PH_SEQS, PH_ROWS, PH_HQ, PH_HKV, PH_PAGE,  // what the plan was made for
  PH_STATUS, PH_TOTAL_ROWS, PH_ITEMS, PH_MERGE_ROWS, PH_PART, PH_FIRST, PH_SPARE,
};

struct PagedShape {
  int32_t seqs, rows, hq, hkv, page, max_pages, num_pages;
};

inline __host__ __device__ int paged_div(int a, int b) { return (a + b - 1) / b; }
inline __host__ __device__ int paged_shift(int page) {
  int s = 0;
  while ((1 << s) < page) ++s;
  return s;
}

// Where a plan's arrays are (in words), and the most items and slots of partial
// results it can have.
struct PlanLayout {
  // [seqs]: offsets of the rows (seqs + 1), tokens before and after, parent, first new page, first page given back,
  // run (its first sequence, or -1), rows of the run that begins here, first row that is merged
  int64_t cu, cached, total, parent, need, back, run, run_rows, merge0;
  int64_t unit;  // [2 seqs][kUnitInts]: own unit, unit of the run that begins here
  int64_t slots, positions, row_seq, merge_rows;  // [rows]
  int64_t items;                                  // [max_items][kItemInts]
  int64_t words;
  int32_t max_items, max_parts, max_slots;
};
// A unit: first item with a part of C blocks, first item with a tile's last part, first slot (-1: none), parts of a tile.
constexpr int kUnitInts = 4;

inline __host__ __device__ PlanLayout plan_layout(const PagedShape& s) {
  PlanLayout L;
  const int64_t n = s.seqs, r = s.rows, g = s.hq / s.hkv;
  int64_t at = kPlanHeader;
  auto take = [&](int64_t words) {
    const int64_t a = at;
    at += (words + 3) / 4 * 4;
    return a;
  };
  L.cu = take(n + 1);
  L.cached = take(n);
  L.total = take(n);
  L.parent = take(n);
  L.need = take(n);
  L.back = take(n);
  L.run = take(n);
  L.run_rows = take(n);
  L.merge0 = take(n);
  L.unit = take(2 * n * kUnitInts);
  L.slots = take(r);
  L.positions = take(r);
  L.row_seq = take(r);
  L.merge_rows = take(r);
  // Every sequence with rows has one tile that may not be full, every run (two sequences or more) one, and parts of
  // C >= all blocks / max_parts blocks are at most max_parts more items. Slots: one per 32 pairs of the units of runs
  // and of their sequences' own; a unit with parts has at most 2 blocks / C of them, of four slots each.
  const int64_t live = n < r ? n : r;
  const int64_t few = g > kSmallPairs ? 0 : (r < live * (kSmallPairs / g) ? r : live * (kSmallPairs / g));
  L.max_parts = 2 * kChipSlots / s.hkv > 1 ? 2 * kChipSlots / s.hkv : 1;
  L.max_items = (int32_t)(r * g / kTilePairs + live + few * g / kTilePairs + live / 2 + L.max_parts);
  L.max_slots = (int32_t)(2 * (few * g / kSlotPairs) + live + live / 2 + 8 * L.max_parts);
  L.items = take((int64_t)L.max_items * kItemInts);
  L.words = at;
  return L;
}

// One item: rows row0 .. of the unit, pairs pair0 .. pair0 + 127 of its
// rows * group; blocks blk0 .. blk1 - 1 of segment A (a_len tokens of sequence
// a_seq, every one visible) and then segment B (b_len tokens of b_seq; row i
// sees those up to b_pos + i); first slot of partial results, or -1: the
// item's results are final.
struct PagedItem {
  int32_t row0, rows, pair0;
  int32_t a_seq, a_len, b_seq, b_len, b_pos;
  int32_t blk0, blk1, slot;
  int32_t pad[5];
};
static_assert(sizeof(PagedItem) == 4 * kItemInts, "item layout");

// ---------------------------------------------------------------------------- construction

struct PlanParams {
  PagedShape s;
  int32_t* table;          // [seqs][max_pages]
  const int32_t* length;   // [seqs]
  const int32_t* parent;   // [seqs] or nullptr
  int32_t* free_pages;     // [num_pages], a ring
  const int32_t* state;    // [2]: first free page in the ring, their number
  const int32_t* fresh;    // [seqs] new tokens, < 0: the sequence ends
  int32_t* length_out;
  int32_t* state_out;
  int32_t* plan;
};

// Blocks of the parts that units are cut into, from the blocks of all tiles
// (each with the blocks of its unit) and the number of tiles, per KV head.
// Few tiles: as many parts as run at once. More of them: parts of half of what
// a slot of the chip has to do, so that items of different lengths fill it.
inline __host__ __device__ int part_blocks(int64_t blocks, int64_t tiles, const PagedShape& s, int max_parts) {
  const int64_t slots = kChipSlots / s.hkv > 1 ? kChipSlots / s.hkv : 1;
  int64_t c;
  if (tiles * 4 < slots) c = (blocks + slots - tiles - 1) / (slots - tiles);
  else c = (blocks + 2 * slots - 1) / (2 * slots) > 8 ? (blocks + 2 * slots - 1) / (2 * slots) : 8;
  const int64_t least = (blocks + max_parts - 1) / max_parts;
  if (c < least) c = least;
  return c < 1 ? 1 : c > INT32_MAX ? INT32_MAX : (int)c;
}

// What a sequence's units are, from the plan's arrays.
struct UnitView {
  const PlanParams& p;
  const PlanLayout& L;
  int g;
  __host__ __device__ UnitView(const PlanParams& p_, const PlanLayout& L_) : p(p_), L(L_), g(p_.s.hq / p_.s.hkv) {}
  __host__ __device__ int rows(int i) const { return p.plan[L.cu + i + 1] - p.plan[L.cu + i]; }
  __host__ __device__ bool small(int i) const {
    const int n = rows(i);
    return n > 0 && p.plan[L.parent + i] >= 0 && (int64_t)n * g <= kSmallPairs;
  }
  // the sequence's rows meet its parent's tokens in the run's unit
  __host__ __device__ bool in_run(int i) const {
    const int r = p.plan[L.run + i];
    return r >= 0 && p.plan[L.run_rows + r] > rows(r);
  }
  // which: 0 the sequence's own unit, 1 the unit of the run that begins with it
  __host__ __device__ PagedItem unit(int i, int which) const {
    PagedItem u;
    u.row0 = p.plan[L.cu + i];
    u.pair0 = 0;
    u.a_seq = u.b_seq = -1;
    u.a_len = u.b_len = u.b_pos = 0;
    u.blk0 = u.blk1 = 0;
    u.slot = -1;
    const int par = p.plan[L.parent + i];
    if (which == 0) {
      u.rows = rows(i);
      u.b_seq = i;
      u.b_len = p.plan[L.total + i];
      u.b_pos = p.plan[L.cached + i];
      if (par >= 0 && u.rows > 0 && !in_run(i)) u.a_seq = par, u.a_len = p.plan[L.total + par];
    } else {
      u.rows = 0;  // (a parent without tokens: nothing to meet)
      if (p.plan[L.run + i] == i && in_run(i) && p.plan[L.total + par] > 0)
        u.rows = p.plan[L.run_rows + i], u.a_seq = par, u.a_len = p.plan[L.total + par];
    }
    return u;
  }
  __host__ __device__ static int blocks(const PagedItem& u) {
    return paged_div(u.a_len, kPagedBlock) + paged_div(u.b_len, kPagedBlock);
  }
  __host__ __device__ int tiles(const PagedItem& u) const { return paged_div(u.rows * g, kTilePairs); }
  __host__ __device__ bool partial(const PagedItem& u, int i, int which, int parts) const {
    return parts > 1 || which == 1 || (u.rows > 0 && in_run(i));
  }
};

// The plan but for what plan_fill writes, by one team of threads: team.tid of
// team.size, barriers, exclusive scans over the threads.
template <class Team>
__host__ __device__ void plan_scan(Team& team, const PlanParams& p) {
  const PagedShape& s = p.s;
  const PlanLayout L = plan_layout(s);
  int32_t* const plan = p.plan;
  const int g = s.hq / s.hkv, page = s.page;
  const int per = paged_div(s.seqs, team.size());
  const int i0 = per * team.tid() < s.seqs ? per * team.tid() : s.seqs;
  const int i1 = i0 + per < s.seqs ? i0 + per : s.seqs;
  const int first = p.state[0], spare = p.state[1];
  const int64_t most = (int64_t)s.max_pages * page;

  // rows, pages needed and given back; what is wrong
  int bad = first < 0 || first >= s.num_pages || spare < 0 || spare > s.num_pages ? PAGES_LENGTH : 0;
  int64_t sums[3] = {0, 0, 0}, before[3], all[3];
  for (int i = i0; i < i1; ++i) {
    const int64_t len = p.length[i], raw = p.fresh[i], n = raw > 0 ? raw : 0;
    int par = p.parent ? p.parent[i] : -1;
    if (len < 0 || len > most) bad |= PAGES_LENGTH;
    else if (len + n > most) bad |= PAGES_LONG;
    int64_t total = len + n;
    if (par >= 0 && n > 0) {
      const bool ok = par < s.seqs && par != i && p.parent[par] < 0 && p.fresh[par] >= 0;
      if (!ok) bad |= PAGES_PARENT;
    }
    plan[L.parent + i] = par < 0 || n == 0 ? -1 : par;
    plan[L.cached + i] = (int32_t)len;
    plan[L.total + i] = (int32_t)(total > INT32_MAX ? INT32_MAX : total);
    sums[0] += n;
    sums[1] += (total + page - 1) / page - (len + page - 1) / page;
    sums[2] += raw < 0 && len > 0 ? (len + page - 1) / page : 0;
  }
  team.template scan<3>(sums, before, all);
  if (all[0] > s.rows) bad |= PAGES_ROWS;
  if (all[1] > spare) bad |= PAGES_SHORT;
  if (all[2] > s.num_pages - spare) bad |= PAGES_LENGTH;
  bad = team.any(bad);
  for (int i = i0; i < i1; ++i) {
    const int64_t len = p.length[i], raw = p.fresh[i], n = bad ? 0 : raw > 0 ? raw : 0;
    plan[L.cu + i] = bad ? 0 : (int32_t)before[0];
    plan[L.need + i] = bad ? 0 : (int32_t)before[1];
    plan[L.back + i] = bad ? -1 : (raw < 0 ? (int32_t)before[2] : -1);
    before[0] += n;
    before[1] += (len + n + page - 1) / page - (len + page - 1) / page;
    before[2] += raw < 0 && len > 0 ? (len + page - 1) / page : 0;
    plan[L.run + i] = plan[L.run_rows + i] = -1;
    if (bad) plan[L.cached + i] = plan[L.total + i] = 0, plan[L.parent + i] = -1;
  }
  if (team.tid() == 0) {
    plan[L.cu + s.seqs] = bad ? 0 : (int32_t)all[0];
    plan[PH_SEQS] = s.seqs;
    plan[PH_ROWS] = s.rows;
    plan[PH_HQ] = s.hq;
    plan[PH_HKV] = s.hkv;
    plan[PH_PAGE] = page;
    plan[PH_STATUS] = bad;
    plan[PH_TOTAL_ROWS] = bad ? 0 : (int32_t)all[0];
    plan[PH_FIRST] = first;
    plan[PH_SPARE] = spare;
  }
  team.sync();  // (lengths and state may be written in place from here on)
  for (int i = i0; i < i1; ++i)
    p.length_out[i] = bad ? p.length[i] : p.fresh[i] < 0 ? 0 : plan[L.total + i];
  if (team.tid() == 0) {
    p.state_out[0] = bad ? first : (int32_t)((first + all[1]) % s.num_pages);
    p.state_out[1] = bad ? spare : (int32_t)(spare - all[1] + all[2]);
  }

  // runs: a small sequence begins one unless the nearest sequence with rows before it is small and of the same parent
  const UnitView view(p, L);
  int last = -1;
  for (int i = i0; i < i1; ++i)
    if (view.rows(i) > 0) last = i;
  int prev = team.scan_max(last);  // nearest sequence with rows before i0
  int begin = -1, q = prev;
  for (int i = i0; i < i1; ++i) {
    if (view.rows(i) == 0) continue;
    if (view.small(i) && !(q >= 0 && view.small(q) && plan[L.parent + q] == plan[L.parent + i])) begin = i;
    q = i;
  }
  int start = team.scan_max(begin);  // the last run that begins before i0
  q = prev;
  for (int i = i0; i < i1; ++i) {
    if (view.rows(i) == 0) continue;
    const bool small = view.small(i), before_small = q >= 0 && view.small(q);
    const bool joins = small && before_small && plan[L.parent + q] == plan[L.parent + i];
    if (before_small && !joins) plan[L.run_rows + start] = plan[L.cu + i] - plan[L.cu + start];
    if (small && !joins) start = i;
    if (small) plan[L.run + i] = start;
    q = i;
  }
  // the run that no sequence with rows follows ends with the rows: the thread of the last sequence closes it
  if (i1 == s.seqs && i0 < i1 && q >= 0 && view.small(q)) plan[L.run_rows + start] = plan[L.cu + s.seqs] - plan[L.cu + start];
  team.sync();

  // blocks of all tiles, and from them the length of a part
  int64_t w[2] = {0, 0}, w_before[2], w_all[2];
  for (int i = i0; i < i1; ++i)
    for (int which = 0; which < 2; ++which) {
      const PagedItem u = view.unit(i, which);
      const int tiles = view.tiles(u);
      w[0] += (int64_t)tiles * view.blocks(u);
      w[1] += tiles;
    }
  team.template scan<2>(w, w_before, w_all);
  const int part = part_blocks(w_all[0], w_all[1], s, L.max_parts);

  // items: the parts of full length first, then the tiles' last ones; slots of partial results; merged rows
  int64_t c[4] = {0, 0, 0, 0}, at[4], sum[4];
  for (int pass = 0; pass < 2; ++pass) {
    for (int i = i0; i < i1; ++i) {
      bool merged = false;
      for (int which = 0; which < 2; ++which) {
        const PagedItem u = view.unit(i, which);
        const int tiles = view.tiles(u), parts = tiles ? paged_div(view.blocks(u), part) : 0;
        const bool partial = tiles && view.partial(u, i, which, parts);
        int32_t* const to = plan + L.unit + (2 * (int64_t)i + which) * kUnitInts;
        if (pass) {
          to[0] = (int32_t)at[0];
          to[1] = (int32_t)(sum[0] + at[1]);
          to[2] = partial ? (int32_t)at[2] : -1;
          to[3] = parts;
          if (which == 0) plan[L.merge0 + i] = partial ? (int32_t)at[3] : -1;
        }
        int64_t* const n = pass ? at : c;
        if (tiles) n[0] += (int64_t)tiles * (parts - 1), n[1] += tiles;
        if (partial) n[2] += (int64_t)parts * paged_div(u.rows * g, kSlotPairs);
        if (which == 0) merged = partial;
      }
      if (merged) (pass ? at : c)[3] += view.rows(i);
    }
    if (!pass) team.template scan<4>(c, at, sum);
  }
  if (team.tid() == 0) {
    plan[PH_PART] = part;
    plan[PH_ITEMS] = (int32_t)(sum[0] + sum[1]);
    plan[PH_MERGE_ROWS] = (int32_t)sum[3];
  }
  team.sync();
}

// The rest of the plan, by `size` threads in wavefronts of `lanes` that need
// not know of one another.
template <class Team>
__host__ __device__ void plan_fill(Team& team, const PlanParams& p, int64_t tid, int64_t size, int lanes) {
  const PagedShape& s = p.s;
  const PlanLayout L = plan_layout(s);
  int32_t* const plan = p.plan;
  const UnitView view(p, L);
  const int g = s.hq / s.hkv, page = s.page, shift = paged_shift(page);
  const int first = plan[PH_FIRST], spare = plan[PH_SPARE], part = plan[PH_PART], rows = plan[PH_TOTAL_ROWS];
  auto ring = [&](int64_t k) { return (int)(k % s.num_pages); };

  // rows: sequence, slot, position; the list of rows to merge
  for (int64_t r = tid; r < s.rows; r += size) {
    int seq = -1, slot = -1, pos = -1;
    if (r < rows) {
      int lo = 0, hi = s.seqs - 1;  // the last sequence that begins at or before r: the one with rows
      while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (plan[L.cu + mid] <= r) lo = mid;
        else hi = mid - 1;
      }
      seq = lo;
      const int off = (int)r - plan[L.cu + seq], cached = plan[L.cached + seq], at = cached + off;
      const int have = (cached + page - 1) >> shift, k = at >> shift;
      const int id = k < have ? p.table[(int64_t)seq * s.max_pages + k]
                              : p.free_pages[ring((int64_t)first + plan[L.need + seq] + k - have)];
      if (id >= 0 && id < s.num_pages) slot = (id << shift) + (at & (page - 1));
      else team.flag(plan + PH_STATUS, PAGES_PAGE);
      const int par = plan[L.parent + seq];
      pos = at + (par >= 0 ? plan[L.total + par] : 0);
      const int m = plan[L.merge0 + seq];
      if (m >= 0) plan[L.merge_rows + m + off] = (int)r;
    }
    plan[L.slots + r] = slot;
    plan[L.positions + r] = pos;
    plan[L.row_seq + r] = seq;
  }

  // sequences, a wavefront each: new pages into the table, ended ones' back to the ring, items
  const int lane = (int)(tid % lanes);
  for (int64_t i = tid / lanes; i < s.seqs; i += size / lanes) {
    const int cached = plan[L.cached + i], have = (cached + page - 1) >> shift;
    int32_t* const row = p.table + i * s.max_pages;
    if (view.rows((int)i) > 0) {
      const int want = (plan[L.total + i] + page - 1) >> shift, need = plan[L.need + i];
      for (int k = have + lane; k < want; k += lanes) row[k] = p.free_pages[ring((int64_t)first + need + k - have)];
    }
    const int back = plan[L.back + i];
    if (back >= 0)
      for (int k = lane; k < have; k += lanes) p.free_pages[ring((int64_t)first + spare + back + k)] = row[k];
    for (int which = 0; which < 2; ++which) {
      const int32_t* const at = plan + L.unit + (2 * i + which) * kUnitInts;
      const PagedItem u = view.unit((int)i, which);
      const int tiles = view.tiles(u), parts = at[3], slots = paged_div(u.rows * g, kSlotPairs);
      for (int k = lane; k < tiles * parts; k += lanes) {
        // a causal unit's last tiles have the most blocks: they come first
        const int t = tiles - 1 - k / parts, c = k % parts;
        PagedItem it = u;
        it.pair0 = t * kTilePairs;
        int end = view.blocks(u);
        if (u.b_len > 0) {  // up to what the tile's last row sees
          const int pairs = u.rows * g, lastpair = it.pair0 + kTilePairs - 1 < pairs - 1 ? it.pair0 + kTilePairs - 1 : pairs - 1;
          end = paged_div(u.a_len, kPagedBlock) + (u.b_pos + lastpair / g) / kPagedBlock + 1;
        }
        it.blk0 = (int)((int64_t)c * part < end ? (int64_t)c * part : end);
        it.blk1 = (int)((int64_t)(c + 1) * part < end ? (int64_t)(c + 1) * part : end);
        if (at[2] >= 0) it.slot = at[2] + c * slots + t * (kTilePairs / kSlotPairs);
        const int to = c < parts - 1 ? at[0] + (k / parts) * (parts - 1) + c : at[1] + k / parts;
        int32_t* const dst = plan + L.items + (int64_t)to * kItemInts;
        const int32_t w[kItemInts] = {it.row0, it.rows, it.pair0, it.a_seq, it.a_len, it.b_seq, it.b_len, it.b_pos,
                                      it.blk0, it.blk1, it.slot, 0, 0, 0, 0, 0};
        for (int j = 0; j < kItemInts; ++j) dst[j] = w[j];
      }
    }
  }
}

// ---------------------------------------------------------------------------- launchers

// How a cache holds its values.
enum : int { CACHE_BF16 = 0, CACHE_E4M3 = 1 };

hipError_t launch_page_plan(const PlanParams& p, bool apart, hipStream_t stream);

struct CacheWriteParams {
  PagedShape s;
  const int32_t* plan;
  const uint16_t *k, *v;            // [rows][hkv][d]
  void *k_cache, *v_cache;          // [num_pages][hkv][page][d], pages `k_stride` (`v_stride`) bytes apart
  int64_t k_stride, v_stride;
  const float *k_scale, *v_scale;   // [hkv] (CACHE_E4M3)
  int32_t d, type;
};
hipError_t launch_cache_write(const CacheWriteParams& p, hipStream_t stream);

struct PagedFwdParams {
  PagedShape s;
  const int32_t* plan;
  const int32_t* table;
  const uint16_t* q;                // [rows][hq][d]
  const void *k_cache, *v_cache;
  int64_t k_stride, v_stride;
  const float *k_scale, *v_scale;
  uint16_t* o;                      // [rows][hq][d]
  float* lse;                       // [hq][rows] or nullptr
  float* part_o;                    // [max_slots][hkv][32][d]
  float* part_lse;                  // [max_slots][hkv][32]
  float scale_log2;
  int32_t d, type, group, max_items, max_slots;
  uint32_t group_magic, hkv_magic;
  int64_t items_at;                 // PlanLayout::items
};
hipError_t launch_paged_fwd(const PagedFwdParams& p, hipStream_t stream);
hipError_t launch_paged_merge(const PagedFwdParams& p, hipStream_t stream);

}  // namespace augtree
