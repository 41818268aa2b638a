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
  PH_STATUS, PH_TOTAL_ROWS, PH_ITEMS, PH_MERGE_ROWS, PH_MOST_PARTS, PH_PART, PH_FIRST, PH_SPARE, PH_NEED, PH_BACK, PH_FULL,
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
  // [seqs]: first row (seqs + 1 of them), tokens before and after, parent and its tokens, pages taken and given back by
  // the sequences before, run (its first sequence, or -1), rows of the run that begins here, rows merged before
  int64_t cu, cached, total, parent, a_len, need, back, run, run_rows, merge0;
  // [2 seqs], own unit and unit of the run that begins here: items with a part of C blocks before the unit's, items with
  // a tile's last part before the unit's, first slot (-1: none), parts of a tile
  int64_t full0, last0, slot0, parts;
  int64_t slots, positions;  // [rows]
  int64_t merge;             // [rows][kMergeInts]
  int64_t items;             // [max_items][kItemInts]
  int64_t words;
  int32_t max_items, max_parts, max_slots;
};
// A row that is merged: the row; then for its own unit and for its run's: slot of the row's first pair's group and that
// pair's place in it (pairs count from there on), slots of a part, parts.
constexpr int kMergeInts = 12;

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
  L.a_len = take(n);
  L.need = take(n);
  L.back = take(n);
  L.run = take(n);
  L.run_rows = take(n);
  L.merge0 = take(n);
  L.full0 = take(2 * n);
  L.last0 = take(2 * n);
  L.slot0 = take(2 * n);
  L.parts = take(2 * n);
  L.slots = take(r);
  L.positions = take(r);
  L.merge = take(r * kMergeInts);
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
  PlanLayout L;
  int32_t* table;          // [seqs][max_pages]
  const int32_t* length;   // [seqs]
  const int32_t* parent;   // [seqs] or nullptr
  int32_t* free_pages;     // [num_pages], a ring
  const int32_t* state;    // [2]: first free page in the ring, their number
  const int32_t* fresh;    // [seqs] new tokens, < 0: the sequence ends
  int32_t* length_out;
  int32_t* state_out;
  int32_t* plan;
  int32_t group, shift;    // query heads of a KV head, log2 of the page size
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
  __host__ __device__ explicit UnitView(const PlanParams& p_) : p(p_) {}
  __host__ __device__ int at(int64_t array, int i) const { return p.plan[array + i]; }
  __host__ __device__ int rows(int i) const { return at(p.L.cu, i + 1) - at(p.L.cu, i); }
  // the sequence's rows meet its parent's tokens in the unit of a run
  __host__ __device__ bool in_run(int i) const {
    const int r = at(p.L.run, i);
    return r >= 0 && at(p.L.run_rows, r) > rows(r);
  }
  // which: 0 the sequence's own unit, 1 the unit of the run that begins with it
  __host__ __device__ PagedItem unit(int i, int which) const {
    PagedItem u;
    u.row0 = at(p.L.cu, i);
    u.pair0 = 0;
    u.a_seq = u.b_seq = -1;
    u.a_len = u.b_len = u.b_pos = 0;
    u.blk0 = u.blk1 = 0;
    u.slot = -1;
    const int n = rows(i), r = at(p.L.run, i);
    const bool run = n > 0 && in_run(i);
    if (which == 0) {
      u.rows = n;
      u.b_seq = i;
      u.b_len = at(p.L.total, i);
      u.b_pos = at(p.L.cached, i);
      if (n > 0 && !run) u.a_seq = at(p.L.parent, i), u.a_len = at(p.L.a_len, i);
    } else {
      u.rows = 0;  // (a parent without tokens: nothing to meet)
      if (run && r == i && at(p.L.a_len, i) > 0)
        u.rows = at(p.L.run_rows, i), u.a_seq = at(p.L.parent, i), u.a_len = at(p.L.a_len, i);
    }
    return u;
  }
  __host__ __device__ static int blocks(const PagedItem& u) {
    return paged_div(u.a_len, kPagedBlock) + paged_div(u.b_len, kPagedBlock);
  }
  __host__ __device__ int tiles(const PagedItem& u) const { return paged_div(u.rows * p.group, kTilePairs); }
};

// Sums of counts that stop at kMostCount, so that no sequence of bad lengths overflows them.
constexpr int32_t kMostCount = 1 << 30;
inline __host__ __device__ int32_t add_count(int32_t a, int32_t b) { return a + b < kMostCount ? a + b : kMostCount; }

// The plan but for what plan_fill writes, by one team of threads: team.tid of
// team.size, barriers, exclusive scans over the threads.
template <class Team>
__host__ __device__ void plan_scan(Team& team, const PlanParams& p) {
  const PagedShape& s = p.s;
  const PlanLayout& L = p.L;
  int32_t* const plan = p.plan;
  const int g = p.group, shift = p.shift, page = s.page;
  const int per = paged_div(s.seqs, team.size());
  const int i0 = per * team.tid() < s.seqs ? per * team.tid() : s.seqs;
  const int i1 = i0 + per < s.seqs ? i0 + per : s.seqs;
  const int first = p.state[0], spare = p.state[1];
  const int most = s.max_pages << shift;
  auto pages = [&](int tokens) { return (tokens + page - 1) >> shift; };

  // a sequence's step, its numbers brought into range; bits of what is wrong with it
  struct One {
    int len, n, need, back, parent, bad;
    bool small;  // may be of a run
  };
  auto look = [&](int i) {
    One o;
    const int len = p.length[i], raw = p.fresh[i], par = p.parent ? p.parent[i] : -1;
    o.bad = len < 0 || len > most ? PAGES_LENGTH : 0;
    o.len = o.bad ? 0 : len;
    o.n = raw <= 0 ? 0 : raw < s.rows + 1 ? raw : s.rows + 1;
    if (raw > most - o.len) o.bad |= PAGES_LONG;
    o.need = pages(o.len + o.n) - pages(o.len);
    o.back = raw < 0 ? pages(o.len) : 0;
    o.parent = par < 0 || o.n == 0 ? -1 : par;
    o.small = o.parent >= 0 && (int64_t)o.n * g <= kSmallPairs;
    return o;
  };
  // of the sequences with rows: the last one's number and, where it may be of a run, its parent, for a scan of maxima
  auto key = [](int i, const One& o) { return (int64_t)(i + 1) << 32 | (uint32_t)(o.small ? o.parent + 1 : 0); };
  auto is_small = [](int64_t k) { return k > 0 && (uint32_t)k != 0; };

  // rows, pages needed and given back; what is wrong
  int bad = first < 0 || first >= s.num_pages || spare < 0 || spare > s.num_pages ? PAGES_LENGTH : 0;
  int32_t sums[3] = {0, 0, 0}, before[3], all[3];
  int64_t last = 0;
  for (int i = i0; i < i1; ++i) {
    const One o = look(i);
    bad |= o.bad;
    int a_len = 0;
    if (o.parent >= 0) {
      const int par = o.parent;
      if (par < s.seqs && par != i && p.parent[par] < 0 && p.fresh[par] >= 0) {
        const One q = look(par);
        a_len = q.len + q.n;
      } else {
        bad |= PAGES_PARENT;
      }
    }
    plan[L.cached + i] = o.len;
    plan[L.total + i] = o.len + o.n;
    plan[L.parent + i] = o.parent;
    plan[L.a_len + i] = a_len;
    sums[0] = add_count(sums[0], o.n);
    sums[1] = add_count(sums[1], o.need);
    sums[2] = add_count(sums[2], o.back);
    if (o.n > 0) last = key(i, o);
  }
  int64_t prev = last;
  team.scan_step(sums, before, all, prev, bad);  // prev: the last sequence with rows before i0
  if (all[0] > s.rows) bad |= PAGES_ROWS;
  if (all[1] > spare) bad |= PAGES_SHORT;
  if (all[2] > s.num_pages - spare) bad |= PAGES_LENGTH;

  // first row and pages of each sequence; runs: a small sequence begins one unless the nearest sequence with rows before
  // it is small and of the same parent
  int begin = -1;
  int64_t q = prev;
  for (int i = i0; i < i1; ++i) {
    const One o = look(i);
    plan[L.cu + i] = bad ? 0 : before[0];
    plan[L.need + i] = bad ? 0 : before[1];
    plan[L.back + i] = bad ? 0 : before[2];
    plan[L.run + i] = plan[L.run_rows + i] = -1;
    before[0] += o.n;
    before[1] += o.need;
    before[2] += o.back;
    if (o.n > 0) {
      const int64_t k = key(i, o);
      if (o.small && (uint32_t)q != (uint32_t)k) begin = i;
      q = k;
    }
  }
  if (team.tid() == 0) {
    const int rows = bad ? 0 : all[0];
    const int32_t head[] = {s.seqs, s.rows, s.hq, s.hkv, page, bad, rows};
    for (int k = 0; k < 7; ++k) plan[PH_SEQS + k] = head[k];
    plan[L.cu + s.seqs] = rows;
    plan[PH_FIRST] = first;
    plan[PH_SPARE] = spare;
    plan[PH_NEED] = bad ? 0 : all[1];
    plan[PH_BACK] = bad ? 0 : all[2];
  }
  int start = team.scan_max(begin);  // the last run that begins before i0
  if (!bad) {
    q = prev;
    int row = i0 < i1 ? plan[L.cu + i0] : 0;
    for (int i = i0; i < i1; ++i) {
      const One o = look(i);
      if (o.n > 0) {
        const int64_t k = key(i, o);
        const bool joins = o.small && (uint32_t)q == (uint32_t)k;
        if (is_small(q) && !joins) plan[L.run_rows + start] = row - plan[L.cu + start];
        if (o.small && !joins) start = i;
        if (o.small) plan[L.run + i] = start;
        q = k;
        row += o.n;
      }
    }
    // the run that no sequence with rows follows ends with the rows: the thread of the last sequence closes it
    if (i1 == s.seqs && i0 < i1 && is_small(q)) plan[L.run_rows + start] = all[0] - plan[L.cu + start];
  }
  team.sync();  // (nobody reads lengths and state from here on: they may be written in place)
  for (int i = i0; i < i1; ++i)
    if (!bad || p.length_out != p.length)
      p.length_out[i] = bad ? p.length[i] : p.fresh[i] < 0 ? 0 : plan[L.total + i];
  if (team.tid() == 0) {
    int to = first + (bad ? 0 : all[1]);
    p.state_out[0] = to >= s.num_pages && !bad ? to - s.num_pages : to;
    p.state_out[1] = bad ? spare : spare - all[1] + all[2];
  }

  // blocks of all tiles, and from them the length of a part
  const UnitView view(p);
  int64_t w[2] = {0, 0};
  for (int i = i0; i < i1; ++i)
    for (int which = 0; which < 2; ++which) {
      const PagedItem u = view.unit(i, which);
      const int tiles = view.tiles(u);
      w[0] += (int64_t)tiles * view.blocks(u);
      w[1] += tiles;
    }
  team.sum(w);
  const int part = part_blocks(w[0], w[1], s, L.max_parts);

  // items: the parts of full length first, then the tiles' last ones; slots of partial results; merged rows
  int32_t c[4] = {0, 0, 0, 0}, at[4], sum[4], most_parts = 0;
  for (int pass = 0; pass < 2; ++pass) {
    int32_t* const n = pass ? at : c;
    for (int i = i0; i < i1; ++i) {
      for (int which = 0; which < 2; ++which) {
        const PagedItem u = view.unit(i, which);
        const int tiles = view.tiles(u), parts = tiles ? paged_div(view.blocks(u), part) : 0;
        const bool partial = tiles && (parts > 1 || which == 1 || view.in_run(i));
        if (pass) {
          const int64_t k = 2 * (int64_t)i + which;
          plan[L.full0 + k] = n[0];
          plan[L.last0 + k] = n[1];
          plan[L.slot0 + k] = partial ? n[2] : -1;
          plan[L.parts + k] = parts;
          if (which == 0) plan[L.merge0 + i] = partial ? n[3] : -1;
        }
        if (tiles) n[0] += tiles * (parts - 1), n[1] += tiles;
        if (partial) n[2] += parts * paged_div(u.rows * g, kSlotPairs);
        if (partial && which == 0) n[3] += u.rows;
        if (partial && parts > most_parts) most_parts = parts;
      }
    }
    if (!pass) team.scan(c, at, sum);
  }
  most_parts = team.max_of(most_parts);
  if (team.tid() == 0) {
    plan[PH_PART] = part;
    plan[PH_FULL] = sum[0];
    plan[PH_ITEMS] = sum[0] + sum[1];
    plan[PH_MERGE_ROWS] = sum[3];
    plan[PH_MOST_PARTS] = most_parts;
  }
  team.sync();
}

// The last of a[0 .. n - 1], which do not decrease, that is at most x (a[0] is).
inline __host__ __device__ int last_at_most(const int32_t* a, int n, int x) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a[mid] <= x) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// The rest of the plan, by `size` threads that need not know of one another:
// rows, pages and items, each found among its sequences by bisection.
template <class Team>
__host__ __device__ void plan_fill(Team& team, const PlanParams& p, int tid, int size) {
  const PagedShape& s = p.s;
  const PlanLayout& L = p.L;
  int32_t* const plan = p.plan;
  const UnitView view(p);
  const int g = p.group, page = s.page, shift = p.shift;
  const int first = plan[PH_FIRST], spare = plan[PH_SPARE], part = plan[PH_PART], rows = plan[PH_TOTAL_ROWS];
  const int need = plan[PH_NEED], back = plan[PH_BACK], full = plan[PH_FULL], items = plan[PH_ITEMS];
  auto ring = [&](int k) { return k < s.num_pages ? k : k - s.num_pages; };

  // rows: slot, position, where the merge finds its parts
  for (int r = tid; r < s.rows; r += size) {
    int slot = -1, pos = -1;
    if (r < rows) {
      const int seq = last_at_most(plan + L.cu, s.seqs, r);
      const int off = r - plan[L.cu + seq], cached = plan[L.cached + seq], at = cached + off;
      const int have = (cached + page - 1) >> shift, k = at >> shift;
      const int id = k < have ? p.table[(int64_t)seq * s.max_pages + k] : p.free_pages[ring(first + plan[L.need + seq] + k - have)];
      if (id >= 0 && id < s.num_pages) slot = (id << shift) + (at & (page - 1));
      else team.flag(plan + PH_STATUS, PAGES_PAGE);
      pos = at + plan[L.a_len + seq];
      const int m = plan[L.merge0 + seq];
      if (m >= 0) {
        int32_t* const dst = plan + L.merge + (int64_t)(m + off) * kMergeInts;
        dst[0] = r;
        for (int u = 0; u < 2; ++u) {
          const int q = u == 0 ? seq : plan[L.run + seq];
          const int slot0 = q < 0 ? -1 : plan[L.slot0 + 2 * (int64_t)q + u];
          const int row0 = q < 0 ? 0 : plan[L.cu + q];
          const int pair = (r - row0) * g;
          dst[1 + 4 * u] = slot0 + pair / kSlotPairs;
          dst[2 + 4 * u] = pair % kSlotPairs;
          dst[3 + 4 * u] = slot0 < 0 ? 0 : paged_div((u == 0 ? view.rows(q) : plan[L.run_rows + q]) * g, kSlotPairs);
          dst[4 + 4 * u] = slot0 < 0 ? 0 : plan[L.parts + 2 * (int64_t)q + u];
        }
      }
    }
    plan[L.slots + r] = slot;
    plan[L.positions + r] = pos;
  }

  // new pages into the table, ended sequences' back to the ring
  for (int k = tid; k < need; k += size) {
    const int i = last_at_most(plan + L.need, s.seqs, k);
    const int have = (plan[L.cached + i] + page - 1) >> shift;
    p.table[(int64_t)i * s.max_pages + have + k - plan[L.need + i]] = p.free_pages[ring(first + k)];
  }
  for (int k = tid; k < back; k += size) {
    const int i = last_at_most(plan + L.back, s.seqs, k);
    p.free_pages[ring(ring(first + spare) + k)] = p.table[(int64_t)i * s.max_pages + k - plan[L.back + i]];
  }

  for (int x = tid; x < items; x += size) {
    const bool whole = x < full;  // a part of `part` blocks, not a tile's last
    const int k = whole ? x : x - full;
    const int unit = last_at_most(plan + (whole ? L.full0 : L.last0), 2 * s.seqs, k);
    PagedItem it = view.unit(unit >> 1, unit & 1);
    const int parts = plan[L.parts + unit], slot0 = plan[L.slot0 + unit];
    const int of_tile = whole ? parts - 1 : 1, j = k - plan[(whole ? L.full0 : L.last0) + unit];
    // a causal unit's last tiles have the most blocks: they come first
    const int t = view.tiles(it) - 1 - j / of_tile, c = whole ? j % of_tile : parts - 1;
    it.pair0 = t * kTilePairs;
    int end = view.blocks(it);
    if (it.b_len > 0) {  // up to what the tile's last row sees
      const int pairs = it.rows * g, lastpair = it.pair0 + kTilePairs - 1 < pairs - 1 ? it.pair0 + kTilePairs - 1 : pairs - 1;
      end = paged_div(it.a_len, kPagedBlock) + (it.b_pos + lastpair / g) / kPagedBlock + 1;
    }
    it.blk0 = (int)((int64_t)c * part < end ? (int64_t)c * part : end);
    it.blk1 = (int)((int64_t)(c + 1) * part < end ? (int64_t)(c + 1) * part : end);
    if (slot0 >= 0) it.slot = slot0 + c * paged_div(it.rows * g, kSlotPairs) + t * (kTilePairs / kSlotPairs);
    int32_t* const dst = plan + L.items + (int64_t)x * kItemInts;
    const int32_t w[kItemInts] = {it.row0, it.rows, it.pair0, it.a_seq, it.a_len, it.b_seq, it.b_len, it.b_pos,
                                  it.blk0, it.blk1, it.slot, 0, 0, 0, 0, 0};
    for (int y = 0; y < kItemInts; ++y) dst[y] = w[y];
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
