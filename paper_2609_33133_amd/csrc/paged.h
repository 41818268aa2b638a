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
// kTilePairs, its keys (in blocks of kPagedBlock) into as few equal parts as
// none of them passes C blocks, and an item is one part of one tile. (Parts of
// C blocks and a shorter last one: a chunk of 1500 and 48 single tokens on two
// KV heads 75 us, with equal ones 72.) Rows of units with several parts, and of
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
// saves no matrix work. 16 branches of a prompt of 16000, 32 / 8 heads, us: nine
// tokens each (36 pairs) 60, as units of their own (a limit of 32) 116; 16 tokens
// 90 and 118; 48 tokens 267, in a run (a limit of 512) 218, but of a prompt of 700
// 23 and 37. Between 65 and 128 pairs a run does not pay everywhere: 32 tokens 162,
// with a limit of 64 154; eight trees of four branches of 32 tokens over 3000 90
// and 68.
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
  PH_SEQS, PH_ROWS, PH_HQ, PH_HKV, PH_PAGE, PH_MAX_PAGES, PH_NUM_PAGES,  // what the plan was made for (PagedShape)
  PH_STATUS, PH_TOTAL_ROWS, PH_ITEMS, PH_MERGE_ROWS, PH_MOST_PARTS, PH_FIRST, PH_SPARE, PH_NEED, PH_BACK, PH_BIG,
};

struct PagedShape {
  int32_t seqs, rows, hq, hkv, page, max_pages, num_pages;
};

// Whether a plan was made for these sizes: a caller may hand over another's.
// (Without branches: the words come by one load, not one after the other.)
inline __host__ __device__ bool plan_is_for(const int32_t* plan, const PagedShape& s) {
  return ((plan[PH_SEQS] ^ s.seqs) | (plan[PH_ROWS] ^ s.rows) | (plan[PH_HQ] ^ s.hq) | (plan[PH_HKV] ^ s.hkv) |
          (plan[PH_PAGE] ^ s.page) | (plan[PH_MAX_PAGES] ^ s.max_pages) | (plan[PH_NUM_PAGES] ^ s.num_pages)) == 0;
}

inline __host__ __device__ int paged_div(int a, int b) { return (a + b - 1) / b; }
inline __host__ __device__ int paged_shift(int page) {
  int s = 0;
  while ((1 << s) < page) ++s;
  return s;
}

// Where a plan's arrays are (in words), and the most items and slots of partial
// results it can have.
struct PlanLayout {
  int64_t cu;                // [seqs + 1] first row
  // work: what the construction keeps (PlanArrays). Of each sequence: first row, tokens before and after, parent and its
  // tokens, pages taken and given back by the sequences before, run (its first sequence, or -1), rows of the run that
  // begins here, rows merged before. Of its own unit and of the unit of the run that begins here: items of units with
  // long parts before the unit's, items of the others before the unit's, first slot (-1: none), parts of a tile.
  int64_t work;
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
  L.work = take(18 * n + 1);
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

// What a plan's tiles come to, per KV head: blocks of those of more than 32
// pairs, of those of at most 32, tiles.
struct TileSums {
  int64_t wide, few, tiles;
};

// The most blocks of the parts that units are cut into (each tile counts with the blocks
// of its unit).
// Fewer tiles than the chip runs at once: as many parts as it does, each tile's
// last one short; but parts of at most twice an even share, so that a few long
// tiles among many short ones are still cut. Nothing limits parts from below
// there. Tiles of at most 32 pairs are bound by the reading of
// their keys, which one workgroup a CU does as fast as two, with half the parts
// to join. More tiles: parts of half of what a slot of the chip has to do, so
// that items of different lengths fill it. (As many parts as make the rounds of the
// chip shortest, counting 3 blocks' time for a part and 6 for its results in memory,
// gained nothing on chunks of 1024 to 6000 tokens, 820 to 1180 TFLOP/s either way.)
// Against the best of half a dozen lengths each, with items in the order of their
// sequences, us: one sequence of 4097 tokens
// 13.4 (13.4), eight branches of a 32768-token prompt 29 (29; with two workgroups
// a CU 32), 256 sequences of 500 to 8000 274 (273), 512 branches in e4m3 236 (231),
// a chunk of 1500 and 48 single tokens on two KV heads 75 (70), two chunks of 7777
// together 1647 (1647). With many tiles a part has eight blocks at least: 64
// sequences' nine tokens over 250 to 500, 32 / 8 heads, 29 us, with three 40, with
// 16 29; over 450 to 900 55, 57 and 45; 16 prompts of 600 to 1200 from nothing 153,
// 148 and 152.
// A tile of a causal unit counts with all blocks of its unit, also those behind
// its last row, and has as many parts: those behind its end are empty, write
// zeros and are joined with weight 0 (a prompt of 1024 from nothing, 8 / 2 heads:
// 90 of 192 items of a KV head).
// Items of at least `big` blocks, the mean, are launched before the others, so
// that the last round of the chip is made of short ones: 256 sequences of 500 to
// 8000 tokens 274 -> 268 us, 512 branches in e4m3 236 -> 225, 16 turns of 150 to
// 700 805 -> 790.
struct Cut {
  int part, big;
};
inline __host__ __device__ Cut part_blocks(const TileSums& w, const PagedShape& s, int max_parts) {
  const int slots = kChipSlots / s.hkv > 1 ? kChipSlots / s.hkv : 1;
  const int64_t blocks = w.wide + w.few;
  // (the GPU has no 64-bit division: of more than 2^31 blocks in thousands, rounded up)
  auto ceil_div = [](int64_t n, int d) {
    if (n <= INT32_MAX - 4096) return (int)(((uint32_t)n + (uint32_t)d - 1) / (uint32_t)d);
    const int64_t k = (n >> 10) + 1;
    const uint32_t q = ((uint32_t)(k < INT32_MAX ? k : INT32_MAX) + (uint32_t)d - 1) / (uint32_t)d;
    return q < INT32_MAX >> 10 ? (int)(q << 10) : (int)INT32_MAX;
  };
  const int once = w.few > w.wide && slots > 1 ? slots / 2 : slots;
  int c;
  if (w.tiles < once) {
    c = ceil_div(blocks, once - (int)w.tiles);
    const int share = ceil_div(blocks, once);
    if (c > 2 * (int64_t)share) c = 2 * share;
  } else {
    c = ceil_div(blocks, 2 * slots);
    if (c < 8) c = 8;
  }
  const int least = ceil_div(blocks, max_parts);
  if (c < least) c = least;
  if (c < 1) c = 1;
  const int mean = w.tiles > 0 && w.tiles <= INT32_MAX ? ceil_div(blocks, (int)w.tiles) : 1;
  return Cut{c, mean <= c ? mean : (c + 1) / 2};
}

// The arrays that the construction works on: the plan's, or copies in faster
// memory where the same workgroup writes all of the plan.
struct PlanArrays {
  int32_t *cu, *cached, *total, *parent, *a_len, *need, *back, *run, *run_rows, *merge0, *big0, *rest0, *slot0, *parts;
  __host__ __device__ static int64_t words(int64_t seqs) { return 18 * seqs + 1; }
  // one after the other, in `words` words
  __host__ __device__ static PlanArrays packed(int32_t* at, int n) {
    PlanArrays a;
    a.cu = at;
    a.cached = a.cu + n + 1;
    a.total = a.cached + n;
    a.parent = a.total + n;
    a.a_len = a.parent + n;
    a.need = a.a_len + n;
    a.back = a.need + n;
    a.run = a.back + n;
    a.run_rows = a.run + n;
    a.merge0 = a.run_rows + n;
    a.big0 = a.merge0 + n;
    a.rest0 = a.big0 + 2 * n;
    a.slot0 = a.rest0 + 2 * n;
    a.parts = a.slot0 + 2 * n;
    return a;
  }
};

// What a sequence's units are.
struct UnitView {
  const PlanArrays& a;
  const int group;
  __host__ __device__ UnitView(const PlanArrays& a_, int group_) : a(a_), group(group_) {}
  // the sequence's rows meet its parent's tokens in the unit of a run
  __host__ __device__ bool in_run(int i) const {
    const int r = a.run[i];
    return r >= 0 && a.run_rows[r] > a.cu[i + 1] - a.cu[i];
  }
  // which: 0 the sequence's own unit, 1 the unit of the run that begins with it
  __host__ __device__ PagedItem unit(int i, int which) const {
    PagedItem u;
    u.row0 = a.cu[i];
    u.pair0 = 0;
    u.a_seq = u.b_seq = -1;
    u.a_len = u.b_len = u.b_pos = 0;
    u.blk0 = u.blk1 = 0;
    u.slot = -1;
    const int n = a.cu[i + 1] - u.row0;
    const bool run = n > 0 && in_run(i);
    if (which == 0) {
      u.rows = n;
      u.b_seq = i;
      u.b_len = a.total[i];
      u.b_pos = a.cached[i];
      if (n > 0 && !run) u.a_seq = a.parent[i], u.a_len = a.a_len[i];
    } else {
      u.rows = 0;  // (a parent without tokens: nothing to meet)
      if (run && a.run[i] == i && a.a_len[i] > 0) u.rows = a.run_rows[i], u.a_seq = a.parent[i], u.a_len = a.a_len[i];
    }
    return u;
  }
  __host__ __device__ static int blocks(const PagedItem& u) {
    return paged_div(u.a_len, kPagedBlock) + paged_div(u.b_len, kPagedBlock);
  }
  __host__ __device__ int tiles(const PagedItem& u) const { return paged_div(u.rows * group, kTilePairs); }
};

// Sums of counts from 0 to kMostCount that stop there, one above the most rows and pages that there is room for (2^30),
// so that no numbers of new tokens overflow them or come out as ones that fit.
constexpr int32_t kMostCount = (1 << 30) + 1;
inline __host__ __device__ int32_t add_count(int32_t a, int32_t b) {
  const uint32_t sum = (uint32_t)a + (uint32_t)b;
  return sum < (uint32_t)kMostCount ? (int32_t)sum : kMostCount;
}

// n / d rounded up, for many n >= 0 by one d >= 1 with n + d < 2^31.
struct CeilDiv {
  int32_t d;
  uint32_t magic;  // 2^32 / d, rounded up: the quotient is right or one too large
  __host__ __device__ explicit CeilDiv(int32_t d_) : d(d_), magic(d_ == 1 ? 0 : (uint32_t)(0xFFFFFFFFu / (uint32_t)d_) + 1) {}
  __host__ __device__ int operator()(int n) const {
    const uint32_t x = (uint32_t)n + d - 1;
    const uint32_t q = d == 1 ? x : (uint32_t)((uint64_t)x * magic >> 32);
    return (int)(q * (uint32_t)d > x ? q - 1 : q);
  }
};

// The plan but for what plan_fill writes, by one team of wavefronts. Each takes
// a range of the sequences, `lanes` neighbours at a time, and knows of the ones
// before by scans over its lanes, a carry from step to step and a scan over the
// wavefronts. ONE: the team has a thread for every sequence, which then looks
// at it once.
template <bool ONE, class Team>
__host__ __device__ void plan_scan(Team& team, const PlanParams& p, const PlanArrays& a) {
  const PagedShape& s = p.s;
  int32_t* const plan = p.plan;
  const int g = p.group, shift = p.shift, page = s.page;
  const int lanes = team.lanes(), steps = ONE ? 1 : paged_div(s.seqs, team.waves() * lanes);
  const int base = team.wave() * steps * lanes + team.lane();
  const int first = p.state[0], spare = p.state[1];
  const int most = s.max_pages << shift;
  // tokens of a sequence after the step, and pages of so many (of one that outgrows its table up to 2^31 + 1)
  auto after = [](int len, int n) { return (uint32_t)len + (uint32_t)n; };
  auto pages = [&](uint32_t tokens) { return (int)((tokens + page - 1) >> shift); };

  // a sequence's step, its numbers brought into range (nothing behind the last sequence); bits of what is wrong with it
  struct One {
    int len, n, need, back, parent, bad;
    bool small;  // may be of a run
  };
  auto look = [&](int i) {
    One o{0, 0, 0, 0, -1, 0, false};
    if (i >= s.seqs) return o;
    const int len = p.length[i], raw = p.fresh[i], par = p.parent ? p.parent[i] : -1;
    o.bad = len < 0 || len > most ? PAGES_LENGTH : 0;
    o.len = o.bad ? 0 : len;
    o.n = raw <= 0 ? 0 : raw < s.rows + 1 ? raw : s.rows + 1;
    if (raw > most - o.len) o.bad |= PAGES_LONG;
    o.need = pages(after(o.len, o.n)) - pages(o.len);
    o.back = raw < 0 ? pages(o.len) : 0;
    o.parent = par < 0 || o.n == 0 ? -1 : par;
    o.small = o.parent >= 0 && (int64_t)o.n * g <= kSmallPairs;
    return o;
  };
  One mine{};
  auto again = [&](int i) { return ONE ? mine : look(i); };
  // of the sequences with rows: the last one's number and, where it may be of a run, its parent, for scans of maxima
  auto key = [](int i, const One& o) {
    return o.n > 0 ? (int64_t)(i + 1) << 32 | (uint32_t)(o.small ? o.parent + 1 : 0) : 0;
  };
  auto is_small = [](int64_t k) { return (uint32_t)k != 0; };
  auto larger = [](int64_t x, int64_t y) { return x > y ? x : y; };

  // rows, pages needed and given back; what is wrong
  int bad = first < 0 || first >= s.num_pages || spare < 0 || spare > s.num_pages ? PAGES_LENGTH : 0;
  int32_t sums[3] = {0, 0, 0}, before[3], all[3];
  int64_t prev = 0;
  for (int j = 0; j < steps; ++j) {
    const int i = base + j * lanes;
    One o = look(i);
    int a_len = 0;
    if (o.parent >= 0) {
      const int par = o.parent;
      if (par < s.seqs && par != i && p.parent[par] < 0 && p.fresh[par] >= 0) {
        const One q = look(par);
        a_len = (int)after(q.len, q.n);
      } else {
        o.bad |= PAGES_PARENT;
      }
    }
    mine = o;
    bad |= o.bad;
    if (i < s.seqs) {
      a.cached[i] = o.len;
      a.total[i] = (int)after(o.len, o.n);
      a.parent[i] = o.parent;
      a.a_len[i] = a_len;
    }
    sums[0] = add_count(sums[0], o.n);
    sums[1] = add_count(sums[1], o.need);
    sums[2] = add_count(sums[2], o.back);
    prev = larger(prev, key(i, o));
  }
  team.scan_waves(sums, before, all, prev, bad);  // prev: the last sequence with rows before this wavefront's
  if (all[0] > s.rows) bad |= PAGES_ROWS;
  if (all[1] > spare) bad |= PAGES_SHORT;
  if (all[2] > s.num_pages - spare) bad |= PAGES_LENGTH;

  // first row and pages of each sequence; runs: a small sequence begins one unless the nearest sequence with rows before
  // it is small and of the same parent
  int start = -1;
  int64_t q = prev;
  for (int j = 0; j < steps; ++j) {
    const int i = base + j * lanes;
    const One o = again(i);
    const int64_t k = key(i, o);
    int32_t v[3] = {o.n, o.need, o.back}, total[3];
    int64_t ahead = k;
    team.scan_lanes(v, total);
    const int64_t k_all = team.last_lanes(ahead);
    if (i < s.seqs) {
      a.cu[i] = plan[p.L.cu + i] = bad ? 0 : before[0] + v[0];
      a.need[i] = bad ? 0 : before[1] + v[1];
      a.back[i] = bad ? 0 : before[2] + v[2];
      a.run[i] = a.run_rows[i] = -1;
      if (o.small && (uint32_t)larger(q, ahead) != (uint32_t)k) start = i;
    }
    for (int c = 0; c < 3; ++c) before[c] = (int)((uint32_t)before[c] + (uint32_t)total[c]);  // (a refused step's may wrap)
    q = larger(q, k_all);
  }
  if (team.tid() == 0) {
    const int rows = bad ? 0 : all[0];
    const int32_t head[] = {s.seqs, s.rows, s.hq, s.hkv, page, s.max_pages, s.num_pages, bad, rows};
    for (int k = 0; k <= PH_TOTAL_ROWS; ++k) plan[k] = head[k];
    a.cu[s.seqs] = plan[p.L.cu + s.seqs] = rows;
    plan[PH_FIRST] = first;
    plan[PH_SPARE] = spare;
    plan[PH_NEED] = bad ? 0 : all[1];
    plan[PH_BACK] = bad ? 0 : all[2];
  }
  start = team.max_waves(start);  // the last run that begins before this wavefront's sequences
  q = prev;
  for (int j = 0; j < steps; ++j) {
    const int i = base + j * lanes;
    const One o = again(i);
    const int64_t k = key(i, o);
    int64_t ahead = k;
    const int64_t k_all = team.last_lanes(ahead);
    const int64_t near = larger(q, ahead);
    const bool joins = o.small && (uint32_t)near == (uint32_t)k;
    int64_t begin = o.small && !joins ? i + 1 : 0;
    const int64_t begin_all = team.last_lanes(begin);
    const int run = begin > 0 ? (int)begin - 1 : start;  // the last that begins before this sequence
    if (!bad && o.n > 0) {
      if (is_small(near) && !joins) a.run_rows[run] = a.cu[i] - a.cu[run];
      if (o.small) a.run[i] = joins ? run : i;
    }
    // the run that no sequence with rows follows ends with the rows
    if (!bad && i == s.seqs - 1 && is_small(larger(near, k))) {
      const int r = o.small && !joins ? i : run;
      a.run_rows[r] = all[0] - a.cu[r];
    }
    q = larger(q, k_all);
    if (begin_all > 0) start = (int)begin_all - 1;
  }
  team.sync();  // (nobody reads lengths and state from here on: they may be written in place)
  for (int j = 0; j < steps; ++j) {
    const int i = base + j * lanes;
    if (i >= s.seqs) break;
    if (!bad) p.length_out[i] = p.fresh[i] < 0 ? 0 : a.total[i];
    else if (p.length_out != p.length) p.length_out[i] = p.length[i];
    if (bad) a.cached[i] = a.total[i] = a.a_len[i] = 0, a.parent[i] = -1;
  }
  if (team.tid() == 0) {
    const int to = first + (bad ? 0 : all[1]);
    p.state_out[0] = to >= s.num_pages && !bad ? to - s.num_pages : to;
    p.state_out[1] = bad ? spare : spare - all[1] + all[2];
  }

  // blocks of all tiles (of the units that UnitView describes), and from them the length of a part
  struct Units {
    int rows[2], blocks[2];
    bool run;
  };
  Units kept{};
  int64_t w[3] = {0, 0, 0};
  for (int j = 0; j < steps; ++j) {
    const int i = base + j * lanes;
    Units x{};
    if (i < s.seqs) {
      const int total = a.total[i], n = total - a.cached[i];
      const int r = a.run[i], run_rows = r >= 0 ? a.run_rows[r] : 0, of_parent = paged_div(a.a_len[i], kPagedBlock);
      x.run = n > 0 && run_rows > n;
      x.rows[0] = n;
      x.blocks[0] = (x.run ? 0 : of_parent) + paged_div(total, kPagedBlock);
      x.rows[1] = x.run && r == i && of_parent > 0 ? run_rows : 0;
      x.blocks[1] = of_parent;
      if (!ONE) {  // for the two passes below, which write what belongs here
        a.big0[2 * i] = x.rows[0];
        a.big0[2 * i + 1] = x.rows[1];
        a.rest0[2 * i] = x.blocks[0];
        a.rest0[2 * i + 1] = x.blocks[1];
        a.merge0[i] = x.run;
      }
    }
    kept = x;
    for (int which = 0; which < 2; ++which) {
      const int tiles = paged_div(x.rows[which] * g, kTilePairs);
      w[x.rows[which] * g <= kSlotPairs] += (int64_t)tiles * x.blocks[which];
      w[2] += tiles;
    }
  }
  team.sum(w);
  const Cut cut = part_blocks(TileSums{w[0], w[1], w[2]}, s, p.L.max_parts);
  const CeilDiv by_part(cut.part);

  // items: of units with long parts first, then the others; slots of partial results; merged rows
  int32_t c[4] = {0, 0, 0, 0}, at[4], sum[4], most_parts = 0;
  for (int pass = 0; pass < 2; ++pass) {
    for (int j = 0; j < steps; ++j) {
      const int i = base + j * lanes;
      Units x = kept;
      if (!ONE) {
        x = Units{};
        if (i < s.seqs) {
          x.rows[0] = a.big0[2 * i];
          x.rows[1] = a.big0[2 * i + 1];
          x.blocks[0] = a.rest0[2 * i];
          x.blocks[1] = a.rest0[2 * i + 1];
          x.run = a.merge0[i] != 0;
        }
      }
      int32_t n[2][4], v[4] = {0, 0, 0, 0}, parts[2];
      for (int which = 0; which < 2; ++which) {
        const int tiles = paged_div(x.rows[which] * g, kTilePairs);
        parts[which] = tiles ? by_part(x.blocks[which]) : 0;
        const bool partial = tiles && (parts[which] > 1 || which == 1 || x.run);
        const bool big = x.blocks[which] >= parts[which] * cut.big;
        n[which][0] = big ? tiles * parts[which] : 0;
        n[which][1] = big ? 0 : tiles * parts[which];
        n[which][2] = partial ? parts[which] * paged_div(x.rows[which] * g, kSlotPairs) : 0;
        n[which][3] = partial && which == 0 ? x.rows[which] : 0;
        for (int k = 0; k < 4; ++k) v[k] += n[which][k];
        if (partial && parts[which] > most_parts) most_parts = parts[which];
      }
      if (!pass) {
        for (int k = 0; k < 4; ++k) c[k] += v[k];
        continue;
      }
      int32_t total[4];
      team.scan_lanes(v, total);
      if (i < s.seqs)
        for (int which = 0; which < 2; ++which) {
          const int k = 2 * i + which;
          for (int y = 0; y < 4; ++y)
            if (which) v[y] += n[0][y];
          a.big0[k] = at[0] + v[0];
          a.rest0[k] = at[1] + v[1];
          a.slot0[k] = n[which][2] ? at[2] + v[2] : -1;
          a.parts[k] = parts[which];
          if (which == 0) a.merge0[i] = n[0][3] ? at[3] + v[3] : -1;
        }
      for (int k = 0; k < 4; ++k) at[k] += total[k];
    }
    if (!pass) team.scan_waves(c, at, sum);
  }
  most_parts = team.max_of(most_parts);
  if (team.tid() == 0) {
    plan[PH_BIG] = sum[0];
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
__host__ __device__ void plan_fill(Team& team, const PlanParams& p, const PlanArrays& a, int tid, int size) {
  const PagedShape& s = p.s;
  int32_t* const plan = p.plan;
  const UnitView view(a, p.group);
  const int g = p.group, page = s.page, shift = p.shift;
  const int first = plan[PH_FIRST], spare = plan[PH_SPARE], rows = plan[PH_TOTAL_ROWS];
  const int need = plan[PH_NEED], back = plan[PH_BACK], bigs = plan[PH_BIG], items = plan[PH_ITEMS];
  auto ring = [&](int k) { return k < s.num_pages ? k : k - s.num_pages; };

  // a row: slot, position, where the merge finds its parts
  auto fill_row = [&](int r) {
    int slot = -1, pos = -1;
    if (r < rows) {
      const int seq = last_at_most(a.cu, s.seqs, r);
      const int off = r - a.cu[seq], cached = a.cached[seq], at = cached + off;
      const int have = (cached + page - 1) >> shift, k = at >> shift;
      const int id = k < have ? p.table[(int64_t)seq * s.max_pages + k] : p.free_pages[ring(first + a.need[seq] + k - have)];
      const int m = a.merge0[seq];
      if (m >= 0) {
        int32_t* const dst = plan + p.L.merge + (int64_t)(m + off) * kMergeInts;
        dst[0] = r;
        for (int u = 0; u < 2; ++u) {
          const int q = u == 0 ? seq : a.run[seq];
          const int slot0 = q < 0 ? -1 : a.slot0[2 * q + u];
          const int row0 = q < 0 ? 0 : a.cu[q];
          const int pair = (r - row0) * g;
          dst[1 + 4 * u] = slot0 + pair / kSlotPairs;
          dst[2 + 4 * u] = pair % kSlotPairs;
          dst[3 + 4 * u] = slot0 < 0 ? 0 : paged_div((u == 0 ? a.cu[q + 1] - row0 : a.run_rows[q]) * g, kSlotPairs);
          dst[4 + 4 * u] = slot0 < 0 ? 0 : a.parts[2 * q + u];
        }
      }
      if (id >= 0 && id < s.num_pages) slot = (id << shift) + (at & (page - 1));
      else team.flag(plan + PH_STATUS, PAGES_PAGE);
      pos = at + a.a_len[seq];
    }
    plan[p.L.slots + r] = slot;
    plan[p.L.positions + r] = pos;
  };
  // a new page into the table; an ended sequence's page back to the ring
  auto fill_need = [&](int k) {
    const int i = last_at_most(a.need, s.seqs, k);
    const int have = (a.cached[i] + page - 1) >> shift;
    p.table[(int64_t)i * s.max_pages + have + k - a.need[i]] = p.free_pages[ring(first + k)];
  };
  auto fill_back = [&](int k) {
    const int i = last_at_most(a.back, s.seqs, k);
    p.free_pages[ring(ring(first + spare) + k)] = p.table[(int64_t)i * s.max_pages + k - a.back[i]];
  };
  auto fill_item = [&](int x) {
    const bool big = x < bigs;
    const int k = big ? x : x - bigs;
    const int32_t* const of = big ? a.big0 : a.rest0;
    const int unit = last_at_most(of, 2 * s.seqs, k);
    PagedItem it = view.unit(unit >> 1, unit & 1);
    const int parts = a.parts[unit], slot0 = a.slot0[unit];
    const int part = paged_div(view.blocks(it), parts), j = k - of[unit];
    // a causal unit's last tiles have the most blocks: they come first; its last parts, which causality shortens, last
    const int tiles = view.tiles(it), c = j / tiles, t = tiles - 1 - (j - c * tiles);
    it.pair0 = t * kTilePairs;
    int end = view.blocks(it);
    if (it.b_len > 0) {  // up to what the tile's last row sees
      const int pairs = it.rows * g, lastpair = it.pair0 + kTilePairs - 1 < pairs - 1 ? it.pair0 + kTilePairs - 1 : pairs - 1;
      end = paged_div(it.a_len, kPagedBlock) + (it.b_pos + lastpair / g) / kPagedBlock + 1;
    }
    it.blk0 = (int)((int64_t)c * part < end ? (int64_t)c * part : end);
    it.blk1 = (int)((int64_t)(c + 1) * part < end ? (int64_t)(c + 1) * part : end);
    if (slot0 >= 0) it.slot = slot0 + c * paged_div(it.rows * g, kSlotPairs) + t * (kTilePairs / kSlotPairs);
    int32_t* const dst = plan + p.L.items + (int64_t)x * kItemInts;
    const int32_t w[kItemInts] = {it.row0, it.rows, it.pair0, it.a_seq, it.a_len, it.b_seq, it.b_len, it.b_pos,
                                  it.blk0, it.blk1, it.slot, 0, 0, 0, 0, 0};
    for (int y = 0; y < kItemInts; ++y) dst[y] = w[y];
  };
  // one after the other through all of it, so that every thread has its share of the kinds
  const int at_back = s.rows + need, at_item = at_back + back, end = at_item + items;
  for (int x = tid; x < end; x += size) {
    if (x < s.rows) fill_row(x);
    else if (x < at_back) fill_need(x - s.rows);
    else if (x < at_item) fill_back(x - at_back);
    else fill_item(x - at_item);
  }
}

// The arrays in the plan itself.
inline __host__ __device__ PlanArrays plan_arrays(const PlanParams& p) { return PlanArrays::packed(p.plan + p.L.work, p.s.seqs); }

// ---------------------------------------------------------------------------- launchers

// How a cache holds its values.
enum : int { CACHE_BF16 = 0, CACHE_E4M3 = 1 };

// apart: the plan's arrays by a second launch, with more than one workgroup; else at most kFillSeqs sequences
constexpr int kFillSeqs = 1024;
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
