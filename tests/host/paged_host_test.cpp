// Host logic of the paged KV cache without a GPU: the construction of a plan
// (paged.h, the same source that the kernels run) by teams of one to nine
// threads, against a plain sequential account of the same step, and the entry
// points of paged.cpp with stand-ins for the launchers, each of which in turn
// reports a HIP error.
//
// Checked on random steps: tables, ring, lengths, slots and positions; that
// items and slots of partial results stay within the plan's room; that every
// (row, head) pair meets every key block it sees exactly once; that pairs with
// several parts find them all where the merge looks, and others have one item;
// that tables, parents, lengths and pages out of range are reported and touch
// nothing.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <condition_variable>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <mutex>
#include <random>
#include <string>
#include <thread>
#include <vector>

#include "augtree.h"
#include "paged.h"

using namespace augtree;

namespace {

int g_errors = 0;
std::mutex g_lock;

void check(bool ok, const char* what) {
  if (ok) return;
  std::lock_guard<std::mutex> l(g_lock);
  if (++g_errors < 40) std::printf("FAILED: %s\n", what);
}

struct Shared {
  explicit Shared(int n_) : n(n_), sums(n_), wide(n_), keys(n_), bits(n_) {}
  const int n;
  std::mutex m;
  std::condition_variable cv;
  int waiting = 0, turn = 0;
  std::vector<std::vector<int32_t>> sums;
  std::vector<std::vector<int64_t>> wide;
  std::vector<int64_t> keys;
  std::vector<int> bits;
  void barrier() {
    std::unique_lock<std::mutex> l(m);
    const int t = turn;
    if (++waiting == n) {
      waiting = 0;
      ++turn;
      cv.notify_all();
    } else {
      cv.wait(l, [&] { return turn != t; });
    }
  }
};

// Threads in place of the kernel's wavefronts, one lane each.
struct ThreadTeam {
  Shared& s;
  int id;
  int tid() const { return id; }
  int lane() const { return 0; }
  int wave() const { return id; }
  int lanes() const { return 1; }
  int waves() const { return s.n; }
  void sync() const { s.barrier(); }
  void flag(int32_t* to, int32_t b) const {
    std::lock_guard<std::mutex> l(g_lock);
    *to |= b;
  }
  template <int K>
  void scan_lanes(int32_t (&v)[K], int32_t (&total)[K]) const {
    for (int k = 0; k < K; ++k) total[k] = v[k], v[k] = 0;
  }
  int64_t last_lanes(int64_t& x) const {
    const int64_t all = x;
    x = 0;
    return all;
  }
  template <int K>
  void scan_waves(const int32_t (&v)[K], int32_t (&before)[K], int32_t (&all)[K]) const {
    int64_t key = 0;
    int b = 0;
    scan_waves(v, before, all, key, b);
  }
  template <int K>
  void scan_waves(const int32_t (&v)[K], int32_t (&before)[K], int32_t (&all)[K], int64_t& key, int& bits) const {
    s.sums[id].assign(v, v + K);
    s.keys[id] = key;
    s.bits[id] = bits;
    s.barrier();
    key = 0;
    for (int t = 0; t < s.n; ++t) {
      if (t < id) key = std::max(key, s.keys[t]);
      bits |= s.bits[t];
    }
    for (int k = 0; k < K; ++k) {
      before[k] = all[k] = 0;
      for (int t = 0; t < s.n; ++t) {
        if (t < id) before[k] = add_count(before[k], s.sums[t][k]);
        all[k] = add_count(all[k], s.sums[t][k]);
      }
    }
    s.barrier();
  }
  int max_waves(int v) const {
    const int32_t none[1] = {0};
    int32_t a[1], b[1];
    int64_t key = v + 1;
    int bits = 0;
    scan_waves(none, a, b, key, bits);
    return (int)key - 1;
  }
  void sum(int64_t (&v)[3]) const {
    s.wide[id].assign(v, v + 3);
    s.barrier();
    for (int k = 0; k < 3; ++k) {
      v[k] = 0;
      for (auto& w : s.wide) v[k] += w[k];
    }
    s.barrier();
  }
  int max_of(int v) const {
    s.keys[id] = v;
    s.barrier();
    for (int64_t k : s.keys) v = std::max(v, (int)k);
    s.barrier();
    return v;
  }
};

struct Step {
  PagedShape s;
  std::vector<int32_t> table, length, parent, ring, state, fresh;
  bool parents = true;
};

struct Result {
  std::vector<int32_t> table, length, ring, state, plan;
};

Result run(const Step& st, int threads, bool in_place) {
  Result r{st.table, st.length, st.ring, st.state, {}};
  const PlanLayout L = plan_layout(st.s);
  r.plan.assign(L.words, -123456);
  std::vector<int32_t> length = st.length, state = st.state;
  PlanParams p;
  std::memset(&p, 0, sizeof(p));
  p.s = st.s;
  p.L = L;
  p.group = st.s.hq / st.s.hkv;
  p.shift = paged_shift(st.s.page);
  p.table = r.table.data();
  p.length = in_place ? r.length.data() : length.data();
  p.parent = st.parents ? st.parent.data() : nullptr;
  p.free_pages = r.ring.data();
  p.state = in_place ? r.state.data() : state.data();
  p.fresh = st.fresh.data();
  p.length_out = r.length.data();
  p.state_out = r.state.data();
  p.plan = r.plan.data();
  // the construction's arrays: in the plan, or elsewhere
  std::vector<int32_t> elsewhere(PlanArrays::words(st.s.seqs), -77);
  const PlanArrays arrays = in_place ? plan_arrays(p) : PlanArrays::packed(elsewhere.data(), st.s.seqs);
  Shared sh(threads);
  std::vector<std::thread> pool;
  for (int t = 0; t < threads; ++t)
    pool.emplace_back([&, t] {
      ThreadTeam team{sh, t};
      if (threads >= st.s.seqs) plan_scan<true>(team, p, arrays);
      else plan_scan<false>(team, p, arrays);
    });
  for (auto& t : pool) t.join();
  // the rest by threads one after the other
  for (int t = threads; t-- > 0;) {
    ThreadTeam team{sh, 0};
    plan_fill(team, p, arrays, t, threads);
  }
  return r;
}

int cdiv(int a, int b) { return (a + b - 1) / b; }

// What the plan says about a good step, against the step itself.
void check_good(const Step& st, const Result& r, const char* label) {
  const PagedShape& s = st.s;
  const PlanLayout L = plan_layout(s);
  const int32_t* plan = r.plan.data();
  const int g = s.hq / s.hkv;
  auto table = st.table;
  auto ring = st.ring;
  auto length = st.length;
  int first = st.state[0], spare = st.state[1];
  const int first0 = first, spare0 = spare;
  int row = 0, back = 0;
  check(plan[PH_STATUS] == 0, label);
  std::vector<int> seq_of, pos_of;
  for (int i = 0; i < s.seqs; ++i) {
    const int n = st.fresh[i] > 0 ? st.fresh[i] : 0;
    check(plan[L.cu + i] == row, "cu");
    for (int k = cdiv(length[i], s.page); k < cdiv(length[i] + n, s.page); ++k) {
      table[(int64_t)i * s.max_pages + k] = st.ring[first];
      first = (first + 1) % s.num_pages;
      --spare;
    }
    for (int j = 0; j < n; ++j) {
      const int at = length[i] + j;
      check(plan[L.slots + row] == table[(int64_t)i * s.max_pages + at / s.page] * s.page + at % s.page, "slot");
      const int par = st.parents ? st.parent[i] : -1;
      check(plan[L.positions + row] == at + (par >= 0 ? st.length[par] + (st.fresh[par] > 0 ? st.fresh[par] : 0) : 0), "position");
      seq_of.push_back(i);
      pos_of.push_back(at);
      ++row;
    }
  }
  check(plan[L.cu + s.seqs] == row && plan[PH_TOTAL_ROWS] == row, "rows");
  for (int i = 0; i < s.seqs; ++i)
    if (st.fresh[i] < 0)
      for (int k = 0; k < cdiv(length[i], s.page); ++k)
        ring[(first0 + spare0 + back++) % s.num_pages] = st.table[(int64_t)i * s.max_pages + k];
  for (int i = 0; i < s.seqs; ++i) length[i] = st.fresh[i] < 0 ? 0 : length[i] + st.fresh[i];
  for (int j = row; j < s.rows; ++j) check(plan[L.slots + j] == -1 && plan[L.positions + j] == -1, "rows behind the last");
  check(r.table == table, "table");
  check(r.ring == ring, "ring");
  check(r.length == length, "lengths");
  check(r.state[0] == first && r.state[1] == spare + back, "state");

  // what every (row, head of a KV head) sees: blocks of its parent, of its own
  const int items = plan[PH_ITEMS];
  check(items >= 0 && items <= L.max_items, "room for items");
  // (pair, segment, block) -> times met; pair -> items, slots
  std::map<std::pair<int, std::pair<int, int>>, int> met;
  std::map<int, std::vector<int>> slots_of;
  std::map<int, int> place[2];  // pair in the sequence's own unit, in the run's
  std::map<int, int> direct;
  std::vector<char> used(L.max_slots, 0);
  for (int k = 0; k < items; ++k) {
    PagedItem it;
    std::memcpy(&it, plan + L.items + (int64_t)k * kItemInts, sizeof(it));
    const int pairs = it.rows * g;
    check(it.rows > 0 && it.pair0 >= 0 && it.pair0 < pairs && it.pair0 % kTilePairs == 0, "pairs of an item");
    check(it.row0 >= 0 && it.row0 + it.rows <= row, "rows of an item");
    check(it.a_seq >= -1 && it.a_seq < s.seqs && it.b_seq >= -1 && it.b_seq < s.seqs, "sequences of an item");
    check((it.a_seq >= 0) == (it.a_len > 0) || it.a_len == 0, "segment A");
    check(it.blk0 >= 0 && it.blk0 <= it.blk1, "blocks of an item");
    const int nA = cdiv(it.a_len, kPagedBlock), nB = cdiv(it.b_len, kPagedBlock);
    check(it.blk1 <= nA + nB, "blocks of an item");
    check(cdiv(it.a_len, s.page) <= s.max_pages && cdiv(it.b_len, s.page) <= s.max_pages, "pages of an item");
    for (int x = it.pair0; x < pairs && x < it.pair0 + kTilePairs; ++x) {
      const int rr = it.row0 + x / g, id = rr * g + x % g;
      if (it.b_seq >= 0) check(seq_of[rr] == it.b_seq && it.b_pos + x / g == pos_of[rr], "position in an item");
      if (it.slot >= 0) {
        const int slot = it.slot + (x - it.pair0) / kSlotPairs;
        check(slot < L.max_slots, "room for slots");
        if ((x - it.pair0) % kSlotPairs == 0) {
          check(slot < L.max_slots && !used[slot], "a slot is used once");
          if (slot < L.max_slots) used[slot] = 1;
        }
        slots_of[id].push_back(slot);
        place[it.b_seq < 0][id] = x;
      } else {
        ++direct[id];
      }
      for (int b = it.blk0; b < it.blk1; ++b) {
        const bool isB = b >= nA;
        const int blk = isB ? b - nA : b;
        if (isB && blk * kPagedBlock > it.b_pos + x / g) continue;  // masked whole
        ++met[{id, {isB ? it.b_seq : it.a_seq, blk}}];
      }
    }
  }
  int64_t pairs_seen = 0;
  for (int rr = 0; rr < row; ++rr) {
    const int i = seq_of[rr], par = st.parents ? st.parent[i] : -1;
    for (int h = 0; h < g; ++h) {
      const int id = rr * g + h;
      for (int b = 0; b <= pos_of[rr] / kPagedBlock; ++b) check((met[{id, {i, b}}]) == 1, "own blocks"), ++pairs_seen;
      if (par >= 0)
        for (int b = 0; b < cdiv(r.length[par], kPagedBlock); ++b) check((met[{id, {par, b}}]) == 1, "parent's blocks"), ++pairs_seen;
      check(direct[id] == (slots_of.count(id) ? 0 : 1), "final or partial");
    }
  }
  check((int64_t)met.size() == pairs_seen, "nothing else is met");
  // the merge's view: the rows it lists, and the slots it finds for them
  std::vector<char> merged(row, 0);
  size_t most = 0;
  check(plan[PH_MERGE_ROWS] <= s.rows, "merged rows");
  for (int m = 0; m < plan[PH_MERGE_ROWS]; ++m) {
    const int32_t* d = plan + L.merge + (int64_t)m * kMergeInts;
    const int rr = d[0];
    const bool fine = rr >= 0 && rr < row;
    check(fine && !merged[rr], "merged rows");
    if (!fine) continue;
    merged[rr] = 1;
    for (int h = 0; h < g; ++h) {
      std::vector<int> want = slots_of[rr * g + h], got;
      for (int u = 0; u < 2; ++u) {
        const int pair = d[2 + 4 * u] + h;
        for (int k = 0; k < d[4 + 4 * u]; ++k) got.push_back(d[1 + 4 * u] + pair / kSlotPairs + k * d[3 + 4 * u]);
        most = std::max(most, (size_t)d[4 + 4 * u]);
      }
      std::sort(want.begin(), want.end());
      std::sort(got.begin(), got.end());
      check(want == got, "the merge finds the parts");
      // and in them the pair's place
      for (int u = 0; u < 2; ++u)
        if (d[4 + 4 * u] > 0) check((d[2 + 4 * u] + h) % kSlotPairs == place[u][rr * g + h] % kSlotPairs, "place in a slot");
    }
  }
  check((int)most == plan[PH_MOST_PARTS], "most parts");
  for (int rr = 0; rr < row; ++rr) check(merged[rr] == (direct[rr * g] ? 0 : 1), "rows to merge");
}

void check_refused(const Step& st, const Result& r, int bits) {
  const PlanLayout L = plan_layout(st.s);
  check((r.plan[PH_STATUS] & bits) == bits, "reported");
  check(r.table == st.table && r.ring == st.ring && r.length == st.length && r.state == st.state, "a refused step changes nothing");
  check(r.plan[PH_ITEMS] == 0 && r.plan[PH_TOTAL_ROWS] == 0 && r.plan[PH_MERGE_ROWS] == 0, "a refused step has no work");
  for (int j = 0; j < st.s.rows; ++j) check(r.plan[L.slots + j] == -1, "a refused step has no slots");
}

Step random_step(std::mt19937& rng) {
  auto in = [&](int a, int b) { return (int)std::uniform_int_distribution<int>(a, b)(rng); };
  Step st;
  const int heads[][2] = {{1, 1}, {4, 2}, {7, 1}, {32, 8}, {6, 2}, {130, 1}, {300, 2}, {12, 12}};
  const int* h = heads[in(0, 7)];
  const int seqs = in(1, 30), page = 16 << in(0, 4);
  const int len = in(0, 1) ? 60 : 900, most_new = in(0, 2) ? 3 : 400;
  st.parents = in(0, 4) > 0;
  st.length.resize(seqs);
  st.fresh.resize(seqs);
  st.parent.assign(seqs, -1);
  std::vector<int> roots;
  int rows = 0, live = 0, need = 0, widest = 1;
  for (int i = 0; i < seqs; ++i) {
    st.length[i] = in(0, 3) ? in(0, len) : 0;
    const int kind = in(0, 5);
    st.fresh[i] = kind == 0 ? 0 : kind == 1 && in(0, 1) ? in(1, most_new) : in(0, 3);
    if (roots.empty() || in(0, 3) == 0) roots.push_back(i);
    else st.parent[i] = roots[in(0, 1) ? (int)roots.size() - 1 : in(0, (int)roots.size() - 1)];
  }
  for (int i = 0; i < seqs; ++i)  // some end; a parent only with all of its children
    if (st.parent[i] >= 0 && in(0, 6) == 0) st.fresh[i] = -in(1, 5);
  for (int t : roots) {
    bool free_to = in(0, 3) == 0;
    for (int i = 0; i < seqs; ++i) free_to = free_to && !(st.parent[i] == t && st.fresh[i] > 0);
    if (free_to) st.fresh[t] = -1;
  }
  if (!st.parents) st.parent.assign(seqs, -1);
  for (int i = 0; i < seqs; ++i) {
    const int n = std::max(0, st.fresh[i]);
    rows += n;
    live += cdiv(st.length[i], page);
    need += cdiv(st.length[i] + n, page) - cdiv(st.length[i], page);
    widest = std::max(widest, cdiv(st.length[i] + n, page));
  }
  const int pages = live + need + in(0, 5) + 1;
  st.s = PagedShape{seqs, rows + in(0, 1) * in(0, 9), h[0], h[1], page, widest + in(0, 2), pages};
  std::vector<int32_t> ids(pages);
  for (int i = 0; i < pages; ++i) ids[i] = i;
  std::shuffle(ids.begin(), ids.end(), rng);
  st.table.resize((size_t)seqs * st.s.max_pages);
  for (auto& x : st.table) x = in(-5, pages + 5);
  int at = 0;
  for (int i = 0; i < seqs; ++i)
    for (int k = 0; k < cdiv(st.length[i], page); ++k) st.table[(size_t)i * st.s.max_pages + k] = ids[at++];
  st.state = {in(0, pages - 1), pages - live};
  st.ring.resize(pages);
  for (auto& x : st.ring) x = in(-5, pages + 5);
  for (int k = 0; k < pages - live; ++k) st.ring[(st.state[0] + k) % pages] = ids[live + k];
  return st;
}

// ---------------------------------------------------------------------------- entry points

std::vector<std::string> g_launches;
int g_fail_at = 0, g_calls = 0;
const char* g_ws;
size_t g_ws_bytes;

hipError_t launched(const char* what) {
  g_launches.push_back(what);
  return ++g_calls == g_fail_at ? hipErrorLaunchFailure : hipSuccess;
}

}  // namespace

namespace augtree {

hipError_t launch_page_plan(const PlanParams& p, bool apart, hipStream_t) {
  check(p.L.words == plan_layout(p.s).words && p.group * p.s.hkv == p.s.hq && 1 << p.shift == p.s.page, "layout");
  check(apart == (p.s.rows > 2048 || p.s.seqs > kFillSeqs), "one launch or two");
  return launched("plan");
}
hipError_t launch_cache_write(const CacheWriteParams&, hipStream_t) { return launched("write"); }
hipError_t launch_paged_fwd(const PagedFwdParams& p, hipStream_t) {
  const PlanLayout L = plan_layout(p.s);
  const size_t pairs = (size_t)L.max_slots * p.s.hkv * kSlotPairs;
  const char *o = reinterpret_cast<const char*>(p.part_o), *l = reinterpret_cast<const char*>(p.part_lse);
  check(o == g_ws && o + pairs * p.d * 4 <= l && l + pairs * 4 <= g_ws + g_ws_bytes, "workspace");
  check(p.max_items == L.max_items && p.max_slots == L.max_slots && p.items_at == L.items, "layout");
  check(p.group * p.s.hkv == p.s.hq, "group");
  return launched("attend");
}
hipError_t launch_paged_merge(const PagedFwdParams&, hipStream_t) { return launched("merge"); }

}  // namespace augtree

namespace {

void entry_points() {
  static int32_t dummy[4];
  char* const base = reinterpret_cast<char*>((uintptr_t)1 << 50);
  auto at = [&](int i) { return base + ((uintptr_t)i << 40); };
  augtree_pages pg = {5, 7, 40, 64, (int32_t*)at(1), (int32_t*)at(2), (int32_t*)at(3), (int32_t*)at(4), (int32_t*)at(5)};
  (void)dummy;
  const int rows = 33, hq = 8, hkv = 2, d = 128;
  const size_t n = augtree_page_plan_size(&pg, rows, hq, hkv);
  check(n > 0, "plan size");
  const int64_t stride = 2 * (int64_t)hkv * 64 * d * 2;
  g_ws = at(8);
  g_ws_bytes = augtree_paged_workspace_size(&pg, rows, hq, hkv, d);
  auto step = [&]() {
    int st = augtree_page_plan(&pg, (int32_t*)at(6), rows, hq, hkv, pg.length, pg.free_state, at(7), n, nullptr);
    if (!st)
      st = augtree_cache_write(&pg, at(7), rows, hq, hkv, d, (uint16_t*)at(9), (uint16_t*)at(10), AUGTREE_CACHE_BF16, at(11),
                               stride, at(11) + stride / 2, stride, nullptr, nullptr, nullptr);
    if (!st)
      st = augtree_paged_fwd(&pg, at(7), rows, hq, hkv, d, 0.1f, (uint16_t*)at(12), AUGTREE_CACHE_BF16, at(11), stride,
                             at(11) + stride / 2, stride, nullptr, nullptr, (uint16_t*)at(13), (float*)at(14), at(8),
                             g_ws_bytes, nullptr);
    return st;
  };
  for (g_fail_at = 0; g_fail_at <= 4; ++g_fail_at) {
    g_calls = 0;
    g_launches.clear();
    const int st = step();
    check(st == (g_fail_at ? AUGTREE_ERR_HIP : AUGTREE_OK), "status of a step");
    check((int)g_launches.size() == (g_fail_at ? g_fail_at : 4), "launches of a step");
    check(!g_fail_at || std::string(augtree_last_error()).find("launch") != std::string::npos, "message");
  }
}

}  // namespace

int main() {
  std::mt19937 rng(11);
  int good = 0, refused = 0;
  for (int k = 0; k < 260; ++k) {
    Step st = random_step(rng);
    const Result r = run(st, 1 + k % 9, k % 2);
    check_good(st, r, "status of a good step");
    const Result again = run(st, 1 + (k + 4) % 9, k % 3 == 0);
    const PlanLayout lay = plan_layout(st.s);
    auto same = [&](int64_t from, int64_t to) { return std::equal(r.plan.begin() + from, r.plan.begin() + to, again.plan.begin() + from); };
    check(same(0, lay.work) && same(lay.slots, lay.words) && again.table == r.table, "the plan does not depend on the team");
    ++good;

    Step b = st;
    const int i = (int)(rng() % st.s.seqs);
    int bits = 0;
    switch (k % 9) {
      case 0: b.state[1] = -1; bits = PAGES_LENGTH; break;
      case 1: b.state[0] = st.s.num_pages; bits = PAGES_LENGTH; break;
      case 2: b.length[i] = -1; bits = PAGES_LENGTH; break;
      case 3: b.length[i] = INT32_MAX; bits = PAGES_LENGTH; break;
      case 4: b.fresh[i] = INT32_MAX; bits = PAGES_LONG | PAGES_ROWS; break;
      case 5: if (st.parents) b.parent[i] = i, b.fresh[i] = 1, bits = PAGES_PARENT; break;
      case 6: if (st.parents) b.parent[i] = st.s.seqs + 3, b.fresh[i] = 2, bits = PAGES_PARENT; break;
      case 7: for (auto& f : b.fresh) f = 1; b.state[1] = 0; for (auto& l : b.length) l = 0; bits = PAGES_SHORT; break;
      case 8: b.fresh[i] = st.s.rows + 1; bits = PAGES_ROWS; break;
    }
    if (bits) {
      check_refused(b, run(b, 1 + k % 5, k % 2), bits);
      ++refused;
    }
    // pages outside the pool: reported, not written, the rest of the plan as before
    Step o = st;
    for (auto& x : o.ring) x = k % 2 ? -7 : st.s.num_pages;
    const Result w = run(o, 3, false);
    const PlanLayout L = plan_layout(st.s);
    bool any = false;
    for (int j = 0; j < w.plan[PH_TOTAL_ROWS]; ++j) {
      const int seq = last_at_most(w.plan.data() + L.cu, st.s.seqs, j), pos = st.length[seq] + j - w.plan[L.cu + seq];
      const bool fresh_page = pos / st.s.page >= cdiv(st.length[seq], st.s.page);
      check(fresh_page ? w.plan[L.slots + j] == -1 : w.plan[L.slots + j] >= 0, "slots outside the pool");
      any = any || fresh_page;
    }
    check(w.plan[PH_STATUS] == (any ? PAGES_PAGE : 0), "pages outside the pool are reported");
  }
  entry_points();
  if (g_errors) {
    std::printf("%d errors\n", g_errors);
    return 1;
  }
  std::printf("ok: %d steps, %d refused\n", good, refused);
  return 0;
}
