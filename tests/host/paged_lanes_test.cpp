// The plan of many sequences (paged.h) by teams of wavefronts of several lanes,
// as the kernel has them, against the account of paged_host_test.cpp: runs that
// cross lanes, wavefronts and the steps in which a wavefront takes its
// sequences, with their items, slots of partial results and merge entries.
#define main paged_host_main
#include "paged_host_test.cpp"
#undef main

#include <memory>

namespace {

// What the lanes of one wavefront exchange.
struct Wave {
  explicit Wave(int lanes) : sync(lanes), v(lanes), key(lanes) {}
  Shared sync;
  std::vector<std::vector<int32_t>> v;
  std::vector<int64_t> key;
};

// Threads in place of the lanes of the kernel's wavefronts.
struct LaneTeam {
  ThreadTeam all;  // every lane as a wavefront of its own: reductions over the team
  Wave& w;
  int n_waves, n_lanes;
  int tid() const { return all.id; }
  int lane() const { return all.id % n_lanes; }
  int wave() const { return all.id / n_lanes; }
  int lanes() const { return n_lanes; }
  int waves() const { return n_waves; }
  void sync() const { all.sync(); }
  void flag(int32_t* to, int32_t b) const { all.flag(to, b); }
  template <int K>
  void scan_lanes(int32_t (&v)[K], int32_t (&total)[K]) const {
    w.v[lane()].assign(v, v + K);
    w.sync.barrier();
    for (int k = 0; k < K; ++k) {
      uint32_t before = 0, sum = 0;
      for (int l = 0; l < n_lanes; ++l) {
        if (l == lane()) before = sum;
        sum += (uint32_t)w.v[l][k];
      }
      v[k] = (int32_t)before;
      total[k] = (int32_t)sum;
    }
    w.sync.barrier();
  }
  // x: 0 or larger than in all lanes before
  int64_t last_lanes(int64_t& x) const {
    w.key[lane()] = x;
    w.sync.barrier();
    int64_t before = 0, last = 0;
    for (int l = 0; l < n_lanes; ++l) {
      if (l == lane()) before = last;
      check(w.key[l] == 0 || w.key[l] > last, "keys grow along a wavefront");
      if (w.key[l]) last = w.key[l];
    }
    w.sync.barrier();
    x = before;
    return last;
  }
  // of the wavefronts before this one, the same for its lanes; of all
  template <int K>
  void scan_waves(const int32_t (&v)[K], int32_t (&before)[K], int32_t (&sum)[K]) const {
    int64_t key = 0;
    int bits = 0;
    scan_waves(v, before, sum, key, bits);
  }
  template <int K>
  void scan_waves(const int32_t (&v)[K], int32_t (&before)[K], int32_t (&sum)[K], int64_t& key, int& bits) const {
    all.scan_waves(v, before, sum, key, bits);  // of the lanes before this one
    for (int k = 0; k < K; ++k) w.v[lane()].resize(K), w.v[lane()][k] = before[k];
    w.key[lane()] = key;
    w.sync.barrier();
    for (int k = 0; k < K; ++k) before[k] = w.v[0][k];
    key = w.key[0];
    w.sync.barrier();
  }
  int max_waves(int v) const {
    const int32_t none[1] = {0};
    int32_t a[1], b[1];
    int64_t key = v + 1;
    int bits = 0;
    scan_waves(none, a, b, key, bits);
    return (int)key - 1;
  }
  void sum(int64_t (&v)[3]) const { all.sum(v); }
  int max_of(int v) const { return all.max_of(v); }
};

Result run_lanes(const Step& st, int waves, int lanes) {
  Result r{st.table, st.length, st.ring, st.state, {}};
  const PlanLayout L = plan_layout(st.s);
  r.plan.assign(L.words, -123456);
  PlanParams p;
  std::memset(&p, 0, sizeof(p));
  p.s = st.s;
  p.L = L;
  p.group = st.s.hq / st.s.hkv;
  p.shift = paged_shift(st.s.page);
  p.table = r.table.data();
  p.length = p.length_out = r.length.data();
  p.parent = st.parent.data();
  p.free_pages = r.ring.data();
  p.state = p.state_out = r.state.data();
  p.fresh = st.fresh.data();
  p.plan = r.plan.data();
  const PlanArrays arrays = plan_arrays(p);
  const int threads = waves * lanes;
  Shared sh(threads);
  std::vector<std::unique_ptr<Wave>> of;
  for (int k = 0; k < waves; ++k) of.push_back(std::make_unique<Wave>(lanes));
  std::vector<std::thread> pool;
  for (int t = 0; t < threads; ++t)
    pool.emplace_back([&, t] {
      LaneTeam team{{sh, t}, *of[t / lanes], waves, lanes};
      if (threads >= st.s.seqs) plan_scan<true>(team, p, arrays);
      else plan_scan<false>(team, p, arrays);
    });
  for (auto& t : pool) t.join();
  for (int t = 0; t < threads; ++t) {
    ThreadTeam team{sh, 0};
    plan_fill(team, p, arrays, t, threads);
  }
  return r;
}

// Trees, one after the other, most of whose branches take a token or a few; some rest, some end, some have many.
Step rollout_step(std::mt19937& rng, int seqs) {
  auto in = [&](int a, int b) { return (int)std::uniform_int_distribution<int>(a, b)(rng); };
  Step st;
  const int heads[][2] = {{1, 1}, {4, 2}, {7, 1}, {32, 8}, {130, 1}};
  const int* h = heads[in(0, 4)];
  const int page = 16 << in(0, 4);
  int root = -1, left = 0, rows = 0, live = 0, need = 0, widest = 1;
  const int most = in(0, 1) ? 40 : 9;
  for (int i = 0; i < seqs; ++i) {
    const bool child = left-- > 0;
    if (!child) root = i, left = in(0, 5) ? in(0, most) : 0;
    st.parent.push_back(child ? root : -1);
    st.length.push_back(in(0, 4) ? in(0, child ? 90 : 200) : 0);
    const int kind = in(0, 19);
    st.fresh.push_back(child ? (kind < 14 ? 1 : kind < 16 ? in(2, 5) : kind < 18 ? 0 : kind < 19 ? -1 : in(20, 90))
                             : (kind < 15 ? 0 : in(1, 40)));
    const int n = std::max(0, st.fresh[i]);
    rows += n;
    live += cdiv(st.length[i], page);
    need += cdiv(st.length[i] + n, page) - cdiv(st.length[i], page);
    widest = std::max(widest, cdiv(st.length[i] + n, page));
  }
  const int pages = live + need + in(1, 5);
  st.s = PagedShape{seqs, rows + in(0, 9), h[0], h[1], page, widest, pages};
  std::vector<int32_t> ids(pages);
  for (int i = 0; i < pages; ++i) ids[i] = i;
  std::shuffle(ids.begin(), ids.end(), rng);
  st.table.assign((size_t)seqs * widest, -1);
  int at = 0;
  for (int i = 0; i < seqs; ++i)
    for (int k = 0; k < cdiv(st.length[i], page); ++k) st.table[(size_t)i * widest + k] = ids[at++];
  st.state = {in(0, pages - 1), pages - live};
  st.ring.assign(pages, -1);
  for (int k = 0; k < pages - live; ++k) st.ring[(st.state[0] + k) % pages] = ids[live + k];
  return st;
}

}  // namespace

int main() {
  std::mt19937 rng(23);
  const int teams[][2] = {{1, 8}, {3, 4}, {4, 8}, {2, 16}, {5, 2}, {1, 1}};
  int runs = 0, steps = 0;
  for (int k = 0; k < 60; ++k) {
    const Step st = rollout_step(rng, 1 + (int)(rng() % (k % 3 ? 60 : 250)));
    const PlanLayout lay = plan_layout(st.s);
    Result first;
    for (int t = 0; t < 3; ++t) {
      const int* team = teams[(k + t) % 6];
      const Result r = run_lanes(st, team[0], team[1]);
      if (t == 0) {
        check_good(st, r, "status of a good step");
        first = r;
      }
      check(std::equal(r.plan.begin(), r.plan.begin() + lay.work, first.plan.begin()) &&
            std::equal(r.plan.begin() + lay.slots, r.plan.end(), first.plan.begin() + lay.slots) && r.table == first.table,
            "the plan does not depend on the team");
    }
    const int32_t* run = first.plan.data() + lay.work;
    const PlanArrays a = PlanArrays::packed(const_cast<int32_t*>(run), st.s.seqs);
    for (int i = 0; i < st.s.seqs; ++i) runs += a.run[i] == i && a.run_rows[i] > st.fresh[i];
    ++steps;
  }
  check(runs > 300, "steps with runs");
  if (g_errors) {
    std::printf("%d errors\n", g_errors);
    return 1;
  }
  std::printf("ok: %d steps, %d runs\n", steps, runs);
  return 0;
}
