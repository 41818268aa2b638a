// Sums of a plan's counts that no room can hold (paged.h), on the team of
// paged_host_test.cpp: they stop above every room instead of passing 32 bits,
// however they are grouped, so that such steps are refused.
#define main paged_host_main
#include "paged_host_test.cpp"
#undef main

namespace {

// A scan over `n` values as the lanes of a wavefront do it: pairs, then pairs of pairs.
int32_t by_pairs(std::vector<int32_t> v) {
  while (v.size() > 1) {
    std::vector<int32_t> w;
    for (size_t i = 0; i < v.size(); i += 2) w.push_back(i + 1 < v.size() ? add_count(v[i], v[i + 1]) : v[i]);
    v.swap(w);
  }
  return v[0];
}

// `seqs` sequences of `cached` tokens that ask for `each` new ones, in a pool that has `spare` pages left; no table, which
// a refused step does not touch.
Step greedy(int seqs, int cached, int each, int rows, int page, int max_pages, int spare) {
  Step st;
  st.s = PagedShape{seqs, rows, 1, 1, page, max_pages, spare};
  st.length.assign(seqs, cached);
  st.fresh.assign(seqs, each);
  st.parent.assign(seqs, -1);
  st.ring.assign(spare, 0);
  st.state = {0, spare};
  return st;
}

}  // namespace

int main() {
  const int32_t room = 1 << 30;  // the most rows, and more than the most pages, that a call may have
  check(add_count(room, 0) == room && add_count(room - 1, 1) == room, "a full room is no more than it");
  check(add_count(room, 1) > room && add_count(room, room) > room && add_count(room + 1, room + 1) > room, "what passes it");
  check(add_count(kMostCount, kMostCount) == kMostCount && add_count(0, kMostCount) == kMostCount, "the end of counting");
  for (int n : {2, 3, 16, 64, 1024})
    for (int32_t x : {room / n + 1, (1 << 21) + 5, room - 1, room, room + 1, kMostCount})
      check(by_pairs(std::vector<int32_t>(n, x)) == (int32_t)std::min<int64_t>((int64_t)n * x, kMostCount), "sums by pairs");

  // new tokens past 2^31, and their pages; each sequence alone has room in its table
  for (int threads : {1, 3, 8})
    for (bool in_place : {false, true}) {
      const Step st = greedy(2500, 0, 1 << 20, 1 << 20, 256, 1 << 12, 64);
      check_refused(st, run(st, threads, in_place), PAGES_ROWS | PAGES_SHORT);
    }
  // lengths at the end of tables of 2^30 tokens
  {
    const Step st = greedy(3, room - 16, 16, 48, 16, 1 << 26, 2);
    check_refused(st, run(st, 2, false), PAGES_SHORT);
  }
  if (g_errors) {
    std::printf("%d errors\n", g_errors);
    return 1;
  }
  std::printf("ok\n");
  return 0;
}
