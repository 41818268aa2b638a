// The backward that is given the forward's workspace (linear.cpp), on the
// stand-ins of linear_host_test.cpp: it needs a table, the reverse states and
// the branches' ends, no room for states that it does not form, and its arrays
// lie inside a workspace of just that size.
#define main linear_host_main
#include "linear_host_test.cpp"
#undef main

int main() {
  std::mt19937 rng(7);
  auto below = [&](int n) { return (int)(rng() % n); };
  auto at = [](int i) { return reinterpret_cast<uint16_t*>((uintptr_t(1) << 50) + (uintptr_t(i) << 44)); };
  auto up = [](size_t n) { return (n + 255) / 256 * 256; };
  int tables = 0, splits = 0;
  for (int round = 0; round < 40; ++round) {
    const int ng = round % 10 == 9 ? 60 : 1 + below(6);
    const bool plain = round % 7 == 3;
    std::vector<int32_t> cp{0}, cb{0}, cr{0};
    for (int t = 0; t < ng; ++t) {
      cp.push_back(cp.back() + 1 + (round % 4 == 0 ? below(60000) : below(700)));
      const int n = plain ? 0 : 1 + below(9);
      cb.push_back(cb.back() + n);
      for (int i = 0; i < n; ++i) cr.push_back(cr.back() + 1 + (round % 5 == 0 ? below(9000) : below(200)));
    }
    const int hkv = 1 + below(8), g = 1 + below(5), d = below(2) ? 64 : 128, nb = cb.back();
    augtree_groups grp = {ng, nb, hkv * g, hkv, d, 0.125f, cp.data(), plain ? nullptr : cb.data(),
                          plain ? nullptr : cr.data()};
    g_grp = &grp;
    std::vector<float> decay(hkv, 0.99f);
    const size_t fwd = augtree_linear_workspace_size(&grp, 0), bwd = augtree_linear_workspace_size(&grp, 1),
                 kept = augtree_linear_workspace_size(&grp, 2);
    const size_t table = up((size_t)(ng + nb) * sizeof(LinSeg)), state = state_bytes();
    const size_t states = fwd - table - up(state * ng);
    check(kept == table + states + up(state * (nb > 1 ? nb : 1)), "table, reverse states and ends");
    check(bwd == kept + states + up(state * ng), "and, without the forward's workspace, its states");
    char* const mem = static_cast<char*>(std::aligned_alloc(256, table));
    auto rs = [&](int i) { return plain ? nullptr : at(i); };
    auto call = [&](size_t bytes, bool with_fwd) {
      g_ws = mem;
      g_ws_bytes = bytes;
      g_calls = g_fail_at = 0;
      g_launches.clear();
      g_ranges.clear();
      return augtree_linear_bwd(&grp, decay.data(), at(0), at(1), at(2), at(3), rs(4), rs(5), rs(6), rs(7), nullptr, at(8),
                                at(9), at(10), rs(11), rs(12), rs(13),
                                with_fwd ? reinterpret_cast<const char*>(at(20)) : nullptr, with_fwd ? fwd : 0, mem, bytes,
                                nullptr);
    };
    check(call(kept, true) == AUGTREE_OK, augtree_last_error());
    int others = 0;
    for (const auto& l : g_launches) {
      if (l == "table") ++tables;
      else ++others, splits += l == "scan_rev_p";
    }
    check(others == 4 || others == 5, "reverse states, scan, dq, dk and dv");
    check(call(bwd, true) == AUGTREE_OK, "a larger workspace serves too");
    check(call(bwd, false) == AUGTREE_OK, augtree_last_error());
    check(call(kept - 1, true) == AUGTREE_ERR_WORKSPACE && g_launches.empty(), "too small");
    check(call(kept, false) == AUGTREE_ERR_WORKSPACE && g_launches.empty(), "too small to form the forward's states");
    std::free(mem);
  }
  if (g_errors) return 1;
  check(tables > 0 && splits > 0, "both forms of the segments and of the scan were met");
  std::printf("ok, %d tables, %d split scans\n", tables, splits);
  return g_errors != 0;
}
