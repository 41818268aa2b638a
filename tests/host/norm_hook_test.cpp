// The launch hook around the head norm's kernels (linear.cpp), on the stand-ins
// of linear_host_test.cpp: called before and after each kernel that a call
// enqueues, the sum of the weight gradients being one of its own, and a failing
// launch, first or second, ends the call.
#define main linear_host_main
#include "linear_host_test.cpp"
#undef main

namespace {
std::vector<std::string> g_hooks;
void hook(const char* role, int phase, void*, void*) {
  g_hooks.push_back(std::string(role) + (phase ? " after " : " before ") + std::to_string(g_calls));
}
}  // namespace

int main() {
  auto at = [](int i) { return reinterpret_cast<uint16_t*>((uintptr_t(1) << 50) + (uintptr_t(i) << 44)); };
  auto f = [&](int i) { return reinterpret_cast<float*>(at(i)); };
  augtree_set_launch_hook(hook, nullptr);
  auto begin = [&](int fail_at) {
    g_calls = 0;
    g_fail_at = fail_at;
    g_launches.clear();
    g_hooks.clear();
  };
  auto bwd = [&](int64_t rows, bool dw, bool db) {
    return augtree_head_norm_bwd(rows, 3, 64, 1, 1e-5f, at(0), nullptr, f(1), f(2), at(3), at(4), nullptr, dw ? f(5) : nullptr,
                                 db ? f(6) : nullptr, at(7), augtree_head_norm_workspace_size(rows, 3, 64), nullptr);
  };
  typedef std::vector<std::string> V;
  const V one{"head_norm_bwd before 0", "head_norm_bwd after 1"};
  const V two{"head_norm_bwd before 0", "head_norm_bwd after 1", "head_norm_sum before 1", "head_norm_sum after 2"};
  begin(0);
  check(augtree_head_norm_fwd(4, 3, 64, 1, 1e-5f, at(0), nullptr, f(1), f(2), at(4), nullptr) == AUGTREE_OK, "forward");
  check(g_hooks == V({"head_norm before 0", "head_norm after 1"}), "hooks of a forward");
  begin(0);
  check(bwd(5, false, false) == AUGTREE_OK && g_hooks == one, "hooks of a backward without sums");
  for (int k = 1; k < 4; ++k) {
    for (int64_t rows : {0, 1, 5000}) {
      begin(0);
      check(bwd(rows, k & 1, k & 2) == AUGTREE_OK && g_hooks == two, "hooks of a backward with sums");
    }
    begin(1);
    check(bwd(5, k & 1, k & 2) == AUGTREE_ERR_HIP && g_hooks == one, "the first launch fails");
    begin(2);
    check(bwd(5, k & 1, k & 2) == AUGTREE_ERR_HIP && g_hooks == two, "the second launch fails");
  }
  if (g_errors) return 1;
  std::printf("ok\n");
  return 0;
}
