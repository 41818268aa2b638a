// Host logic of the linear-attention layer (linear.cpp) without a GPU: stand-ins
// for its kernel launchers check every launch against the batch it was called
// for. Random batches of trees go through every entry point; each launch in turn
// reports a HIP error.
//
// Checked: the segments (inline, or as the table launches wrote them) name every
// row of the batch once and every branch's tree; blocks are numbered without
// gaps and cut at multiples of 64 rows that follow from the tree alone; all
// state arrays lie inside the workspace, apart from one another; launches come in
// the order that hands states from prompts to branches and back.
#include <hip/hip_runtime_api.h>

#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>
#include <string>
#include <vector>

#include "augtree.h"
#include "linear.h"

using namespace augtree;

namespace {

const augtree_groups* g_grp;
char* g_ws;
size_t g_ws_bytes;
std::vector<std::string> g_launches;
int g_fail_at = 0, g_calls = 0, g_errors = 0;
std::vector<std::pair<const char*, size_t>> g_ranges;

void check(bool ok, const char* what) {
  if (!ok) {
    std::printf("FAILED: %s\n", what);
    ++g_errors;
  }
}

hipError_t launched(const std::string& what) {
  g_launches.push_back(what);
  return ++g_calls == g_fail_at ? hipErrorLaunchFailure : hipSuccess;
}

void inside(const void* p, size_t bytes, const char* what) {
  const char* c = static_cast<const char*>(p);
  check(c >= g_ws && c + bytes <= g_ws + g_ws_bytes, what);
  check(reinterpret_cast<uintptr_t>(p) % 256 == 0, "alignment in the workspace");
  for (const auto& r : g_ranges)
    check((c == r.first && bytes == r.second) || c + bytes <= r.first || r.first + r.second <= c, "arrays overlap");
  g_ranges.push_back({c, bytes});
}

size_t state_bytes() { return (size_t)g_grp->num_kv_heads * g_grp->head_dim * g_grp->head_dim * 4; }

void check_batch(const LinBatch& b) {
  const augtree_groups& g = *g_grp;
  const int ng = g.num_groups, nb = g.num_branches;
  check(b.num_trees == ng && b.num_branches == nb && b.heads_kv == g.num_kv_heads, "counts");
  check(b.group * g.num_kv_heads == g.num_q_heads, "group");
  check((b.segs == nullptr) == (ng + nb <= kLinInlineSegs), "inline or table");
  const LinSeg* s = b.segs ? b.segs : b.inl;
  int block = 0;
  for (int i = 0; i < ng + nb; ++i) {
    const bool prompt = i < ng;
    const int j = prompt ? i : i - ng;
    const int32_t* cu = prompt ? g.cu_prompt : g.cu_resp;
    check(s[i].row0 == cu[j] && s[i].len == cu[j + 1] - cu[j], "rows of a segment");
    check(s[i].block0 == block, "block numbers");
    check(s[i].rows % kLinChunk == 0 && s[i].rows >= kLinChunk, "rows of a block");
    const int n = (s[i].len + s[i].rows - 1) / s[i].rows;
    check(s[i].rows == kLinChunk || (int64_t)n * (s[i].rows - kLinChunk) < s[i].len, "even blocks");
    block += n;
    if (prompt) {
      check(nb == 0 ? s[i].link == 0 : s[i].link == g.cu_branch[j], "first branch");
    } else {
      const int t = s[i].link;
      check(t >= 0 && t < ng && j >= g.cu_branch[t] && j < g.cu_branch[t + 1], "tree of a branch");
    }
  }
  check(block == b.num_blocks, "number of blocks");
}

}  // namespace

namespace augtree {

hipError_t launch_lin_table(const LinTable& t, hipStream_t) {
  check(t.n > 0 && t.n <= kLinTableWords, "table words");
  const char* c = reinterpret_cast<const char*>(t.dst);
  check(c >= g_ws && c + 4 * (size_t)t.n <= g_ws + g_ws_bytes, "table inside the workspace");
  std::memcpy(t.dst, t.words, 4 * (size_t)t.n);
  return launched("table");
}
hipError_t launch_lin_state(const LinStateParams& p, int d, bool reverse, hipStream_t) {
  check(d == g_grp->head_dim, "head_dim");
  check_batch(p.b);
  check(p.heads_y == (reverse ? g_grp->num_q_heads : g_grp->num_kv_heads), "heads of y");
  inside(p.states, state_bytes() * p.b.num_blocks, "states");
  return launched(reverse ? "state_rev" : "state");
}
hipError_t launch_lin_scan(const LinScanParams& p, int, bool reverse, int part, hipStream_t) {
  check_batch(p.b);
  inside(p.states, state_bytes() * p.b.num_blocks, "states");
  const size_t ends = reverse ? (p.b.num_branches ? p.b.num_branches : 1) : p.b.num_trees;
  inside(p.ends, state_bytes() * ends, "ends");
  return launched(std::string(reverse ? "scan_rev" : "scan") + (part == 0 ? "" : part == 1 ? "_p" : "_r"));
}
hipError_t launch_lin_out(const LinOutParams& p, int, hipStream_t) {
  check_batch(p.b);
  inside(p.states, state_bytes() * p.b.num_blocks, "states");
  return launched("out");
}
hipError_t launch_lin_dq(const LinGradParams& p, int, hipStream_t) {
  check_batch(p.b);
  return launched("dq");
}
hipError_t launch_lin_dkv(const LinGradParams& p, int, hipStream_t) {
  check_batch(p.b);
  inside(p.states_rev, state_bytes() * p.b.num_blocks, "reverse states");
  return launched("dkv");
}
hipError_t launch_lin_step(const LinStepParams&, int, hipStream_t) { return launched("step"); }
hipError_t launch_head_norm_fwd(const HeadNormParams&, hipStream_t) { return launched("norm"); }
hipError_t launch_head_norm_bwd(const HeadNormParams&, hipStream_t) { return launched("norm_bwd"); }

}  // namespace augtree

int main() {
  std::mt19937 rng(5);
  auto below = [&](int n) { return (int)(rng() % n); };
  // addresses that stand for tensors: far apart, never read
  auto at = [](int i) { return reinterpret_cast<uint16_t*>((uintptr_t(1) << 50) + (uintptr_t(i) << 44)); };
  int calls = 0, tables = 0, splits = 0;
  for (int round = 0; round < 60; ++round) {
    const int ng = round % 10 == 9 ? 60 : 1 + below(6);
    const bool plain = round % 7 == 3;
    std::vector<int32_t> cp{0}, cb{0}, cr{0};
    for (int t = 0; t < ng; ++t) {
      cp.push_back(cp.back() + 1 + (round % 4 == 0 ? below(60000) : below(700)));
      const int n = plain ? 0 : 1 + below(9);
      cb.push_back(cb.back() + n);
      for (int i = 0; i < n; ++i) cr.push_back(cr.back() + 1 + (round % 5 == 0 ? below(9000) : below(200)));
    }
    const int hkv = 1 + below(8), g = 1 + below(5), d = below(2) ? 64 : 128;
    augtree_groups grp = {ng, cb.back(), hkv * g, hkv, d, 0.125f, cp.data(), plain ? nullptr : cb.data(),
                          plain ? nullptr : cr.data()};
    g_grp = &grp;
    std::vector<float> decay(hkv, 0.99f);
    for (int backward = 0; backward < 2; ++backward) {
      const size_t need = augtree_linear_workspace_size(&grp, backward), fwd = augtree_linear_workspace_size(&grp, 0);
      check(need > 0, "workspace size");
      // only the segment table is written here: the states need no memory behind their addresses
      const size_t table = ((size_t)(ng + cb.back()) * sizeof(LinSeg) + 255) / 256 * 256;
      char* const mem = static_cast<char*>(std::aligned_alloc(256, table));
      auto rs = [&](int i) { return plain ? nullptr : at(i); };
      int launches = 0;
      for (int fail_at = 0; fail_at <= launches; ++fail_at) {
        g_ws = mem;
        g_ws_bytes = need;
        g_calls = 0;
        g_fail_at = fail_at;
        g_launches.clear();
        g_ranges.clear();
        // (mem stands for the whole workspace: addresses behind the table are formed, not used)
        const char* fwd_ws = reinterpret_cast<const char*>(at(20));
        const bool kept = backward && round % 2;
        const int st =
            backward
                ? augtree_linear_bwd(&grp, decay.data(), at(0), at(1), at(2), at(3), rs(4), rs(5), rs(6), rs(7), nullptr,
                                     at(8), at(9), at(10), rs(11), rs(12), rs(13), kept ? fwd_ws : nullptr, kept ? fwd : 0,
                                     mem, need, nullptr)
                : augtree_linear_fwd(&grp, decay.data(), at(0), at(1), at(2), rs(3), rs(4), rs(5), nullptr, at(6), rs(7),
                                     round % 3 ? reinterpret_cast<float*>(at(8)) : nullptr,
                                     round % 3 ? reinterpret_cast<float*>(rs(9)) : nullptr, mem, need, nullptr);
        ++calls;
        if (fail_at) {
          check(st == AUGTREE_ERR_HIP && std::strlen(augtree_last_error()) > 0, "a failed launch is reported");
          check((int)g_launches.size() == fail_at, "nothing is launched after a failed launch");
          continue;
        }
        check(st == AUGTREE_OK, augtree_last_error());
        launches = (int)g_launches.size();
        std::string order;
        for (const auto& l : g_launches) {
          if (l == "table") ++tables;
          else order += l + " ";
        }
        const bool split = order.find("_p") != std::string::npos;
        splits += split;
        std::string want;
        if (!kept) want += split ? "state scan_p scan_r " : "state scan ";
        if (backward) want += split ? "state_rev scan_rev_r scan_rev_p dq dkv " : "state_rev scan_rev dq dkv ";
        else want += "out ";
        check(order == want, order.c_str());
      }
      std::free(mem);
    }
  }
  if (g_errors) return 1;
  check(tables > 0 && splits > 0, "both forms of the segments and of the scan were met");
  std::printf("ok, %d calls, %d tables, %d split scans\n", calls, tables, splits);
  return 0;
}
