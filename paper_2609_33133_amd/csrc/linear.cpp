// Host side of the linear-attention layer: argument validation, segment
// tables, workspace layout and launches.
//
// The segment table travels in the kernel arguments; a batch of more than
// kLinInlineSegs segments has it written into the workspace by small kernels
// that carry it in theirs. So every call enqueues kernels only.
#include "linear.h"

#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstring>
#include <exception>
#include <vector>

#include "../../include/augtree.h"
#include "internal.h"

using namespace augtree;

namespace {

template <class... A>
int fail(int status, const char* fmt, A... a) {
  char buf[512];
  std::snprintf(buf, sizeof(buf), fmt, a...);
  return fail_status(status, buf);
}

int hip_ok(hipError_t e, const char* what) {
  return e == hipSuccess ? AUGTREE_OK : fail(AUGTREE_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

// Calls the launch hook around one kernel launch.
struct Hook {
  const char* role;
  hipStream_t stream;
  Hook(const char* r, hipStream_t s) : role(r), stream(s) { launch_hook(role, 0, stream); }
  ~Hook() { launch_hook(role, 1, stream); }
};

// No C++ exception crosses the ABI (the tables are vectors).
template <class F>
int guarded(F f) {
  try {
    return f();
  } catch (const std::exception& e) {
    return fail(AUGTREE_ERR_INVALID_ARGUMENT, "host allocation failed: %s", e.what());
  }
}

int check_ptr(const void* p, const char* name, bool required, size_t align = 16) {
  if (!p) return required ? fail(AUGTREE_ERR_INVALID_ARGUMENT, "null pointer: %s", name) : AUGTREE_OK;
  if (reinterpret_cast<uintptr_t>(p) % align)
    return fail(AUGTREE_ERR_MISALIGNED, "pointer %s is not %d-byte aligned", name, (int)align);
  return AUGTREE_OK;
}

int check_heads(int hq, int hkv, int d, float scale, const float* decay) {
  if (hq < 1 || hkv < 1) return fail(AUGTREE_ERR_INVALID_ARGUMENT, "head counts must be >= 1");
  if (hq % hkv) return fail(AUGTREE_ERR_UNSUPPORTED, "num_q_heads %d not a multiple of num_kv_heads %d", hq, hkv);
  if (hq > 65536) return fail(AUGTREE_ERR_UNSUPPORTED, "num_q_heads %d > 65536", hq);  // 64 rows within 2^31 bytes
  if (hkv > kLinMaxHeads) return fail(AUGTREE_ERR_UNSUPPORTED, "num_kv_heads %d > %d", hkv, kLinMaxHeads);
  if (d != 64 && d != 128) return fail(AUGTREE_ERR_UNSUPPORTED, "head_dim %d not in {64,128}", d);
  if (!(scale > 0.f) || !std::isfinite(scale))
    return fail(AUGTREE_ERR_INVALID_ARGUMENT, "softmax_scale must be finite and > 0");
  if (!decay) return fail(AUGTREE_ERR_INVALID_ARGUMENT, "null pointer: decay");
  for (int h = 0; h < hkv; ++h)
    if (!(decay[h] > 0.f && decay[h] <= 1.f))
      return fail(AUGTREE_ERR_INVALID_ARGUMENT, "decay[%d] = %g not in (0, 1]", h, (double)decay[h]);
  return AUGTREE_OK;
}

int check_offsets(const int32_t* cu, int n, const char* name) {
  if (!cu) return fail(AUGTREE_ERR_INVALID_ARGUMENT, "null offset array: %s", name);
  if (cu[0] != 0) return fail(AUGTREE_ERR_INVALID_ARGUMENT, "%s must start at 0", name);
  for (int i = 0; i < n; ++i)
    if (cu[i + 1] <= cu[i])
      return fail(AUGTREE_ERR_INVALID_ARGUMENT, "%s: length %d is not positive or offsets decrease", name, i);
  return AUGTREE_OK;
}

// num_branches == 0: prompts only, cu_branch and cu_resp are not read
int check_batch(const augtree_groups* g, const float* decay) {
  if (!g) return fail(AUGTREE_ERR_INVALID_ARGUMENT, "null descriptor");
  if (g->num_groups < 1 || g->num_branches < 0)
    return fail(AUGTREE_ERR_INVALID_ARGUMENT, "num_groups=%d must be >= 1, num_branches=%d >= 0", g->num_groups,
                g->num_branches);
  int st = check_offsets(g->cu_prompt, g->num_groups, "cu_prompt");
  if (!st && g->num_branches > 0) {
    st = check_offsets(g->cu_branch, g->num_groups, "cu_branch");
    if (!st && g->cu_branch[g->num_groups] != g->num_branches)
      return fail(AUGTREE_ERR_INVALID_ARGUMENT, "cu_branch[num_groups]=%d != num_branches=%d",
                  g->cu_branch[g->num_groups], g->num_branches);
    if (!st) st = check_offsets(g->cu_resp, g->num_branches, "cu_resp");
  }
  return st ? st : check_heads(g->num_q_heads, g->num_kv_heads, g->head_dim, g->softmax_scale, decay);
}

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Rounds of `units` workgroups with at most `per_cu` on each of 256 CUs; w of them on a CU take sqrt(w) times
// as long as one (measured: 1.42 for two, 2.0 for four).
double rounds(int64_t units, int per_cu) {
  const int64_t rest = units % (256 * per_cu);
  return (double)(units / (256 * per_cu)) * std::sqrt((double)per_cu) + std::sqrt((double)cdiv(rest, 256));
}

// Rows of a tree's blocks: those for which this model of a training step's kernels gives the shortest time. A
// workgroup of the output kernel takes `row` us a row and 2 d / (1 + group) rows' time for its state; dq and
// the state kernels come to 1.75 of that; dk and dv take 0.9 a row and twice the state, with workgroups that
// fill twice the room; each of the two scans moves the states once in and out at 4.7 TB/s, but takes 0.12 us
// for every block of its longest chain. Measured: over 88 random trees of up to 30 k rows and seven head layouts
// the rows chosen take 0.6 % longer on average than the best of 64, 128, 192, 256, 384, 512, 768 and 1024; with
// d = 128 4.8 % at most, with d = 64 (17 of them) 1.9 % on average and once 16 % (8 k rows with short branches,
// 16 / 4 heads). A training step of 32768 rows with eight branches of 2048, 32 / 8 heads, d = 128, takes 1059 us
// with the 832 rows chosen, 1110 with 512, 1150 with 1024. The tree alone decides, so that its results do not
// depend on the batch.
int block_rows(const augtree_groups* g, int tree) {
  const int d = g->head_dim, hkv = g->num_kv_heads, nb = g->num_branches, group = g->num_q_heads / hkv;
  const double row = group * (d == 128 ? 0.033 : 0.025), state = 2.0 * d / (1 + group);
  auto blocks = [](int32_t len, uint32_t rows) { return ((uint32_t)len + rows - 1) / rows; };
  int best = 0;
  double best_cost = 0;
  for (int rows = kLinChunk; rows <= 1024; rows += kLinChunk) {
    const int64_t prompt = blocks(g->cu_prompt[tree + 1] - g->cu_prompt[tree], rows);
    int64_t units = prompt, longest = 0;
    for (int b = nb ? g->cu_branch[tree] : 0; nb && b < g->cu_branch[tree + 1]; ++b) {
      const int64_t n = blocks(g->cu_resp[b + 1] - g->cu_resp[b], rows);
      units += n;
      longest = std::max(longest, n);
    }
    units *= hkv;
    const double cost = 2.75 * row * (rows + state) * rounds(units, d == 128 ? 2 : 4) +
                        0.9 * row * (rows + 2 * state) * rounds(units, d == 128 ? 1 : 2) +
                        2 * std::max((double)units * d * d * 8 / 4.7e6, 0.12 * (double)(prompt + longest));
    if (!best || cost < best_cost) best = rows, best_cost = cost;
  }
  return best;
}

constexpr int64_t kScanBlocks = 32;

struct Layout {
  std::vector<LinSeg> segs;
  int64_t blocks = 0, longest = 0;  // of the batch; of the tree with the most
  size_t states = 0, tree = 0;  // bytes: states of all blocks; one state per tree
};

size_t align_up(size_t n) { return (n + 255) / 256 * 256; }

// (A launch has fewer than 2^32 threads: the state and the scan kernels' are the most.)
int make_layout(const augtree_groups* g, Layout* L) {
  const int ng = g->num_groups, nb = g->num_branches;
  L->segs.resize((size_t)ng + nb);
  int64_t blocks = 0;
  // A segment is cut evenly, into the number of blocks that block_rows of a block would make: the branches' blocks, which
  // start last, are then no longer than they have to be (that step: 1076 us against 1081).
  auto add = [&](int i, int row0, int len, int link, int rows) {
    const int64_t n = cdiv(len, rows);
    LinSeg& s = L->segs[i];
    s.row0 = row0;
    s.len = len;
    s.link = link;
    s.rows = n ? (int32_t)(cdiv(cdiv(len, n), kLinChunk) * kLinChunk) : kLinChunk;
    s.block0 = (int32_t)std::min<int64_t>(blocks, INT32_MAX);
    const int64_t own = cdiv(len, s.rows);
    blocks += own;
    return own;
  };
  std::vector<int> rows(ng);
  std::vector<int64_t> own(ng);
  for (int t = 0; t < ng; ++t) {
    rows[t] = block_rows(g, t);
    own[t] = add(t, g->cu_prompt[t], g->cu_prompt[t + 1] - g->cu_prompt[t], nb ? g->cu_branch[t] : 0, rows[t]);
  }
  for (int t = 0; nb && t < ng; ++t)
    for (int b = g->cu_branch[t]; b < g->cu_branch[t + 1]; ++b)
      own[t] += add(ng + b, g->cu_resp[b], g->cu_resp[b + 1] - g->cu_resp[b], t, rows[t]);
  L->longest = *std::max_element(own.begin(), own.end());
  const int64_t hkv = g->num_kv_heads, d = g->head_dim;
  if (blocks * hkv * 4 * d > UINT32_MAX || (ng + (int64_t)nb) * hkv * (d * d / 1024) * 256 > UINT32_MAX)
    return fail(AUGTREE_ERR_UNSUPPORTED, "%lld blocks, %lld prompts and branches of %d KV heads exceed a launch",
                (long long)blocks, (long long)ng + nb, g->num_kv_heads);
  L->blocks = blocks;
  const size_t state = (size_t)g->num_kv_heads * g->head_dim * g->head_dim * sizeof(float);
  L->states = align_up(state * (size_t)blocks);
  L->tree = state;
  return AUGTREE_OK;
}

// What a workspace is for: a forward, a backward, a backward that is given the forward's workspace.
enum Use { kForward = 0, kBackward = 1, kBackwardKept = 2 };
Use use_of(int backward) { return backward == kBackwardKept ? kBackwardKept : backward ? kBackward : kForward; }

size_t workspace_bytes(const augtree_groups* g, const Layout& L, Use use) {
  size_t n = align_up(L.segs.size() * sizeof(LinSeg));
  if (use != kBackwardKept) n += L.states + align_up(L.tree * g->num_groups);
  if (use != kForward) n += L.states + align_up(L.tree * (size_t)std::max(1, g->num_branches));
  return n;
}

// A call: the batch in kernel form, the workspace handed out piece by piece.
struct Call {
  const augtree_groups* g;
  Layout L;
  LinBatch b;
  char* ws;
  hipStream_t stream;

  template <class T>
  T* take(size_t bytes) {
    T* p = reinterpret_cast<T*>(ws);
    ws += align_up(bytes);
    return p;
  }

  // after validation: segment table, inline or through the workspace
  int begin(const float* decay) {
    std::memset(&b, 0, sizeof(b));
    const size_t n = L.segs.size();
    b.num_trees = g->num_groups;
    b.num_branches = g->num_branches;
    b.num_blocks = (int32_t)L.blocks;
    b.heads_kv = g->num_kv_heads;
    b.group = g->num_q_heads / g->num_kv_heads;
    for (int h = 0; h < b.heads_kv; ++h) b.log2_decay[h] = (float)std::log2((double)decay[h]);
    LinSeg* table = take<LinSeg>(n * sizeof(LinSeg));
    if (n <= (size_t)kLinInlineSegs) {
      std::copy(L.segs.begin(), L.segs.end(), b.inl);
      return AUGTREE_OK;
    }
    b.segs = table;
    const size_t words = n * (sizeof(LinSeg) / 4);
    const int32_t* src = reinterpret_cast<const int32_t*>(L.segs.data());
    for (size_t at = 0; at < words; at += kLinTableWords) {
      LinTable t;
      t.dst = reinterpret_cast<int32_t*>(table) + at;
      t.n = (int32_t)std::min<size_t>(kLinTableWords, words - at);
      std::memcpy(t.words, src + at, (size_t)t.n * 4);
      Hook h("linear_table", stream);
      if (int st = hip_ok(launch_lin_table(t, stream), "segment table launch")) return st;
    }
    return AUGTREE_OK;
  }

  // states[block] <- what reaches the block
  int states(bool reverse, const uint16_t* const y[2], const uint16_t* const z[2], const float* init, float* states,
             float* ends, float* out_p, float* out_r) {
    const bool branches = g->num_branches > 0;
    LinStateParams s;
    std::memset(&s, 0, sizeof(s));
    for (int i = 0; i < 2; ++i) s.y[i] = y[i], s.z[i] = z[i];
    s.heads_y = reverse ? g->num_q_heads : g->num_kv_heads;
    s.states = states;
    // nobody reads a prompt's own end without branches (a start in reverse), nor a branch's unless it is handed out
    s.skip_prompt = reverse || (!branches && !out_p);
    s.skip_branch = !reverse && !out_r;
    s.b = b;
    {
      Hook h(reverse ? "linear_state_rev" : "linear_state", stream);
      if (int st = hip_ok(launch_lin_state(s, g->head_dim, reverse, stream), "state launch")) return st;
    }
    LinScanParams c;
    std::memset(&c, 0, sizeof(c));
    c.states = states;
    c.init = init;
    c.ends = ends;
    c.out_p = out_p;
    c.out_r = out_r;
    c.b = b;
    // A tree's blocks are scanned by one launch, its branches one after the other, where they are few; else prompts and
    // branches get a launch each, in which the branches run side by side (32 / 8 heads, d = 128, both scans of a step,
    // one launch against two: two trees of 27 and 29 blocks 28 us against 32; 64 blocks, 8 branches, 41 against 36).
    const bool split = branches && L.longest > kScanBlocks;
    for (int k = 0; k < (split ? 2 : 1); ++k) {
      const int part = !split ? 0 : (k == 0) != reverse ? 1 : 2;
      Hook h(reverse ? "linear_scan_rev" : "linear_scan", stream);
      if (int st = hip_ok(launch_lin_scan(c, g->head_dim, reverse, part, stream), "scan launch")) return st;
    }
    return AUGTREE_OK;
  }
};

int check_ws(const void* ws, size_t have, size_t need) {
  if (!ws || have < need)
    return fail(AUGTREE_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", ws ? have : (size_t)0, need);
  return check_ptr(ws, "ws", true, 256);
}

struct Named {
  const void* p;
  const char* name;
};

int check_all(const Named* v, int n, bool required) {
  for (int i = 0; i < n; ++i)
    if (int st = check_ptr(v[i].p, v[i].name, required)) return st;
  return AUGTREE_OK;
}

bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a && b && na && nb && x < y + nb && y < x + na;
}

// A tensor of a call, for the check that outputs are apart from all else. An `in_place` output may be an `in_place`
// input itself.
struct Span {
  const void* p;
  size_t bytes;
  const char* name;
  bool in_place = false;
};

int check_apart(const Span* in, int n_in, const Span* out, int n_out) {
  for (int i = 0; i < n_out; ++i) {
    for (int j = 0; j < n_in; ++j)
      if (overlap(out[i].p, out[i].bytes, in[j].p, in[j].bytes) &&
          !(out[i].in_place && in[j].in_place && out[i].p == in[j].p))
        return fail(AUGTREE_ERR_INVALID_ARGUMENT, "%s overlaps %s", out[i].name, in[j].name);
    for (int j = 0; j < i; ++j)
      if (overlap(out[i].p, out[i].bytes, out[j].p, out[j].bytes))
        return fail(AUGTREE_ERR_INVALID_ARGUMENT, "%s overlaps %s", out[i].name, out[j].name);
  }
  return AUGTREE_OK;
}

// bytes of a batch's tensors: q and k rows of prompts and responses, states of trees and branches
struct Sizes {
  size_t qp, kp, qr, kr, sp, sr;
  explicit Sizes(const augtree_groups* g) {
    const size_t row = 2 * (size_t)g->head_dim, tp = g->cu_prompt[g->num_groups],
                 tr = g->num_branches ? g->cu_resp[g->num_branches] : 0;
    const size_t state = (size_t)g->num_kv_heads * g->head_dim * g->head_dim * sizeof(float);
    qp = tp * row * g->num_q_heads;
    kp = tp * row * g->num_kv_heads;
    qr = tr * row * g->num_q_heads;
    kr = tr * row * g->num_kv_heads;
    sp = state * g->num_groups;
    sr = state * g->num_branches;
  }
};

}  // namespace

extern "C" {

size_t augtree_linear_workspace_size(const augtree_groups* grp, int backward) {
  size_t n = 0;
  guarded([&]() -> int {
    static const std::vector<float> ones(kLinMaxHeads, 1.f);
    if (int st = check_batch(grp, ones.data())) return st;
    Layout L;
    if (int st = make_layout(grp, &L)) return st;
    n = workspace_bytes(grp, L, use_of(backward));
    return fail_status(AUGTREE_OK, "");
  });
  return n;
}

int augtree_linear_fwd(const augtree_groups* grp, const float* decay, const uint16_t* q_p, const uint16_t* k_p,
                       const uint16_t* v_p, const uint16_t* q_r, const uint16_t* k_r, const uint16_t* v_r,
                       const float* state, uint16_t* o_p, uint16_t* o_r, float* state_p, float* state_r, void* ws,
                       size_t ws_bytes, void* stream) {
  return guarded([&]() -> int {
    int st = check_batch(grp, decay);
    if (st) return st;
    const bool br = grp->num_branches > 0;
    const Named prompt[] = {{q_p, "q_p"}, {k_p, "k_p"}, {v_p, "v_p"}, {o_p, "o_p"}};
    const Named resp[] = {{q_r, "q_r"}, {k_r, "k_r"}, {v_r, "v_r"}, {o_r, "o_r"}};
    const Named opt[] = {{state, "state"}, {state_p, "state_p"}, {state_r, "state_r"}};
    if ((st = check_all(prompt, 4, true)) || (br && (st = check_all(resp, 4, true))) || (st = check_all(opt, 3, false)))
      return st;
    if (!br && state_r) return fail(AUGTREE_ERR_INVALID_ARGUMENT, "state_r without branches");
    const Sizes z(grp);
    const Span ins[] = {{q_p, z.qp, "q_p"}, {k_p, z.kp, "k_p"}, {v_p, z.kp, "v_p"}, {q_r, z.qr, "q_r"},
                        {k_r, z.kr, "k_r"}, {v_r, z.kr, "v_r"}, {state, z.sp, "state", true}};
    const Span outs[] = {{o_p, z.qp, "o_p"}, {o_r, z.qr, "o_r"}, {state_p, z.sp, "state_p", true},
                         {state_r, z.sr, "state_r"}, {ws, ws_bytes, "ws"}};
    if ((st = check_apart(ins, 7, outs, 5))) return st;
    Call c;
    c.g = grp;
    if ((st = make_layout(grp, &c.L)) || (st = check_ws(ws, ws_bytes, workspace_bytes(grp, c.L, kForward))) ||
        (st = augtree_check_device()))
      return st;
    c.ws = static_cast<char*>(ws);
    c.stream = static_cast<hipStream_t>(stream);
    if ((st = c.begin(decay))) return st;
    float* const states = c.take<float>(c.L.states);
    float* const tree = c.take<float>(c.L.tree * grp->num_groups);
    const uint16_t *const q[2] = {q_p, q_r}, *const k[2] = {k_p, k_r}, *const v[2] = {v_p, v_r};
    uint16_t* const o[2] = {o_p, o_r};
    if ((st = c.states(false, k, v, state, states, tree, state_p, state_r))) return st;
    LinOutParams p;
    std::memset(&p, 0, sizeof(p));
    for (int i = 0; i < 2; ++i) p.q[i] = q[i], p.k[i] = k[i], p.v[i] = v[i], p.o[i] = o[i];
    p.states = states;
    p.scale = grp->softmax_scale;
    p.b = c.b;
    Hook h("linear_out", c.stream);
    if ((st = hip_ok(launch_lin_out(p, grp->head_dim, c.stream), "output launch"))) return st;
    return fail_status(AUGTREE_OK, "");
  });
}

int augtree_linear_bwd(const augtree_groups* grp, const float* decay, const uint16_t* q_p, const uint16_t* k_p,
                       const uint16_t* v_p, const uint16_t* do_p, const uint16_t* q_r, const uint16_t* k_r,
                       const uint16_t* v_r, const uint16_t* do_r, const float* state, uint16_t* dq_p, uint16_t* dk_p,
                       uint16_t* dv_p, uint16_t* dq_r, uint16_t* dk_r, uint16_t* dv_r, const void* fwd_ws,
                       size_t fwd_ws_bytes, void* ws, size_t ws_bytes, void* stream) {
  return guarded([&]() -> int {
    int st = check_batch(grp, decay);
    if (st) return st;
    const bool br = grp->num_branches > 0;
    const Named prompt[] = {{q_p, "q_p"}, {k_p, "k_p"}, {v_p, "v_p"}, {do_p, "do_p"}, {dq_p, "dq_p"}, {dk_p, "dk_p"},
                            {dv_p, "dv_p"}};
    const Named resp[] = {{q_r, "q_r"}, {k_r, "k_r"}, {v_r, "v_r"}, {do_r, "do_r"}, {dq_r, "dq_r"}, {dk_r, "dk_r"},
                          {dv_r, "dv_r"}};
    if ((st = check_all(prompt, 7, true)) || (br && (st = check_all(resp, 7, true))) ||
        (st = check_ptr(state, "state", false)))
      return st;
    const Sizes z(grp);
    const Span ins[] = {{q_p, z.qp, "q_p"},   {k_p, z.kp, "k_p"}, {v_p, z.kp, "v_p"}, {do_p, z.qp, "do_p"}, {q_r, z.qr, "q_r"},
                        {k_r, z.kr, "k_r"},   {v_r, z.kr, "v_r"}, {do_r, z.qr, "do_r"}, {state, z.sp, "state"},
                        {fwd_ws, fwd_ws_bytes, "fwd_ws"}};
    const Span outs[] = {{dq_p, z.qp, "dq_p"}, {dk_p, z.kp, "dk_p"}, {dv_p, z.kp, "dv_p"}, {dq_r, z.qr, "dq_r"},
                         {dk_r, z.kr, "dk_r"}, {dv_r, z.kr, "dv_r"}, {ws, ws_bytes, "ws"}};
    if ((st = check_apart(ins, 10, outs, 7))) return st;
    Call c;
    c.g = grp;
    if ((st = make_layout(grp, &c.L)) ||
        (st = check_ws(ws, ws_bytes, workspace_bytes(grp, c.L, fwd_ws ? kBackwardKept : kBackward))) ||
        (fwd_ws && (st = check_ws(fwd_ws, fwd_ws_bytes, workspace_bytes(grp, c.L, kForward)))))
      return st;
    if ((st = augtree_check_device())) return st;
    c.ws = static_cast<char*>(ws);
    c.stream = static_cast<hipStream_t>(stream);
    if ((st = c.begin(decay))) return st;
    const uint16_t *const q[2] = {q_p, q_r}, *const k[2] = {k_p, k_r}, *const v[2] = {v_p, v_r},
                   *const g[2] = {do_p, do_r};
    uint16_t *const dq[2] = {dq_p, dq_r}, *const dk[2] = {dk_p, dk_r}, *const dv[2] = {dv_p, dv_r};
    const float* fwd = nullptr;
    if (fwd_ws) {
      fwd = reinterpret_cast<const float*>(static_cast<const char*>(fwd_ws) + align_up(c.L.segs.size() * sizeof(LinSeg)));
    } else {
      float* const own = c.take<float>(c.L.states);
      float* const tree = c.take<float>(c.L.tree * grp->num_groups);
      fwd = own;
      if ((st = c.states(false, k, v, state, own, tree, nullptr, nullptr))) return st;
    }
    float* const rev = c.take<float>(c.L.states);
    float* const ends = c.take<float>(c.L.tree * std::max(1, grp->num_branches));
    if ((st = c.states(true, q, g, nullptr, rev, ends, nullptr, nullptr))) return st;
    LinGradParams p;
    std::memset(&p, 0, sizeof(p));
    for (int i = 0; i < 2; ++i) {
      p.q[i] = q[i], p.k[i] = k[i], p.v[i] = v[i], p.dout[i] = g[i];
      p.dq[i] = dq[i], p.dk[i] = dk[i], p.dv[i] = dv[i];
    }
    p.states = fwd;
    p.states_rev = rev;
    p.scale = grp->softmax_scale;
    p.b = c.b;
    {
      Hook h("linear_dq", c.stream);
      if ((st = hip_ok(launch_lin_dq(p, grp->head_dim, c.stream), "dq launch"))) return st;
    }
    Hook h("linear_dkv", c.stream);
    if ((st = hip_ok(launch_lin_dkv(p, grp->head_dim, c.stream), "dk/dv launch"))) return st;
    return fail_status(AUGTREE_OK, "");
  });
}

int augtree_linear_step(int32_t rows, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, float scale,
                        const float* decay, const uint16_t* q, const uint16_t* k, const uint16_t* v, int32_t n_states,
                        const float* state_in, const int32_t* src, float* state_out, uint16_t* o, void* stream) {
  int st = check_heads(num_q_heads, num_kv_heads, head_dim, scale, decay);
  if (st) return st;
  if (rows < 0 || n_states < 0)
    return fail(AUGTREE_ERR_INVALID_ARGUMENT, "rows=%d n_states=%d must be >= 0", rows, n_states);
  if (!src && n_states < rows)
    return fail(AUGTREE_ERR_INVALID_ARGUMENT, "%d states for %d rows without src", n_states, rows);
  if ((int64_t)rows * num_kv_heads * (head_dim / 64) * 256 > UINT32_MAX)
    return fail(AUGTREE_ERR_UNSUPPORTED, "%d rows of %d KV heads exceed a launch", rows, num_kv_heads);
  if (rows == 0) return fail_status(AUGTREE_OK, "");
  const Named need[] = {{q, "q"}, {k, "k"}, {v, "v"}, {state_out, "state_out"}, {o, "o"}};
  if ((st = check_all(need, 5, true)) || (st = check_ptr(state_in, "state_in", n_states > 0)) ||
      (st = check_ptr(src, "src", false, 4)))
    return st;
  const size_t state = (size_t)num_kv_heads * head_dim * head_dim * sizeof(float);
  const size_t nq = 2 * (size_t)rows * num_q_heads * head_dim, nk = 2 * (size_t)rows * num_kv_heads * head_dim;
  const bool in_place = !src;  // with src a row could read what another one wrote
  const Span ins[] = {{q, nq, "q"}, {k, nk, "k"}, {v, nk, "v"}, {state_in, state * n_states, "state_in", in_place},
                      {src, 4 * (size_t)rows, "src"}};
  const Span outs[] = {{state_out, state * rows, "state_out", in_place}, {o, nq, "o"}};
  if ((st = check_apart(ins, 5, outs, 2))) return st;
  if ((st = augtree_check_device())) return st;
  LinStepParams p;
  std::memset(&p, 0, sizeof(p));
  p.q = q;
  p.k = k;
  p.v = v;
  p.state_in = state_in;
  p.src = src;
  p.state_out = state_out;
  p.o = o;
  p.rows = rows;
  p.n_states = n_states;
  p.heads_kv = num_kv_heads;
  p.group = num_q_heads / num_kv_heads;
  p.scale = scale;
  std::copy(decay, decay + num_kv_heads, p.decay);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  Hook h("linear_step", s);
  if ((st = hip_ok(launch_lin_step(p, head_dim, s), "step launch"))) return st;
  return fail_status(AUGTREE_OK, "");
}

}  // extern "C"

namespace {

int check_norm(int64_t rows, int heads, int d, int activation, float eps) {
  if (rows < 0) return fail(AUGTREE_ERR_INVALID_ARGUMENT, "rows=%lld must be >= 0", (long long)rows);
  if (heads < 1 || heads > 65535) return fail(AUGTREE_ERR_UNSUPPORTED, "heads %d not in [1, 65535]", heads);
  if (d < 8 || d % 8 || d > kHeadNormMaxDim)
    return fail(AUGTREE_ERR_UNSUPPORTED, "head_dim %d not a multiple of 8 in [8, %d]", d, kHeadNormMaxDim);
  if (activation != AUGTREE_ACT_NONE && activation != AUGTREE_ACT_SILU)
    return fail(AUGTREE_ERR_INVALID_ARGUMENT, "unknown activation %d", activation);
  if (!(eps > 0.f) || !std::isfinite(eps)) return fail(AUGTREE_ERR_INVALID_ARGUMENT, "eps must be finite and > 0");
  if (rows > ((int64_t)1 << 47) / ((int64_t)heads * d))
    return fail(AUGTREE_ERR_UNSUPPORTED, "%lld rows of %d x %d", (long long)rows, heads, d);
  return AUGTREE_OK;
}

}  // namespace

extern "C" {

size_t augtree_head_norm_workspace_size(int64_t rows, int32_t heads, int32_t head_dim) {
  if (check_norm(rows, heads, head_dim, AUGTREE_ACT_NONE, 1.f)) return 0;
  fail_status(AUGTREE_OK, "");
  return align_up((size_t)head_norm_bwd_grid(rows, heads, head_dim).parts * 2 * heads * head_dim * sizeof(float));
}

int augtree_head_norm_fwd(int64_t rows, int32_t heads, int32_t head_dim, int activation, float eps, const uint16_t* x,
                          const uint16_t* gate, const float* weight, const float* bias, uint16_t* y, void* stream) {
  int st = check_norm(rows, heads, head_dim, activation, eps);
  if (st) return st;
  if (rows == 0) return fail_status(AUGTREE_OK, "");
  const Named need[] = {{x, "x"}, {y, "y"}}, opt[] = {{gate, "gate"}, {weight, "weight"}, {bias, "bias"}};
  if ((st = check_all(need, 2, true)) || (st = check_all(opt, 3, false))) return st;
  const size_t row = (size_t)heads * head_dim, all = 2 * row * rows;
  const Span ins[] = {{x, all, "x", true}, {gate, all, "gate", true}, {weight, 4 * row, "weight"}, {bias, 4 * row, "bias"}};
  const Span outs[] = {{y, all, "y", true}};
  if ((st = check_apart(ins, 4, outs, 1)) || (st = augtree_check_device())) return st;
  HeadNormParams p;
  std::memset(&p, 0, sizeof(p));
  p.x = x;
  p.gate = gate;
  p.weight = weight;
  p.bias = bias;
  p.y = y;
  p.rows = rows;
  p.heads = heads;
  p.d = head_dim;
  p.silu = activation == AUGTREE_ACT_SILU;
  p.eps = eps;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  Hook h("head_norm", s);
  if ((st = hip_ok(launch_head_norm_fwd(p, s), "head norm launch"))) return st;
  return fail_status(AUGTREE_OK, "");
}

int augtree_head_norm_bwd(int64_t rows, int32_t heads, int32_t head_dim, int activation, float eps, const uint16_t* x,
                          const uint16_t* gate, const float* weight, const float* bias, const uint16_t* dy,
                          uint16_t* dx, uint16_t* dgate, float* dweight, float* dbias, void* ws, size_t ws_bytes,
                          void* stream) {
  int st = check_norm(rows, heads, head_dim, activation, eps);
  if (st) return st;
  const Named need[] = {{x, "x"}, {dy, "dy"}, {dx, "dx"}};
  const Named opt[] = {{gate, "gate"}, {weight, "weight"}, {bias, "bias"}, {dgate, "dgate"}, {dweight, "dweight"},
                       {dbias, "dbias"}};
  if (rows > 0 && (st = check_all(need, 3, true))) return st;
  if ((st = check_all(opt, 6, false))) return st;
  if (rows > 0 && !gate != !dgate) return fail(AUGTREE_ERR_INVALID_ARGUMENT, "gate and dgate go together");
  const bool sums = dweight || dbias;
  if (rows == 0 && !sums) return fail_status(AUGTREE_OK, "");
  if (sums && (st = check_ws(ws, ws_bytes, augtree_head_norm_workspace_size(rows, heads, head_dim)))) return st;
  const size_t row = (size_t)heads * head_dim, all = 2 * row * rows;
  const Span ins[] = {{x, all, "x", true}, {gate, all, "gate", true}, {dy, all, "dy", true}, {weight, 4 * row, "weight"},
                      {bias, 4 * row, "bias"}};
  const Span outs[] = {{dx, all, "dx", true}, {dgate, all, "dgate", true}, {dweight, 4 * row, "dweight"},
                       {dbias, 4 * row, "dbias"}, {sums ? ws : nullptr, ws_bytes, "ws"}};
  if ((st = check_apart(ins, 5, outs, 5)) || (st = augtree_check_device())) return st;
  HeadNormParams p;
  std::memset(&p, 0, sizeof(p));
  p.x = x;
  p.gate = gate;
  p.dy = dy;
  p.weight = weight;
  p.bias = bias;
  p.dx = dx;
  p.dgate = dgate;
  p.dweight = dweight;
  p.dbias = dbias;
  p.part = sums ? static_cast<float*>(ws) : nullptr;
  p.rows = rows;
  p.heads = heads;
  p.d = head_dim;
  p.silu = activation == AUGTREE_ACT_SILU;
  p.eps = eps;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  {
    Hook h("head_norm_bwd", s);
    if ((st = hip_ok(launch_head_norm_bwd(p, s), "head norm backward launch"))) return st;
  }
  if (sums) {
    p.sum = 1;
    Hook h("head_norm_sum", s);
    if ((st = hip_ok(launch_head_norm_bwd(p, s), "head norm sum launch"))) return st;
  }
  return fail_status(AUGTREE_OK, "");
}

}  // extern "C"
