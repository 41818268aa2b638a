// Shared declarations of the linear-attention layer: its kernels' parameters
// and launchers (host and device).
#pragma once

#include <hip/hip_runtime_api.h>
#include <stdint.h>

namespace augtree {

// A segment: the rows of one prompt, or of one branch. A batch lists its
// prompts first, then its branches. Segments are cut into blocks of `rows`
// rows (a multiple of kLinChunk; the last one shorter), numbered through the
// batch; every block has one state per KV head in the workspace.
struct LinSeg {
  int32_t row0, len;  // first row in the prompt (response) tensors, rows
  int32_t block0;     // number of its first block
  int32_t link;       // prompt: its first branch; branch: its tree
  int32_t rows;       // rows of a block
};

constexpr int kLinChunk = 64;       // rows a workgroup takes at a time
constexpr int kLinInlineSegs = 128; // segments carried in the kernel arguments
constexpr int kLinMaxHeads = 256;   // KV heads (their decays travel in the kernel arguments)

// The batch as the kernels see it.
struct LinBatch {
  const LinSeg* segs;  // device copy, or nullptr: `inl`
  int32_t num_trees, num_branches, num_blocks;
  int32_t heads_kv, group;       // KV heads, query heads of each
  float log2_decay[kLinMaxHeads];
  LinSeg inl[kLinInlineSegs];
};

// States of blocks: every block's own sum_j w_j y_j z_j^T over its rows, w_j
// the decay from row j to the block's last row (reverse: first row), summed
// over the `heads_y` / heads_kv heads of a KV head.
struct LinStateParams {
  const uint16_t* y[2];  // [0] prompt rows, [1] response rows
  const uint16_t* z[2];
  int32_t heads_y;       // heads of y and z
  float* states;         // [num_blocks][heads_kv][d][d]
  int32_t skip_prompt, skip_branch;  // leave out the last block (reverse: first) of prompts / branches
  LinBatch b;
};

// The same states, in place, from each block's own to what reaches its first
// row (reverse: its last): a scan over the blocks of a segment.
struct LinScanParams {
  float* states;
  const float* init;    // [num_trees] states that prompts begin from (forward), or nullptr: zero
  float* ends;          // forward: [num_trees] prompts' ends; reverse: [num_branches] branches' ends
  float* out_p;         // forward: user's copies of the prompts' and branches' ends, or nullptr
  float* out_r;
  LinBatch b;
};

// o from q, k, v and the states that reach the blocks.
struct LinOutParams {
  const uint16_t *q[2], *k[2], *v[2];
  uint16_t* o[2];
  const float* states;
  float scale;
  LinBatch b;
};

// dq, dk, dv from q, k, v, do and the states in both directions.
struct LinGradParams {
  const uint16_t *q[2], *k[2], *v[2], *dout[2];
  uint16_t *dq[2], *dk[2], *dv[2];
  const float *states, *states_rev;
  float scale;
  LinBatch b;
};

static_assert(sizeof(LinStateParams) <= 4096 && sizeof(LinScanParams) <= 4096 && sizeof(LinOutParams) <= 4096 &&
                  sizeof(LinGradParams) <= 4096,
              "kernel arguments");

// writes n words (at most kLinTableWords) to dst
constexpr int kLinTableWords = 960;
struct LinTable {
  int32_t* dst;
  int32_t n;
  int32_t words[kLinTableWords];
};
static_assert(sizeof(LinTable) <= 4096, "kernel arguments");

hipError_t launch_lin_table(const LinTable& t, hipStream_t stream);
hipError_t launch_lin_state(const LinStateParams& p, int head_dim, bool reverse, hipStream_t stream);
// part: 0 whole trees, 1 prompts, 2 branches (1 and 2 hand over through `ends`, in the order of the direction)
hipError_t launch_lin_scan(const LinScanParams& p, int head_dim, bool reverse, int part, hipStream_t stream);
hipError_t launch_lin_out(const LinOutParams& p, int head_dim, hipStream_t stream);
hipError_t launch_lin_dq(const LinGradParams& p, int head_dim, hipStream_t stream);
hipError_t launch_lin_dkv(const LinGradParams& p, int head_dim, hipStream_t stream);

struct LinStepParams {
  const uint16_t *q, *k, *v;
  const float* state_in;   // [n_states][heads_kv][d][d]
  const int32_t* src;      // [rows] or nullptr: row r reads state r
  float* state_out;        // [rows][heads_kv][d][d]
  uint16_t* o;
  int32_t rows, n_states, heads_kv, group;
  float scale;
  float decay[kLinMaxHeads];
};
hipError_t launch_lin_step(const LinStepParams& p, int head_dim, hipStream_t stream);

struct HeadNormParams {
  const uint16_t *x, *gate, *dy;  // [rows][heads][d]
  const float *weight, *bias;     // [heads][d] or nullptr
  uint16_t *y, *dx, *dgate;
  float *dweight, *dbias;         // [heads][d]
  float* part;                    // [parts][2][heads][d], or nullptr: no weight or bias gradient
  int64_t rows;
  int32_t heads, d;
  int32_t silu;
  int32_t sum;                    // backward: 0 the rows' gradients and the parts, 1 the sum of the parts
  float eps;
};
// Workgroups: row_parts x head_blocks (about `want` at most) of `heads` heads. In
// the backward they leave `parts` partial sums of the weight and bias gradients.
struct HeadNormGrid {
  int heads, head_blocks, row_parts, parts;
};
constexpr int kHeadNormMaxDim = 1024;
inline HeadNormGrid head_norm_grid(int64_t rows, int heads, int d, int want) {
  int lanes = 1;
  while (lanes < d / 8 && lanes < 64) lanes *= 2;
  const int groups = 256 / lanes;
  HeadNormGrid g;
  g.heads = heads < groups ? heads : groups;
  g.head_blocks = (heads + g.heads - 1) / g.heads;
  const int sharing = groups / g.heads;  // groups of lanes that share a head's rows
  int64_t parts = want / g.head_blocks;
  if (parts * sharing > rows) parts = (rows + sharing - 1) / sharing;
  g.row_parts = parts < 1 ? 1 : (int)parts;
  g.parts = g.row_parts * sharing;
  return g;
}
inline HeadNormGrid head_norm_bwd_grid(int64_t rows, int heads, int d) { return head_norm_grid(rows, heads, d, 1024); }
hipError_t launch_head_norm_fwd(const HeadNormParams& p, hipStream_t stream);
hipError_t launch_head_norm_bwd(const HeadNormParams& p, hipStream_t stream);

}  // namespace augtree
