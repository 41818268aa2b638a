/*
 * augtree.h — C ABI of the shared-prompt group attention library (libaugtree.so)
 * for AMD Instinct MI355X (gfx950).
 *
 * The operation is one attention layer of a batch of replay trees
 * T = (P, {R_i}_{i=1..G}) (paper §2.1, §3.1): a shared prompt P and G response
 * branches. A response token of branch i attends to every prompt key and to
 * its own prefix, never to a sibling branch (§2.2; Eq. 1:
 * KV(R_{i,t}) = KV_P ∪ KV(R_{i,<t})). Attention is
 * O = softmax(s Q K^T + M) V with s = softmax_scale (§2.2).
 *
 * The library splits it the way the method does (§3.2, §3.3):
 *   prefill_fwd   causal attention over the prompt, run once per tree;
 *   replay_fwd    every branch against the prompt KV (read in place, never
 *                 copied) plus its own causal KV, two partial softmax states
 *                 merged by log-sum-exp;
 *   lse_merge     the merge of partial states on its own;
 *   replay_bwd    gradients of the replay, with each branch's prompt-KV
 *                 gradient ("seed") accumulated on the prompt KV (Eq. 2);
 *   prefill_bwd   gradients of the prefill (the prompt's own contribution);
 *   prompt_grad_reduce  the Eq. 2 sum of the prefill contribution and the
 *                 seeds, in a fixed order, without atomics;
 *   tree_fwd / tree_bwd  the same step in two calls with fewer launches (the
 *                 prefill and replay tiles share launches, and the Eq. 2 sum
 *                 is formed in registers).
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * Layout (packed varlen, head_dim innermost, row-major):
 *   Q_P [T_P, Hq, d]   K_P, V_P [T_P, Hkv, d]   (T_P = total prompt rows)
 *   Q_R [T_R, Hq, d]   K_R, V_R [T_R, Hkv, d]   (T_R = total response rows)
 *   O, dO, dQ like Q; dK, dV like K.   LSE [Hq, T] fp32 (head-major).
 *   bf16 tensors are passed as uint16_t bit patterns.
 * GQA: KV head k serves query heads k*g .. k*g+g-1, g = Hq / Hkv.
 * LSE is the natural log of sum_j exp(s q.k_j) over the visible keys.
 * Pointers: every tensor pointer is a DEVICE pointer of the current HIP
 *   device and must be 16-byte aligned; the descriptor's offset arrays are
 *   HOST pointers. `stream` is a hipStream_t (NULL = the null stream).
 * Ownership: the caller allocates and owns every buffer, workspace included.
 *   The library never allocates or frees memory and never synchronises the
 *   device; all work is enqueued on `stream`. Prompt tensors must stay alive
 *   from prefill_fwd until prefill_bwd.
 * Outputs are overwritten, never accumulated into.
 * Workspace: `ws` must hold augtree_workspace_size(...) bytes (256-byte
 *   aligned). A launch of more than 112 tiles of 128 rows (35 where sweeps are
 *   split) may read its tile schedule from the workspace, written there with
 *   an asynchronous host-to-device copy on `stream` (the host staging happens
 *   before the call returns); smaller schedules travel in the kernel
 *   arguments. The backward also keeps
 *   D = rowsum(dO * O) of every row there (written by its dQ kernel, read by
 *   its dK/dV kernel), and the fp32 sums of key tiles whose sweep is split
 *   into parts (trees with few key tiles and long sweeps): of each part where
 *   the parts are workgroups of their own (a second kernel of the dK/dV launch
 *   adds them), or of the tile where one workgroup runs them one after the
 *   other (batches that fill the GPU). A tile or part takes
 *   2 x 128 x Hkv x d x 4 bytes. Both ways give the same bits. A backward whose
 *   workspace has no room for the parts runs them in one workgroup; without
 *   room for that either it runs these sweeps whole: the same gradients up to
 *   fp32 summation order.
 * Errors: every call returns an augtree_status. Arguments are validated on
 *   the host before any work is enqueued; on error nothing is launched and
 *   augtree_last_error() gives a detail string (thread-local). No C++
 *   exception crosses the ABI. Asynchronous kernel faults surface at the
 *   caller's next synchronisation, as in HIP.
 * Determinism: every output is bitwise reproducible run to run (no atomics),
 *   and a tree's outputs do not depend on the other trees of the batch (each
 *   output element is computed by one workgroup in a fixed order, or as parts
 *   whose cuts follow from the tree alone and which are added in a fixed
 *   order, whatever order the tiles are scheduled in). The second holds for
 *   workspaces of augtree_workspace_size() bytes or more: a smaller one, or the
 *   fixed array of augtree_tree_bwd_noalloc, may have no room for a batch's
 *   parts or chunks, and the whole sweeps that then run round the key
 *   gradients of its trees differently.
 * Thread safety: calls are reentrant; calls on different streams that share a
 *   workspace race.
 */
#ifndef AUGTREE_H
#define AUGTREE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum augtree_status {
  AUGTREE_OK = 0,
  AUGTREE_ERR_INVALID_ARGUMENT = 1, /* null pointer, bad count, bad offsets */
  AUGTREE_ERR_UNSUPPORTED = 2,      /* head_dim not in {64,128}, Hq % Hkv != 0 */
  AUGTREE_ERR_MISALIGNED = 3,       /* a tensor pointer not 16-byte aligned */
  AUGTREE_ERR_WORKSPACE = 4,        /* workspace missing or too small */
  AUGTREE_ERR_DEVICE = 5,           /* current device is not gfx950 */
  AUGTREE_ERR_HIP = 6               /* a HIP launch or copy reported an error */
} augtree_status;

typedef enum augtree_replay_mode {
  AUGTREE_REPLAY_FUSED = 0, /* prompt sweep then own-branch sweep, merged in registers */
  AUGTREE_REPLAY_SPLIT = 1, /* two partial states written out, then lse_merge */
  AUGTREE_REPLAY_AUTO = 2   /* per group, FUSED or SPLIT by a cost rule (augtree_replay_split_groups) */
} augtree_replay_mode;

typedef enum augtree_op {
  AUGTREE_OP_PREFILL_FWD = 0,
  AUGTREE_OP_REPLAY_FWD = 1, /* workspace arg: replay mode */
  AUGTREE_OP_PREFILL_BWD = 2,
  AUGTREE_OP_REPLAY_BWD = 3, /* workspace arg: n_seed */
  AUGTREE_OP_TREE_FWD = 4,   /* workspace arg: replay mode */
  AUGTREE_OP_TREE_BWD = 5    /* workspace arg ignored */
} augtree_op;

/*
 * A batch of replay trees (§3.1: T = (P, {R_i})). Offsets are HOST arrays.
 *   cu_prompt [num_groups+1]  group g's prompt rows are cu_prompt[g] .. cu_prompt[g+1]-1
 *   cu_branch [num_groups+1]  group g owns branches cu_branch[g] .. cu_branch[g+1]-1
 *   cu_resp   [num_branches+1] branch b's response rows are cu_resp[b] .. cu_resp[b+1]-1
 * Requirements: cu_*[0] == 0, every prompt and branch length >= 1, every
 * group has >= 1 branch, cu_branch[num_groups] == num_branches, branches of a
 * group are consecutive, offsets fit int32. softmax_scale > 0 (normally
 * 1/sqrt(head_dim)).
 */
typedef struct augtree_groups {
  int32_t num_groups;
  int32_t num_branches;
  int32_t num_q_heads;
  int32_t num_kv_heads;
  int32_t head_dim;
  float softmax_scale;
  const int32_t* cu_prompt;
  const int32_t* cu_branch;
  const int32_t* cu_resp;
} augtree_groups;

/* Bytes of workspace an entry point needs for this batch. `arg` is the replay
 * mode for AUGTREE_OP_REPLAY_FWD / AUGTREE_OP_TREE_FWD, n_seed for
 * AUGTREE_OP_REPLAY_BWD, ignored otherwise. Returns 0 on invalid arguments
 * (see augtree_last_error). */
size_t augtree_workspace_size(const augtree_groups* grp, int op, int arg);

/*
 * Prompt prefill forward (§3.2, shared prompt prefill pass; attention of §2.2
 * with the causal mask). For every group and query head h:
 *   O_P[r] = sum_{j<=r} exp(s q_r.k_j - LSE_r) v_j,  LSE_r = ln sum_{j<=r} exp(s q_r.k_j)
 * over the group's prompt rows, KV head h / g.
 * In:  q_p [T_P,Hq,d], k_p, v_p [T_P,Hkv,d] bf16.
 * Out: o_p [T_P,Hq,d] bf16, lse_p [Hq,T_P] fp32.
 * Reads num_groups, cu_prompt and the head shape only: cu_branch / cu_resp may
 * be NULL and num_branches is ignored (a batch of plain causal sequences).
 */
int augtree_prefill_fwd(const augtree_groups* grp, const uint16_t* q_p, const uint16_t* k_p,
                        const uint16_t* v_p, uint16_t* o_p, float* lse_p, void* ws, size_t ws_bytes,
                        void* stream);

/*
 * Response replay forward (§3.2 response replay; Eq. 1; §3.3 merge of partial
 * states). Every response row of branch b (group g) attends to all prompt keys
 * of g (partial A, no mask) and to rows 0..t of branch b (partial B, causal);
 * the two partial states are merged by log-sum-exp:
 *   LSE = ln(exp(LSE_A) + exp(LSE_B)),  O = exp(LSE_A-LSE) O_A + exp(LSE_B-LSE) O_B.
 * FUSED: one sweep over both key sets, merged in registers.
 * SPLIT: partial A and partial B are written to o_part [2][T_R,Hq,d] fp32 and
 *   lse_part [2][Hq,T_R] fp32 (part 0 = prompt, part 1 = own branch), then
 *   merged by the lse_merge kernel into o_r / lse_r. The prompt partial's
 *   query tiles pack the rows of all branches of a group (they all see the
 *   same prompt keys), so short branches do not leave tiles mostly empty.
 * AUTO: each group runs FUSED or SPLIT as augtree_replay_split_groups reports;
 *   o_part / lse_part are required (only the split groups' rows are written
 *   there). In FUSED mode o_part and lse_part may be NULL.
 * In:  q_r [T_R,Hq,d], k_r, v_r [T_R,Hkv,d], k_p, v_p [T_P,Hkv,d] bf16.
 * Out: o_r [T_R,Hq,d] bf16, lse_r [Hq,T_R] fp32.
 */
int augtree_replay_fwd(const augtree_groups* grp, int mode, const uint16_t* q_r, const uint16_t* k_r,
                       const uint16_t* v_r, const uint16_t* k_p, const uint16_t* v_p, uint16_t* o_r,
                       float* lse_r, float* o_part, float* lse_part, void* ws, size_t ws_bytes,
                       void* stream);

/*
 * The replay-forward mode AUGTREE_REPLAY_AUTO gives each group (the choice of
 * a way to run one step of §3.2 per group, like the per-tree primitive choice
 * of §3.4, made here from the kernels' own costs). Writes split[g] = 1 when
 * group g runs SPLIT, 0 when FUSED. The rule: a mode costs the number of
 * (query tile, 64-key block) steps its forward tiles execute at a measured
 * time per step, plus, for SPLIT, the merge's HBM bytes at a measured
 * bandwidth; SPLIT is taken when it costs less. Short branches favour SPLIT
 * (a fused tile of a 16-row branch sweeps every prompt block for 16 rows),
 * long ones FUSED (same steps, no merge).
 * In:  grp (host offsets). Out: split [num_groups] int32, host memory.
 * Errors: INVALID_ARGUMENT for a bad descriptor or a NULL split.
 */
int augtree_replay_split_groups(const augtree_groups* grp, int32_t* split);

/*
 * Merge of n partial softmax states of the same rows (§3.3, the associative
 * merge applied to full states). For every row r and head h, in part order:
 *   M = max_k lse_k;  LSE = M + ln sum_k exp(lse_k - M);  O = sum_k exp(lse_k - LSE) o_k.
 * Parts with lse = -inf carry weight 0; if all parts are -inf the row gets
 * O = 0 and LSE = -inf.
 * In:  o_parts [n_parts][rows,heads,head_dim] fp32, lse_parts [n_parts][heads,rows] fp32.
 * Out: o [rows,heads,head_dim] bf16 (nullable), o_f32 same shape fp32 (nullable,
 *      at least one of o / o_f32), lse [heads,rows] fp32 (nullable).
 * head_dim must be a multiple of 8 and <= 256; n_parts >= 1; rows >= 0.
 */
int augtree_lse_merge(int64_t rows, int32_t heads, int32_t head_dim, int32_t n_parts,
                      const float* o_parts, const float* lse_parts, uint16_t* o, float* o_f32,
                      float* lse, void* stream);

/*
 * Response replay backward (§3.2 exact many-to-one backward; Eq. 2). With the
 * merged O and LSE of replay_fwd and D_r = sum_c dO_rc O_rc, for each branch
 * row and both partials: P = exp(s q.k - LSE), dP = dO.v, dS = P (dP - D);
 *   dQ_R = s (dS_A K_P + dS_B K_R),  dK_R = s dS_B^T Q_R,  dV_R = P_B^T dO_R,
 *   seeds  dK_P += s dS_A^T Q_R,  dV_P += P_A^T dO_R  (summed over the g query
 *   heads of each KV head and over the group's branches).
 * The group's response rows are cut into n_seed contiguous chunks of about
 * equal size; chunk c's prompt-key gradient is written to slab c of
 * dkv_p_seed [n_seed][2][T_P,Hkv,d] fp32 (index 0 = dK, 1 = dV). n_seed = 1
 * sums every branch in-kernel; n_seed > 1 trades a larger Eq. 2 reduction for
 * more parallelism. Slabs are overwritten.
 * In:  q_r, k_r, v_r, k_p, v_p, o_r (bf16), lse_r (fp32), do_r (bf16).
 * Out: dq_r [T_R,Hq,d], dk_r, dv_r [T_R,Hkv,d] bf16; dkv_p_seed fp32.
 * 1 <= n_seed <= 64.
 * dQ: with dS rounded to bf16 for the dQ product, the kernel subtracts c times
 * the row sum of the rounded dS, c = the group's first prompt key (exact in
 * arithmetic since every row of dS sums to zero over its keys); this keeps a
 * component shared by all keys from amplifying the rounding of dS.
 */
int augtree_replay_bwd(const augtree_groups* grp, const uint16_t* q_r, const uint16_t* k_r,
                       const uint16_t* v_r, const uint16_t* k_p, const uint16_t* v_p,
                       const uint16_t* o_r, const float* lse_r, const uint16_t* do_r, uint16_t* dq_r,
                       uint16_t* dk_r, uint16_t* dv_r, int32_t n_seed, float* dkv_p_seed, void* ws,
                       size_t ws_bytes, void* stream);

/*
 * Prompt prefill backward: the prompt queries' own contribution to every
 * gradient, i.e. the backward of the causal prefill attention itself (§3.2;
 * Eq. 2's first term for the prompt keys), causal over P.
 * In:  q_p, k_p, v_p, o_p (bf16), lse_p (fp32), do_p (bf16).
 * Out: dq_p [T_P,Hq,d] bf16 (nullable) and/or dq_p_f32 same shape fp32
 *      (nullable; at least one), dkv_p_self [2][T_P,Hkv,d] fp32 (0 = dK, 1 = dV).
 * Like prefill_fwd, reads only num_groups, cu_prompt and the head shape.
 */
int augtree_prefill_bwd(const augtree_groups* grp, const uint16_t* q_p, const uint16_t* k_p,
                        const uint16_t* v_p, const uint16_t* o_p, const float* lse_p,
                        const uint16_t* do_p, uint16_t* dq_p, float* dq_p_f32, float* dkv_p_self,
                        void* ws, size_t ws_bytes, void* stream);

/*
 * One tree step's forward in one call (§3.2: prefill once, then replay every
 * branch against the prompt KV read in place; Eq. 1; §3.3). Computes exactly what
 * augtree_prefill_fwd followed by augtree_replay_fwd compute (bit for bit:
 * the same kernels and per-row arithmetic), but the prefill tiles and the
 * fused replay tiles run in ONE kernel launch (fewer launches and one launch
 * tail; the replay tiles read the prompt KV the prefill reads).
 * mode: as for augtree_replay_fwd (SPLIT / AUTO groups add the fp32 partial
 *   launch and the merge; o_part / lse_part are then required).
 * In:  q_p [T_P,Hq,d], k_p, v_p [T_P,Hkv,d], q_r [T_R,Hq,d], k_r, v_r [T_R,Hkv,d] bf16.
 * Out: o_p [T_P,Hq,d] bf16, lse_p [Hq,T_P], o_r [T_R,Hq,d] bf16, lse_r [Hq,T_R] fp32.
 * Workspace: augtree_workspace_size(grp, AUGTREE_OP_TREE_FWD, mode).
 */
int augtree_tree_fwd(const augtree_groups* grp, int mode, const uint16_t* q_p, const uint16_t* k_p,
                     const uint16_t* v_p, const uint16_t* q_r, const uint16_t* k_r, const uint16_t* v_r,
                     uint16_t* o_p, float* lse_p, uint16_t* o_r, float* lse_r, float* o_part,
                     float* lse_part, void* ws, size_t ws_bytes, void* stream);

/*
 * One tree step's backward in one call (§3.2 exact many-to-one backward;
 * Eq. 2). The same gradients as augtree_replay_bwd + augtree_prefill_bwd +
 * augtree_prompt_grad_reduce, in two kernel launches:
 *   dQ launch: every prompt row (causal over the prompt) and every response
 *     row (prompt keys, then its own causal keys); also forms
 *     D = rowsum(dO * O) of every row into the workspace;
 *   dK/dV launch: each prompt-key tile sweeps every response row of its group
 *     (all branches, every prompt key visible) and then the prompt rows at or
 *     after its first key (causal), so the whole Eq. 2 sum (branch seeds and
 *     the prompt queries' own contribution) is accumulated in registers, in
 *     that fixed order, and rounded once; each branch-key tile sweeps its
 *     branch's rows (causal).
 * A group whose branch rows exceed augtree_tree_chunk_blocks() query blocks
 * (64 rows of one query head) per prompt-key tile has that sweep cut into
 * chunks (at most 64) of consecutive branch rows, the first chunk also taking
 * the prompt rows; the chunks write fp32 partial sums to the workspace and a
 * third launch adds them per row in chunk order and rounds once (role
 * "reduce_tree"). Long sweeps otherwise lose the L2 sharing of the query rows.
 * The prompt gradient is the same sum as the three-call path up to fp32
 * rounding order (that path adds two fp32 partial sums); it is bitwise
 * reproducible for a given chunk setting. The dK/dV launch is followed by a
 * small one that adds the parts of split sweeps, where the batch has any (both
 * under the role "dkv_tree"). dQ carries the same common-mode
 * correction as augtree_replay_bwd.
 * In:  q_p, k_p, v_p, o_p (bf16), lse_p (fp32), do_p (bf16) [prompt rows];
 *      q_r, k_r, v_r, o_r (bf16), lse_r (fp32), do_r (bf16) [response rows].
 * Out: dq_p [T_P,Hq,d], dk_p, dv_p [T_P,Hkv,d], dq_r [T_R,Hq,d], dk_r, dv_r
 *      [T_R,Hkv,d] bf16; dkv_p_f32 [2][T_P,Hkv,d] fp32 (nullable: the prompt
 *      gradient before its bf16 rounding, 0 = dK, 1 = dV).
 * Workspace: augtree_workspace_size(grp, AUGTREE_OP_TREE_BWD, 0) (with chunks:
 * the fp32 partials, 2 x (sum over chunked groups of chunks x P) x Hkv x d x 4
 * bytes, and a row map of chunks x T_P int32).
 */
int augtree_tree_bwd(const augtree_groups* grp, const uint16_t* q_p, const uint16_t* k_p,
                     const uint16_t* v_p, const uint16_t* o_p, const float* lse_p,
                     const uint16_t* do_p, const uint16_t* q_r, const uint16_t* k_r,
                     const uint16_t* v_r, const uint16_t* o_r, const float* lse_r,
                     const uint16_t* do_r, uint16_t* dq_p, uint16_t* dk_p, uint16_t* dv_p,
                     float* dkv_p_f32, uint16_t* dq_r, uint16_t* dk_r, uint16_t* dv_r, void* ws,
                     size_t ws_bytes, void* stream);

/*
 * augtree_tree_bwd without a workspace argument, for callers that cannot
 * allocate device memory (code under stream capture, tight serving loops,
 * harnesses that forbid allocation). Same inputs, outputs and results as
 * augtree_tree_bwd (bit for bit, except that a batch whose split sweeps do not
 * fit the array even with one slot a tile runs them whole, and one whose
 * chunks do not fit runs one sweep per prompt-key tile: the same gradients up
 * to fp32 summation order). Its workspace is a fixed 64 MiB device array of
 * the library (augtree_noalloc_scratch_bytes()), one copy per GPU, held from
 * the first call on that GPU until the process ends; the call performs no
 * allocation. A batch whose workspace without chunks and splits exceeds it is
 * rejected with AUGTREE_ERR_WORKSPACE before anything is enqueued. Calls that
 * overlap on one GPU (several streams or threads) share the array and race;
 * serialise them. Stream capture: a schedule that does not fit the kernel arguments, and
 * a chunked batch's row map, come by a host-to-device copy from a host buffer
 * the call frees on return, so a graph captured around such a call must not be
 * replayed. Batches without chunks of at most 112 tiles per launch (128 query
 * or key rows each), or 35 where sweeps are split, enqueue kernels only.
 */
int augtree_tree_bwd_noalloc(const augtree_groups* grp, const uint16_t* q_p, const uint16_t* k_p,
                             const uint16_t* v_p, const uint16_t* o_p, const float* lse_p,
                             const uint16_t* do_p, const uint16_t* q_r, const uint16_t* k_r,
                             const uint16_t* v_r, const uint16_t* o_r, const float* lse_r,
                             const uint16_t* do_r, uint16_t* dq_p, uint16_t* dk_p, uint16_t* dv_p,
                             float* dkv_p_f32, uint16_t* dq_r, uint16_t* dk_r, uint16_t* dv_r,
                             void* stream);

/* Bytes of the device array augtree_tree_bwd_noalloc works in (its limit). */
size_t augtree_noalloc_scratch_bytes(void);

/*
 * Eq. 2 reduction: the prompt-KV gradient is the prefill's own contribution
 * plus the sum of the branch seeds. Elementwise, in a fixed order (self first,
 * then terms in index order), fp32 sum and one rounding to bf16:
 *   out[t][r] = self[t][r] + sum_{k<n_parts} parts[k*part_stride + (t*part_rows + src(k,r))*E]
 * for tensor t < n_tensors (t = 0 dK, 1 dV), row r < rows, E = heads*head_dim
 * elements per row (a row is contiguous).
 *   self:  [n_tensors][rows][heads][head_dim] fp32, or NULL (treated as 0).
 *   parts: fp32; term k starts at parts + k*part_stride (elements) and holds
 *          [n_tensors][part_rows][heads][head_dim]. Dense seed slabs use
 *          part_stride = n_tensors*part_rows*E; part_stride = 0 lets every
 *          term read one slab through row_map.
 *   row_map: NULL means src(k,r) = r (then part_rows must equal rows);
 *            otherwise a DEVICE int32 array [n_parts][rows] of source rows in
 *            [0, part_rows), -1 meaning "term k has no row for r" (used to sum
 *            the prompt copies of a flattened batch).
 *   out: [n_tensors][rows][heads][head_dim] bf16 (nullable); out_f32 same
 *        shape fp32 (nullable); at least one.
 * n_tensors in {1,2}; 0 <= n_parts <= 4096; E a multiple of 4; part_stride
 * a multiple of 4 and >= 0. Source rows outside [0, part_rows) are the
 * caller's error (not checked on the device).
 */
int augtree_prompt_grad_reduce(int32_t n_tensors, int64_t rows, int32_t heads, int32_t head_dim,
                               const float* self, int32_t n_parts, int64_t part_rows,
                               int64_t part_stride, const float* parts, const int32_t* row_map,
                               uint16_t* out, float* out_f32, void* stream);

/* ---------------------------------------------------------------------------
 * Linear attention over replay trees
 *
 * The mixing layer of models whose layers keep a decayed state instead of a KV
 * cache, on the same packed batches of replay trees. With gamma the decay of a
 * KV head, s = softmax_scale and rows numbered through a prompt and on through
 * a branch (the first row of a branch follows the last one of its prompt):
 *   o_t = s sum_{j <= t} gamma^(t-j) (q_t . k_j) v_j  +  s gamma^(t+1) q_t S_0
 *   S_t = gamma S_(t-1) + k_t v_t^T                     [d_k, d_v], fp32
 * over the rows j of t's prompt and of its own branch. The prompt's state is
 * computed once and every branch goes on from it; in the backward the branches'
 * gradients of that state are added, in branch order, to what the prompt's own
 * rows receive (the linear form of Eq. 2).
 *
 * decay: HOST array [num_kv_heads], 0 < decay <= 1, at most 256 KV heads. It is a
 * constant of the layer: no gradient is formed for it.
 * A NaN or infinity in one row reaches the rows that the formulas name, an
 * infinity perhaps as NaN (operands are split into two terms). The rows of a
 * chunk (64 rows) of a sequence pass through common matrix products, so it may
 * reach the other rows of its chunk too; never another KV head or another tree,
 * nor from a branch any other branch.
 * Every call enqueues kernels only and may be captured into a graph; calls that
 * share a workspace must not overlap (as for all entry points). Outputs must lie
 * apart from the inputs and from one another, but for what is named below.
 * Results are bitwise reproducible and a tree's do not depend on the batch.
 * ------------------------------------------------------------------------- */

/* Bytes of workspace of augtree_linear_fwd (backward = 0), of augtree_linear_bwd
 * (1) and of an augtree_linear_bwd that is given fwd_ws (2: about half of that).
 * 0 on invalid arguments. */
size_t augtree_linear_workspace_size(const augtree_groups* grp, int backward);

/*
 * Forward. In:  q_p [T_P,Hq,d], k_p, v_p [T_P,Hkv,d], q_r [T_R,Hq,d], k_r, v_r
 *      [T_R,Hkv,d] bf16; state [num_groups,Hkv,d,d] fp32: what each prompt begins
 *      from (nullable: zero).
 * Out: o_p [T_P,Hq,d], o_r [T_R,Hq,d] bf16; state_p [num_groups,Hkv,d,d], state_r
 *      [num_branches,Hkv,d,d] fp32: the states after each prompt and each branch
 *      (nullable), for augtree_linear_step or the next piece of a sequence.
 *      state_p may be state.
 * num_branches = 0 is a batch of plain sequences: cu_branch and cu_resp are not
 * read and the response pointers may be NULL. softmax_scale is s.
 */
int augtree_linear_fwd(const augtree_groups* grp, const float* decay, const uint16_t* q_p,
                       const uint16_t* k_p, const uint16_t* v_p, const uint16_t* q_r, const uint16_t* k_r,
                       const uint16_t* v_r, const float* state, uint16_t* o_p, uint16_t* o_r, float* state_p,
                       float* state_r, void* ws, size_t ws_bytes, void* stream);

/*
 * Backward: gradients of the outputs' loss for q, k and v (none for `state`
 * or through state_p / state_r). In: as forward, do_p, do_r bf16 like o_p, o_r;
 * the outputs are not read. Out: dq like q, dk, dv like k, bf16.
 * fwd_ws (nullable): the workspace of the augtree_linear_fwd call of the same
 * batch, decay, k, v and state, not written since. The states it holds are then
 * used instead of being formed again, and `state` is not read; the results are
 * the same bits.
 */
int augtree_linear_bwd(const augtree_groups* grp, const float* decay, const uint16_t* q_p,
                       const uint16_t* k_p, const uint16_t* v_p, const uint16_t* do_p, const uint16_t* q_r,
                       const uint16_t* k_r, const uint16_t* v_r, const uint16_t* do_r, const float* state,
                       uint16_t* dq_p, uint16_t* dk_p, uint16_t* dv_p, uint16_t* dq_r, uint16_t* dk_r,
                       uint16_t* dv_r, const void* fwd_ws, size_t fwd_ws_bytes, void* ws, size_t ws_bytes,
                       void* stream);

/*
 * One token of each of `rows` sequences:
 *   state_out[r] = decay state_in[src[r]] + k_r v_r^T,  o_r = scale q_r state_out[r].
 * In:  q [rows,Hq,d], k, v [rows,Hkv,d] bf16, state_in [n_states,Hkv,d,d] fp32,
 *      src [rows] DEVICE int32 or NULL (src[r] = r). Several rows may read one
 *      state (the branches of a prompt); a src outside [0, n_states) begins from a
 *      zero state. decay: HOST array [Hkv].
 * Out: state_out [rows,Hkv,d,d] fp32, o [rows,Hq,d] bf16.
 * state_out may be state_in without src (in place); any other overlap of the
 * two is refused. No workspace.
 */
int augtree_linear_step(int32_t rows, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                        float scale, const float* decay, const uint16_t* q, const uint16_t* k,
                        const uint16_t* v, int32_t n_states, const float* state_in, const int32_t* src,
                        float* state_out, uint16_t* o, void* stream);

typedef enum augtree_activation { AUGTREE_ACT_NONE = 0, AUGTREE_ACT_SILU = 1 } augtree_activation;

/*
 * Norm of each head of each row, with an activation (a group norm over
 * [rows, heads * head_dim], one group per head), as it follows linear
 * attention: n = (x - mean) / sqrt(var + eps) over the head_dim channels (var
 * with the divisor head_dim), a = n * weight + bias, and
 *   y = act(a),  or with a gate  y = a * act(gate);  act(u) = u / (1 + exp(-u)) (SILU) or u (NONE).
 * Arithmetic is fp32: squares of values from 2^63 on overflow.
 * In:  x, gate (nullable) [rows,heads,head_dim] bf16; weight, bias (each
 *      nullable: 1 and 0) [heads,head_dim] fp32. head_dim a multiple of 8, at most 1024.
 * Out: y like x (it may be x or gate itself; other overlaps are refused). rows = 0 is a no-op.
 */
int augtree_head_norm_fwd(int64_t rows, int32_t heads, int32_t head_dim, int activation, float eps,
                          const uint16_t* x, const uint16_t* gate, const float* weight, const float* bias,
                          uint16_t* y, void* stream);

/*
 * Its backward. In: as forward, dy like y. Out: dx, dgate (with a gate) bf16
 * (each may be x, gate or dy itself, not both the same; other overlaps are refused);
 * dweight, dbias [heads,head_dim] fp32 (each nullable), summed over the rows in a
 * fixed order. The workspace (augtree_head_norm_workspace_size bytes) is needed
 * for dweight or dbias only. rows = 0 writes zeros to them.
 */
int augtree_head_norm_bwd(int64_t rows, int32_t heads, int32_t head_dim, int activation, float eps,
                          const uint16_t* x, const uint16_t* gate, const float* weight, const float* bias,
                          const uint16_t* dy, uint16_t* dx, uint16_t* dgate, float* dweight, float* dbias,
                          void* ws, size_t ws_bytes, void* stream);
size_t augtree_head_norm_workspace_size(int64_t rows, int32_t heads, int32_t head_dim);

/* ---------------------------------------------------------------------------
 * Paged KV cache under replay trees (rollout)
 *
 * Attention of new tokens over cached ones, for the sampling that fills the
 * trees which the calls above train on. Keys and values of one layer lie in a
 * pool of pages of page_size tokens, [num_pages][Hkv][page_size][d]; a
 * sequence's tokens are named by its row of the page table. A sequence may have
 * a parent (a branch its prompt): its tokens then see all tokens of the parent,
 * whose pages stay where they are and belong to the parent alone, and after
 * them its own, causally. A parent has no parent itself.
 *
 * A step: augtree_page_plan once, for all layers; then per layer
 * augtree_cache_write and augtree_paged_fwd with that plan. Lengths, tables and
 * plans stay on the GPU, every call enqueues kernels only and may be captured
 * into a graph and replayed. Calls that share a plan being written, or a
 * workspace, must not overlap. Results are bitwise reproducible; their last bits
 * follow from the batch: from how work is cut, and from the scores of rows that are
 * computed together, which move the reference of their exponents together.
 * A NaN or infinity in a row of q stays in that row and head. In a token of K or V
 * it reaches the rows that see the token, in the query heads of its KV head (in V:
 * in its channel), and in V perhaps earlier new rows of the same sequence, at most
 * 94 tokens before it: a wavefront multiplies the 64 keys that its last row is among
 * with all of its up to 32 rows, and 0 times NaN is NaN. Never another sequence but
 * a parent's branches. (A result that it reaches need not be NaN.)
 * ------------------------------------------------------------------------- */

/* Tables of a cache (DEVICE arrays, owned by the caller), shared by all layers. */
typedef struct augtree_pages {
  int32_t num_seqs;    /* rows of the table, at most 2^20 */
  int32_t max_pages;   /* entries of a row; max_pages * page_size <= 2^30 */
  int32_t num_pages;   /* pages of the pool; num_pages * page_size <= 2^30 */
  int32_t page_size;   /* tokens of a page: 16, 32, 64, 128 or 256 */
  int32_t* table;      /* [num_seqs][max_pages]: page of each page_size tokens of a sequence */
  int32_t* length;     /* [num_seqs]: cached tokens */
  int32_t* parent;     /* [num_seqs], < 0: none; NULL: nobody has one */
  int32_t* free_pages; /* [num_pages]: a ring of free pages */
  int32_t* free_state; /* [2]: position of the first free page in the ring, number of free pages */
} augtree_pages;

/* Bits of a plan's status word; 0: the plan is good. A plan with any of them (but
 * AUGTREE_PAGES_PAGE) has no rows: lengths, the ring and the caches stay as they
 * were, and the calls that take it do nothing. */
typedef enum augtree_pages_status {
  AUGTREE_PAGES_SHORT = 1,  /* fewer free pages than the new tokens need */
  AUGTREE_PAGES_LONG = 2,   /* a sequence outgrows its row of the table */
  AUGTREE_PAGES_ROWS = 4,   /* more new tokens than `rows` */
  AUGTREE_PAGES_LENGTH = 8, /* a length < 0 or past the table; a free_state out of range, or more pages given back than are in use */
  AUGTREE_PAGES_PARENT = 16, /* a sequence with new tokens whose parent is no sequence, itself, has a parent or ends in this call */
  AUGTREE_PAGES_PAGE = 32   /* a page of the new tokens is outside the pool: these are not written */
} augtree_pages_status;

/* Fields of a plan that a caller may read, as offsets in int32 words (augtree_page_plan_offset). */
typedef enum augtree_plan_field {
  AUGTREE_PLAN_STATUS = 0,    /* [1] augtree_pages_status */
  AUGTREE_PLAN_CU_ROWS = 1,   /* [num_seqs + 1] first row of each sequence's new tokens */
  AUGTREE_PLAN_SLOTS = 2,     /* [rows] page * page_size + place in the page; -1 behind the last row */
  AUGTREE_PLAN_POSITIONS = 3  /* [rows] tokens before it, its parent's among them; -1 behind the last row */
} augtree_plan_field;

/* Bytes of a plan for at most `rows` new tokens, 0 on invalid arguments; the offset of a field, -1 on invalid arguments. */
size_t augtree_page_plan_size(const augtree_pages* pages, int32_t rows, int32_t num_q_heads, int32_t num_kv_heads);
int64_t augtree_page_plan_offset(const augtree_pages* pages, int32_t rows, int32_t num_q_heads, int32_t num_kv_heads,
                                 int field);

/*
 * Plans a step. In: new_rows [num_seqs] DEVICE int32: new tokens of each sequence
 * (0: none; < 0: the sequence has ended, its pages go back and its length becomes
 * 0), `pages`. The new tokens are numbered sequence by sequence. Out: the table's
 * new entries (free pages in ring order, sequence by sequence), the ring's
 * entries behind its last one (ended sequences' pages, in order; they are free
 * for the next call; a parent's go with it, so its children end before or with
 * it), length_out [num_seqs], free_state_out [2] (each may be the array it
 * follows from), the plan. A parent's new tokens of the same step are among those
 * that its children's see.
 * `rows` may exceed the number of new tokens (a captured graph's room): rows
 * behind the last one are left as they are by the calls that take the plan.
 * Neighbouring sequences of one parent share its reading where they have few rows each.
 */
int augtree_page_plan(const augtree_pages* pages, const int32_t* new_rows, int32_t rows, int32_t num_q_heads,
                      int32_t num_kv_heads, int32_t* length_out, int32_t* free_state_out, void* plan,
                      size_t plan_bytes, void* stream);

/* How a cache holds its values: bf16, or OCP e4m3 bytes that stand for byte * scale, with a scale per KV head. */
typedef enum augtree_cache_type { AUGTREE_CACHE_BF16 = 0, AUGTREE_CACHE_E4M3 = 1 } augtree_cache_type;

/*
 * Keys and values of the new tokens, k, v [rows,Hkv,d] bf16, into their slots.
 * Caches: [num_pages][Hkv][page_size][d], pages k_page_stride (v_page_stride)
 * BYTES apart (a multiple of 16, at least a page), so that both may be views of
 * one tensor. e4m3: value / scale, rounded to nearest even, at most 448 in
 * magnitude (NaN stays NaN); k_scale, v_scale [Hkv] DEVICE fp32, > 0 and finite,
 * not read for bf16.
 */
int augtree_cache_write(const augtree_pages* pages, const void* plan, int32_t rows, int32_t num_q_heads,
                        int32_t num_kv_heads, int32_t head_dim, const uint16_t* k, const uint16_t* v, int cache_type,
                        void* k_cache, int64_t k_page_stride, void* v_cache, int64_t v_page_stride,
                        const float* k_scale, const float* v_scale, void* stream);

/*
 * Attention of the new tokens, which have been written: o_t = sum_j softmax_j(s
 * q_t.k_j) v_j over all tokens of the sequence's parent and its own tokens up to
 * t. In: q [rows,Hq,d] bf16, the caches. Out: o like q; lse [Hq,rows] fp32
 * (nullable). What stands in a page behind a sequence's last token is not read
 * into any result; a table entry outside the pool reads as zeros.
 */
int augtree_paged_fwd(const augtree_pages* pages, const void* plan, int32_t rows, int32_t num_q_heads,
                      int32_t num_kv_heads, int32_t head_dim, float softmax_scale, const uint16_t* q, int cache_type,
                      const void* k_cache, int64_t k_page_stride, const void* v_cache, int64_t v_page_stride,
                      const float* k_scale, const float* v_scale, uint16_t* o, float* lse, void* ws, size_t ws_bytes,
                      void* stream);
/* Bytes of `ws`, 0 on invalid arguments: room for the most partial results that any plan of these sizes can have, in
 * slots of 32 (row, head) pairs of every KV head: one at least for each sequence that may have new tokens, and 8192 / Hkv
 * beside them. One token at 32 / 8 heads, d = 128: 135 MB, of which a token over 4097 writes 0.4. */
size_t augtree_paged_workspace_size(const augtree_pages* pages, int32_t rows, int32_t num_q_heads,
                                    int32_t num_kv_heads, int32_t head_dim);

/*
 * Launch hook (instrumentation; not part of the method). When set, `hook` is
 * called on the calling thread immediately before (phase 0) and after
 * (phase 1) every kernel launch the library enqueues from that thread, with a
 * static role name ("fwd_prefill", "fwd_replay", "fwd_tree", "fwd_replay_split",
 * "lse_merge", "dq_prefill", "dkv_prefill", "dq_replay", "dkv_replay", "dq_tree",
 * "dkv_tree", "grad_reduce", "reduce_tree", "linear_table", "linear_state",
 * "linear_state_rev", "linear_scan", "linear_scan_rev", "linear_out", "linear_dq",
 * "linear_dkv", "linear_step", "head_norm", "head_norm_bwd", "head_norm_sum",
 * "page_plan", "cache_write", "paged_fwd", "paged_merge")
 * and the stream the kernel is enqueued on, so that a caller can record HIP
 * events around single kernels. The hook must not call back into the library. NULL removes it.
 * Per thread; the library keeps no other state.
 */
typedef void (*augtree_launch_hook)(const char* role, int phase, void* stream, void* user);
void augtree_set_launch_hook(augtree_launch_hook hook, void* user);

/*
 * Tuning of augtree_tree_bwd (process-wide; schedules and workspace sizes
 * computed after the call use it): the most query blocks (64 rows x one
 * query head) one prompt-key tile sweeps over a group's branch rows before
 * the sweep is cut into chunks. blocks >= 1 sets it, 0 restores the default
 * (1024); negative: AUGTREE_ERR_INVALID_ARGUMENT.
 */
int augtree_set_tree_chunk_blocks(int32_t blocks);
int32_t augtree_tree_chunk_blocks(void);

/* Static text of a status code. */
const char* augtree_status_string(int status);

/* Detail of the last error on the calling thread ("" if none). */
const char* augtree_last_error(void);

/* AUGTREE_OK if the current HIP device is gfx950, AUGTREE_ERR_DEVICE otherwise. */
int augtree_check_device(void);

/* Library version string. */
const char* augtree_version(void);

#ifdef __cplusplus
}
#endif

#endif /* AUGTREE_H */
