// Forward attention kernel for gfx950: prompt prefill, fused response replay
// and the split-mode partials (§3.2, Eq. 1, §3.3).
//
// One workgroup = 4 wavefronts = 128 (query row, head) pairs of one KV head
// (QRows); each wavefront owns 32 of them (one per lane column of the S^T
// accumulator). The workgroup sweeps 64-key blocks of segment A (the prompt
// KV, every key visible) and then of segment B (causal). Continuing the
// online softmax across the two segments is the log-sum-exp merge of the two
// partial states done in registers; a tile with only one segment produces one
// partial state (split mode).
//
// The step of a 64-key block is FwdCore's (fwd_core.h). K and V tiles are double-buffered in LDS (separate arrays, loop
// unrolled by two, so the compiler can tell the buffer being filled from the
// one being read) and copied there directly from global memory
// (buffer_load ... lds), so no registers hold staged data. Two workgroups
// share a CU (two wavefronts per SIMD).
#include "common.h"
#include "fwd_core.h"
#include "kernels.h"

namespace augtree {

namespace {

constexpr int BN = kFwdBlockN;  // keys per block

template <int D, bool OUT32>
__global__ __launch_bounds__(256, 2) void attn_fwd_kernel(FwdParams p) {
  __shared__ __bf16 k_buf0[BN * D], k_buf1[BN * D], v_buf0[BN * D], v_buf1[BN * D];
  int unit, hh;
  if (!xcd_unit(p.n_units, p.group, p.group_magic, unit, hh)) return;
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hf = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);  // uniform: scalar branches below
  const int tile_id = fast_div(unit, p.hkv, p.hkv_magic);
  const int kvh = unit - tile_id * p.hkv;
  const QTile t = load_tile(p.tiles, p.inl, tile_id);
  const QRows rows(t, p.group, p.group_magic, hh, wave, l32);
  if (!rows.any) return;
  // prompt rows (prefill) or response rows (replay): tensors of the tile
  const bool prow = (t.flags & QT_PROMPT_ROWS) != 0;
  const uint16_t* const qsrc = prow ? p.q[1] : p.q[0];
  const uint16_t* const kb = prow ? p.kb[1] : p.kb[0];
  const uint16_t* const vb = prow ? p.vb[1] : p.vb[0];
  const int qi = rows.row;
  const int64_t qstride = (int64_t)p.hq * D;
  const int64_t kvstride = (int64_t)p.hkv * D;
  // this lane's elements in Q: uniform start of the tile's rows of KV head
  // kvh, plus the pair's offset
  const int64_t qbase = t.q_row0 * qstride + (int64_t)kvh * p.group * D;
  const int64_t qoff = pair_offset<D>(qi, rows.head, p.hq);

  const int nA = (t.a_len + BN - 1) / BN;
  // segment B up to the workgroup's last row
  const int nB = t.b_len > 0 ? (t.b_qpos + rows.last) / BN + 1 : 0;
  const int nblk = nA + nB;

  TileCopy<BN, D, 4> cp;
  cp.init(kvstride);
  // K / V of both segments at the segment's first row and this KV head
  const char* const ka0 = reinterpret_cast<const char*>(p.ka + (int64_t)t.a_row0 * kvstride + kvh * D);
  const char* const va0 = reinterpret_cast<const char*>(p.va + (int64_t)t.a_row0 * kvstride + kvh * D);
  const char* const kb0p = reinterpret_cast<const char*>(kb + (int64_t)t.b_row0 * kvstride + kvh * D);
  const char* const vb0p = reinterpret_cast<const char*>(vb + (int64_t)t.b_row0 * kvstride + kvh * D);
  // Load cursors of K and V: the next block of each to be copied into LDS,
  // stepped in place, so that a block's scalar work is a few adds (the
  // eight wavefronts of a CU share one scalar unit)
  struct KvCursor {
    int isB, kb0, len;  // segment (0: A, 1: B), the block's first key in it, the segment's length
    const char* src;    // the block's first key row, KV head kvh
  };
  const int row_bytes = (int)(kvstride * 2);
  KvCursor kcur = nA > 0 ? KvCursor{0, 0, t.a_len, ka0} : KvCursor{1, 0, t.b_len, kb0p};
  KvCursor vcur = nA > 0 ? KvCursor{0, 0, t.a_len, va0} : KvCursor{1, 0, t.b_len, vb0p};
  // copy the cursor's block into dst and step the cursor (past the end of
  // segment B: never loaded)
  auto load_next = [&](KvCursor& c, const char* seg_b, __bf16* dst) {
    cp.issue_bytes(dst, reinterpret_cast<const uint16_t*>(c.src), min(BN, c.len - c.kb0) * row_bytes);
    int64_t step = (int64_t)BN * row_bytes;
    c.kb0 += BN;
    if (c.kb0 >= c.len && c.isB == 0) {
      step = seg_b - c.src;
      c.isB = 1;
      c.kb0 = 0;
      c.len = t.b_len;
    }
    c.src += step;
  };
  auto load_k = [&](__bf16* dst) { load_next(kcur, kb0p, dst); };
  auto load_v = [&](__bf16* dst) { load_next(vcur, vb0p, dst); };

  // the first blocks' copies go out before anything else is computed: K(b + 1)
  // and V(b) are resident while block b is processed
  if (nblk > 0) {
    load_k(k_buf0);
    load_v(v_buf0);
    if (nblk > 1) load_k(k_buf1);
  }

  FwdCore<D> core;
  core.hf = hf;
  core.load_q(qsrc + qbase + qoff);
  core.init(p.scale_log2, l32, lane);
  const int qpos_lo = t.b_qpos + rows.wlo;  // causal: the wavefront's first query position

  // a causal block whose keys all follow the wavefront's queries (and every
  // later block) contributes nothing; neither does any block to a wavefront
  // without rows
  const int nlive = !rows.wave_any ? 0 : t.b_len > 0 ? nA + (t.b_qpos + rows.whi) / BN + 1 : nA;
  auto skipped = [&](int b) { return b >= nlive; };

  auto step = [&](int b, f32x16& s0, f32x16& s1, const __bf16* kn, const __bf16* vl, f32x16& n0, f32x16& n1) {
    const bool isB = b >= nA;
    const int kb0 = (isB ? b - nA : b) * BN;
    const int len = isB ? t.b_len : t.a_len;
    auto masked = [&] { return (kb0 + BN > len) || (isB && (kb0 + BN - 1 > qpos_lo)); };
    auto limit = [&] { return min(len - 1, isB ? t.b_qpos + qi : len - 1) - kb0; };  // last visible key of the block
    core.step(masked, limit, s0, s1, kn, vl, n0, n1);
  };

  // iteration b loads K(b + 2) over K(b) and V(b + 1) over V(b - 1)
  f32x16 sa0, sa1, sb0, sb1;
  wait_vmem();
  __syncthreads();
  core.s_mfma(k_buf0, sa0, sa1);
  pace_lds_mfma<D / 8, 1, FWD_DEPTH>();
  __syncthreads();
  for (int b = 0; b < nblk; b += 2) {
    if (b + 2 < nblk) load_k(k_buf0);
    if (b + 1 < nblk) load_v(v_buf1);
    if (!skipped(b)) step(b, sa0, sa1, k_buf1, v_buf0, sb0, sb1);
    wait_vmem();
    __syncthreads();
    if (b + 1 < nblk) {
      if (b + 3 < nblk) load_k(k_buf1);
      if (b + 2 < nblk) load_v(v_buf0);
      if (!skipped(b + 1)) step(b + 1, sb0, sb1, k_buf0, v_buf1, sa0, sa1);
      wait_vmem();
      __syncthreads();
    }
  }

  const float l_tot = pair_sum(core.l_run);
  const bool part1 = (t.flags & QT_PART1) != 0;
  // (the lane's row again, instead of registers held over the sweep)
  const QRows er(t, p.group, p.group_magic, hh, wave, (int)opaque(l32));
  if (er.valid && hf == 0) {
    float* lse;
    int64_t lrows;
    if constexpr (OUT32) {
      lse = p.lse[0] + (part1 ? p.lse_part : 0);
      lrows = p.lse_rows[0];
    } else {
      lse = prow ? p.lse[1] : p.lse[0];
      lrows = prow ? p.lse_rows[1] : p.lse_rows[0];
    }
    lse[(int64_t)(kvh * p.group + er.head) * lrows + t.q_row0 + er.row] = (core.m_run * core.c + __log2f(l_tot)) * kLn2;
  }
  if (!rows.wave_any) return;
  // through this wavefront's own buffer (nothing is in flight any more)
  char* const buf = reinterpret_cast<char*>(wave == 0 ? k_buf0 : wave == 1 ? k_buf1 : wave == 2 ? v_buf0 : v_buf1);
  const float inv = 1.f / l_tot;
  if constexpr (OUT32)
    store_pairs<D>(buf, core.oacc, inv, p.o32 + (part1 ? p.o32_part : 0) + qbase, qstride, t, p.group, p.group_magic, hh,
                   wave, lane);
  else
    store_pairs<D>(buf, core.oacc, inv, reinterpret_cast<__bf16*>(prow ? p.o[1] : p.o[0]) + qbase, qstride, t, p.group, p.group_magic, hh, wave,
                   lane);
}

}  // namespace

hipError_t launch_attn_fwd(const FwdParams& p0, int n_tiles, bool out_f32, hipStream_t stream) {
  if (n_tiles == 0) return hipSuccess;
  FwdParams p = p0;
  p.n_units = n_tiles * p.hkv;
  p.hkv_magic = div_magic(p.hkv);
  p.group_magic = div_magic(p.group);
  const dim3 grid((unsigned)xcd_grid(p.n_units, p.group)), block(256);
  if (p.head_dim == 128) {
    if (out_f32) hipLaunchKernelGGL((attn_fwd_kernel<128, true>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((attn_fwd_kernel<128, false>), grid, block, 0, stream, p);
  } else {
    if (out_f32) hipLaunchKernelGGL((attn_fwd_kernel<64, true>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((attn_fwd_kernel<64, false>), grid, block, 0, stream, p);
  }
  return hipGetLastError();
}

}  // namespace augtree
