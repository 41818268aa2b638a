// Linear attention with a decay per KV head over replay trees.
//
// Every product of the layer has one form. With the rows of a segment in
// order, gamma the decay and |t - j| the distance of two rows,
//   out_t = sum_{j <= t} gamma^(t-j) (x_t . y_j) z_j          (forward in time)
//   out_t = sum_{j >= t} gamma^(j-t) (x_t . y_j) z_j          (reverse)
// where (x, y, z, out) is (q, k, v, o) and (do, v, k, dq) forward, (k, q, do,
// dv) and (v, do, q, dk) reverse. A segment is cut into blocks, a block into
// chunks of 64 rows. Inside a chunk the sum is two matrix products with the
// decayed, masked P = (x y^T) between; what lies before the chunk (after it, in
// reverse) reaches it through the state S = sum_j gamma^(edge-j) y_j z_j^T,
// [d, d] in fp32. Three steps: each block's own state (lin_state_kernel), a scan
// of the blocks' states along a segment and from the prompt into its branches,
// or from the branches back onto the prompt (lin_scan_kernel), and the outputs,
// every block from the state that reaches it (lin_out_kernel).
//
// A workgroup has one wavefront for every 32 columns of z. The state's columns
// stay in that wavefront's accumulators (rows: y, column of the lane: z) and
// serve from there as an operand of the next product, whose k index runs over
// y: the row order of `perm` below makes registers 8s .. 8s+7 of a lane hold 8
// consecutive rows of y, so that x is read from LDS in its plain order.
//
// Roundings to bf16, all of them operands of matrix products: P (2^-9 of an
// element); the decayed z of the state's update and the state itself as an
// operand are each split into two bf16 terms (2^-17), or z into three (2^-25)
// where the state is handed out in fp32.
#include "common.h"
#include "linear.h"

namespace augtree {
namespace {

constexpr int C = kLinChunk;

// ---------------------------------------------------------------------------- the batch

struct Block {
  int seg, row0, len;
  int index, count;  // of its segment's blocks
  bool prompt;
};

__device__ __forceinline__ const LinSeg* segments(const LinBatch& b) { return b.segs ? b.segs : b.inl; }

__device__ __forceinline__ Block find_block(const LinBatch& b, int block) {
  const LinSeg* s = segments(b);
  int lo = 0, hi = b.num_trees + b.num_branches;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (s[mid].block0 <= block) lo = mid;
    else hi = mid;
  }
  Block r;
  const int at = (block - s[lo].block0) * s[lo].rows;
  r.seg = lo;
  r.row0 = s[lo].row0 + at;
  r.len = min(s[lo].rows, s[lo].len - at);
  r.index = block - s[lo].block0;
  r.count = (s[lo].len + s[lo].rows - 1) / s[lo].rows;
  r.prompt = lo < b.num_trees;
  return r;
}

// ---------------------------------------------------------------------------- operands

// Transpose reads of a swizzled [64, D] tile (TrOffsets of common.h), of the
// 32 columns from c0 on. PERM exchanges the second and third group of four
// columns in every 16, which gives accumulator register i of half-wave hf the
// column 16 (i / 8) + 8 hf + i % 8 of the 32.
template <int D, bool PERM>
struct ColumnReader {
  int o[2];
  __device__ __forceinline__ void init(int c0, int lane) {
    const int grp = lane >> 4, j = lane & 15;
    const int row = 4 * (grp >> 1) + (j >> 2);
    const int q = j & 3, qp = PERM ? ((q & 1) << 1) | (q >> 1) : q;
    const int col = c0 + 16 * (grp & 1) + 4 * qp;
    o[0] = 2 * toff<D>(row, col);
    o[1] = 2 * toff<D>(row + 8, col);
  }
  // rows 16 m .. 16 m + 15: elements 0..3 are rows 16 m + 4 hf + 0..3, 4..7 are 8 further on
  __device__ __forceinline__ bf16x8 read(const __bf16* tile, int m) const {
    const char* t = reinterpret_cast<const char*>(tile) + m * 16 * D * 2;
    const s16x4 a = lds_tr16(reinterpret_cast<const __bf16*>(t + o[0]));
    const s16x4 b = lds_tr16(reinterpret_cast<const __bf16*>(t + o[1]));
    bf16x8 r;
    __builtin_memcpy(&r, &a, 8);
    __builtin_memcpy(reinterpret_cast<char*>(&r) + 8, &b, 8);
    return r;
  }
};

// v = hi + lo up to 2^-17 of v
__device__ __forceinline__ void split2(const float* v, bf16x8& hi, bf16x8& lo) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    hi[e] = (__bf16)v[e];
    lo[e] = (__bf16)(v[e] - (float)hi[e]);
  }
}

// The decays of a workgroup in LDS. row[r]: from row r of a chunk of n rows to
// its end (reverse: to its start), the weights of the state's update; rows from
// n on weigh nothing. pair[32 + k]: over a distance of k rows, 0 for k < 0.
struct Decays {
  float row[C];
  float pair[32 + C];
};

template <bool REV>
__device__ __forceinline__ void set_row_decays(Decays& t, float lg, int n) {
  const int r = threadIdx.x;
  if (r < C) t.row[r] = r < n ? exp2f(lg * (float)(REV ? r : n - 1 - r)) : 0.f;
}
__device__ __forceinline__ void set_pair_decays(Decays& t, float lg) {
  const int i = threadIdx.x;
  if (i < 32 + C) t.pair[i] = i < 32 ? 0.f : exp2f(lg * (float)(i - 32));
}

// s += Y^T (w Z) of one chunk: rows y (of all of Y's D columns, permuted),
// columns z (32 of this wavefront). TERMS bf16 terms of the weighted z.
template <int D, int TERMS>
__device__ __forceinline__ void update_state(f32x16* s, const __bf16* yt, const __bf16* zt,
                                             const ColumnReader<D, true>* yr, const ColumnReader<D, false>& zr,
                                             const float* w, int hf) {
#pragma unroll
  for (int m = 0; m < 4; ++m) {
    const bf16x8 z = zr.read(zt, m);
    const f32x4 w0 = *reinterpret_cast<const f32x4*>(w + 16 * m + 4 * hf);
    const f32x4 w1 = *reinterpret_cast<const f32x4*>(w + 16 * m + 8 + 4 * hf);
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = (float)z[e] * (e < 4 ? w0[e] : w1[e - 4]);
    bf16x8 b[3];
    split2(f, b[0], b[1]);
    if constexpr (TERMS == 3) {
#pragma unroll
      for (int e = 0; e < 8; ++e) b[2][e] = (__bf16)(f[e] - (float)b[0][e] - (float)b[1][e]);
    }
#pragma unroll
    for (int t = 0; t < D / 32; ++t) {
      const bf16x8 a = yr[t].read(yt, m);
#pragma unroll
      for (int k = 0; k < TERMS; ++k) s[t] = mfma32(a, b[k], s[t]);
    }
  }
}

// row of the state (y column) that register i of tile t holds
__device__ __forceinline__ int state_row(int t, int i, int hf) { return 32 * t + 16 * (i >> 3) + 8 * hf + (i & 7); }

// ---------------------------------------------------------------------------- blocks' own states

template <int D, bool REV, int TERMS>
__global__ __launch_bounds__(2 * D, 2) void lin_state_kernel(LinStateParams p) {
  constexpr int NW = D / 32;
  __shared__ __attribute__((aligned(1024))) __bf16 yt[C * D];
  __shared__ __attribute__((aligned(1024))) __bf16 zt[C * D];
  __shared__ __attribute__((aligned(16))) Decays decays;
  const int block = blockIdx.x / p.b.heads_kv, kvh = blockIdx.x - block * p.b.heads_kv;
  const Block bl = find_block(p.b, block);
  const bool edge = REV ? bl.index == 0 : bl.index == bl.count - 1;
  if (edge && (bl.prompt ? p.skip_prompt : p.skip_branch)) return;

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), hf = lane >> 5;
  const float lg = p.b.log2_decay[kvh];
  const int side = bl.prompt ? 0 : 1, gy = p.heads_y / p.b.heads_kv;
  const int64_t stride = (int64_t)p.heads_y * D;
  const uint16_t* y = p.y[side] + bl.row0 * stride + (int64_t)kvh * gy * D;
  const uint16_t* z = p.z[side] + bl.row0 * stride + (int64_t)kvh * gy * D;
  TileCopy<C, D, NW> copy;
  copy.init(stride);
  ColumnReader<D, true> yr[NW];
  ColumnReader<D, false> zr;
#pragma unroll
  for (int t = 0; t < NW; ++t) yr[t].init(32 * t, lane);
  zr.init(32 * wave, lane);
  f32x16 s[NW];
#pragma unroll
  for (int t = 0; t < NW; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) s[t][i] = 0.f;

  int row_n = -1;
  const int chunks = (bl.len + C - 1) / C;
  for (int ci = 0; ci < chunks; ++ci) {
    const int c = REV ? chunks - 1 - ci : ci, n = min(C, bl.len - c * C);
    const float fade = exp2f(lg * (float)n);
#pragma unroll
    for (int t = 0; t < NW; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[t][i] *= fade;
    for (int h = 0; h < gy; ++h) {
      __syncthreads();
      if (n != row_n) set_row_decays<REV>(decays, lg, n), row_n = n;
      copy.issue_at(yt, y + c * C * stride + h * D, n, stride);
      copy.issue_at(zt, z + c * C * stride + h * D, n, stride);
      wait_vmem();
      __syncthreads();
      update_state<D, TERMS>(s, yt, zt, yr, zr, decays.row, hf);
    }
  }
  float* out = p.states + ((int64_t)block * p.b.heads_kv + kvh) * D * D + 32 * wave + (lane & 31);
#pragma unroll
  for (int t = 0; t < NW; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) out[state_row(t, i, hf) * D] = s[t][i];
}

// ---------------------------------------------------------------------------- scan

// One workgroup: 1024 elements of the states of one segment and KV head.
template <bool REV>
__global__ __launch_bounds__(256) void lin_scan_kernel(LinScanParams p, int prompts, int elems) {
  const int slices = elems / 1024;
  const int unit = blockIdx.x / slices, slice = blockIdx.x - unit * slices;
  const int seg_i = unit / p.b.heads_kv, kvh = unit - seg_i * p.b.heads_kv;
  const LinSeg* segs = segments(p.b);
  const LinSeg sg = segs[prompts ? seg_i : p.b.num_trees + seg_i];
  const float lg = p.b.log2_decay[kvh];
  const int64_t per = (int64_t)p.b.heads_kv * elems;                        // one block's (tree's) states
  const int64_t at = (int64_t)kvh * elems + slice * 1024 + threadIdx.x * 4;  // this thread's four elements of them
  auto ld = [&](const float* base, int64_t i) { return *reinterpret_cast<const f32x4*>(base + i * per + at); };
  auto st = [&](float* base, int64_t i, f32x4 v) { *reinterpret_cast<f32x4*>(base + i * per + at) = v; };

  f32x4 carry = {0.f, 0.f, 0.f, 0.f};
  if (!REV) {
    if (!prompts) carry = ld(p.tree, sg.link);
    else if (p.init) carry = ld(p.init, seg_i);
  } else if (prompts) {
    const int b1 = seg_i + 1 < p.b.num_trees ? segs[seg_i + 1].link : p.b.num_branches;
    for (int b = sg.link; b < b1; ++b) carry += ld(p.tree, b);
  }
  const int count = (sg.len + sg.rows - 1) / sg.rows;
  const int skip = prompts ? p.skip_prompt : p.skip_branch;
  for (int i = 0; i < count; ++i) {
    const int j = REV ? count - 1 - i : i;
    const int len = min(sg.rows, sg.len - j * sg.rows);
    const int64_t b = sg.block0 + j;
    if (skip && i == count - 1) {
      st(p.states, b, carry);
      break;
    }
    const f32x4 own = ld(p.states, b);
    st(p.states, b, carry);
    carry = carry * exp2f(lg * (float)len) + own;
  }
  if (skip) return;
  if (!REV) {
    if (prompts) {
      st(p.tree, seg_i, carry);
      if (p.out_p) st(p.out_p, seg_i, carry);
    } else if (p.out_r) {
      st(p.out_r, seg_i, carry);
    }
  } else if (!prompts) {
    st(p.tree, seg_i, carry);
  }
}

// ---------------------------------------------------------------------------- outputs

// Forward: x and out have `group` heads for each head of y and z. Reverse: y
// and z have, and their terms are summed.
template <int D, bool REV, bool TS>
__global__ __launch_bounds__(2 * D, 2) void lin_out_kernel(LinOutParams p) {
  constexpr int NW = D / 32;
  __shared__ __attribute__((aligned(1024))) __bf16 xt[C * D];
  __shared__ __attribute__((aligned(1024))) __bf16 yt[C * D];
  __shared__ __attribute__((aligned(1024))) __bf16 zt[C * D];
  __shared__ __attribute__((aligned(1024))) __bf16 pt[C * C];
  __shared__ __attribute__((aligned(16))) Decays decays;
  const int block = blockIdx.x / p.b.heads_kv, kvh = blockIdx.x - block * p.b.heads_kv;
  const Block bl = find_block(p.b, block);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int hf = lane >> 5, l32 = lane & 31;
  const float lg = p.b.log2_decay[kvh];
  const int side = bl.prompt ? 0 : 1, g = p.b.group;
  const int64_t stride_q = (int64_t)p.b.heads_kv * g * D, stride_kv = (int64_t)p.b.heads_kv * D;
  const int64_t stride_x = REV ? stride_kv : stride_q, stride_y = REV ? stride_q : stride_kv;
  const int64_t off_x = bl.row0 * stride_x + (int64_t)kvh * (REV ? 1 : g) * D;
  const int64_t off_y = bl.row0 * stride_y + (int64_t)kvh * (REV ? g : 1) * D;
  const uint16_t* x = p.x[side] + off_x;
  const uint16_t* y = p.y[side] + off_y;
  const uint16_t* z = p.z[side] + off_y;
  uint16_t* out = p.out[side] + off_x;
  TileCopy<C, D, NW> copy_x, copy_y;
  copy_x.init(stride_x);
  copy_y.init(stride_y);
  ColumnReader<D, true> yr[NW];
  ColumnReader<D, false> zr;
#pragma unroll
  for (int t = 0; t < NW; ++t) yr[t].init(32 * t, lane);
  zr.init(32 * wave, lane);
  RowOffsets<D> rows;  // of the chunk's first 32 rows; the other 32 lie 64 D bytes further on (same swizzle)
  rows.init(l32, hf);
  auto row8 = [&](const __bf16* tile, int half, int ks) { return lds_row8_at<D>(tile + half * 32 * D, rows.o[ks]); };
  set_pair_decays(decays, lg);

  // the state that reaches the block
  f32x16 s[NW];
  {
    const float* st = p.states + ((int64_t)block * p.b.heads_kv + kvh) * D * D;
    const int col = 32 * wave + l32;
#pragma unroll
    for (int t = 0; t < NW; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int r = state_row(t, i, hf);
        s[t][i] = TS ? st[col * D + r] : st[r * D + col];
      }
  }

  // Tiles of P^T, [32 y] x [32 x]: the diagonal ones and the one off it. With
  // four wavefronts 0, 1 and 2 take one each, with two wavefront 0 both
  // diagonal ones.
  const bool diag = NW == 4 ? wave != 1 : wave == 0;
  const float* const pw = decays.pair + 32 + (REV ? 4 * hf - l32 : l32 - 4 * hf) + (diag ? 0 : 32);
  auto p_tile = [&](int ty, int tx) {
    f32x16 acc;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0.f;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
      acc = mfma32(row8(yt, ty, ks), row8(xt, tx, ks), acc);
#pragma unroll
    for (int qd = 0; qd < 4; ++qd) {
      typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
      bf16x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = (__bf16)(acc[4 * qd + e] * pw[REV ? 8 * qd + e : -8 * qd - e]);
      // k step 2 ty + qd / 2, in the order of the transposed z: chunk 2 m + hf, half qd % 2
      *reinterpret_cast<bf16x4*>(pt + toff<64>(32 * tx + l32, 8 * (2 * (2 * ty + (qd >> 1)) + hf)) + 4 * (qd & 1)) = v;
    }
  };
  int prow[2];
#pragma unroll
  for (int tx = 0; tx < 2; ++tx) prow[tx] = 32 * tx + l32;

  int row_n = -1;
  f32x16 acc[2];
  const int chunks = (bl.len + C - 1) / C;
  for (int ci = 0; ci < chunks; ++ci) {
    const int c = REV ? chunks - 1 - ci : ci, n = min(C, bl.len - c * C);
    const float fade = exp2f(lg * (float)n);
    // the state as an operand (forward: of all heads; reverse: once, where it is used)
    bf16x8 hi[NW][2], lo[NW][2];
    auto split_state = [&](int t, int k) {
      float f[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = s[t][8 * k + e];
      split2(f, hi[t][k], lo[t][k]);
    };
    if (!REV) {
#pragma unroll
      for (int t = 0; t < NW; ++t)
#pragma unroll
        for (int k = 0; k < 2; ++k) split_state(t, k);
    }
    for (int h = 0; h < g; ++h) {
      __syncthreads();
      if (n != row_n) set_row_decays<REV>(decays, lg, n), row_n = n;
      if (!REV || h == 0) copy_x.issue_at(xt, x + c * C * stride_x + (REV ? 0 : h) * D, n, stride_x);
      if (REV || h == 0) {
        copy_y.issue_at(yt, y + c * C * stride_y + (REV ? h : 0) * D, n, stride_y);
        copy_y.issue_at(zt, z + c * C * stride_y + (REV ? h : 0) * D, n, stride_y);
      }
      wait_vmem();
      __syncthreads();
      if constexpr (NW == 4) {
        if (wave == 0) p_tile(0, 0);
        else if (wave == 1) p_tile(REV ? 1 : 0, REV ? 0 : 1);
        else if (wave == 2) p_tile(1, 1);
      } else {
        if (wave == 0) p_tile(0, 0), p_tile(1, 1);
        else p_tile(REV ? 1 : 0, REV ? 0 : 1);
      }
      if (!REV || h == 0) {
        // out^T [z, x] = S^T X^T
#pragma unroll
        for (int tx = 0; tx < 2; ++tx)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[tx][i] = 0.f;
#pragma unroll
        for (int t = 0; t < NW; ++t)
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            if (REV) split_state(t, k);
#pragma unroll
            for (int tx = 0; tx < 2; ++tx) {
              const bf16x8 xv = row8(xt, tx, 2 * t + k);
              acc[tx] = mfma32(hi[t][k], xv, acc[tx]);
              acc[tx] = mfma32(lo[t][k], xv, acc[tx]);
            }
          }
#pragma unroll
        for (int tx = 0; tx < 2; ++tx) {
          const int r = 32 * tx + l32;
          const float lead = exp2f(lg * (float)(REV ? max(n - r, 0) : r + 1));
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[tx][i] *= lead;
        }
      }
      if (REV && h == 0) {
#pragma unroll
        for (int t = 0; t < NW; ++t)
#pragma unroll
          for (int i = 0; i < 16; ++i) s[t][i] *= fade;
      }
      __syncthreads();
      // out^T += Z^T P^T
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        const bf16x8 zv = zr.read(zt, m);
#pragma unroll
        for (int tx = 0; tx < 2; ++tx)
          if (REV ? (tx == 0 || m >= 2) : (tx == 1 || m < 2))
            acc[tx] = mfma32(zv, *reinterpret_cast<const bf16x8*>(pt + toff<64>(prow[tx], 8 * (2 * m + hf))), acc[tx]);
      }
      if (REV) update_state<D, 2>(s, yt, zt, yr, zr, decays.row, hf);
      if (!REV || h == g - 1) {
        uint16_t* const o = out + c * C * stride_x + (REV ? 0 : h) * D + 32 * wave + 8 * hf;
#pragma unroll
        for (int tx = 0; tx < 2; ++tx) {
          uint32_t d[8];  // registers 2i, 2i + 1 as bf16
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
            const bf16x2 v = {(__bf16)(acc[tx][2 * i] * p.scale), (__bf16)(acc[tx][2 * i + 1] * p.scale)};
            __builtin_memcpy(&d[i], &v, 4);
          }
          const int r = 32 * tx + l32;
#pragma unroll
          for (int pr = 0; pr < 2; ++pr) {
            // the half-waves exchange four columns: each then has eight consecutive ones
            const auto e0 = __builtin_amdgcn_permlane32_swap(d[4 * pr], d[4 * pr + 2], false, false);
            const auto e1 = __builtin_amdgcn_permlane32_swap(d[4 * pr + 1], d[4 * pr + 3], false, false);
            const raw16 v = {e0[0], e1[0], e0[1], e1[1]};
            if (r < n) *reinterpret_cast<raw16*>(o + r * stride_x + 16 * pr) = v;
          }
        }
      }
    }
    if (!REV && ci + 1 < chunks) {
#pragma unroll
      for (int t = 0; t < NW; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[t][i] *= fade;
      update_state<D, 2>(s, yt, zt, yr, zr, decays.row, hf);
    }
  }
}

__global__ __launch_bounds__(256) void lin_table_kernel(LinTable t) {
  for (int i = threadIdx.x; i < t.n; i += 256) t.dst[i] = t.words[i];
}

}  // namespace

hipError_t launch_lin_table(const LinTable& t, hipStream_t stream) {
  lin_table_kernel<<<1, 256, 0, stream>>>(t);
  return hipGetLastError();
}

hipError_t launch_lin_state(const LinStateParams& p, int head_dim, bool reverse, bool exact, hipStream_t stream) {
  const dim3 grid(p.b.num_blocks * p.b.heads_kv);
  if (head_dim == 128) {
    if (reverse) lin_state_kernel<128, true, 2><<<grid, 256, 0, stream>>>(p);
    else if (exact) lin_state_kernel<128, false, 3><<<grid, 256, 0, stream>>>(p);
    else lin_state_kernel<128, false, 2><<<grid, 256, 0, stream>>>(p);
  } else {
    if (reverse) lin_state_kernel<64, true, 2><<<grid, 128, 0, stream>>>(p);
    else if (exact) lin_state_kernel<64, false, 3><<<grid, 128, 0, stream>>>(p);
    else lin_state_kernel<64, false, 2><<<grid, 128, 0, stream>>>(p);
  }
  return hipGetLastError();
}

hipError_t launch_lin_scan(const LinScanParams& p, int head_dim, bool reverse, bool prompts, hipStream_t stream) {
  const int elems = head_dim * head_dim, segs = prompts ? p.b.num_trees : p.b.num_branches;
  const dim3 grid(segs * p.b.heads_kv * (elems / 1024));
  if (reverse) lin_scan_kernel<true><<<grid, 256, 0, stream>>>(p, prompts, elems);
  else lin_scan_kernel<false><<<grid, 256, 0, stream>>>(p, prompts, elems);
  return hipGetLastError();
}

hipError_t launch_lin_out(const LinOutParams& p, int head_dim, bool reverse, bool transposed, hipStream_t stream) {
  const dim3 grid(p.b.num_blocks * p.b.heads_kv);
  if (head_dim == 128) {
    if (!reverse && !transposed) lin_out_kernel<128, false, false><<<grid, 256, 0, stream>>>(p);
    else if (!reverse) lin_out_kernel<128, false, true><<<grid, 256, 0, stream>>>(p);
    else if (!transposed) lin_out_kernel<128, true, false><<<grid, 256, 0, stream>>>(p);
    else lin_out_kernel<128, true, true><<<grid, 256, 0, stream>>>(p);
  } else {
    if (!reverse && !transposed) lin_out_kernel<64, false, false><<<grid, 128, 0, stream>>>(p);
    else if (!reverse) lin_out_kernel<64, false, true><<<grid, 128, 0, stream>>>(p);
    else if (!transposed) lin_out_kernel<64, true, false><<<grid, 128, 0, stream>>>(p);
    else lin_out_kernel<64, true, true><<<grid, 128, 0, stream>>>(p);
  }
  return hipGetLastError();
}

}  // namespace augtree
