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
// every block from the state that reaches it (lin_out_kernel, lin_grad_kernel).
//
// Each wavefront owns columns of z (16 in the state kernel, 32 in the others).
// The state's columns stay in its accumulators (rows: y, column of the lane: z)
// and serve from there as an operand of the next product, whose k index runs
// over y.
//
// Roundings to bf16, all of them operands of matrix products: P, the decayed z of
// the state's update and the state itself as an operand are each split into two
// bf16 terms (2^-17 of an element), or z into three (2^-25) in the forward's
// states, which are handed out in fp32. So results are as exact as their own
// rounding; the low terms are 45 % of the matrix instructions and cost about a
// sixth of the time.
//
// What bounds it (49152 rows, 32 / 8 heads, d = 128; a copy reaches 4.9 TB/s
// here): the forward's output kernel moves 1.0 GB in 250 us, 4.2 TB/s, the state
// kernels 0.2 GB in 55 us forward and 0.8 GB in 167 us in reverse, 3.6 and 4.8
// TB/s. The gradient kernel moves 2.3 GB past the L2s (1.7 read: dv and dk share
// theirs, dq runs the other way through time) in 660 us, 3.6 TB/s, and has about
// as much work on the CU: a wavefront needs 6900 cycles for 64 rows of a head,
// beside one of another workgroup on its SIMD. Of these, two such wavefronts keep
// the matrix cores busy for 3600, the LDS for 3000 and the vector unit for about
// as many. The clock is what the chip's power leaves, 1.4 to 1.9 GHz of 2.4. Other
// shapes of it took the same time within 3 %: 8 wavefronts of 16 columns (four on
// a SIMD instead of two, but 2.4 times the LDS reads), P in 32 x 32 tiles,
// wavefront priorities, three barriers a head instead of two.
#include "common.h"
#include "linear.h"

namespace augtree {
namespace {

constexpr int C = kLinChunk;
typedef uint32_t u32x2 __attribute__((ext_vector_type(2), may_alias));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------------------- the batch

struct Block {
  int row0, len;
  bool prompt, first, last;  // of a prompt; the first, the last block of its segment
};

// Segment i. From the kernel arguments or the device copy, each by an access of
// its own kind, and made uniform (scalar registers).
__device__ __forceinline__ LinSeg load_segment(const LinBatch& b, int i) {
  const LinSeg s = b.segs ? b.segs[i] : b.inl[i];
  return {__builtin_amdgcn_readfirstlane(s.row0), __builtin_amdgcn_readfirstlane(s.len),
          __builtin_amdgcn_readfirstlane(s.block0), __builtin_amdgcn_readfirstlane(s.link),
          __builtin_amdgcn_readfirstlane(s.rows)};
}

__device__ __forceinline__ Block find_block(const LinBatch& b, int block) {
  int lo = 0, hi = b.num_trees + b.num_branches;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    const int first = __builtin_amdgcn_readfirstlane(b.segs ? b.segs[mid].block0 : b.inl[mid].block0);
    if (first <= block) lo = mid;
    else hi = mid;
  }
  const LinSeg s = load_segment(b, lo);
  Block r;
  const int at = (block - s.block0) * s.rows;
  r.row0 = s.row0 + at;
  r.len = min(s.rows, s.len - at);
  r.first = at == 0;
  r.last = s.len - at <= s.rows;
  r.prompt = lo < b.num_trees;
  return r;
}

// ---------------------------------------------------------------------------- operands
//
// 16x16x32 products: lane l holds row (column) l % 16 of the first (second)
// operand, k indices 8 (l / 16) .. + 7; of the result column l % 16, rows
// 4 (l / 16) + 0..3.
__device__ __forceinline__ f32x4 mfma16(const bf16x8& a, const bf16x8& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// LDS tiles: row-major, the 16-byte pieces of a row exchanged by an exclusive or
// with swz16(row). The LDS serves a 16-byte read in groups of 16 lanes that take
// rows 0-3 and 12-15 from one quarter of the wavefront and rows 4-11 from the
// next one, whose piece differs in bit 0; and a transpose read in groups of 32,
// four rows and two neighbouring pieces from one quarter and the rows 8 further
// on from the next. The order 0, 2, 3, 1 of the middle bits keeps both free of
// bank conflicts. (With the order 0, 1, 2, 3, made for 32x32 products, 45 % of
// the LDS cycles here were conflicts.)
template <int D>
__device__ __forceinline__ int swz16(int row) {
  const int g = (0x78 >> ((row >> 1) & 6)) & 3;  // 0, 2, 3, 1 for rows 0-3, 4-7, 8-11, 12-15
  if constexpr (D == 128) return ((row & 3) << 2) | g;
  else return (((row >> 1) & 1) << 2) | g;
}

// element offset of (row, col); col % 4 == 0 keeps 8-byte accesses inside one piece
template <int D>
__device__ __forceinline__ int loff(int row, int col) {
  return row * D + (((col >> 3) ^ swz16<D>(row)) << 3) + (col & 7);
}

// An operand whose k index runs down the rows of a swizzled [64, D] tile: 16
// columns, of which lane j of 16 names the four from `col` on in row j / 4 and
// receives one in four rows (transpose reads). Rows 32 m + 8 (lane / 16) + 0..7
// are read in two pieces of four, which lie 4 rows apart: row bit 2 and, in the
// swizzle, piece bit 1.
template <int D>
__device__ __forceinline__ int column_base(int col, int lane) {
  return 2 * loff<D>(8 * (lane >> 4) + ((lane & 15) >> 2), col);
}
// `base`: byte offset of the named columns; `flip`: bytes by which the columns wanted differ from them (bits of the
// swizzled piece, so an exclusive or)
template <int D>
__device__ __forceinline__ bf16x8 read_columns(const __bf16* tile, int base, int flip, int m) {
  const char* t = reinterpret_cast<const char*>(tile) + m * 32 * D * 2;
  constexpr int kFourRows = D == 128 ? 4 * 256 + 32 : 4 * 128 + 32;
  const s16x4 a = lds_tr16(reinterpret_cast<const __bf16*>(t + (base ^ flip)));
  const s16x4 b = lds_tr16(reinterpret_cast<const __bf16*>(t + (base ^ flip ^ kFourRows)));
  bf16x8 r;
  __builtin_memcpy(&r, &a, 8);
  __builtin_memcpy(reinterpret_cast<char*>(&r) + 8, &b, 8);
  return r;
}

// The compiler keeps such sums of a base and a constant over a loop, a register
// each; behind this it forms them where they are used.
__device__ __forceinline__ int here(int base) {
  asm volatile("" : "+v"(base));
  return base;
}

// a and b as bf16, a in the low half: one instruction. (An inline asm of it would
// hide from the compiler that a matrix instruction reading the result has to wait.)
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const f32x2 v = {a, b};
  const bf16x2 w = __builtin_convertvector(v, bf16x2);
  uint32_t r;
  __builtin_memcpy(&r, &w, 4);
  return r;
}

// v = hi + lo up to 2^-17 of v (NEXT: what is left of v stays in it)
template <bool NEXT = false>
__device__ __forceinline__ void split2(float* v, bf16x8& hi, bf16x8& lo) {
  uint32_t h[4], l[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float &a = v[2 * e], &b = v[2 * e + 1];
    h[e] = bf16_pair(a, b);
    a -= __uint_as_float(h[e] << 16);
    b -= __uint_as_float(h[e] & 0xffff0000u);
    l[e] = bf16_pair(a, b);
    if (NEXT) {
      a -= __uint_as_float(l[e] << 16);
      b -= __uint_as_float(l[e] & 0xffff0000u);
    }
  }
  __builtin_memcpy(&hi, h, 16);
  __builtin_memcpy(&lo, l, 16);
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
template <int THREADS>
__device__ __forceinline__ void set_pair_decays(Decays& t, float lg) {
  static_assert(THREADS >= 32 + C, "one element a thread");
  const int i = threadIdx.x;
  if (i < 32 + C) t.pair[i] = i < 32 ? 0.f : exp2f(lg * (float)(i - 32));
}

// s += Y^T (w Z) of one chunk: rows y (of all of Y's D columns), columns z (16 of
// this wavefront, in zf). TERMS bf16 terms of the weighted z.
template <int D, int TERMS>
__device__ __forceinline__ void update_state(f32x4* s, const __bf16* yt, const bf16x8* zf, int ybase, const float* w,
                                             int q) {
  const int yb = here(ybase);
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    const f32x4 w0 = *reinterpret_cast<const f32x4*>(w + 32 * m + 8 * q);
    const f32x4 w1 = *reinterpret_cast<const f32x4*>(w + 32 * m + 8 * q + 4);
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = (float)zf[m][e] * (e < 4 ? w0[e] : w1[e - 4]);
    bf16x8 b[3];
    split2<TERMS == 3>(f, b[0], b[1]);
    if constexpr (TERMS == 3) {
      uint32_t r[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) r[e] = bf16_pair(f[2 * e], f[2 * e + 1]);
      __builtin_memcpy(&b[2], r, 16);
    }
#pragma unroll
    for (int t = 0; t < D / 16; ++t) {
      const bf16x8 a = read_columns<D>(yt, yb, 32 * t, m);
#pragma unroll
      for (int k = 0; k < TERMS; ++k) s[t] = mfma16(a, b[k], s[t]);
    }
  }
}

template <int NT>
__device__ __forceinline__ void scale_state(f32x4* s, float f) {
#pragma unroll
  for (int t = 0; t < NT; ++t) s[t] *= f;
}

// A [64, D] tile on its way from memory to LDS through registers: fetch()
// issues the loads, put() waits for them and writes the swizzled tile. The loads
// of the next tiles are in flight while a chunk is worked on (they arrive before
// they are waited for: 150 cycles of a step of 6900 go to that and the barrier),
// and LDS holds one tile of each operand, so that two workgroups fit a CU. Rows
// from n on are zeros.
template <int D, int NW>
struct TileStage {
  static constexpr int CH = D / 8, RPI = 64 / CH, ROWS = NW * RPI, NI = C / ROWS;  // pieces of a row; rows of a pass
  static_assert(ROWS % 16 == 0, "a multiple of the swizzle's period");
  raw16 r[NI];
  __device__ __forceinline__ static int row() {
    return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * RPI + (threadIdx.x & 63) / CH;
  }
  // byte offset of this lane's first piece in the tensor's rows (of `stride` elements)
  __device__ __forceinline__ static uint32_t source(int64_t stride) {
    return (uint32_t)(2 * row() * stride) + 16 * ((threadIdx.x & 63) % CH);
  }
  __device__ __forceinline__ static int target() {
    return 2 * row() * D + ((((threadIdx.x & 63) % CH) ^ swz16<D>(row())) << 4);
  }
  __device__ __forceinline__ void fetch(const uint16_t* base, uint32_t src, int n, int64_t stride) {
#if defined(__HIP_DEVICE_COMPILE__)
    const __amdgpu_buffer_rsrc_t rsrc =
        __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, (int)(2 * n * stride), 0x00020000);
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const auto v = __builtin_amdgcn_raw_buffer_load_b128(rsrc, src + i * (uint32_t)(2 * ROWS * stride), 0, 0);
      __builtin_memcpy(&r[i], &v, 16);
    }
#endif
  }
  __device__ __forceinline__ void put(__bf16* tile, int dst) const {
    char* t = reinterpret_cast<char*>(tile) + dst;
#pragma unroll
    for (int i = 0; i < NI; ++i) *reinterpret_cast<raw16*>(t + i * 2 * ROWS * D) = r[i];
  }
};

// ---------------------------------------------------------------------------- blocks' own states

template <int D, bool REV>
__global__ __launch_bounds__(4 * D, 4) void lin_state_kernel(LinStateParams p) {
  constexpr int NT = D / 16;            // tiles of the state's rows, and wavefronts
  constexpr int TERMS = REV ? 2 : 3;    // forward states may be handed out
  __shared__ __attribute__((aligned(1024))) __bf16 yt[C * D];
  __shared__ __attribute__((aligned(1024))) __bf16 zt[C * D];
  __shared__ __attribute__((aligned(16))) Decays decays;
  const int block = blockIdx.x / p.b.heads_kv, kvh = blockIdx.x - block * p.b.heads_kv;
  const Block bl = find_block(p.b, block);
  const bool edge = REV ? bl.first : bl.last;
  if (edge && (bl.prompt ? p.skip_prompt : p.skip_branch)) return;

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4;
  const float lg = p.b.log2_decay[kvh];
  const int side = bl.prompt ? 0 : 1, gy = p.heads_y / p.b.heads_kv;
  const int64_t stride = (int64_t)p.heads_y * D;
  const uint16_t* y = p.y[side] + bl.row0 * stride + (int64_t)kvh * gy * D;
  const uint16_t* z = p.z[side] + bl.row0 * stride + (int64_t)kvh * gy * D;
  typedef TileStage<D, NT> Stage;
  Stage sy, sz;
  const uint32_t src = Stage::source(stride);
  const int dst = Stage::target();
  const int ybase = column_base<D>(4 * (lane & 3), lane), zbase = column_base<D>(16 * wave + 4 * (lane & 3), lane);
  f32x4 s[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) s[t] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int chunks = (bl.len + C - 1) / C;
  auto fetch = [&](int ci, int h) {
    const int c = REV ? chunks - 1 - ci : ci, n = min(C, bl.len - c * C);
    const int64_t at = c * C * stride + h * D;
    sy.fetch(y + at, src, n, stride);
    sz.fetch(z + at, src, n, stride);
  };
  fetch(0, 0);
  int row_n = -1;
  for (int ci = 0; ci < chunks; ++ci) {
    const int c = REV ? chunks - 1 - ci : ci, n = min(C, bl.len - c * C);
    scale_state<NT>(s, exp2f(lg * (float)n));
    for (int h = 0; h < gy; ++h) {
      __syncthreads();
      sy.put(yt, dst);
      sz.put(zt, dst);
      if (n != row_n) set_row_decays<REV>(decays, lg, n), row_n = n;
      __syncthreads();
      if (h + 1 < gy) fetch(ci, h + 1);
      else if (ci + 1 < chunks) fetch(ci + 1, 0);
      const bf16x8 zf[2] = {read_columns<D>(zt, zbase, 0, 0), read_columns<D>(zt, zbase, 0, 1)};
      update_state<D, TERMS>(s, yt, zf, ybase, decays.row, q);
    }
  }
  float* out = p.states + ((int64_t)block * p.b.heads_kv + kvh) * D * D + 16 * wave + (lane & 15);
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) out[(16 * t + 4 * q + i) * D] = s[t][i];
}

// ---------------------------------------------------------------------------- scan

// A thread carries four elements of the states of one KV head through blocks.
struct Scan {
  const LinScanParams& p;
  int64_t per, at;  // elements of one block's (tree's) states; this thread's place in them
  float lg;
  __device__ __forceinline__ f32x4 load(const float* base, int64_t i) const {
    return *reinterpret_cast<const f32x4*>(base + i * per + at);
  }
  __device__ __forceinline__ void store(float* base, int64_t i, f32x4 v) const {
    *reinterpret_cast<f32x4*>(base + i * per + at) = v;
  }
  // One segment: every block's own state is replaced by the carry that reaches it. Eight blocks are loaded ahead, which
  // hides most of the way to memory: 64 blocks of 0.5 MB, read and written in a chain, take 25 us. Workgroups of one
  // wavefront instead of four (more CUs with work) took the same.
  template <bool REV>
  __device__ __forceinline__ f32x4 segment(const LinSeg& s, f32x4 carry, bool skip) const {
    constexpr int kAhead = 8;
    const int count = (s.len + s.rows - 1) / s.rows, last = count - 1;
    for (int i0 = 0; i0 < count; i0 += kAhead) {
      f32x4 own[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int i = i0 + k;
        if (i < count) own[k] = load(p.states, s.block0 + (REV ? last - i : i));
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int i = i0 + k, j = REV ? last - i : i;
        if (i >= count) break;
        store(p.states, s.block0 + j, carry);
        if (i == last && skip) break;  // its own state was left out
        carry = carry * exp2f(lg * (float)min(s.rows, s.len - j * s.rows)) + own[k];
      }
    }
    return carry;
  }
};

// A workgroup takes 1024 elements of the states of one KV head of a tree. `part`:
// 0 the whole tree, 1 its prompt alone, 2 one branch of it (the grid then has a
// workgroup for every branch).
template <bool REV>
__global__ __launch_bounds__(256) void lin_scan_kernel(LinScanParams p, int part, int elems) {
  const int slices = elems / 1024;
  const int unit = blockIdx.x / slices, slice = blockIdx.x - unit * slices;
  const int i = unit / p.b.heads_kv, kvh = unit - i * p.b.heads_kv;
  const Scan scan = {p, (int64_t)p.b.heads_kv * elems, (int64_t)kvh * elems + slice * 1024 + threadIdx.x * 4,
                     p.b.log2_decay[kvh]};
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  if (part == 2) {
    const LinSeg s = load_segment(p.b, p.b.num_trees + i);
    if (REV) {
      scan.store(p.ends, i, scan.segment<true>(s, zero, false));
    } else {
      const f32x4 end = scan.segment<false>(s, scan.load(p.ends, s.link), p.skip_branch);
      if (p.out_r) scan.store(p.out_r, i, end);
    }
    return;
  }
  const LinSeg prompt = load_segment(p.b, i);
  const int b0 = prompt.link, b1 = i + 1 < p.b.num_trees ? load_segment(p.b, i + 1).link : p.b.num_branches;
  if (REV) {
    f32x4 carry = zero;
    for (int b = b0; b < b1; ++b)
      carry += part == 1 ? scan.load(p.ends, b)
                         : scan.segment<true>(load_segment(p.b, p.b.num_trees + b), zero, false);
    scan.segment<true>(prompt, carry, p.skip_prompt);
  } else {
    const f32x4 end = scan.segment<false>(prompt, p.init ? scan.load(p.init, i) : zero, p.skip_prompt);
    if (p.out_p) scan.store(p.out_p, i, end);
    if (part == 1) {
      scan.store(p.ends, i, end);
    } else {
      for (int b = b0; b < b1; ++b) {
        const f32x4 e = scan.segment<false>(load_segment(p.b, p.b.num_trees + b), end, p.skip_branch);
        if (p.out_r) scan.store(p.out_r, b, e);
      }
    }
  }
}

// ---------------------------------------------------------------------------- outputs

// The product of one block and KV head (see the top of the file). Forward: x
// and out have `group` heads for each head of y and z. Reverse: y and z have,
// and their terms are summed.
struct Product {
  const uint16_t *x, *y, *z;
  uint16_t* out;
  const float* state;  // of the block and KV head
};

// Rows 32 tx + l32 (< n) of a chunk, 32 columns from `out` on. The buffer's range
// ends behind row n - 1, so later rows are not written.
template <int D>
__device__ __forceinline__ void store_rows(uint16_t* out, const f32x16* acc, float scale, int n, int64_t stride, int l32,
                                           int hf) {
#if defined(__HIP_DEVICE_COMPILE__)
  const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)out, 0, (int)(2 * n * stride), 0x00020000);
  const uint32_t at = 2 * (uint32_t)(l32 * stride) + 16 * hf;
#pragma unroll
  for (int tx = 0; tx < 2; ++tx) {
    uint32_t d[8];  // registers 2i, 2i + 1
#pragma unroll
    for (int i = 0; i < 8; ++i) d[i] = bf16_pair(acc[tx][2 * i] * scale, acc[tx][2 * i + 1] * scale);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      // the half-waves exchange four columns: each then has eight consecutive ones
      const auto e0 = __builtin_amdgcn_permlane32_swap(d[4 * k], d[4 * k + 2], false, false);
      const auto e1 = __builtin_amdgcn_permlane32_swap(d[4 * k + 1], d[4 * k + 3], false, false);
      const u32x4 v = {e0[0], e1[0], e0[1], e1[1]};
      __builtin_amdgcn_raw_buffer_store_b128(v, rsrc, at + 32 * k + tx * (uint32_t)(64 * stride), 0, 0);
    }
  }
#endif
}

template <int D>
struct OutShared {
  __attribute__((aligned(1024))) __bf16 xt[C * D];
  __attribute__((aligned(1024))) __bf16 yt[C * D];
  __attribute__((aligned(1024))) __bf16 zt[C * D];
  // P as two bf16 terms, x by y in 32 x 32 tiles: (0, 0), the one off the diagonal, (1, 1)
  __attribute__((aligned(1024))) __bf16 pt[2][3][32 * 32];
  Decays decays;
};

// 32x32x16 products (see common.h): lane l holds row (column) l % 32, k indices
// 8 (l / 32) .. + 7; register i of the result column l % 32, row acc_row(i, l / 32).

// As read_columns, for 32 columns: rows 16 m + 4 hf + 0..3 and 8 further on.
template <int D>
__device__ __forceinline__ int column32_base(int col, int lane) {
  return 2 * loff<D>(4 * (lane >> 5) + ((lane & 15) >> 2), col);
}
template <int D>
__device__ __forceinline__ bf16x8 read_columns32(const __bf16* tile, int base, int flip, int m) {
  const char* t = reinterpret_cast<const char*>(tile) + m * 16 * D * 2;
  // rows 8 further on: row bit 3 and, in the swizzle (0, 2, 3, 1), both middle bits: 0 <-> 3, 2 <-> 1
  constexpr int kEightRows = 8 * 2 * D + 48;
  const s16x4 a = lds_tr16(reinterpret_cast<const __bf16*>(t + (base ^ flip)));
  const s16x4 b = lds_tr16(reinterpret_cast<const __bf16*>(t + (base ^ flip ^ kEightRows)));
  bf16x8 r;
  __builtin_memcpy(&r, &a, 8);
  __builtin_memcpy(reinterpret_cast<char*>(&r) + 8, &b, 8);
  return r;
}

// Rows of the state in the accumulators: register i of tile t in half hf. The
// columns of y are read with the second and third four of every 16 exchanged, so
// that registers 8 s .. 8 s + 7 hold 8 consecutive ones and x is read plainly.
__device__ __forceinline__ int state32_row(int t, int i, int hf) { return 32 * t + 16 * (i >> 3) + 8 * hf + (i & 7); }

// element offset of the 16-byte piece `ch` (0..3) of row r of a [32, 32] tile of P
__device__ __forceinline__ int poff(int r, int ch) { return 32 * r + 8 * (ch ^ ((r >> 2) & 3)); }

template <int D, bool REV, bool TS>
__device__ __forceinline__ void lin_out(OutShared<D>& sh, const LinBatch& batch, float scale, const Block& bl, int kvh,
                                        const Product& pr) {
  constexpr int NW = D / 32;  // wavefronts, and tiles of the state's rows
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int hf = lane >> 5, l32 = lane & 31;
  const float lg = batch.log2_decay[kvh];
  const int g = batch.group;
  const int64_t stride_q = (int64_t)batch.heads_kv * g * D, stride_kv = (int64_t)batch.heads_kv * D;
  const int64_t stride_x = REV ? stride_kv : stride_q, stride_y = REV ? stride_q : stride_kv;
  const int64_t off_x = bl.row0 * stride_x + (int64_t)kvh * (REV ? 1 : g) * D;
  const int64_t off_y = bl.row0 * stride_y + (int64_t)kvh * (REV ? g : 1) * D;
  const uint16_t* const x = pr.x + off_x;
  const uint16_t* const y = pr.y + off_y;
  const uint16_t* const z = pr.z + off_y;
  uint16_t* const out = pr.out + off_x;
  typedef TileStage<D, NW> Stage;
  Stage s0, s1, s2;  // forward: x, y, z; reverse: y, z, x
  const uint32_t src_x = Stage::source(stride_x), src_y = Stage::source(stride_y);
  const int dst = Stage::target();

  const int chunks = (bl.len + C - 1) / C;
  auto chunk_of = [&](int ci) { return REV ? chunks - 1 - ci : ci; };
  auto rows_of = [&](int c) { return min(C, bl.len - c * C); };
  auto fetch_x = [&](Stage& a, int ci, int h) {
    const int c = chunk_of(ci);
    a.fetch(x + c * C * stride_x + h * D, src_x, rows_of(c), stride_x);
  };
  auto fetch_yz = [&](Stage& a, Stage& b, int ci, int h) {
    const int c = chunk_of(ci);
    a.fetch(y + c * C * stride_y + h * D, src_y, rows_of(c), stride_y);
    b.fetch(z + c * C * stride_y + h * D, src_y, rows_of(c), stride_y);
  };
  if (REV) fetch_x(s2, 0, 0), fetch_yz(s0, s1, 0, 0);
  else fetch_yz(s1, s2, 0, 0), fetch_x(s0, 0, 0);

  // bytes: this lane's four columns of y (exchanged order) and z, its row of a tile's first 32, its row of a tile of P
  const int c4 = 16 * ((lane >> 4) & 1);
  const int ybase = column32_base<D>(c4 + 4 * (((lane & 1) << 1) | ((lane >> 1) & 1)), lane);
  const int zbase = column32_base<D>(32 * wave + c4 + 4 * (lane & 3), lane);
  const int rbase = 2 * loff<D>(l32, 8 * hf);
  const int pbase = 2 * poff(l32, hf);
  set_pair_decays<2 * D>(sh.decays, lg);
  // the 16 x 16 tiles of P beside the diagonal that are masked stay zero
  for (int i = threadIdx.x; i < 2 * 3 * 32 * 32 / 8; i += 2 * D) reinterpret_cast<raw16*>(sh.pt)[i] = raw16{0u, 0u, 0u, 0u};

  // the state that reaches the block
  f32x16 s[NW];
  {
    const int col = 32 * wave + l32;
#pragma unroll
    for (int t = 0; t < NW; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int r = state32_row(t, i, hf);
        s[t][i] = TS ? pr.state[col * D + r] : pr.state[r * D + col];
      }
  }

  // row l32 of a tile's half `half`, 8 columns from 16 ks + 8 hf on
  auto read8 = [&](const __bf16* tile, int base, int half, int ks) {
    return *reinterpret_cast<const bf16x8*>(reinterpret_cast<const char*>(tile) + half * 64 * D + (base ^ (32 * ks)));
  };
  // P^T in 16 x 16 tiles (16x16x32 products, a lane having one x and four y), of which the 10 on and beside the diagonal
  // are dealt to the wavefronts: tile k is (i, j), j <= i, with i (i + 1) / 2 + j = k. (The three 32 x 32 tiles they make
  // up leave one of four wavefronts without one.)
  const int q = lane >> 4, l16 = lane & 15;
  const int rbase16 = 2 * loff<D>(l16, 8 * q);
  auto p_tile = [&](int ty, int tx) {
    const int rb = here(rbase16);
    const char* const yt = reinterpret_cast<const char*>(sh.yt) + ty * 32 * D;
    const char* const xt = reinterpret_cast<const char*>(sh.xt) + tx * 32 * D;
    f32x4 a = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks)
      a = mfma16(*reinterpret_cast<const bf16x8*>(yt + (rb ^ (64 * ks))),
                 *reinterpret_cast<const bf16x8*>(xt + (rb ^ (64 * ks))), a);
    const float* const pw = sh.decays.pair + 32 + (REV ? 16 * (ty - tx) + 4 * q - l16 : 16 * (tx - ty) + l16 - 4 * q);
    u32x2 v, u;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const float f0 = a[2 * e] * pw[REV ? 2 * e : -2 * e], f1 = a[2 * e + 1] * pw[REV ? 2 * e + 1 : -2 * e - 1];
      v[e] = bf16_pair(f0, f1);
      u[e] = bf16_pair(f0 - __uint_as_float(v[e] << 16), f1 - __uint_as_float(v[e] & 0xffff0000u));
    }
    // in the order of the transposed z: y = 4 q of k step ty % 2 is piece 2 (ty % 2) + q % 2, half q / 2
    const int k = (ty >> 1) == (tx >> 1) ? 2 * (tx >> 1) : 1;
    const int o = poff(16 * (tx & 1) + l16, 2 * (ty & 1) + (q & 1)) + 4 * (q >> 1);
    *reinterpret_cast<u32x2*>(sh.pt[0][k] + o) = v;
    *reinterpret_cast<u32x2*>(sh.pt[1][k] + o) = u;
  };
  auto p_tiles = [&]() {
#pragma unroll
    for (int r = 0; r < (10 + NW - 1) / NW; ++r) {
      const int k = r * NW + wave;
      if (k >= 10) break;
      const int i = (k >= 1) + (k >= 3) + (k >= 6), j = k - i * (i + 1) / 2;
      if (REV) p_tile(i, j);
      else p_tile(j, i);
    }
  };

  f32x16 acc[2];
  // acc = out^T [z, x] of what reaches the chunk: S^T X^T, the state as two bf16 terms, and its decay to each row
  auto from_state = [&](int n) {
    const int xb = here(rbase);
#pragma unroll
    for (int tx = 0; tx < 2; ++tx)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[tx][i] = 0.f;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      float f[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = s[ks >> 1][8 * (ks & 1) + e];
      bf16x8 hi, lo;
      split2(f, hi, lo);
      const bf16x8 x0 = read8(sh.xt, xb, 0, ks), x1 = read8(sh.xt, xb, 1, ks);
      acc[0] = mfma32(hi, x0, acc[0]);
      acc[1] = mfma32(hi, x1, acc[1]);
      acc[0] = mfma32(lo, x0, acc[0]);
      acc[1] = mfma32(lo, x1, acc[1]);
    }
#pragma unroll
    for (int tx = 0; tx < 2; ++tx) {
      const int r = 32 * tx + l32;
      const float lead = exp2f(lg * (float)(REV ? max(n - r, 0) : r + 1));
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[tx][i] *= lead;
    }
  };
  // acc += Z^T P^T
  auto from_chunk = [&](const bf16x8* zf) {
    const int pb = here(pbase);
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int tx = 0; tx < 2; ++tx) {
          const int ty = m >> 1;
          if (REV ? ty < tx : ty > tx) continue;  // masked
          const char* t = reinterpret_cast<const char*>(sh.pt[k][ty == tx ? 2 * tx : 1]);
          acc[tx] = mfma32(zf[m], *reinterpret_cast<const bf16x8*>(t + (pb ^ (32 * (m & 1)))), acc[tx]);
        }
  };
  // s += Y^T (w Z)
  auto update = [&](const bf16x8* zf) {
    const int yb = here(ybase);
    const float* const w = sh.decays.row + 4 * hf;
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const f32x4 w0 = *reinterpret_cast<const f32x4*>(w + 16 * m), w1 = *reinterpret_cast<const f32x4*>(w + 16 * m + 8);
      float f[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = (float)zf[m][e] * (e < 4 ? w0[e] : w1[e - 4]);
      bf16x8 hi, lo;
      split2(f, hi, lo);
#pragma unroll
      for (int t = 0; t < NW; ++t) {
        const bf16x8 a = read_columns32<D>(sh.yt, yb, 64 * t, m);
        s[t] = mfma32(a, hi, s[t]);
        s[t] = mfma32(a, lo, s[t]);
      }
    }
  };
  auto fade_state = [&](float f) {
#pragma unroll
    for (int t = 0; t < NW; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[t][i] *= f;
  };
  auto store = [&](int c, int h, int n) {
    store_rows<D>(out + c * C * stride_x + h * D + 32 * wave, acc, scale, n, stride_x, l32, hf);
  };

  // Two barriers a head: behind the first its tiles are in LDS, behind the second P is, and all that reads the tiles has
  // read them (forward: but for y and z, once a chunk), so that the next ones may be written beside the product with P.
  int row_n = -1;
  for (int ci = 0; ci < chunks; ++ci) {
    const int c = chunk_of(ci), n = rows_of(c);
    const bool more = ci + 1 < chunks;
    const float fade = exp2f(lg * (float)n);
    if constexpr (REV) {
      s2.put(sh.xt, dst);
      if (n != row_n) set_row_decays<REV>(sh.decays, lg, n), row_n = n;
      if (ci == 0) s0.put(sh.yt, dst), s1.put(sh.zt, dst);
      for (int h = 0; h < g; ++h) {
        __syncthreads();
        if (h + 1 < g) fetch_yz(s0, s1, ci, h + 1);
        else if (more) fetch_yz(s0, s1, ci + 1, 0), fetch_x(s2, ci + 1, 0);
        if (h == 0) {
          from_state(n);
          fade_state(fade);
        }
        bf16x8 zf[4];
#pragma unroll
        for (int m = 0; m < 4; ++m) zf[m] = read_columns32<D>(sh.zt, zbase, 0, m);
        p_tiles();
        update(zf);
        __syncthreads();
        if (more || h + 1 < g) s0.put(sh.yt, dst), s1.put(sh.zt, dst);
        from_chunk(zf);
      }
      store(c, 0, n);
    } else {
      if (ci > 0) __syncthreads();  // y has been read by the state's update
      s1.put(sh.yt, dst);
      s2.put(sh.zt, dst);
      if (n != row_n) set_row_decays<REV>(sh.decays, lg, n), row_n = n;
      bf16x8 zf[4];
      for (int h = 0; h < g; ++h) {
        s0.put(sh.xt, dst);
        __syncthreads();
        if (h + 1 < g) fetch_x(s0, ci, h + 1);
        else if (more) fetch_x(s0, ci + 1, 0), fetch_yz(s1, s2, ci + 1, 0);
        if (h == 0) {
#pragma unroll
          for (int m = 0; m < 4; ++m) zf[m] = read_columns32<D>(sh.zt, zbase, 0, m);
        }
        p_tiles();
        // (the state's two terms are formed again for every head: kept over the loop they take registers, which then
        // spill. The empty asm keeps the compiler from doing that.)
#pragma unroll
        for (int t = 0; t < NW; ++t) asm volatile("" : "+v"(s[t]));
        from_state(n);
        __syncthreads();
        from_chunk(zf);
        store(c, h, n);
      }
      if (more) {
        fade_state(fade);
        update(zf);
      }
    }
  }
}

template <int D>
__global__ __launch_bounds__(2 * D, 2) void lin_out_kernel(LinOutParams p) {
  __shared__ OutShared<D> sh;
  const int block = blockIdx.x / p.b.heads_kv, kvh = blockIdx.x - block * p.b.heads_kv;
  const Block bl = find_block(p.b, block);
  const int side = bl.prompt ? 0 : 1;
  const float* state = p.states + ((int64_t)block * p.b.heads_kv + kvh) * D * D;
  const Product pr = {p.q[side], p.k[side], p.v[side], p.o[side], state};
  lin_out<D, false, false>(sh, p.b, p.scale, bl, kvh, pr);
}

// dq, dv and dk: three workgroups a block and KV head, one after the other on
// one XCD (workgroups go to the 8 XCDs in turn), so that what they share of q,
// k, v and do comes from memory once.
template <int D>
__global__ __launch_bounds__(2 * D, 2) void lin_grad_kernel(LinGradParams p) {
  __shared__ OutShared<D> sh;
  const int j = blockIdx.x >> 3, unit = (j / 3) * 8 + (blockIdx.x & 7), role = j % 3;
  if (unit >= p.b.num_blocks * p.b.heads_kv) return;
  const int block = unit / p.b.heads_kv, kvh = unit - block * p.b.heads_kv;
  const Block bl = find_block(p.b, block);
  const int side = bl.prompt ? 0 : 1;
  const int64_t at = ((int64_t)block * p.b.heads_kv + kvh) * D * D;
  if (role == 0) {
    const Product pr = {p.dout[side], p.v[side], p.k[side], p.dq[side], p.states + at};
    lin_out<D, false, true>(sh, p.b, p.scale, bl, kvh, pr);
  } else if (role == 1) {
    const Product pr = {p.k[side], p.q[side], p.dout[side], p.dv[side], p.states_rev + at};
    lin_out<D, true, false>(sh, p.b, p.scale, bl, kvh, pr);
  } else {
    const Product pr = {p.v[side], p.dout[side], p.q[side], p.dk[side], p.states_rev + at};
    lin_out<D, true, true>(sh, p.b, p.scale, bl, kvh, pr);
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

hipError_t launch_lin_state(const LinStateParams& p, int head_dim, bool reverse, hipStream_t stream) {
  const dim3 grid(p.b.num_blocks * p.b.heads_kv);
  if (head_dim == 128) {
    if (reverse) lin_state_kernel<128, true><<<grid, 512, 0, stream>>>(p);
    else lin_state_kernel<128, false><<<grid, 512, 0, stream>>>(p);
  } else {
    if (reverse) lin_state_kernel<64, true><<<grid, 256, 0, stream>>>(p);
    else lin_state_kernel<64, false><<<grid, 256, 0, stream>>>(p);
  }
  return hipGetLastError();
}

hipError_t launch_lin_scan(const LinScanParams& p, int head_dim, bool reverse, int part, hipStream_t stream) {
  const int elems = head_dim * head_dim, units = part == 2 ? p.b.num_branches : p.b.num_trees;
  const dim3 grid(units * p.b.heads_kv * (elems / 1024));
  if (reverse) lin_scan_kernel<true><<<grid, 256, 0, stream>>>(p, part, elems);
  else lin_scan_kernel<false><<<grid, 256, 0, stream>>>(p, part, elems);
  return hipGetLastError();
}

hipError_t launch_lin_out(const LinOutParams& p, int head_dim, hipStream_t stream) {
  const dim3 grid(p.b.num_blocks * p.b.heads_kv);
  if (head_dim == 128) lin_out_kernel<128><<<grid, 256, 0, stream>>>(p);
  else lin_out_kernel<64><<<grid, 128, 0, stream>>>(p);
  return hipGetLastError();
}

hipError_t launch_lin_grad(const LinGradParams& p, int head_dim, hipStream_t stream) {
  const dim3 grid((p.b.num_blocks * p.b.heads_kv + 7) / 8 * 24);
  if (head_dim == 128) lin_grad_kernel<128><<<grid, 256, 0, stream>>>(p);
  else lin_grad_kernel<64><<<grid, 128, 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace augtree
