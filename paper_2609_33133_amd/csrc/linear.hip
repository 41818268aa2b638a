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
// every block from the state that reaches it (lin_out_kernel, lin_dq_kernel,
// lin_dkv_kernel).
//
// Each wavefront owns columns of z (16 in the state kernel, 32 in the others).
// The state's columns stay in its accumulators (rows: y, column of the lane: z)
// and serve from there as an operand of the next product, whose k index runs
// over y. (The kernel for dk and dv hands it on through LDS: see there.)
//
// Roundings to bf16, all of them operands of matrix products: P, the decayed z of
// the state's update and the state itself as an operand are each split into two
// bf16 terms (2^-17 of an element), or z into three (2^-25) in the forward's
// states, which are handed out in fp32. So results are as exact as their own
// rounding; the low terms are 45 % of the matrix instructions and cost about a
// sixth of the time.
//
// What bounds it (49152 rows, 32 / 8 heads, d = 128, in a steady run; a copy
// reaches 4.9 TB/s here): the output and dq kernels move 1.0 GB each in 235 and 238
// us, 4.4 TB/s, the state kernels 0.2 GB in 55 us forward and 0.8 GB in 166 us in
// reverse, 3.8 and 4.9 TB/s. The kernel for dk and dv moves 1.2 GB in 330 us, 3.7
// TB/s; its matrix cores are busy for 41 % of that and its LDS for 37 %, in phases
// that barriers part.
// The clock is what the chip's power leaves, 1.4 to 2.0 GHz of 2.4. Taken or left
// within 3 % of the time: P in 32 x 32 tiles, 8 wavefronts of 16 columns, wavefront
// priorities, tiles fetched half a step earlier, operands of a product with P all
// read ahead of it.
#include <type_traits>

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

// The segment of a block: the last one that does not begin behind it. All lanes of a wavefront look at once, at 64
// segments that part the ones in question, so that 4096 take two loads in a row
// (halving them: 541 us for a training step of 32 trees with 16 short branches each, 8 / 2 heads, where this takes 511).
__device__ __forceinline__ Block find_block(const LinBatch& b, int block) {
  int lo = 0, n = b.num_trees + b.num_branches;
  while (n > 1) {
    const int step = (n + 63) >> 6, i = (int)(threadIdx.x & 63) * step;
    int first = INT32_MAX;
    if (i < n) first = b.segs ? b.segs[lo + i].block0 : b.inl[lo + i].block0;
    const int at = (__popcll(__ballot(first <= block)) - 1) * step;
    lo += at;
    n = min(step, n - at);
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
// they are waited for: 200 cycles of a step of 5500 go to that and the barrier),
// and LDS holds one tile of each operand. Rows from n on are zeros.
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
  // One segment: every block's own state is replaced by the carry that reaches it. While a group of eight blocks is
  // worked on the next one is on its way: from sixteen blocks on without a branch, behind which the wait for a load would
  // take in all that are on their way.
  template <bool REV>
  __device__ __forceinline__ f32x4 segment(const LinSeg& s, f32x4 carry) const {
    constexpr int kAhead = 8;
    const int count = (s.len + s.rows - 1) / s.rows, last = count - 1;
    const float fade = exp2f(lg * (float)s.rows), short_fade = exp2f(lg * (float)(s.len - last * s.rows));
    auto block = [&](int i) { return REV ? last - i : i; };
    auto pass = [&](f32x4 own, int i) {
      store(p.states, s.block0 + block(i), carry);
      carry = carry * (block(i) == last ? short_fade : fade) + own;
    };
    f32x4 a[kAhead], b[kAhead];
    int i0 = 0;
    if (count >= 2 * kAhead) {
      auto fetch = [&](f32x4* own, int i) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k) own[k] = load(p.states, s.block0 + block(min(i + k, last)));
      };
      fetch(a, 0);
      for (; i0 + 2 * kAhead <= count; i0 += 2 * kAhead) {
        fetch(b, i0 + kAhead);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) pass(a[k], i0 + k);
        fetch(a, i0 + 2 * kAhead);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) pass(b[k], i0 + kAhead + k);
      }
    }
    for (; i0 < count; i0 += kAhead) {
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        if (i0 + k < count) a[k] = load(p.states, s.block0 + block(i0 + k));
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        if (i0 + k < count) pass(a[k], i0 + k);
    }
    return carry;
  }
};

// Where the state kernel left a segment's last block out, what is found there ends in a carry that nobody reads.
//
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
      scan.store(p.ends, i, scan.segment<true>(s, zero));
    } else {
      const f32x4 end = scan.segment<false>(s, scan.load(p.ends, s.link));
      if (p.out_r) scan.store(p.out_r, i, end);
    }
    return;
  }
  const LinSeg prompt = load_segment(p.b, i);
  const int b0 = prompt.link, b1 = i + 1 < p.b.num_trees ? load_segment(p.b, i + 1).link : p.b.num_branches;
  if (REV) {
    f32x4 carry = zero;
    if (part == 0) {
      for (int b = b0; b < b1; ++b) carry += scan.segment<true>(load_segment(p.b, p.b.num_trees + b), zero);
    } else {
      for (int b = b0; b < b1; b += 8) {
        f32x4 e[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (b + k < b1) e[k] = scan.load(p.ends, b + k);
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (b + k < b1) carry += e[k];
      }
    }
    scan.segment<true>(prompt, carry);
  } else {
    const f32x4 end = scan.segment<false>(prompt, p.init ? scan.load(p.init, i) : zero);
    if (p.out_p) scan.store(p.out_p, i, end);
    if (part == 1) {
      scan.store(p.ends, i, end);
    } else {
      for (int b = b0; b < b1; ++b) {
        const f32x4 e = scan.segment<false>(load_segment(p.b, p.b.num_trees + b), end);
        if (p.out_r) scan.store(p.out_r, b, e);
      }
    }
  }
}

// ---------------------------------------------------------------------------- outputs

// The product of one block and KV head, forward in time (see the top of the
// file): x and out have `group` heads for each head of y and z.
struct Product {
  const uint16_t *x, *y, *z;
  uint16_t* out;
  const float* state;  // of the block and KV head
};

// Rows 32 tx + l32 (< n) of a chunk, 32 columns from `out` on. The buffer's range
// ends behind row n - 1, so later rows are not written.
template <int D>
__device__ __forceinline__ void store_rows(uint16_t* out, const f32x16* acc, float scale, int n, int64_t stride,
                                           int l32, int hf) {
#if defined(__HIP_DEVICE_COMPILE__)
  const __amdgpu_buffer_rsrc_t rsrc =
      __builtin_amdgcn_make_buffer_rsrc((void*)out, 0, (int)(2 * n * stride), 0x00020000);
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

// 8 elements from byte `at` of a tile
__device__ __forceinline__ bf16x8 read8(const __bf16* tile, int at) {
  return *reinterpret_cast<const bf16x8*>(reinterpret_cast<const char*>(tile) + at);
}

// P as two bf16 terms, x by y in 32 x 32 tiles: (0, 0), the one off the diagonal, (1, 1)
typedef __bf16 PTiles[2][3][32 * 32];
// element offset of the 16-byte piece `ch` (0..3) of row r of such a tile
__device__ __forceinline__ int poff(int r, int ch) { return 32 * r + 8 * (ch ^ ((r >> 2) & 3)); }

// This lane's four elements (x l16, y 4 q .. + 3) of the 16 x 16 tile (tx, ty), in the order of the transposed z:
// y = 4 q of k step ty % 2 is piece 2 (ty % 2) + q % 2, half q / 2.
// w: their decays.
__device__ __forceinline__ void put_p(PTiles& pt, int tx, int ty, const f32x4& a, const float* w, int q, int l16) {
  u32x2 v, u;
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const float f0 = a[2 * e] * w[2 * e], f1 = a[2 * e + 1] * w[2 * e + 1];
    v[e] = bf16_pair(f0, f1);
    u[e] = bf16_pair(f0 - __uint_as_float(v[e] << 16), f1 - __uint_as_float(v[e] & 0xffff0000u));
  }
  const int k = (ty >> 1) == (tx >> 1) ? 2 * (tx >> 1) : 1;
  const int o = poff(16 * (tx & 1) + l16, 2 * (ty & 1) + (q & 1)) + 4 * (q >> 1);
  *reinterpret_cast<u32x2*>(pt[0][k] + o) = v;
  *reinterpret_cast<u32x2*>(pt[1][k] + o) = u;
}

template <int THREADS>
__device__ __forceinline__ void clear(void* p, int bytes) {
  for (int i = threadIdx.x; i < bytes / 16; i += THREADS) static_cast<raw16*>(p)[i] = raw16{0u, 0u, 0u, 0u};
}

template <int N>
using Int = std::integral_constant<int, N>;

template <int D>
struct OutShared {
  __attribute__((aligned(1024))) __bf16 xt[C * D];
  __attribute__((aligned(1024))) __bf16 yt[C * D];
  __attribute__((aligned(1024))) __bf16 zt[C * D];
  __attribute__((aligned(1024))) PTiles pt;
  Decays decays;
};

template <int D, bool TS>
__device__ __forceinline__ void lin_out(OutShared<D>& sh, const LinBatch& batch, float scale, const Block& bl, int kvh,
                                        const Product& pr) {
  constexpr int NW = D / 32;  // wavefronts, and tiles of the state's rows
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int hf = lane >> 5, l32 = lane & 31;
  const float lg = batch.log2_decay[kvh];
  const int g = batch.group;
  const int64_t stride_x = (int64_t)batch.heads_kv * g * D, stride_y = (int64_t)batch.heads_kv * D;
  const int64_t off_x = bl.row0 * stride_x + (int64_t)kvh * g * D, off_y = bl.row0 * stride_y + (int64_t)kvh * D;
  const uint16_t* const x = pr.x + off_x;
  const uint16_t* const y = pr.y + off_y;
  const uint16_t* const z = pr.z + off_y;
  uint16_t* const out = pr.out + off_x;
  typedef TileStage<D, NW> Stage;
  Stage sx, sy, sz;
  const uint32_t src_x = Stage::source(stride_x), src_y = Stage::source(stride_y);
  const int dst = Stage::target();

  const int chunks = (bl.len + C - 1) / C;
  auto rows_of = [&](int c) { return c < chunks ? min(C, bl.len - c * C) : 0; };
  // (Nothing is fetched behind the last head, by a range of no rows: under a branch the registers of both ways would be
  // copied, and the copies wait for the loads.)
  int fetched = 0, head = 0;  // chunk and head of the next fetch of x
  auto fetch_x = [&]() {
    sx.fetch(x + fetched * C * stride_x + head * D, src_x, rows_of(fetched), stride_x);
    if (++head == g) head = 0, ++fetched;
  };
  auto fetch_yz = [&](int c) {
    sy.fetch(y + c * C * stride_y, src_y, rows_of(c), stride_y);
    sz.fetch(z + c * C * stride_y, src_y, rows_of(c), stride_y);
  };
  fetch_yz(0);
  fetch_x();

  // bytes: this lane's four columns of y (exchanged order) and z, its row of a tile's first 32, its row of a tile of P
  const int c4 = 16 * ((lane >> 4) & 1);
  const int ybase = column32_base<D>(c4 + 4 * (((lane & 1) << 1) | ((lane >> 1) & 1)), lane);
  const int zbase = column32_base<D>(32 * wave + c4 + 4 * (lane & 3), lane);
  const int rbase = 2 * loff<D>(l32, 8 * hf);
  const int pbase = 2 * poff(l32, hf);
  set_pair_decays<2 * D>(sh.decays, lg);
  // the 16 x 16 tiles of P beside the diagonal that are masked stay zero
  clear<2 * D>(&sh.pt, sizeof(sh.pt));

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

  // P^T in 16 x 16 tiles (16x16x32 products, a lane having one x and four y), of which the 10 on and beside the diagonal
  // are dealt to the wavefronts: tile k is (tx, ty), ty <= tx, with tx (tx + 1) / 2 + ty = k. (The three 32 x 32 tiles
  // they make up leave one of four wavefronts without one.) A wavefront forms its tiles k0, k0 + NW, ... side by side.
  const int q = lane >> 4, l16 = lane & 15;
  const int rbase16 = 2 * loff<D>(l16, 8 * q);
  auto p_tiles = [&](auto count, int k0) {
    constexpr int N = decltype(count)::value;
    const int rb = here(rbase16);
    int tx[N], ty[N];
    f32x4 a[N];
    float w[N][4];
#pragma unroll
    for (int r = 0; r < N; ++r) {
      const int k = k0 + r * NW;
      tx[r] = (k >= 1) + (k >= 3) + (k >= 6);
      ty[r] = k - tx[r] * (tx[r] + 1) / 2;
      a[r] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 4; ++e) w[r][e] = sh.decays.pair[32 + 16 * (tx[r] - ty[r]) + l16 - 4 * q - e];
    }
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks)
#pragma unroll
      for (int r = 0; r < N; ++r)
        a[r] = mfma16(read8(sh.yt + ty[r] * 16 * D, rb ^ (64 * ks)), read8(sh.xt + tx[r] * 16 * D, rb ^ (64 * ks)),
                      a[r]);
#pragma unroll
    for (int r = 0; r < N; ++r) put_p(sh.pt, tx[r], ty[r], a[r], w[r], q, l16);
  };

  f32x16 acc[2];
  // acc = out^T [z, x] of what reaches the chunk: S^T X^T, the state as two bf16 terms, and its decay to each row
  auto from_state = [&]() {
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
      const bf16x8 x0 = read8(sh.xt, xb ^ (32 * ks)), x1 = read8(sh.xt + 32 * D, xb ^ (32 * ks));
      acc[0] = mfma32(hi, x0, acc[0]);
      acc[1] = mfma32(hi, x1, acc[1]);
      acc[0] = mfma32(lo, x0, acc[0]);
      acc[1] = mfma32(lo, x1, acc[1]);
    }
#pragma unroll
    for (int tx = 0; tx < 2; ++tx) {
      const int r = 32 * tx + l32;
      const float lead = exp2f(lg * (float)(r + 1));
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
          if (ty > tx) continue;  // masked
          acc[tx] = mfma32(zf[m], read8(sh.pt[k][ty == tx ? 2 * tx : 1], pb ^ (32 * (m & 1))), acc[tx]);
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
  // Two barriers a head: behind the first its tiles are in LDS, behind the second P is, and all that reads x (and, with
  // the chunk's last head, y) has read it.
  int row_n = -1;
  for (int c = 0; c < chunks; ++c) {
    const int n = rows_of(c);
    if (c > 0) __syncthreads();  // y has been read by the state's update
    sy.put(sh.yt, dst);
    sz.put(sh.zt, dst);
    if (c + 1 < chunks) fetch_yz(c + 1);
    if (n != row_n) set_row_decays<false>(sh.decays, lg, n), row_n = n;
    bf16x8 zf[4];
    for (int h = 0; h < g; ++h) {
      sx.put(sh.xt, dst);
      __syncthreads();
      fetch_x();
      if (h == 0) {
#pragma unroll
        for (int m = 0; m < 4; ++m) zf[m] = read_columns32<D>(sh.zt, zbase, 0, m);
      }
      if (NW == 2) p_tiles(Int<5>{}, wave);
      else if (wave < 2) p_tiles(Int<3>{}, wave);
      else p_tiles(Int<2>{}, wave);
      // (the state's two terms are formed again for every head: kept over the loop they take registers, which then
      // spill. The empty asm keeps the compiler from doing that.)
#pragma unroll
      for (int t = 0; t < NW; ++t) asm volatile("" : "+v"(s[t]));
      from_state();
      __syncthreads();
      from_chunk(zf);
      store_rows<D>(out + c * C * stride_x + h * D + 32 * wave, acc, scale, n, stride_x, l32, hf);
    }
    if (c + 1 < chunks) {
      fade_state(exp2f(lg * (float)n));
      update(zf);
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
  lin_out<D, false>(sh, p.b, p.scale, bl, kvh, pr);
}

template <int D>
__global__ __launch_bounds__(2 * D, 2) void lin_dq_kernel(LinGradParams p) {
  __shared__ OutShared<D> sh;
  const int block = blockIdx.x / p.b.heads_kv, kvh = blockIdx.x - block * p.b.heads_kv;
  const Block bl = find_block(p.b, block);
  const int side = bl.prompt ? 0 : 1;
  const float* const state = p.states + ((int64_t)block * p.b.heads_kv + kvh) * D * D;
  const Product pr = {p.dout[side], p.v[side], p.k[side], p.dq[side], state};
  lin_out<D, true>(sh, p.b, p.scale, bl, kvh, pr);
}

// ---------------------------------------------------------------------------- dk and dv

// Both sum over the query heads and run backwards in time, and their states are
// one and the transpose of it: dv_t = k_t S, dk_t = v_t S^T with S = sum q_j do_j^T.
// So a workgroup forms both, with two kinds of wavefronts that take 32 columns each:
// those of dv own columns of S, as the accumulators of its update, and those of dk
// form P for both. Between chunks S goes through LDS as two bf16 terms, where dv's
// wavefronts read it by rows and dk's by columns. The two kinds share SIMDs: one is
// busy with matrix products where the other waits for LDS or converts. (Workgroups
// of their own for dk and dv, two a CU, each with a state and P: 1160 us for forward
// and backward of those 49152 rows where this took 1065.)
template <int D>
struct DkvShared {
  __attribute__((aligned(1024))) __bf16 kt[C * D];
  __attribute__((aligned(1024))) __bf16 vt[C * D];
  __attribute__((aligned(1024))) __bf16 qt[C * D];
  __attribute__((aligned(1024))) __bf16 gt[C * D];     // do
  __attribute__((aligned(1024))) PTiles pt[2];         // of dv, of dk
  // S^T as two bf16 terms: a row for each column of do (the second and third four of every 16 exchanged)
  __attribute__((aligned(1024))) __bf16 st[2][D * D];
  Decays decays;
};

template <int D, bool OF_K>
__device__ __forceinline__ void lin_dkv(DkvShared<D>& sh, const LinGradParams& p, const Block& bl, int block, int kvh,
                                        int wave) {
  constexpr int NW = D / 32;  // wavefronts of either kind, and tiles of the state's rows
  const int side = bl.prompt ? 0 : 1;
  const int lane = threadIdx.x & 63;
  const int hf = lane >> 5, l32 = lane & 31, q4 = lane >> 4, l16 = lane & 15;
  const float lg = p.b.log2_decay[kvh];
  const int g = p.b.group;
  const int64_t stride_q = (int64_t)p.b.heads_kv * g * D, stride_k = (int64_t)p.b.heads_kv * D;
  const int64_t off_q = bl.row0 * stride_q + (int64_t)kvh * g * D, off_k = bl.row0 * stride_k + (int64_t)kvh * D;
  const uint16_t *const qp = p.q[side] + off_q, *const gp = p.dout[side] + off_q;
  const uint16_t *const kp = p.k[side] + off_k, *const vp = p.v[side] + off_k;
  uint16_t* const out = (OF_K ? p.dk[side] : p.dv[side]) + off_k;

  typedef TileStage<D, 2 * NW> Stage;
  Stage sq, sg, sk, sv;
  const uint32_t src_q = Stage::source(stride_q), src_k = Stage::source(stride_k);
  const int dst = Stage::target();
  const int chunks = (bl.len + C - 1) / C;
  auto rows_of = [&](int c) { return min(C, bl.len - c * C); };
  // (Nothing is fetched behind the last head, by a range of no rows: under a branch the registers of both ways would be
  // copied, and the copies wait for the loads.)
  int fetched = 0, head = 0;  // chunk and head of the next fetch
  auto fetch_q = [&]() {
    const int c = chunks - 1 - fetched, n = fetched < chunks ? rows_of(c) : 0;
    sq.fetch(qp + c * C * stride_q + head * D, src_q, n, stride_q);
    sg.fetch(gp + c * C * stride_q + head * D, src_q, n, stride_q);
    const int next = head + 1 == g;
    head = __builtin_amdgcn_readfirstlane(next ? 0 : head + 1);
    fetched = __builtin_amdgcn_readfirstlane(fetched + next);
  };
  auto fetch_k = [&](int ci) {
    const int c = chunks - 1 - ci, n = ci < chunks ? rows_of(c) : 0;
    sk.fetch(kp + c * C * stride_k, src_k, n, stride_k);
    sv.fetch(vp + c * C * stride_k, src_k, n, stride_k);
  };
  auto put_q = [&]() {
    sq.put(sh.qt, dst);
    sg.put(sh.gt, dst);
    fetch_q();
  };
  fetch_k(0);
  fetch_q();

  const int c4 = 16 * ((lane >> 4) & 1);
  const int ybase = column32_base<D>(c4 + 4 * (((lane & 1) << 1) | ((lane >> 1) & 1)), lane);
  const int zbase = column32_base<D>(32 * wave + c4 + 4 * (lane & 3), lane);
  const int rbase = 2 * loff<D>(l32, 8 * hf), rbase16 = 2 * loff<D>(l16, 8 * q4);
  const int pbase = 2 * poff(l32, hf);
  const int g4 = (l32 >> 2) & 3;
  const int srow = 32 * wave + (l32 & 19) + 4 * (((g4 & 1) << 1) | (g4 >> 1));
  const int sbase = 2 * loff<D>(srow, 8 * hf);
  set_pair_decays<4 * D>(sh.decays, lg);
  clear<4 * D>(&sh.pt, sizeof(sh.pt));

  f32x16 s[NW];  // dv: the state that reaches the chunk
  auto put_state = [&]() {
    const int sb = here(sbase);
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      float f[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = s[ks >> 1][8 * (ks & 1) + e];
      bf16x8 hi, lo;
      split2(f, hi, lo);
      *reinterpret_cast<bf16x8*>(reinterpret_cast<char*>(sh.st[0]) + (sb ^ (32 * ks))) = hi;
      *reinterpret_cast<bf16x8*>(reinterpret_cast<char*>(sh.st[1]) + (sb ^ (32 * ks))) = lo;
    }
  };
  if constexpr (!OF_K) {
    const float* const in = p.states_rev + ((int64_t)block * p.b.heads_kv + kvh) * D * D;
#pragma unroll
    for (int t = 0; t < NW; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[t][i] = in[state32_row(t, i, hf) * D + 32 * wave + l32];
    put_state();
  }

  bf16x8 xr[4][D / 32];  // dk: x of the chunk's tiles of P, the same for all heads
  // P^T of two rows of 16 x 16 tiles (y) against those of x before them and at their own place
  auto p_rows = [&](auto r0, auto r1, int which) {
    constexpr int R0 = decltype(r0)::value, R1 = decltype(r1)::value;
    static_assert(R0 > R1, "the longer row first");
    const __bf16* const yt = which ? sh.gt : sh.qt;
    const int rb = here(rbase16);
    f32x4 a[R0 + R1 + 2];
#pragma unroll
    for (int t = 0; t < R0 + R1 + 2; ++t) a[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks) {
      const int at = rb ^ (64 * ks);
      const bf16x8 y0 = read8(yt + R0 * 16 * D, at), y1 = read8(yt + R1 * 16 * D, at);
#pragma unroll
      for (int t = 0; t <= R0; ++t) {
        a[t] = mfma16(y0, xr[t][ks], a[t]);
        if (t <= R1) a[R0 + 1 + t] = mfma16(y1, xr[t][ks], a[R0 + 1 + t]);
      }
    }
    const float* const pw = sh.decays.pair + 32 + 4 * q4 - l16;
    float w[R0 + 1][4];
#pragma unroll
    for (int t = 0; t <= R0; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) w[t][e] = pw[16 * t + e];
#pragma unroll
    for (int t = 0; t < R0 + R1 + 2; ++t) {
      const int ty = t <= R0 ? R0 : R1, tx = t <= R0 ? t : t - R0 - 1;
      put_p(sh.pt[which], tx, ty, a[t], w[ty - tx], q4, l16);
    }
  };

  put_q();
  f32x16 acc[2];  // out^T [column, row]
  // Two barriers a head, the same for both kinds of wavefronts: behind the first its tiles and S are in LDS, behind the
  // second P is, and tiles and S have been read.
  int row_n = -1;
  for (int ci = 0; ci < chunks; ++ci) {
    const int c = chunks - 1 - ci, n = rows_of(c);
    const bool more = ci + 1 < chunks;
    sk.put(sh.kt, dst);
    sv.put(sh.vt, dst);
    if (more) fetch_k(ci + 1);
    if (n != row_n) set_row_decays<true>(sh.decays, lg, n), row_n = n;
    for (int h = 0; h < g; ++h) {
      __syncthreads();
      if (h == 0) {
#pragma unroll
        for (int tx = 0; tx < 2; ++tx)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[tx][i] = 0.f;
        const int xb = here(rbase), sb = here(OF_K ? zbase : sbase);
        const __bf16* const xt = OF_K ? sh.vt : sh.kt;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          bf16x8 hi, lo;
          if constexpr (OF_K) hi = read_columns32<D>(sh.st[0], sb, 0, ks), lo = read_columns32<D>(sh.st[1], sb, 0, ks);
          else hi = read8(sh.st[0], sb ^ (32 * ks)), lo = read8(sh.st[1], sb ^ (32 * ks));
          const bf16x8 x0 = read8(xt, xb ^ (32 * ks)), x1 = read8(xt + 32 * D, xb ^ (32 * ks));
          acc[0] = mfma32(hi, x0, acc[0]);
          acc[1] = mfma32(hi, x1, acc[1]);
          acc[0] = mfma32(lo, x0, acc[0]);
          acc[1] = mfma32(lo, x1, acc[1]);
        }
#pragma unroll
        for (int tx = 0; tx < 2; ++tx) {
          const float lead = exp2f(lg * (float)max(n - 32 * tx - l32, 0));
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[tx][i] *= lead;
        }
      }
      bf16x8 zf[4];
#pragma unroll
      for (int m = 0; m < 4; ++m) zf[m] = read_columns32<D>(OF_K ? sh.qt : sh.gt, zbase, 0, m);
      if constexpr (OF_K) {
        if (h == 0) {
          const __bf16* const xt = wave & 1 ? sh.vt : sh.kt;
          const int rb = here(rbase16);
#pragma unroll
          for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int ks = 0; ks < D / 32; ++ks) xr[t][ks] = read8(xt + t * 16 * D, rb ^ (64 * ks));
        }
        if (NW == 2 || wave < 2) p_rows(Int<3>{}, Int<0>{}, wave & 1);
        if (NW == 2 || wave >= 2) p_rows(Int<2>{}, Int<1>{}, wave & 1);
      } else {
        if (h == 0) {
          const float fade = exp2f(lg * (float)n);
#pragma unroll
          for (int t = 0; t < NW; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[t][i] *= fade;
        }
        const int yb = here(ybase);
        const float* const w = sh.decays.row + 4 * hf;
        // (operands of the next 16 rows are read, and their z weighed, beside the products of these)
        bf16x8 a[2][NW], hi[2], lo[2];
        auto operands = [&](int m) {
#pragma unroll
          for (int t = 0; t < NW; ++t) a[m & 1][t] = read_columns32<D>(sh.qt, yb, 64 * t, m);
        };
        auto weigh = [&](int m) {
          const f32x4 w0 = *reinterpret_cast<const f32x4*>(w + 16 * m);
          const f32x4 w1 = *reinterpret_cast<const f32x4*>(w + 16 * m + 8);
          float f[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) f[e] = (float)zf[m][e] * (e < 4 ? w0[e] : w1[e - 4]);
          split2(f, hi[m & 1], lo[m & 1]);
        };
        operands(0);
        weigh(0);
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          if (m < 3) operands(m + 1);
          __builtin_amdgcn_sched_barrier(0);
          if (m < 3) weigh(m + 1);
#pragma unroll
          for (int t = 0; t < NW; ++t) s[t] = mfma32(a[m & 1][t], hi[m & 1], s[t]);
#pragma unroll
          for (int t = 0; t < NW; ++t) s[t] = mfma32(a[m & 1][t], lo[m & 1], s[t]);
        }
      }
      __syncthreads();
      put_q();
      const int pb = here(pbase);
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
          for (int tx = 0; tx < 2; ++tx) {
            const int ty = m >> 1;
            if (ty < tx) continue;  // masked
            acc[tx] = mfma32(zf[m], read8(sh.pt[OF_K][k][ty == tx ? 2 * tx : 1], pb ^ (32 * (m & 1))), acc[tx]);
          }
    }
    if constexpr (!OF_K)
      if (more) put_state();
    store_rows<D>(out + c * C * stride_k + 32 * wave, acc, p.scale, n, stride_k, l32, hf);
  }
}

template <int D>
__global__ __launch_bounds__(4 * D, 2) void lin_dkv_kernel(LinGradParams p) {
  __shared__ DkvShared<D> sh;
  const int block = blockIdx.x / p.b.heads_kv, kvh = blockIdx.x - block * p.b.heads_kv;
  const Block bl = find_block(p.b, block);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (wave < D / 32) lin_dkv<D, false>(sh, p, bl, block, kvh, wave);
  else lin_dkv<D, true>(sh, p, bl, block, kvh, wave - D / 32);
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

hipError_t launch_lin_dq(const LinGradParams& p, int head_dim, hipStream_t stream) {
  const dim3 grid(p.b.num_blocks * p.b.heads_kv);
  if (head_dim == 128) lin_dq_kernel<128><<<grid, 256, 0, stream>>>(p);
  else lin_dq_kernel<64><<<grid, 128, 0, stream>>>(p);
  return hipGetLastError();
}

hipError_t launch_lin_dkv(const LinGradParams& p, int head_dim, hipStream_t stream) {
  const dim3 grid(p.b.num_blocks * p.b.heads_kv);
  if (head_dim == 128) lin_dkv_kernel<128><<<grid, 512, 0, stream>>>(p);
  else lin_dkv_kernel<64><<<grid, 256, 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace augtree
