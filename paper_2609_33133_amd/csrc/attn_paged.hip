// Attention of new tokens over a paged KV cache for gfx950.
//
// One workgroup = 4 wavefronts = one item of the plan (paged.h) for one KV head:
// 128 (row, head) pairs, 32 per wavefront, against a range of 64-key blocks of
// segment A (a parent's tokens, every key visible) and segment B (the sequence's
// own, causal). The step of a block is FwdCore's (fwd_core.h), which the
// forward over packed rows runs too; here a block's rows are found through the
// page table, at most 64 of whose entries a wavefront holds at a time, one per
// lane. A block's copies go page by page where pages are shorter than it, and
// rows behind a segment's last token are zeros by the copies' range check, so
// what stands there is never read. Bound by LDS bandwidth and the matrix cores
// together: two chunks of 7777 tokens together, over 7.7k and 23k tokens (32 / 8
// heads, d = 128), in 1.60 to 1.68 ms, 1.11 to 1.17 PFLOP/s.
//
// e4m3 caches: tiles stay bytes and every wavefront makes its operands bf16
// (exactly) as it reads them, K by 16-byte reads that serve two MFMAs, V^T by 8-bit
// transpose reads. The scales of K and V multiply the softmax scale and the result.
// The four wavefronts convert the same tile four times over, but LDS bandwidth is
// what a step is short of: in clocks of 128 bytes a step of a workgroup takes 1280
// in bf16, 640 this way, and 1536 with tiles that the wavefront which fetched them
// widens in LDS. 16384 tokens 1975 us (bf16 1915, widened in LDS 2250, there a step
// ahead beside the second product 2270, V alone from bytes 2155).
#include <type_traits>

#include "common.h"
#include "fwd_core.h"
#include "paged.h"

namespace augtree {

namespace {

constexpr int BN = kFwdBlockN;
static_assert(BN == kPagedBlock && kTilePairs == kPairsPerWorkgroup, "the plan's items are cut to the kernel's tiles");

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Eight e4m3 values as bf16, exactly.
__device__ __forceinline__ bf16x8 widen8(int lo, int hi) {
  bf16x8 y;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(k ? hi : lo, 1.f, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(k ? hi : lo, 1.f, true);
    y[4 * k] = a[0];
    y[4 * k + 1] = a[1];
    y[4 * k + 2] = b[0];
    y[4 * k + 3] = b[1];
  }
  return y;
}

// Swizzle of 16-byte chunks in a tile of byte rows.
template <int RB>
__device__ __forceinline__ int swz8(int row) {
  return RB == 128 ? (row >> 1) & 7 : (row >> 2) & 3;
}
// The 8-bit transpose read of V^T from such a tile (inside a 16-lane group, lane j addresses 8 bytes of row j / 2 and
// receives one column of the 8 rows): this lane's offset for columns 32 db .. + 31, keys in the order of the accumulators
template <int RB>
__device__ __forceinline__ int tr8_offset(int lane, int db) {
  const int grp = lane >> 4, j = lane & 15, r8 = j >> 1, row = 4 * (grp >> 1) + (r8 & 3) + 8 * (r8 >> 2);
  return row * RB + (((2 * db + (grp & 1)) ^ swz8<RB>(row)) << 4) + 8 * (j & 1);
}
// The first of the 8 columns that half-wave hf holds of step ks of a product with byte rows: 16 bytes of a row serve two
// steps, so that they come by one read.
__device__ __forceinline__ int byte_column(int ks, int hf) { return ks / 2 * 32 + hf * 16 + ks % 2 * 8; }
__device__ __forceinline__ bf16x8 read_tr8(const char* at) {
  typedef int v2i __attribute__((ext_vector_type(2)));
  const v2i x = __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) v2i*)(at));
  return widen8(x[0], x[1]);
}

// s_waitcnt vmcnt(N): all but the last N vector-memory accesses of this wavefront have completed
template <int N>
__device__ __forceinline__ void wait_vmem_but() {
  __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14));
}
// what this wavefront read from LDS has arrived: a copy may overwrite it
__device__ __forceinline__ void wait_lds() {
  wave_lds_fence();
  __builtin_amdgcn_s_waitcnt(0xC07F);
  wave_lds_fence();
}
// Scheduling of N MFMAs that take operands from bytes: a read for every PER of them, DEPTH reads ahead, and the four
// conversions of each.
template <int N, int PER, int DEPTH>
__device__ __forceinline__ void pace_bytes() {
  __builtin_amdgcn_sched_group_barrier(0x100, DEPTH, 0);
  __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    if (i % PER == 0 && i / PER < N / PER - DEPTH) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);
  }
}

// Copies of 64-key blocks of one KV head from a cache into LDS, by four
// wavefronts. BIG: a page holds a block or more; else a quarter of one or more.
//
// Where a block (a quarter) lies is computed lane by lane, for a window of 64 of
// them at a time: its byte offset in either cache and its valid bytes. A copy
// then costs three lane reads and an addition on the scalar unit, which eight
// wavefronts share. (With the offsets formed on the scalar unit, block by block
// and for both page sizes, a step of a wavefront had 493 scalar instructions
// where the packed forward has 127, and a chunk of 7777 tokens took 2150 us for
// 1856.)
template <int D, bool E4M3, bool BIG>
struct PageCopy {
  static constexpr int ROWB = E4M3 ? D : 2 * D;    // bytes of a row
  static constexpr int RPI = 1024 / ROWB;          // rows of one copy instruction
  static constexpr int PER_WAVE = BN / RPI / 4;    // instructions of a block and wavefront
  static constexpr int EPB = BIG ? 1 : 4;          // entries of a block
  const PagedFwdParams& p;
  const PagedItem& it;
  int nA, wave, lane, head_off;
  int voff[BIG ? PER_WAVE : 1];  // this lane's byte offset from the entry's first row
  int win;                       // first block of the window
  int k_lo, k_hi, v_lo, v_hi;    // this lane's entry: its offsets
  int bytes;                     // and its valid bytes

  __device__ __forceinline__ PageCopy(const PagedFwdParams& p_, const PagedItem& it_, int nA_, int kvh, int wave_, int lane_)
      : p(p_), it(it_), nA(nA_), wave(wave_), lane(lane_), head_off(kvh * (p_.s.page * ROWB)) {
    constexpr int CH = ROWB / 16;
#pragma unroll
    for (int k = 0; k < (BIG ? PER_WAVE : 1); ++k) {
      const int r = (wave + 4 * k) * RPI + lane / CH;
      // straight into the swizzled tile (bf16: TileCopy's)
      voff[k] = (BIG ? r : r & 15) * ROWB + (((lane % CH) ^ (E4M3 ? swz8<ROWB>(r) : swz<D>(r))) << 4);
    }
    window(it.blk0);
  }

  __device__ __forceinline__ void window(int blk0) {
    win = blk0;
    const int blk = blk0 + lane / EPB, shift = __builtin_ctz(p.s.page);
    const bool isB = blk >= nA;
    const int key = (isB ? blk - nA : blk) * BN + (lane % EPB) * (BN / EPB), len = isB ? it.b_len : it.a_len;
    const int seq = max(isB ? it.b_seq : it.a_seq, 0);
    const int left = len - key;  // keys from the entry's first one on (none behind the item)
    int id = -1;
    if (left > 0) id = p.table[(int64_t)seq * p.s.max_pages + (key >> shift)];
    const bool ok = (uint32_t)id < (uint32_t)p.s.num_pages;
    bytes = ok ? min(BN / EPB, left) * ROWB : 0;
    const int64_t at = head_off + (key & (p.s.page - 1)) * ROWB;
    const int64_t k = ok ? id * p.k_stride + at : 0, v = ok ? id * p.v_stride + at : 0;
    k_lo = (int)k;
    k_hi = (int)(k >> 32);
    v_lo = (int)v;
    v_hi = (int)(v >> 32);
  }

  // the window holds block blk and the one before it
  __device__ __forceinline__ void ensure(int blk) {
    if (blk - win >= 64 / EPB) window(blk - 1);
  }

  __device__ __forceinline__ void copy(const void* cache, int lo, int hi, int blk, void* tile) const {
#if defined(__HIP_DEVICE_COMPILE__)
    char* const lds = static_cast<char*>(tile);
    __amdgpu_buffer_rsrc_t rsrc;
#pragma unroll
    for (int k = 0; k < PER_WAVE; ++k) {
      if (!BIG || k == 0) {
        const int e = (blk - win) * EPB + (BIG ? 0 : (wave + 4 * k) * RPI / 16);
        const uint32_t l = __builtin_amdgcn_readlane(lo, e), h = __builtin_amdgcn_readlane(hi, e);
        const char* const base = static_cast<const char*>(cache) + (int64_t)((uint64_t)h << 32 | l);
        rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, __builtin_amdgcn_readlane(bytes, e), 0x00020000);
      }
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)(lds + (wave + 4 * k) * 1024), 16,
                                               voff[BIG ? k : 0], 0, 0, 0);
    }
#endif
  }
  __device__ __forceinline__ void copy_k(int blk, void* tile) const { copy(p.k_cache, k_lo, k_hi, blk, tile); }
  __device__ __forceinline__ void copy_v(int blk, void* tile) const { copy(p.v_cache, v_lo, v_hi, blk, tile); }
};

// ---------------------------------------------------------------------------- items of few pairs

// An item of at most 32 pairs (single tokens: a few heads of one row, or of the
// rows of a run) is bound by the reading of its keys, so its wavefronts share
// them instead of the pairs: each takes every fourth block of KEYS keys, 8 KB of
// K and of V, for all pairs, on its own and without barriers. K of its next
// block is fetched as soon as the scores of this one are formed, V as soon as
// they are applied, so that one of the two is always on its way: with two
// workgroups on a CU at least 64 KB. The page ids of the block after the next
// one are read a step ahead. The wavefronts' states are joined in LDS at the
// end.
//
// Tiles: per wavefront 4 KB in each of the kernel's four arrays (in arrays of
// their own K and V can be told apart by the compiler, which would otherwise
// wait for the one on its way before it reads the other): bf16, d = 128: 64
// columns each; else half of the keys each. bf16 tiles are [32][64], swizzled
// as such. e4m3 tiles stay bytes: their operands become bf16 (exactly) as they
// are read, V^T with the 8-bit transpose read (inside a 16-lane group, lane j
// addresses 8 bytes of row j / 2 and receives one column of the 8 rows).
template <int D, bool E4M3>
struct FewTiles {
  static constexpr int ROWB = E4M3 ? D : 2 * D;        // bytes of a row in the cache
  static constexpr int KEYS = 8192 / ROWB;             // keys of a block
  static constexpr bool BY_COLS = !E4M3 && D == 128;   // the halves of a tile: columns, or keys
  static constexpr int RB = BY_COLS ? ROWB / 2 : ROWB; // bytes of a row of a half
  static constexpr int RPI = 1024 / RB;                // rows of one copy instruction
  static constexpr int GROUPS = KEYS / RPI;            // groups of keys that are looked up on their own
  static constexpr int SUB = KEYS / 32;                // 32-key tiles
  static_assert(GROUPS <= 8 && RPI <= 16, "a copy instruction stays inside a page");

  int voff[2];     // this lane's byte offset from an instruction's first row, even and odd instructions
  int koff[8];     // K operand of 16 columns, e4m3: of 32 (bytes inside a half)
  int voff_tr[4][2];  // V^T operand of 32 columns

  __device__ __forceinline__ void init(int lane) {
    const int l32 = lane & 31, hf = lane >> 5;
    constexpr int CH = RB / 16;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int r = lane / CH, row = k * RPI + r;
      voff[k] = r * ROWB + (((lane % CH) ^ (E4M3 ? swz8<RB>(row) : swz<64>(row))) << 4);
    }
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
      if constexpr (!E4M3) koff[ks] = ks < 4 ? 2 * toff<64>(l32, ks * 16 + hf * 8) : 0;
      else koff[ks] = ks < D / 32 ? l32 * RB + (((2 * ks + hf) ^ swz8<RB>(l32)) << 4) : 0;
    }
    if constexpr (!E4M3) {
      TrOffsets<64> t;
      t.init(0, lane);
#pragma unroll
      for (int db = 0; db < 2; ++db) voff_tr[db][0] = t.o[db][0], voff_tr[db][1] = t.o[db][1];
    } else {
#pragma unroll
      for (int db = 0; db < D / 32; ++db) voff_tr[db][0] = tr8_offset<RB>(lane, db);
    }
  }

  // K rows 32 t + l32, columns of steps ks and ks + 1 (ks is even); h0, h1: the tile's halves
  __device__ __forceinline__ void k_operands(const char* h0, const char* h1, int t, int ks, bf16x8& x0, bf16x8& x1) const {
    if constexpr (!E4M3) {
      const bool second = BY_COLS ? ks >= 4 : t >= 1;
      const char* const at = second ? h1 : h0;
      x0 = *reinterpret_cast<const bf16x8*>(at + koff[BY_COLS ? ks % 4 : ks]);
      x1 = *reinterpret_cast<const bf16x8*>(at + koff[BY_COLS ? ks % 4 + 1 : ks + 1]);
    } else {
      const int row0 = RB == 128 ? 0 : (t & 1) * 32;
      const raw16 x = *reinterpret_cast<const raw16*>(((RB == 128 ? t : t >> 1) ? h1 : h0) + row0 * RB + koff[ks / 2]);
      x0 = widen8(x[0], x[1]);
      x1 = widen8(x[2], x[3]);
    }
  }
  // V^T: columns 32 db + l32, keys 32 t + 16 m + the ones that accumulator registers 8 m .. 8 m + 7 hold
  __device__ __forceinline__ bf16x8 v_operand(const char* h0, const char* h1, int t, int m, int db) const {
    if constexpr (!E4M3) {
      const bool second = BY_COLS ? db >= 2 : t >= 1;
      const char* const at = (second ? h1 : h0) + m * 16 * 128;
      const int k = BY_COLS ? db % 2 : db;
      const s16x4 a = lds_tr16(reinterpret_cast<const __bf16*>(at + voff_tr[k][0]));
      const s16x4 b = lds_tr16(reinterpret_cast<const __bf16*>(at + voff_tr[k][1]));
      bf16x8 r;
      __builtin_memcpy(&r, &a, 8);
      __builtin_memcpy(reinterpret_cast<char*>(&r) + 8, &b, 8);
      return r;
    } else {
      const int row0 = (RB == 128 ? 0 : (t & 1) * 32) + 16 * m;
      return read_tr8(((RB == 128 ? t : t >> 1) ? h1 : h0) + row0 * RB + voff_tr[db][0]);
    }
  }

  // copies keys key .. key + KEYS - 1 (those from `lim` on: zeros); ids: lane g has the page of key + g * RPI, and works
  // out where these keys lie (on the scalar unit, which eight wavefronts share: five tokens of 33 sequences, pages of 16,
  // 15.0 us with their merge, this way 13.5)
  __device__ __forceinline__ void copy(char* h0, char* h1, const char* cache, int64_t stride, int head_off, int ids, int key,
                                       int lim, int page, int num_pages, int lane) const {
#if defined(__HIP_DEVICE_COMPILE__)
    const int first = key + (lane & 7) * RPI;
    const bool ok = (uint32_t)ids < (uint32_t)num_pages;
    const int64_t off = (ok ? ids : 0) * stride + (head_off + (first & (page - 1)) * ROWB);
    const int bytes = ok ? max(0, min(RPI, lim - first)) * ROWB : 0;
#pragma unroll
    for (int gr = 0; gr < GROUPS; ++gr) {
      const uint32_t lo = __builtin_amdgcn_readlane((int)off, gr), hi = __builtin_amdgcn_readlane((int)(off >> 32), gr);
      const char* const base = cache + (int64_t)((uint64_t)hi << 32 | lo);
      const __amdgpu_buffer_rsrc_t rsrc =
          __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, __builtin_amdgcn_readlane(bytes, gr), 0x00020000);
      if constexpr (BY_COLS) {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)(h0 + gr * 1024), 16,
                                                 voff[gr & 1], 0, 0, 0);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)(h1 + gr * 1024), 16,
                                                 voff[gr & 1] + RB, 0, 0, 0);
      } else {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            rsrc, (__attribute__((address_space(3))) void*)((gr < GROUPS / 2 ? h0 : h1) + (gr % (GROUPS / 2)) * 1024), 16,
            voff[gr & 1], 0, 0, 0);
      }
    }
#endif
  }
};

template <int D, bool E4M3>
__device__ __forceinline__ void attend_few(const PagedFwdParams& p, const PagedItem& it, int kvh, __bf16* k0, __bf16* k1,
                                           __bf16* v0, __bf16* v1, float (*stat)[4][kSlotPairs]) {
  typedef FewTiles<D, E4M3> Tiles;
  constexpr int KEYS = Tiles::KEYS, SUB = Tiles::SUB;
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hf = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = p.group, pairs = it.rows * g, shift = __builtin_ctz(p.s.page);
  const int64_t qbase = ((int64_t)it.row0 * p.s.hq + kvh * g) * D;
  // this wavefront's 4 KB of each array
  char* const ka = reinterpret_cast<char*>(k0) + wave * 4096;
  char* const kb = reinterpret_cast<char*>(k1) + wave * 4096;
  char* const va = reinterpret_cast<char*>(v0) + wave * 4096;
  char* const vb = reinterpret_cast<char*>(v1) + wave * 4096;
  // keys of the item: a0 .. a1 - 1 of segment A, b0 .. b1 - 1 of segment B
  const int nA64 = (it.a_len + BN - 1) / BN;
  const int a0 = min(it.blk0, nA64) * BN, a1 = min(min(it.blk1, nA64) * BN, it.a_len);
  const int b0 = max(it.blk0 - nA64, 0) * BN, b1 = min(max(it.blk1 - nA64, 0) * BN, it.b_len);
  const int nA = max(0, a1 - a0 + KEYS - 1) / KEYS, n = nA + max(0, b1 - b0 + KEYS - 1) / KEYS;
  const int32_t* const row_a = p.table + (int64_t)max(it.a_seq, 0) * p.s.max_pages;
  const int32_t* const row_b = p.table + (int64_t)max(it.b_seq, 0) * p.s.max_pages;
  auto first_key = [&](int j) { return j < nA ? a0 + j * KEYS : b0 + (j - nA) * KEYS; };
  auto last_key = [&](int j) { return j < nA ? a1 : b1; };
  // (behind the last block: entries that nobody uses, so that the count of loads on their way stays the same)
  auto page_ids = [&](int j) {
    const int k = first_key(min(j, n - 1)) + (lane & 7) * Tiles::RPI;
    return (j < nA ? row_a : row_b)[min(k >> shift, p.s.max_pages - 1)];
  };
  const char* const kc = static_cast<const char*>(p.k_cache);
  const char* const vc = static_cast<const char*>(p.v_cache);
  const int head_off = kvh * (p.s.page * Tiles::ROWB);

  Tiles tiles;
  tiles.init(lane);
  int j = wave;
  float c = p.scale_log2;  // (e4m3: the scale follows)
  float m_run = -INFINITY, l_run = 0.f;
  f32x16 oacc[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) oacc[db][i] = 0.f;
  const int pair = min(l32, pairs - 1), qrow = fast_div(pair, g, p.group_magic);
  bf16x8 qreg[D / 16];
  int ids_next = 0;
  if (j < n) {
    const int ids = page_ids(j);
    ids_next = page_ids(j + 4);
    const uint16_t* const q = p.q + qbase + pair_offset<D>(qrow, pair - qrow * g, p.s.hq);
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) qreg[ks] = as_bf16x8(ldg16(q + (E4M3 ? byte_column(ks, hf) : ks * 16 + hf * 8)));
    float k_scale = 1.f;
    if constexpr (E4M3) k_scale = p.k_scale[kvh];
    tiles.copy(ka, kb, kc, p.k_stride, head_off, ids, first_key(j), last_key(j), p.s.page, p.s.num_pages, lane);
    tiles.copy(va, vb, vc, p.v_stride, head_off, ids, first_key(j), last_key(j), p.s.page, p.s.num_pages, lane);
    wait_vmem_but<16>();  // all but the copies (else the compiler would wait for Q and the scale in every step)
    if constexpr (E4M3) {
      asm volatile("" : "+v"(k_scale));
      c *= k_scale;
    }
  }
  // One block; MORE: another one of this wavefront follows, whose copies go out.
  auto step = [&](auto more) {
    constexpr bool MORE = decltype(more)::value;
    const int key = first_key(j), lim = last_key(j);
    const bool isB = j >= nA;
    wait_vmem_but<8>();  // all but V of this block
    wave_lds_fence();
    f32x16 s[SUB];
#pragma unroll
    for (int t = 0; t < SUB; ++t) {
      f32x16 s1;  // two chains of MFMAs
#pragma unroll
      for (int i = 0; i < 16; ++i) s[t][i] = s1[i] = 0.f;
#pragma unroll
      for (int ks = 0; ks < D / 16; ks += 2) {
        bf16x8 x0, x1;
        tiles.k_operands(ka, kb, t, ks, x0, x1);
        s[t] = mfma32(x0, qreg[ks], s[t]);
        s1 = mfma32(x1, qreg[ks + 1], s1);
      }
      if constexpr (!E4M3) pace_lds_mfma<D / 16, 1, 4>();
      s[t] += s1;
      __builtin_amdgcn_sched_barrier(0);  // (the operands of one tile at a time: two workgroups a CU)
    }
    wait_lds();
    const int ids_now = ids_next;
    if constexpr (MORE) {
      ids_next = page_ids(j + 8);
      tiles.copy(ka, kb, kc, p.k_stride, head_off, ids_now, first_key(j + 4), last_key(j + 4), p.s.page, p.s.num_pages, lane);
    }
    if (key + KEYS > lim || (isB && key + KEYS - 1 > it.b_pos)) {
      const int seen = min(lim - 1, isB ? it.b_pos + qrow : lim - 1) - key;  // last visible key of the block
#pragma unroll
      for (int t = 0; t < SUB; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (32 * t + acc_row(i, hf) > seen) s[t][i] = -INFINITY;
    }
    float mx = s[0][0];
#pragma unroll
    for (int t = 0; t < SUB; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[t][i]);
    mx = pair_max<MaxWritten>(mx);
    if (__any(mx * c > m_run * c + RESCALE_MARGIN_LOG2)) {
      const float mnew = MaxWritten::of(m_run, mx);
      const float alpha = (mnew == -INFINITY) ? 1.f : __builtin_amdgcn_exp2f((m_run - mnew) * c);
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) oacc[db][i] *= alpha;
      m_run = mnew;
    }
    const float ms = (m_run == -INFINITY) ? 0.f : m_run * c;
    bf16x8 pb[SUB][2];
#pragma unroll
    for (int t = 0; t < SUB; ++t) {
      float l4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[t][i] = __builtin_amdgcn_exp2f(s[t][i] * c - ms);
        l4[i & 3] += s[t][i];
      }
      l_run += (l4[0] + l4[1]) + (l4[2] + l4[3]);
      pb[t][0] = to_bf16x8(s[t], 0);
      pb[t][1] = to_bf16x8(s[t], 8);
    }
    __builtin_amdgcn_sched_barrier(0);  // (the softmax runs while V is on its way)
    if constexpr (MORE) wait_vmem_but<9>();  // all but K of the next block and the page ids after it
    else wait_vmem();
    wave_lds_fence();
#pragma unroll
    for (int t = 0; t < SUB; ++t) {
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int db = 0; db < D / 32; ++db) oacc[db] = mfma32(tiles.v_operand(va, vb, t, m, db), pb[t][m], oacc[db]);
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (MORE) {
      wait_lds();
      tiles.copy(va, vb, vc, p.v_stride, head_off, ids_now, first_key(j + 4), last_key(j + 4), p.s.page, p.s.num_pages, lane);
    }
  };
  for (; j + 4 < n; j += 4) step(std::true_type());
  if (j < n) step(std::false_type());

  // the four states of each pair, joined: wavefront w writes its outputs to array w
  c = p.scale_log2;  // (a wavefront without blocks joins too)
  if constexpr (E4M3) c *= p.k_scale[kvh];
  const float l_tot = pair_sum(l_run);
  __syncthreads();
  char* const mine = reinterpret_cast<char*>(wave == 0 ? k0 : wave == 1 ? k1 : wave == 2 ? v0 : v1);
  constexpr int CPR = D / 4;  // 16-byte chunks of a pair's output
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int g4 = 0; g4 < 4; ++g4) {
      const f32x4 v = {oacc[db][g4 * 4], oacc[db][g4 * 4 + 1], oacc[db][g4 * 4 + 2], oacc[db][g4 * 4 + 3]};
      const int ch = db * 8 + g4 * 2 + hf;
      *reinterpret_cast<f32x4*>(mine + l32 * (D * 4) + ((ch ^ (l32 & (CPR - 1))) << 4)) = v;
    }
  if (hf == 0) {
    stat[0][wave][l32] = l_tot > 0.f ? m_run : -INFINITY;
    stat[1][wave][l32] = l_tot;
  }
  __syncthreads();
  const int ch = lane % CPR;
  float vscale = 1.f;
  if constexpr (E4M3) vscale = p.v_scale[kvh];
  for (int x = wave * (64 / CPR) + lane / CPR; x < pairs; x += 4 * (64 / CPR)) {
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) top = fmaxf(top, stat[0][w][x]);
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const char* const o = reinterpret_cast<const char*>(w == 0 ? k0 : w == 1 ? k1 : w == 2 ? v0 : v1);
      const float m = stat[0][w][x], wt = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - top) * c);
      acc += *reinterpret_cast<const f32x4*>(o + x * (D * 4) + ((ch ^ (x & (CPR - 1))) << 4)) * wt;
      sum += stat[1][w][x] * wt;
    }
    const float inv = sum > 0.f ? vscale / sum : 0.f;
    const float lse = sum > 0.f ? (top * c + __log2f(sum)) * kLn2 : -INFINITY;
    if (it.slot < 0) {
      typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
      bf16x4 y;
#pragma unroll
      for (int k = 0; k < 4; ++k) y[k] = (__bf16)(acc[k] * inv);
      const int r = fast_div(x, g, p.group_magic);
      *reinterpret_cast<bf16x4*>(p.o + qbase + pair_offset<D>(r, x - r * g, p.s.hq) + ch * 4) = y;
      if (p.lse && ch == 0) p.lse[(int64_t)(kvh * g + x - r * g) * p.s.rows + it.row0 + r] = lse;
    } else if (it.slot < p.max_slots) {
      const int64_t at = ((int64_t)it.slot * p.s.hkv + kvh) * kSlotPairs + x;
      *reinterpret_cast<f32x4*>(p.part_o + at * D + ch * 4) = acc * inv;
      if (ch == 0) p.part_lse[at] = lse;
    }
  }
}

template <int D, bool E4M3, bool BIG>
__global__ __launch_bounds__(256, 2) void attn_paged_kernel(PagedFwdParams p) {
  // (16 KB each: tiles of 64 keys, or of items of few pairs)
  __shared__ __bf16 k_buf0[BN * 128], k_buf1[BN * 128], v_buf0[BN * 128], v_buf1[BN * 128];
  __shared__ float stat[2][4][kSlotPairs];
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hf = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);  // uniform: scalar branches below
  const int unit = blockIdx.x;
  const int item = fast_div(unit, p.s.hkv, p.hkv_magic);
  const int kvh = unit - item * p.s.hkv;
  const int32_t* const plan = p.plan;
  PagedItem it;
  {
    int32_t w[kItemInts];
    const int32_t* const src = plan + p.items_at + (int64_t)item * kItemInts;
#pragma unroll
    for (int k = 0; k < kItemInts; ++k) w[k] = __builtin_amdgcn_readfirstlane(src[k]);
    __builtin_memcpy(&it, w, sizeof(it));
  }
  const bool fits = plan_is_for(plan, p.s);
  if (!fits | (item >= plan[PH_ITEMS])) return;
  if (it.rows * p.group <= kSlotPairs) {
    attend_few<D, E4M3>(p, it, kvh, k_buf0, k_buf1, v_buf0, v_buf1, stat);
    return;
  }
  QTile t;
  t.q_row0 = it.row0;
  t.q_len = it.rows;
  const int sub = it.pair0 / kTilePairs;
  const QRows rows(t, p.group, p.group_magic, sub, wave, l32);
  const int64_t qstride = (int64_t)p.s.hq * D;
  const int64_t qbase = it.row0 * qstride + (int64_t)kvh * p.group * D;

  const int nA = (it.a_len + BN - 1) / BN;
  const int nblk = it.blk1;  // blocks blk0 .. blk1 - 1 of A and then B

  const int b0 = it.blk0;
  FwdCore<D, MaxWritten> core;  // (a chunk of 7777 tokens 1630 us; with the compiler's maxima 1670)
  core.hf = hf;
  if (b0 < nblk) {
    PageCopy<D, E4M3, BIG> cp(p, it, nA, kvh, wave, lane);
    // the first blocks' copies go out before anything else is computed: K(b + 1)
    // and V(b) are resident while block b is processed
    cp.copy_k(b0, k_buf0);
    cp.copy_v(b0, v_buf0);
    if (b0 + 1 < nblk) cp.copy_k(b0 + 1, k_buf1);

    const uint16_t* const q = p.q + qbase + pair_offset<D>(rows.row, rows.head, p.s.hq);
    if constexpr (E4M3) {
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) core.qreg[ks] = as_bf16x8(ldg16(q + byte_column(ks, hf)));
    } else {
      core.load_q(q);
    }
    float scale = p.scale_log2;
    if constexpr (E4M3) scale *= p.k_scale[kvh];
    core.init(scale, l32, lane);

    const int qpos_lo = it.b_pos + rows.wlo;  // causal: the wavefront's first query position
    const int qi = rows.row;
    // a causal block whose keys all follow the wavefront's queries (and every
    // later block) contributes nothing; neither does any block to a wavefront
    // without rows
    const int nlive = !rows.wave_any ? 0 : it.b_len > 0 ? nA + (it.b_pos + rows.whi) / BN + 1 : nA;
    // the block needs a mask; the last visible key in it
    auto first_of = [&](int b) { return (b >= nA ? b - nA : b) * BN; };
    auto masked_in = [&](int b) {
      const int kb0 = first_of(b);
      return (kb0 + BN > (b >= nA ? it.b_len : it.a_len)) || (b >= nA && (kb0 + BN - 1 > qpos_lo));
    };
    auto limit_in = [&](int b) {
      return (b >= nA ? min(it.b_len - 1, it.b_pos + qi) : it.a_len - 1) - first_of(b);
    };

    f32x16 sa0, sa1, sb0, sb1;
    wait_vmem();
    __syncthreads();
    int k8[D / 32], tr8[D / 32];  // e4m3: operands from byte tiles
    if constexpr (E4M3) {
#pragma unroll
      for (int ks = 0; ks < D / 32; ++ks) k8[ks] = l32 * D + (((2 * ks + hf) ^ swz8<D>(l32)) << 4);
#pragma unroll
      for (int db = 0; db < D / 32; ++db) tr8[db] = tr8_offset<D>(lane, db);
    }
    auto scores = [&](const __bf16* kl, f32x16& s0, f32x16& s1) {
      if constexpr (!E4M3) {
        core.s_mfma(kl, s0, s1);
      } else {
        const char* const kb = reinterpret_cast<const char*>(kl);
#pragma unroll
        for (int i = 0; i < 16; ++i) { s0[i] = 0.f; s1[i] = 0.f; }
#pragma unroll
        for (int ks = 0; ks < D / 32; ++ks) {
          const raw16 x = *reinterpret_cast<const raw16*>(kb + k8[ks]), y = *reinterpret_cast<const raw16*>(kb + 32 * D + k8[ks]);
          s0 = mfma32(widen8(x[0], x[1]), core.qreg[2 * ks], s0);
          s1 = mfma32(widen8(y[0], y[1]), core.qreg[2 * ks], s1);
          s0 = mfma32(widen8(x[2], x[3]), core.qreg[2 * ks + 1], s0);
          s1 = mfma32(widen8(y[2], y[3]), core.qreg[2 * ks + 1], s1);
        }
      }
    };
    scores(k_buf0, sa0, sa1);
    if constexpr (!E4M3) pace_lds_mfma<D / 8, 1, FWD_DEPTH>();
    __syncthreads();
    // iteration b loads K(b + 2) over K(b) and V(b + 1) over V(b - 1)
    auto step = [&](int b, f32x16& s0, f32x16& s1, const __bf16* kn, const __bf16* vl, f32x16& n0, f32x16& n1) {
      auto masked = [&] { return masked_in(b); };
      auto limit = [&] { return limit_in(b); };
      if constexpr (!E4M3) {
        core.step(masked, limit, s0, s1, kn, vl, n0, n1);
      } else {
        bf16x8 pb[4];
        core.softmax(masked, limit, s0, s1, [&] { scores(kn, n0, n1); }, pb);
        set_wave_priority<1>();
        const char* const vb = reinterpret_cast<const char*>(vl);
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
#pragma unroll
          for (int db = 0; db < D / 32; ++db)
            core.oacc[db] = mfma32(read_tr8(vb + ks * 16 * D + tr8[db]), pb[ks], core.oacc[db]);
        pace_bytes<D / 8, 1, PV_DEPTH>();
        set_wave_priority<0>();
      }
    };
    for (int b = b0; b < nblk; b += 2) {
      cp.ensure(b + 2);
      if (b + 2 < nblk) cp.copy_k(b + 2, k_buf0);
      if (b + 1 < nblk) cp.copy_v(b + 1, v_buf1);
      if (b < nlive) step(b, sa0, sa1, k_buf1, v_buf0, sb0, sb1);
      wait_vmem();
      __syncthreads();
      if (b + 1 < nblk) {
        cp.ensure(b + 3);
        if (b + 3 < nblk) cp.copy_k(b + 3, k_buf1);
        if (b + 2 < nblk) cp.copy_v(b + 2, v_buf0);
        if (b + 1 < nlive) step(b + 1, sb0, sb1, k_buf0, v_buf1, sa0, sa1);
        wait_vmem();
        __syncthreads();
      }
    }
  } else {  // a part that ends before the tile's last row begins
    core.init(p.scale_log2, l32, lane);
  }

  if (!rows.wave_any) return;
  const float l_tot = pair_sum(core.l_run);
  const float lse = l_tot > 0.f ? (core.m_run * core.c + __log2f(l_tot)) * kLn2 : -INFINITY;
  float inv = l_tot > 0.f ? 1.f / l_tot : 0.f;
  if constexpr (E4M3) inv *= p.v_scale[kvh];
  // (the lane's row again, instead of registers held over the sweep)
  const QRows er(t, p.group, p.group_magic, sub, wave, (int)opaque(l32));
  // through this wavefront's own buffer (nothing is in flight any more)
  char* const buf = reinterpret_cast<char*>(wave == 0 ? k_buf0 : wave == 1 ? k_buf1 : wave == 2 ? v_buf0 : v_buf1);
  if (it.slot < 0) {
    if (p.lse && er.valid && hf == 0)
      p.lse[(int64_t)(kvh * p.group + er.head) * p.s.rows + it.row0 + er.row] = lse;
    store_pairs<D>(buf, core.oacc, inv, reinterpret_cast<__bf16*>(p.o) + qbase, qstride, t, p.group, p.group_magic, sub,
                   wave, lane);
  } else if (it.slot + wave < p.max_slots) {
    const int64_t slot = ((int64_t)(it.slot + wave) * p.s.hkv + kvh) * kSlotPairs;
    if (er.valid && hf == 0) p.part_lse[slot + l32] = lse;
    QTile pt;  // 32 pairs as 32 rows of one head
    pt.q_len = min(kSlotPairs, it.rows * p.group - it.pair0 - wave * kSlotPairs);
    store_pairs<D>(buf, core.oacc, inv, p.part_o + slot * D, (int64_t)D, pt, 1, 0u, 0, 0, lane);
  }
}

template <int D, bool E4M3, bool BIG>
void launch(dim3 grid, const PagedFwdParams& p, hipStream_t stream) {
  attn_paged_kernel<D, E4M3, BIG><<<grid, 256, 0, stream>>>(p);
}

}  // namespace

hipError_t launch_paged_fwd(const PagedFwdParams& p, hipStream_t stream) {
  const dim3 grid((unsigned)((int64_t)p.max_items * p.s.hkv));
  const bool big = p.s.page >= kPagedBlock, e4m3 = p.type == CACHE_E4M3;
  if (p.d == 128) {
    if (big) e4m3 ? launch<128, true, true>(grid, p, stream) : launch<128, false, true>(grid, p, stream);
    else e4m3 ? launch<128, true, false>(grid, p, stream) : launch<128, false, false>(grid, p, stream);
  } else {
    if (big) e4m3 ? launch<64, true, true>(grid, p, stream) : launch<64, false, true>(grid, p, stream);
    else e4m3 ? launch<64, true, false>(grid, p, stream) : launch<64, false, false>(grid, p, stream);
  }
  return hipGetLastError();
}

}  // namespace augtree
