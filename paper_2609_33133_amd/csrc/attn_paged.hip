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
// what stands there is never read.
//
// e4m3 caches: the copies bring the bytes into a staging area, each lane then
// turns its own 16 into bf16 (exactly) and puts them into the tile. The scales
// of K and V multiply the softmax scale and the result.
#include "common.h"
#include "fwd_core.h"
#include "paged.h"

namespace augtree {

namespace {

constexpr int BN = kFwdBlockN;
static_assert(BN == kPagedBlock && kTilePairs == kPairsPerWorkgroup, "the plan's items are cut to the kernel's tiles");

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// A position in a sequence's keys: the next block that is copied.
struct PageCursor {
  const int32_t* row;  // the segment's page table
  int key, len;        // the block's first key; the segment's tokens
  bool isB;
  int win;             // first page of the window of 64 table entries
  int ids;             // this lane's entry of the window
};

// Copies of 64-key blocks of one KV head from a cache into LDS, by four
// wavefronts.
template <int D, bool E4M3>
struct PageCopy {
  static constexpr int ROWB = E4M3 ? D : 2 * D;    // bytes of a row
  static constexpr int RPI = 1024 / ROWB;          // rows of one copy instruction
  static constexpr int PER_WAVE = BN / RPI / 4;    // instructions of a block and wavefront
  const int32_t* table;
  int max_pages, num_pages, shift;
  int b_seq, b_len;
  int wave, lane;
  int voff[PER_WAVE];  // this lane's byte offset from the block's first row

  __device__ __forceinline__ void init(const PagedFwdParams& p, int b_seq_, int b_len_, int wave_, int lane_) {
    table = p.table;
    max_pages = p.s.max_pages;
    num_pages = p.s.num_pages;
    shift = __builtin_ctz(p.s.page);
    b_seq = b_seq_;
    b_len = b_len_;
    wave = wave_;
    lane = lane_;
    constexpr int CH = ROWB / 16;
#pragma unroll
    for (int k = 0; k < PER_WAVE; ++k) {
      const int r = (wave + 4 * k) * RPI + lane / CH;
      // bf16: straight into the swizzled tile (TileCopy); e4m3: as it lies
      voff[k] = r * ROWB + ((E4M3 ? lane % CH : (lane % CH) ^ swz<D>(r)) << 4);
    }
  }

  __device__ __forceinline__ void window(PageCursor& c) const {
    c.win = c.key >> shift;
    c.ids = c.win + lane < max_pages ? c.row[c.win + lane] : -1;
  }

  __device__ __forceinline__ PageCursor at(const PagedItem& it, int nA) const {
    PageCursor c;
    c.isB = it.blk0 >= nA;
    c.row = table + (int64_t)(c.isB ? b_seq : it.a_seq) * max_pages;
    c.key = (c.isB ? it.blk0 - nA : it.blk0) * BN;
    c.len = c.isB ? b_len : it.a_len;
    window(c);
    return c;
  }

  // copies the cursor's block and steps the cursor
  __device__ __forceinline__ void next(PageCursor& c, const char* cache, int64_t stride, int head_off, char* lds) const {
#if defined(__HIP_DEVICE_COMPILE__)
    const int page = 1 << shift;
    if (shift >= 6) {  // one page holds the block
      const int id = __builtin_amdgcn_readlane(c.ids, (c.key >> shift) - c.win);
      const bool ok = (uint32_t)id < (uint32_t)num_pages;
      const char* const base = cache + (ok ? id : 0) * stride + head_off + (c.key & (page - 1)) * ROWB;
      const int n = ok ? min(BN, c.len - c.key) * ROWB : 0;
      const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, n, 0x00020000);
#pragma unroll
      for (int k = 0; k < PER_WAVE; ++k)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            rsrc, (__attribute__((address_space(3))) void*)(lds + (wave + 4 * k) * 1024), 16, voff[k], 0, 0, 0);
    } else {
#pragma unroll
      for (int k = 0; k < PER_WAVE; ++k) {
        const int r0 = (wave + 4 * k) * RPI, key = c.key + r0;  // the instruction's first row
        const int id = __builtin_amdgcn_readlane(c.ids, (key >> shift) - c.win);
        const bool ok = (uint32_t)id < (uint32_t)num_pages;
        // the address that the block's first row would have in this page; only the instruction's rows are read
        const char* const base = cache + (ok ? id : 0) * stride + head_off + ((key & (page - 1)) - r0) * ROWB;
        const int n = ok && c.len > key ? (r0 + min(RPI, c.len - key)) * ROWB : 0;
        const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, n, 0x00020000);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            rsrc, (__attribute__((address_space(3))) void*)(lds + (wave + 4 * k) * 1024), 16, voff[k], 0, 0, 0);
      }
    }
#endif
    c.key += BN;
    if (c.key >= c.len && !c.isB && b_len > 0) {
      c.isB = true;
      c.key = 0;
      c.len = b_len;
      c.row = table + (int64_t)b_seq * max_pages;
      window(c);
    } else if (((c.key + BN - 1) >> shift) - c.win >= 64) {
      window(c);
    }
  }

  // e4m3: this wavefront's staged rows as bf16 into the swizzled tile
  __device__ __forceinline__ void widen(const char* staged, __bf16* tile) const {
    if constexpr (E4M3) {
      constexpr int CH = ROWB / 16;
#pragma unroll
      for (int k = 0; k < PER_WAVE; ++k) {
        const raw16 x = *reinterpret_cast<const raw16*>(staged + (wave + 4 * k) * 1024 + lane * 16);
        const int r = (wave + 4 * k) * RPI + lane / CH, col = (lane % CH) * 16;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          bf16x8 y;
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[2 * h + j], 1.f, false);
            const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[2 * h + j], 1.f, true);
            y[4 * j] = a[0];
            y[4 * j + 1] = a[1];
            y[4 * j + 2] = b[0];
            y[4 * j + 3] = b[1];
          }
          *reinterpret_cast<bf16x8*>(tile + toff<D>(r, col + 8 * h)) = y;
        }
      }
    }
  }
};

template <int D, bool E4M3>
__global__ __launch_bounds__(256, 2) void attn_paged_kernel(PagedFwdParams p) {
  __shared__ __bf16 k_buf0[BN * D], k_buf1[BN * D], v_buf0[BN * D], v_buf1[BN * D];
  // bytes of an e4m3 cache on their way (K, V)
  __shared__ char stage_k[E4M3 ? BN * D : 16], stage_v[E4M3 ? BN * D : 16];
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
  if (item >= plan[PH_ITEMS] || plan[PH_SEQS] != p.s.seqs || plan[PH_ROWS] != p.s.rows || plan[PH_HQ] != p.s.hq ||
      plan[PH_HKV] != p.s.hkv || plan[PH_PAGE] != p.s.page)
    return;
  QTile t;
  t.q_row0 = it.row0;
  t.q_len = it.rows;
  const int sub = it.pair0 / kTilePairs;
  const QRows rows(t, p.group, p.group_magic, sub, wave, l32);
  const int64_t qstride = (int64_t)p.s.hq * D;
  const int64_t qbase = it.row0 * qstride + (int64_t)kvh * p.group * D;

  const int nA = (it.a_len + BN - 1) / BN;
  const int nblk = it.blk1;  // blocks blk0 .. blk1 - 1 of A and then B

  PageCopy<D, E4M3> cp;
  cp.init(p, it.b_seq, it.b_len, wave, lane);
  const char* const kc = static_cast<const char*>(p.k_cache);
  const char* const vc = static_cast<const char*>(p.v_cache);
  const int head_off = kvh * (p.s.page * PageCopy<D, E4M3>::ROWB);
  const int b0 = it.blk0;
  FwdCore<D> core;
  core.hf = hf;
  if (b0 < nblk) {
    PageCursor kcur = cp.at(it, nA), vcur = kcur;
    // e4m3: through the staging areas, `dst` is filled by land_k / land_v
    auto load_k = [&](__bf16* dst) { cp.next(kcur, kc, p.k_stride, head_off, E4M3 ? stage_k : reinterpret_cast<char*>(dst)); };
    auto load_v = [&](__bf16* dst) { cp.next(vcur, vc, p.v_stride, head_off, E4M3 ? stage_v : reinterpret_cast<char*>(dst)); };
    auto land_k = [&](__bf16* dst) { cp.widen(stage_k, dst); };
    auto land_v = [&](__bf16* dst) { cp.widen(stage_v, dst); };

    // the first blocks' copies go out before anything else is computed: K(b + 1)
    // and V(b) are resident while block b is processed
    load_k(k_buf0);
    load_v(v_buf0);
    if constexpr (E4M3) {
      wait_vmem();
      land_k(k_buf0);
      land_v(v_buf0);
      wave_lds_fence();
    }
    if (b0 + 1 < nblk) load_k(k_buf1);

    core.load_q(p.q + qbase + pair_offset<D>(rows.row, rows.head, p.s.hq));
    float scale = p.scale_log2;
    if constexpr (E4M3) scale *= p.k_scale[kvh];
    core.init(scale, l32, lane);

    const int qpos_lo = it.b_pos + rows.wlo;  // causal: the wavefront's first query position
    const int qi = rows.row;
    // a causal block whose keys all follow the wavefront's queries (and every
    // later block) contributes nothing; neither does any block to a wavefront
    // without rows
    const int nlive = !rows.wave_any ? 0 : it.b_len > 0 ? nA + (it.b_pos + rows.whi) / BN + 1 : nA;
    auto step = [&](int b, f32x16& s0, f32x16& s1, const __bf16* kn, const __bf16* vl, f32x16& n0, f32x16& n1) {
      const bool isB = b >= nA;
      const int kb0 = (isB ? b - nA : b) * BN;
      const int len = isB ? it.b_len : it.a_len;
      auto masked = [&] { return (kb0 + BN > len) || (isB && (kb0 + BN - 1 > qpos_lo)); };
      auto limit = [&] { return min(len - 1, isB ? it.b_pos + qi : len - 1) - kb0; };  // last visible key of the block
      core.step(masked, limit, s0, s1, kn, vl, n0, n1);
    };

    // iteration b loads K(b + 2) over K(b) and V(b + 1) over V(b - 1)
    f32x16 sa0, sa1, sb0, sb1;
    wait_vmem();
    if constexpr (E4M3) {
      if (b0 + 1 < nblk) land_k(k_buf1);
      wave_lds_fence();
    }
    __syncthreads();
    core.s_mfma(k_buf0, sa0, sa1);
    pace_lds_mfma<D / 8, 1, FWD_DEPTH>();
    __syncthreads();
    for (int b = b0; b < nblk; b += 2) {
      if (b + 2 < nblk) load_k(k_buf0);
      if (b + 1 < nblk) load_v(v_buf1);
      if (b < nlive) step(b, sa0, sa1, k_buf1, v_buf0, sb0, sb1);
      wait_vmem();
      if constexpr (E4M3) {
        if (b + 2 < nblk) land_k(k_buf0);
        if (b + 1 < nblk) land_v(v_buf1);
        wave_lds_fence();
      }
      __syncthreads();
      if (b + 1 < nblk) {
        if (b + 3 < nblk) load_k(k_buf1);
        if (b + 2 < nblk) load_v(v_buf0);
        if (b + 1 < nlive) step(b + 1, sb0, sb1, k_buf0, v_buf1, sa0, sa1);
        wait_vmem();
        if constexpr (E4M3) {
          if (b + 3 < nblk) land_k(k_buf1);
          if (b + 2 < nblk) land_v(v_buf0);
          wave_lds_fence();
        }
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

}  // namespace

hipError_t launch_paged_fwd(const PagedFwdParams& p, hipStream_t stream) {
  const dim3 grid((unsigned)((int64_t)p.max_items * p.s.hkv)), block(256);
  if (p.d == 128) {
    if (p.type == CACHE_E4M3) attn_paged_kernel<128, true><<<grid, block, 0, stream>>>(p);
    else attn_paged_kernel<128, false><<<grid, block, 0, stream>>>(p);
  } else {
    if (p.type == CACHE_E4M3) attn_paged_kernel<64, true><<<grid, block, 0, stream>>>(p);
    else attn_paged_kernel<64, false><<<grid, block, 0, stream>>>(p);
  }
  return hipGetLastError();
}

}  // namespace augtree
