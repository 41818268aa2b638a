// The paged KV cache's plan and write kernels, and the merge of partial results
// of its attention.
#include <type_traits>

#include "common.h"
#include "paged.h"

namespace augtree {
namespace {

constexpr int kPlanThreads = 1024;
// Parts of a row up to which one group of lanes joins them, with more a workgroup.
// Attention and merge, us, by a workgroup and (a limit of 48) by a group: one
// sequence of 4096 in 22 parts 11.2 and 14.0, eight branches of 32768 in 23 34.3
// and 37.1, a chunk of 120 over 9000 in 48 24.4 and 30.4, 64 branches of 9000 in 18
// 33.2 and 32.2. A limit of six: the same as 16.
constexpr int kMergeAlone = 16;

// x of the lane that a DPP control names, 0 where it names none.
template <int CTRL, int ROWS>
__device__ __forceinline__ int32_t dpp(int32_t x) {
  return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false);
}
// f(x, value of an earlier lane) for an inclusive scan over the wavefront (N = 64) or each 16 lanes: rows of 16 by
// shifts, then the rows' last lanes to the rows behind
template <int N, class F>
__device__ __forceinline__ void scan_by_dpp(F f) {
  f(std::integral_constant<int, 0x111>(), std::integral_constant<int, 0xf>());
  f(std::integral_constant<int, 0x112>(), std::integral_constant<int, 0xf>());
  f(std::integral_constant<int, 0x114>(), std::integral_constant<int, 0xf>());
  f(std::integral_constant<int, 0x118>(), std::integral_constant<int, 0xf>());
  if constexpr (N == 64) {
    f(std::integral_constant<int, 0x142>(), std::integral_constant<int, 0xa>());
    f(std::integral_constant<int, 0x143>(), std::integral_constant<int, 0xc>());
  }
}
template <int N>
__device__ __forceinline__ int32_t sums(int32_t x) {
  scan_by_dpp<N>([&](auto ctrl, auto rows) { x = add_count(x, dpp<decltype(ctrl)::value, decltype(rows)::value>(x)); });
  return x;
}
template <int N>
__device__ __forceinline__ int64_t sums64(int64_t x) {
  scan_by_dpp<N>([&](auto ctrl, auto rows) {
    const uint32_t lo = dpp<decltype(ctrl)::value, decltype(rows)::value>((int32_t)x);
    const uint32_t hi = dpp<decltype(ctrl)::value, decltype(rows)::value>((int32_t)(x >> 32));
    x += (int64_t)((uint64_t)hi << 32 | lo);
  });
  return x;
}
template <int N>
__device__ __forceinline__ int64_t maxima(int64_t x) {  // of x >= 0
  scan_by_dpp<N>([&](auto ctrl, auto rows) {
    const uint32_t lo = dpp<decltype(ctrl)::value, decltype(rows)::value>((int32_t)x);
    const uint32_t hi = dpp<decltype(ctrl)::value, decltype(rows)::value>((int32_t)(x >> 32));
    const int64_t y = (int64_t)((uint64_t)hi << 32 | lo);
    x = y > x ? y : x;
  });
  return x;
}
__device__ __forceinline__ int64_t lane64(int64_t x, int lane) {
  const uint32_t lo = __builtin_amdgcn_readlane((int32_t)x, lane), hi = __builtin_amdgcn_readlane((int32_t)(x >> 32), lane);
  return (int64_t)((uint64_t)hi << 32 | lo);
}

// The wavefronts of one workgroup, for plan_scan. Each reduction puts one value
// per wavefront into LDS of its own turn's half, so that two barriers apart no
// wavefront still reads what the next turn writes; every wavefront then scans
// these values, one per lane. All instructions run on one CU, so they count:
// scans by LDS shuffles, and totals added up by every thread in a loop, took
// 11 of 29 us for 576 sequences, sums that stop and 64-bit maxima inside a
// wavefront 3 of 35 for 4352.
struct GroupTeam {
  static constexpr int kWaves = kPlanThreads / 64;
  struct Turn {
    int64_t key[kWaves];
    int32_t v[4][kWaves], bits[kWaves];
  };
  Turn* lds;  // [2]
  int turn = 0;
  __device__ int tid() const { return threadIdx.x; }
  __device__ int lane() const { return threadIdx.x & 63; }
  __device__ int wave() const { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }
  __device__ int lanes() const { return 64; }
  __device__ int waves() const { return kWaves; }
  __device__ void sync() const { __syncthreads(); }
  __device__ void flag(int32_t* to, int32_t bits) const { atomicOr(to, bits); }
  __device__ Turn* next() { return lds + (turn ^= 1); }

  // v: of the lanes before this one; total: of all lanes
  template <int K>
  __device__ void scan_lanes(int32_t (&v)[K], int32_t (&total)[K]) const {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      uint32_t x = v[k];  // (a step whose sums pass kMostCount is refused: these may wrap)
      scan_by_dpp<64>([&](auto ctrl, auto rows) { x += dpp<decltype(ctrl)::value, decltype(rows)::value>(x); });
      v[k] = x - v[k];
      total[k] = __builtin_amdgcn_readlane(x, 63);
    }
  }
  // x: 0 or larger than in all lanes before; the last of the lanes before that is not 0, or 0; returns that of all lanes
  __device__ int64_t last_lanes(int64_t& x) const {
    const uint64_t set = __ballot(x != 0), mine = set & ((uint64_t(1) << lane()) - 1);
    const int64_t all = set ? lane64(x, 63 - __builtin_clzll(set)) : 0;
    const int at = 4 * (63 - __builtin_clzll(mine | 1));
    const uint32_t lo = __builtin_amdgcn_ds_bpermute(at, (int32_t)x), hi = __builtin_amdgcn_ds_bpermute(at, (int32_t)(x >> 32));
    x = mine ? (int64_t)((uint64_t)hi << 32 | lo) : 0;
    return all;
  }
  // sums over the threads: of the wavefronts before this one, of all
  template <int K>
  __device__ void scan_waves(const int32_t (&v)[K], int32_t (&before)[K], int32_t (&all)[K]) {
    Turn* const t = next();
    const int w = wave();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int32_t x = sums<64>(v[k]);
      if (lane() == 63) t->v[k][w] = x;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int32_t y = sums<kWaves>(lane() < kWaves ? t->v[k][lane()] : 0);
      before[k] = w > 0 ? __builtin_amdgcn_readlane(y, w - 1) : 0;
      all[k] = __builtin_amdgcn_readlane(y, kWaves - 1);
    }
  }
  // the same, the largest key (>= 0) of the wavefronts before this one, and the bits of all
  template <int K>
  __device__ void scan_waves(const int32_t (&v)[K], int32_t (&before)[K], int32_t (&all)[K], int64_t& key, int& bits) {
    const int64_t m = maxima<64>(key);
#pragma unroll
    for (int b = 1; b <= PAGES_PAGE; b *= 2)
      if (__any(bits & b)) bits |= b;
    Turn* const t = lds + (turn ^ 1);
    const int w = wave();
    if (lane() == 63) {
      t->key[w] = m;
      t->bits[w] = bits;
    }
    scan_waves(v, before, all);
    const int64_t y = maxima<kWaves>(lane() < kWaves ? t->key[lane()] : 0);
    key = w > 0 ? lane64(y, w - 1) : 0;
    const int other = lane() < kWaves ? t->bits[lane()] : 0;
#pragma unroll
    for (int b = 1; b <= PAGES_PAGE; b *= 2)
      if (__any(other & b)) bits |= b;
  }
  // the largest value of the wavefronts before this one, -1 at least
  __device__ int max_waves(int v) {
    Turn* const t = next();
    const int w = wave();
    const int64_t x = maxima<64>((int64_t)v + 1);
    if (lane() == 63) t->key[w] = x;
    __syncthreads();
    const int64_t y = maxima<kWaves>(lane() < kWaves ? t->key[lane()] : 0);
    return w > 0 ? (int)lane64(y, w - 1) - 1 : -1;
  }
  __device__ int max_of(int v) {  // of v >= 0
    Turn* const t = next();
    const int64_t x = maxima<64>(v);
    if (lane() == 63) t->key[wave()] = x;
    __syncthreads();
    return (int)lane64(maxima<kWaves>(lane() < kWaves ? t->key[lane()] : 0), kWaves - 1);
  }
  __device__ void sum(int64_t (&v)[3]) {
    Turn* const t = next();
    int64_t* const at[] = {t->key, reinterpret_cast<int64_t*>(t->v[0]), reinterpret_cast<int64_t*>(t->v[2])};
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      const int64_t x = sums64<64>(v[k]);
      if (lane() == 63) at[k][wave()] = x;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 3; ++k) v[k] = lane64(sums64<kWaves>(lane() < kWaves ? at[k][lane()] : 0), kWaves - 1);
  }
};

// One workgroup: the scans over the sequences and, where the rest is little
// (FILL: at most kFillSeqs sequences), that too, with all arrays in LDS. Bound
// by latency: a dozen barriers and the memory round trips between them. 576
// sequences with 496 rows and 585 items 13.3 us, 4352 sequences 33 us and 10 us
// for the second launch (12 with threads for the rows alone).
template <bool FILL>
__global__ __launch_bounds__(kPlanThreads) void page_plan_kernel(PlanParams p) {
  __shared__ GroupTeam::Turn lds[2];
  GroupTeam team{lds};
  if constexpr (FILL) {
    __shared__ int32_t work[18 * kFillSeqs + 1];
    const PlanArrays a = PlanArrays::packed(work, p.s.seqs);
    plan_scan<true>(team, p, a);
    plan_fill(team, p, a, threadIdx.x, kPlanThreads);
  } else {
    plan_scan<false>(team, p, plan_arrays(p));
  }
}

__global__ __launch_bounds__(256) void page_fill_kernel(PlanParams p) {
  GroupTeam team{nullptr};
  plan_fill(team, p, plan_arrays(p), blockIdx.x * 256 + threadIdx.x, gridDim.x * 256);
}

// x / s correctly rounded, from y = 1 / s correctly rounded: q = x y is off by
// less than a unit in the last place, and so is the quotient of its exact
// remainder from making it right (Markstein's theorem). For s of which neither y
// nor a remainder leaves the normal range, and quotients in e4m3's; any larger
// one (or NaN) is returned as x y.
__device__ __forceinline__ float quotient(float x, float s, float y) {
  const float q = x * y;
  // (the sign: of a -0 the remainder is +0)
  return __builtin_fabsf(q) < 512.f ? __builtin_copysignf(__builtin_fmaf(__builtin_fmaf(-q, s, x), y, q), q) : q;
}
// Four floats as e4m3, rounded to nearest even; what passes 448 becomes 448,
// NaN stays NaN (a minimum of the two would make it 448).
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, float c, float d) {
  auto in_range = [](float x) { return x > 448.f ? 448.f : x < -448.f ? -448.f : x; };
  int w = 0;
  w = __builtin_amdgcn_cvt_pk_fp8_f32(in_range(a), in_range(b), w, false);
  return __builtin_amdgcn_cvt_pk_fp8_f32(in_range(c), in_range(d), w, true);
}

// Rows of K (y = 0) and V (y = 1) into their slots; a thread writes 16 bytes.
// Bound by HBM: 82660 rows of 4 heads of 128 into e4m3, 254 MB, in 45 us, 5.7 TB/s
// (eight values a thread and a division each: 62 us); 256 rows of 8 heads in 3 us,
// the time of a launch.
template <bool E4M3>
__global__ __launch_bounds__(256) void cache_write_kernel(CacheWriteParams p, int64_t slots) {
  constexpr int N = E4M3 ? 16 : 8;  // values of a thread
  if (!plan_is_for(p.plan, p.s)) return;
  const int of_head = p.d / N, chunks = p.s.hkv * of_head;  // of a row
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = i / chunks;
  if (row >= p.s.rows) return;
  const int slot = p.plan[slots + row];
  if (slot < 0) return;
  const int c = (int)(i - row * chunks), h = c / of_head, e = (c - h * of_head) * N;
  const bool isv = blockIdx.y != 0;
  const int shift = __builtin_ctz(p.s.page);
  const int page = slot >> shift, off = slot & (p.s.page - 1);
  const uint16_t* const src = (isv ? p.v : p.k) + i * N;
  char* const dst = static_cast<char*>(isv ? p.v_cache : p.k_cache) + page * (isv ? p.v_stride : p.k_stride);
  const int64_t at = ((int64_t)h * p.s.page + off) * p.d + e;
  if constexpr (!E4M3) {
    *reinterpret_cast<uint4*>(dst + 2 * at) = ldg16(src);
  } else {
    const uint4 x[2] = {ldg16(src), ldg16(src + 8)};
    const float scale = (isv ? p.v_scale : p.k_scale)[h], inverse = 1.f / scale;
    const bool plain = scale > 0x1p-60f && scale < 0x1p60f;
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float f[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float v = __uint_as_float(half16(x[j >> 1], (j & 1) * 4 + k) << 16);
        f[k] = plain ? quotient(v, scale, inverse) : v / scale;
      }
      w[j] = to_e4m3(f[0], f[1], f[2], f[3]);
    }
    *reinterpret_cast<uint4*>(dst + at) = uint4{w[0], w[1], w[2], w[3]};
  }
}

// One pair of a merge: where its parts lie, and what they come to so far.
template <int D>
struct MergePair {
  const PagedFwdParams& p;
  int32_t d[kMergeInts];  // the row's entry of the plan
  int head, kvh, lane;
  float top = -INFINITY, sum = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};

  __device__ __forceinline__ MergePair(const PagedFwdParams& p_, const int32_t* merge, uint32_t i, int lane_)
      : p(p_), lane(lane_) {
    const uint32_t m = i / (uint32_t)p.s.hq;  // (fewer than 2^30 pairs)
    head = (int)(i - m * p.s.hq);
    kvh = fast_div(head, p.group, p.group_magic);
    const int4* const src = reinterpret_cast<const int4*>(merge + (int64_t)m * kMergeInts);  // (arrays of a plan are 16-byte aligned)
#pragma unroll
    for (int k = 0; k < kMergeInts / 4; ++k) {
      const int4 w = src[k];
      d[4 * k] = w.x;
      d[4 * k + 1] = w.y;
      d[4 * k + 2] = w.z;
      d[4 * k + 3] = w.w;
    }
  }
  __device__ __forceinline__ int parts() const { return d[4] + d[8]; }
  // the parts phase, phase + share, .. of both units
  __device__ __forceinline__ void add(int phase, int share) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int pair = d[2 + 4 * u] + head - kvh * p.group, parts = d[4 + 4 * u];
      // the pair's place in slots of 32 pairs, per KV head; from part to part
      const int64_t first = ((int64_t)(d[1 + 4 * u] + pair / kSlotPairs) * p.s.hkv + kvh) * kSlotPairs + pair % kSlotPairs;
      const int64_t step = (int64_t)d[3 + 4 * u] * p.s.hkv * kSlotPairs;
      // four parts at a time, so that their loads are on their way together
      for (int k = phase; k < parts; k += 4 * share) {
        float l[4];
        f32x4 o[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int kk = k + j * share;
          const int64_t at = first + (kk < parts ? kk : k) * step;
          l[j] = p.part_lse[at];
          o[j] = *reinterpret_cast<const f32x4*>(p.part_o + at * D + lane * 4);
          if (kk >= parts) l[j] = -INFINITY;
        }
        const float t = fmaxf(fmaxf(fmaxf(l[0], l[1]), fmaxf(l[2], l[3])), top);
        if (t == -INFINITY) continue;  // parts that the row sees nothing of
        const float back = __expf(top - t);
        acc = acc * back;
        sum *= back;
        top = t;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float w = __expf(l[j] - t);
          acc += o[j] * w;
          sum += w;
        }
      }
    }
  }
  __device__ __forceinline__ void store() const {
    const float inv = 1.f / sum;
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    bf16x4 y;
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = (__bf16)(acc[j] * inv);
    const int row = d[0];
    *reinterpret_cast<bf16x4*>(p.o + ((int64_t)row * p.s.hq + head) * D + lane * 4) = y;
    if (p.lse && lane == 0) p.lse[(int64_t)head * p.s.rows + row] = top + __logf(sum);
  }
};

// Joins the partial results of a row: o = sum_p w_p o_p / sum_p w_p, w_p =
// exp(lse_p - max lse), lse = max + log sum_p w_p, over the parts of its
// sequence's own unit and of its run's. D / 4 lanes take a (row, head) pair;
// pairs of more than kMergeAlone parts are taken by a workgroup, each of whose
// groups of lanes joins every eighth (d = 64: sixteenth) part. The loads of four
// parts are on their way together: 32 pairs of 22 parts take 4 us, 256 of 24 4.4
// us, 16384 of two 13 us. (By one group, one part after the other, 32 pairs of 33
// parts took 25 us.)
template <int D>
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedFwdParams p, int64_t merge_at) {
  constexpr int LANES = D / 4, GROUPS = 256 / LANES;
  __shared__ f32x4 part_acc[GROUPS][LANES];
  __shared__ float part_top[GROUPS], part_sum[GROUPS];
  const int32_t* const plan = p.plan;
  if (!plan_is_for(plan, p.s)) return;
  const int32_t* const merge = plan + merge_at;
  const uint32_t pairs = (uint32_t)plan[PH_MERGE_ROWS] * p.s.hq;
  const int lane = threadIdx.x % LANES, grp = threadIdx.x / LANES;
  const bool some_together = plan[PH_MOST_PARTS] * 2 > kMergeAlone;  // (of one unit, of which a row has two)
  for (uint32_t i = blockIdx.x * GROUPS + grp; i < pairs; i += gridDim.x * GROUPS) {
    MergePair<D> x(p, merge, i, lane);
    if (some_together && x.parts() > kMergeAlone) continue;
    x.add(0, 1);
    x.store();
  }
  if (!some_together) return;
  for (uint32_t i = blockIdx.x; i < pairs; i += gridDim.x) {
    MergePair<D> x(p, merge, i, lane);
    if (x.parts() <= kMergeAlone) continue;  // (the same for the whole workgroup)
    x.add(grp, GROUPS);
    part_acc[grp][lane] = x.acc;
    if (lane == 0) {
      part_top[grp] = x.top;
      part_sum[grp] = x.sum;
    }
    __syncthreads();
    if (grp == 0) {
      for (int k = 1; k < GROUPS; ++k) x.top = fmaxf(x.top, part_top[k]);
      const float w0 = __expf(part_top[0] - x.top);
      x.acc = x.acc * w0;
      x.sum *= w0;
      for (int k = 1; k < GROUPS; ++k) {
        const float w = __expf(part_top[k] - x.top);
        x.acc += part_acc[k][lane] * w;
        x.sum += part_sum[k] * w;
      }
      x.store();
    }
    __syncthreads();
  }
}

}  // namespace

hipError_t launch_page_plan(const PlanParams& p, bool apart, hipStream_t stream) {
  if (!apart) {
    page_plan_kernel<true><<<1, kPlanThreads, 0, stream>>>(p);
    return hipGetLastError();
  }
  page_plan_kernel<false><<<1, kPlanThreads, 0, stream>>>(p);
  if (hipError_t e = hipGetLastError()) return e;
  // a thread for every row and item, and for the pages of rows that fill theirs
  const int64_t most = (int64_t)p.s.rows + p.L.max_items + p.s.rows / p.s.page;
  page_fill_kernel<<<most < 1024 * 256 ? (unsigned)((most + 255) / 256) : 1024, 256, 0, stream>>>(p);
  return hipGetLastError();
}

hipError_t launch_cache_write(const CacheWriteParams& p, hipStream_t stream) {
  const int64_t threads = (int64_t)p.s.rows * p.s.hkv * (p.d / (p.type == CACHE_E4M3 ? 16 : 8)), slots = plan_layout(p.s).slots;
  const dim3 grid((unsigned)((threads + 255) / 256), 2);
  if (p.type == CACHE_E4M3) cache_write_kernel<true><<<grid, 256, 0, stream>>>(p, slots);
  else cache_write_kernel<false><<<grid, 256, 0, stream>>>(p, slots);
  return hipGetLastError();
}

hipError_t launch_paged_merge(const PagedFwdParams& p, hipStream_t stream) {
  const int64_t merge_at = plan_layout(p.s).merge, pairs = (int64_t)p.s.rows * p.s.hq;
  const unsigned grid = (unsigned)(pairs < 4096 ? pairs : 4096);
  if (p.d == 128) paged_merge_kernel<128><<<grid, 256, 0, stream>>>(p, merge_at);
  else paged_merge_kernel<64><<<grid, 256, 0, stream>>>(p, merge_at);
  return hipGetLastError();
}

}  // namespace augtree
