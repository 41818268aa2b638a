// The paged KV cache's plan and write kernels, and the merge of partial results
// of its attention.
#include "common.h"
#include "paged.h"

namespace augtree {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kMergeAlone = 16;  // parts of a row up to which one group of lanes joins them

// The threads of one workgroup, for plan_scan. Each reduction puts one value
// per wavefront into LDS of its own turn's half, so that two barriers apart no
// wavefront still reads what the next turn writes.
struct GroupTeam {
  struct Wave {
    int64_t key;
    int32_t v[4], bits;
  };
  Wave (*lds)[kPlanThreads / 64];  // [2]
  int turn = 0;
  __device__ int tid() const { return threadIdx.x; }
  __device__ int size() const { return kPlanThreads; }
  __device__ void sync() const { __syncthreads(); }
  __device__ void flag(int32_t* to, int32_t bits) const { atomicOr(to, bits); }
  __device__ Wave* next() { return lds[turn ^= 1]; }

  template <int K>
  __device__ static void wave_scan(int32_t (&x)[K]) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int32_t y = __shfl_up(x[k], d);
        if (lane >= d) x[k] = add_count(x[k], y);
      }
    }
  }
  // sums over the threads before this one, and over all
  template <int K>
  __device__ void scan(const int32_t (&v)[K], int32_t (&before)[K], int32_t (&all)[K]) {
    int64_t none = 0;
    int bits = 0;
    scan_step(v, before, all, none, bits);
  }
  // the same, the largest key of the threads before this one (0 at least), and the bits of all
  template <int K>
  __device__ void scan_step(const int32_t (&v)[K], int32_t (&before)[K], int32_t (&all)[K], int64_t& key, int& bits) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Wave* const to = next();
    int32_t x[K];
#pragma unroll
    for (int k = 0; k < K; ++k) x[k] = v[k];
    wave_scan(x);
    int64_t m = key;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int64_t y = __shfl_up((long long)m, d);
      if (lane >= d && y > m) m = y;
    }
#pragma unroll
    for (int b = 1; b <= PAGES_PAGE; b *= 2)
      if (__any(bits & b)) bits |= b;
    if (lane == 63) {
#pragma unroll
      for (int k = 0; k < K; ++k) to[wave].v[k] = x[k];
      to[wave].key = m;
      to[wave].bits = bits;
    }
    __syncthreads();
    const int64_t up = __shfl_up((long long)m, 1);
    key = lane == 0 ? 0 : up;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      before[k] = x[k] - v[k];  // (exact where the sum has not stopped: a step whose sums stop is refused)
      all[k] = 0;
    }
    for (int w = 0; w < kPlanThreads / 64; ++w) {
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int32_t y = to[w].v[k];
        if (w < wave) before[k] = add_count(before[k], y);
        all[k] = add_count(all[k], y);
      }
      if (w < wave && to[w].key > key) key = to[w].key;
      bits |= to[w].bits;
    }
  }
  // the largest value of the threads before this one, -1 at least
  __device__ int scan_max(int v) {
    const int32_t none[1] = {0};
    int32_t a[1], b[1];
    int64_t key = v + 1;
    int bits = 0;
    scan_step(none, a, b, key, bits);
    return (int)key - 1;
  }
  __device__ void sum(int64_t (&v)[2]) {
    Wave* const to = next();
#pragma unroll
    for (int d = 32; d > 0; d /= 2) {
      v[0] += __shfl_xor((long long)v[0], d);
      v[1] += __shfl_xor((long long)v[1], d);
    }
    if ((threadIdx.x & 63) == 0) {
      to[threadIdx.x >> 6].key = v[0];
      __builtin_memcpy(to[threadIdx.x >> 6].v, &v[1], 8);
    }
    __syncthreads();
    v[0] = v[1] = 0;
    for (int w = 0; w < kPlanThreads / 64; ++w) {
      int64_t y;
      __builtin_memcpy(&y, to[w].v, 8);
      v[0] += to[w].key;
      v[1] += y;
    }
  }
  __device__ int max_of(int v) {
    Wave* const to = next();
#pragma unroll
    for (int d = 32; d > 0; d /= 2) v = max(v, __shfl_xor(v, d));
    if ((threadIdx.x & 63) == 0) to[threadIdx.x >> 6].v[0] = v;
    __syncthreads();
    for (int w = 0; w < kPlanThreads / 64; ++w) v = max(v, to[w].v[0]);
    return v;
  }
};

// One workgroup: the scans over the sequences and, where the rest is little
// (FILL: at most kFillSeqs sequences), that too, with all arrays in LDS. Bound
// by latency: a dozen barriers and the memory round trips between them. TODO_FIGURE
template <bool FILL>
__global__ __launch_bounds__(kPlanThreads) void page_plan_kernel(PlanParams p) {
  __shared__ GroupTeam::Wave lds[2][kPlanThreads / 64];
  GroupTeam team{lds};
  if constexpr (FILL) {
    __shared__ int32_t work[18 * kFillSeqs + 1];
    const PlanArrays a = PlanArrays::packed(work, p.s.seqs);
    plan_scan(team, p, a);
    plan_fill(team, p, a, threadIdx.x, kPlanThreads);
  } else {
    plan_scan(team, p, plan_arrays(p));
  }
}

__global__ __launch_bounds__(256) void page_fill_kernel(PlanParams p) {
  GroupTeam team{nullptr};
  plan_fill(team, p, plan_arrays(p), blockIdx.x * 256 + threadIdx.x, gridDim.x * 256);
}

__device__ __forceinline__ bool plan_is_for(const int32_t* plan, const PagedShape& s) {
  return plan[PH_SEQS] == s.seqs && plan[PH_ROWS] == s.rows && plan[PH_HQ] == s.hq && plan[PH_HKV] == s.hkv &&
         plan[PH_PAGE] == s.page;
}

// Four floats as e4m3, rounded to nearest even; what passes 448 becomes 448,
// NaN stays NaN (a minimum of the two would make it 448).
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, float c, float d) {
  auto in_range = [](float x) { return x > 448.f ? 448.f : x < -448.f ? -448.f : x; };
  int w = 0;
  w = __builtin_amdgcn_cvt_pk_fp8_f32(in_range(a), in_range(b), w, false);
  return __builtin_amdgcn_cvt_pk_fp8_f32(in_range(c), in_range(d), w, true);
}

// Rows of K (y = 0) and V (y = 1) into their slots, 16 bytes of bf16 a thread.
// Bound by HBM.
template <bool E4M3>
__global__ __launch_bounds__(256) void cache_write_kernel(CacheWriteParams p, PlanLayout L) {
  if (!plan_is_for(p.plan, p.s)) return;
  const int chunks = p.s.hkv * (p.d / 8);  // of a row
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = i / chunks;
  if (row >= p.s.rows) return;
  const int slot = p.plan[L.slots + row];
  if (slot < 0) return;
  const int c = (int)(i - row * chunks), h = c / (p.d / 8), e = (c - h * (p.d / 8)) * 8;
  const bool isv = blockIdx.y != 0;
  const int shift = __builtin_ctz(p.s.page);
  const int page = slot >> shift, off = slot & (p.s.page - 1);
  const uint4 x = ldg16((isv ? p.v : p.k) + i * 8);
  char* const dst = static_cast<char*>(isv ? p.v_cache : p.k_cache) + page * (isv ? p.v_stride : p.k_stride);
  const int64_t at = ((int64_t)h * p.s.page + off) * p.d + e;
  if constexpr (!E4M3) {
    *reinterpret_cast<uint4*>(dst + 2 * at) = x;
  } else {
    const float scale = (isv ? p.v_scale : p.k_scale)[h];
    float f[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = __uint_as_float(half16(x, j) << 16) / scale;
    uint2 w;
    w.x = to_e4m3(f[0], f[1], f[2], f[3]);
    w.y = to_e4m3(f[4], f[5], f[6], f[7]);
    *reinterpret_cast<uint2*>(dst + at) = w;
  }
}

// Joins the partial results of a row: o = sum_p w_p o_p / sum_p w_p, w_p =
// exp(lse_p - max lse), lse = max + log sum_p w_p, over the parts of its
// sequence's own unit and of its run's. D / 4 lanes take a (row, head) pair and,
// of its parts, every `share`-th: one group of lanes all of them where the plan
// has few parts a row, else the workgroup's groups together.
template <int D>
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedFwdParams p, int64_t merge_at) {
  constexpr int LANES = D / 4, GROUPS = 256 / LANES;
  __shared__ f32x4 part_acc[GROUPS][LANES];
  __shared__ float part_top[GROUPS], part_sum[GROUPS];
  const int32_t* const plan = p.plan;
  if (!plan_is_for(plan, p.s)) return;
  const int64_t pairs = (int64_t)plan[PH_MERGE_ROWS] * p.s.hq;
  const int lane = threadIdx.x % LANES, grp = threadIdx.x / LANES, g = p.group;
  const int share = plan[PH_MOST_PARTS] > kMergeAlone ? GROUPS : 1;
  const int per = GROUPS / share, mine = share > 1 ? 0 : grp, phase = share > 1 ? grp : 0;
  for (int64_t i0 = (int64_t)blockIdx.x * per; i0 < pairs; i0 += (int64_t)gridDim.x * per) {
    const int64_t i = i0 + mine;
    const bool any = i < pairs;
    const int64_t m = any ? i / p.s.hq : 0;
    const int head = any ? (int)(i - m * p.s.hq) : 0, kvh = head / g;
    const int32_t* const d = plan + merge_at + m * kMergeInts;
    const int row = d[0];
    float top = -INFINITY, sum = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    if (any)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int pair = d[2 + 4 * u] + head - kvh * g, parts = d[4 + 4 * u];
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
    if (share > 1) {
      part_acc[grp][lane] = acc;
      if (lane == 0) {
        part_top[grp] = top;
        part_sum[grp] = sum;
      }
      __syncthreads();
      if (grp == 0) {
        for (int k = 1; k < GROUPS; ++k) top = fmaxf(top, part_top[k]);
        const float w0 = __expf(part_top[0] - top);
        acc = acc * w0;
        sum *= w0;
        for (int k = 1; k < GROUPS; ++k) {
          const float w = __expf(part_top[k] - top);
          acc += part_acc[k][lane] * w;
          sum += part_sum[k] * w;
        }
      }
      __syncthreads();
      if (grp != 0) continue;
    }
    if (!any) continue;
    const float inv = 1.f / sum;
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    bf16x4 y;
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = (__bf16)(acc[j] * inv);
    *reinterpret_cast<bf16x4*>(p.o + ((int64_t)row * p.s.hq + head) * D + lane * 4) = y;
    if (p.lse && lane == 0) p.lse[(int64_t)head * p.s.rows + row] = top + __logf(sum);
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
  const int most = p.s.rows > p.L.max_items ? p.s.rows : p.L.max_items;
  page_fill_kernel<<<most < 1024 * 256 ? (most + 255) / 256 : 1024, 256, 0, stream>>>(p);
  return hipGetLastError();
}

hipError_t launch_cache_write(const CacheWriteParams& p, hipStream_t stream) {
  const int64_t threads = (int64_t)p.s.rows * p.s.hkv * (p.d / 8);
  const dim3 grid((unsigned)((threads + 255) / 256), 2);
  const PlanLayout L = plan_layout(p.s);
  if (p.type == CACHE_E4M3) cache_write_kernel<true><<<grid, 256, 0, stream>>>(p, L);
  else cache_write_kernel<false><<<grid, 256, 0, stream>>>(p, L);
  return hipGetLastError();
}

hipError_t launch_paged_merge(const PagedFwdParams& p, hipStream_t stream) {
  const int64_t merge_at = plan_layout(p.s).merge, pairs = (int64_t)p.s.rows * p.s.hq;
  const unsigned grid = (unsigned)(pairs < 2048 ? pairs : 2048);
  if (p.d == 128) paged_merge_kernel<128><<<grid, 256, 0, stream>>>(p, merge_at);
  else paged_merge_kernel<64><<<grid, 256, 0, stream>>>(p, merge_at);
  return hipGetLastError();
}

}  // namespace augtree
