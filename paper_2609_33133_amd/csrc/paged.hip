// The paged KV cache's plan and write kernels, and the merge of partial results
// of its attention.
#include "common.h"
#include "paged.h"

namespace augtree {
namespace {

constexpr int kPlanThreads = 1024;

// The threads of one workgroup, for plan_scan.
struct GroupTeam {
  int64_t* sums;   // [wavefronts][4] of LDS
  int* maxs;       // [wavefronts]
  __device__ int tid() const { return threadIdx.x; }
  __device__ int size() const { return blockDim.x; }
  __device__ void sync() const { __syncthreads(); }
  __device__ int any(int bits) const {
    int r = 0;
#pragma unroll
    for (int b = 0; b < 6; ++b)
      if (__syncthreads_or(bits & (1 << b))) r |= 1 << b;
    return r;
  }
  __device__ void flag(int32_t* to, int32_t bits) const { atomicOr(to, bits); }
  // sums over the threads before this one, and over all
  template <int K>
  __device__ void scan(const int64_t (&v)[K], int64_t (&before)[K], int64_t (&all)[K]) const {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    int64_t x[K];
#pragma unroll
    for (int k = 0; k < K; ++k) x[k] = v[k];
    for (int d = 1; d < 64; d *= 2) {
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int64_t y = __shfl_up((long long)x[k], d);
        if (lane >= d) x[k] += y;
      }
    }
    __syncthreads();  // the last scan's sums have been read
    if (lane == 63)
#pragma unroll
      for (int k = 0; k < K; ++k) sums[wave * 4 + k] = x[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      before[k] = x[k] - v[k];
      all[k] = 0;
    }
    for (int w = 0; w < waves; ++w)
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int64_t y = sums[w * 4 + k];
        if (w < wave) before[k] += y;
        all[k] += y;
      }
  }
  // the largest value of the threads before this one, -1 at least
  __device__ int scan_max(int v) const {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int x = v;
    for (int d = 1; d < 64; d *= 2) {
      const int y = __shfl_up(x, d);
      if (lane >= d) x = max(x, y);
    }
    __syncthreads();
    if (lane == 63) maxs[wave] = x;
    __syncthreads();
    int r = __shfl_up(x, 1);
    if (lane == 0) r = -1;
    for (int w = 0; w < wave; ++w) r = max(r, maxs[w]);
    return r;
  }
};

// One workgroup: the scans over the sequences and, where the rest is little
// (FILL), that too. Bound by latency: a dozen barriers and the memory round
// trips between them.
template <bool FILL>
__global__ __launch_bounds__(kPlanThreads) void page_plan_kernel(PlanParams p) {
  __shared__ int64_t sums[kPlanThreads / 64 * 4];
  __shared__ int maxs[kPlanThreads / 64];
  GroupTeam team{sums, maxs};
  plan_scan(team, p);
  if constexpr (FILL) plan_fill(team, p, threadIdx.x, kPlanThreads, 64);
}

__global__ __launch_bounds__(256) void page_fill_kernel(PlanParams p) {
  GroupTeam team{nullptr, nullptr};
  plan_fill(team, p, (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256, 64);
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
// sequence's own unit and of its run's. D / 4 lanes take a (row, head) pair.
template <int D>
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedFwdParams p, PlanLayout L) {
  constexpr int LANES = D / 4;
  if (!plan_is_for(p.plan, p.s)) return;
  const int32_t* const plan = p.plan;
  const int64_t pairs = (int64_t)plan[PH_MERGE_ROWS] * p.s.hq;
  const int lane = threadIdx.x % LANES, g = p.group;
  for (int64_t i = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES; i < pairs;
       i += (int64_t)gridDim.x * (256 / LANES)) {
    const int64_t m = i / p.s.hq;
    const int head = (int)(i - m * p.s.hq), kvh = head / g;
    const int row = plan[L.merge_rows + m], seq = plan[L.row_seq + row], run = plan[L.run + seq];
    // the two units: first slot of the pair's group of 32, slots of a part, parts
    int64_t slot[2] = {0, 0};
    int step[2] = {0, 0}, parts[2] = {0, 0}, at[2] = {0, 0};
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int s = u == 0 ? seq : run;
      if (s < 0) continue;
      const int32_t* const unit = plan + L.unit + (2 * (int64_t)s + u) * kUnitInts;
      const int row0 = plan[L.cu + s], rows = u == 0 ? plan[L.cu + s + 1] - row0 : plan[L.run_rows + s];
      const int pair = (row - row0) * g + head % g;
      if (unit[2] < 0) continue;
      step[u] = paged_div(rows * g, kSlotPairs);
      slot[u] = unit[2] + pair / kSlotPairs;
      at[u] = pair % kSlotPairs;
      parts[u] = unit[3];
    }
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < 2; ++u)
      for (int k = 0; k < parts[u]; ++k)
        top = fmaxf(top, p.part_lse[((slot[u] + (int64_t)k * step[u]) * p.s.hkv + kvh) * kSlotPairs + at[u]]);
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    float sum = 0.f;
#pragma unroll
    for (int u = 0; u < 2; ++u)
      for (int k = 0; k < parts[u]; ++k) {
        const int64_t at32 = ((slot[u] + (int64_t)k * step[u]) * p.s.hkv + kvh) * kSlotPairs + at[u];
        const float l = p.part_lse[at32];
        if (l == -INFINITY) continue;  // a part that the row sees nothing of
        const float w = __expf(l - top);
        acc += *reinterpret_cast<const f32x4*>(p.part_o + at32 * D + lane * 4) * w;
        sum += w;
      }
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
  const int64_t rows = (p.s.rows + 255) / 256, seqs = ((int64_t)p.s.seqs + 3) / 4;
  const int64_t want = rows > seqs ? rows : seqs;
  page_fill_kernel<<<(unsigned)(want < 1024 ? want : 1024), 256, 0, stream>>>(p);
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
  const PlanLayout L = plan_layout(p.s);
  const int64_t pairs = (int64_t)p.s.rows * p.s.hq, per = 256 / (p.d / 4);
  const int64_t want = (pairs + per - 1) / per;
  const unsigned grid = (unsigned)(want < 2048 ? want : 2048);
  if (p.d == 128) paged_merge_kernel<128><<<grid, 256, 0, stream>>>(p, L);
  else paged_merge_kernel<64><<<grid, 256, 0, stream>>>(p, L);
  return hipGetLastError();
}

}  // namespace augtree
