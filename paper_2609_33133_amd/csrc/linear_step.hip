// One token of linear attention for every row: S' = gamma S + k v^T,
// o_h = scale q_h S'. The states are read and written once, 8 d^2 bytes per row
// and KV head against 2 d^2 (1 + group) multiply-adds, so the kernel is bound
// by HBM. All arithmetic is fp32. A state is held in registers between its read
// and its write, so nothing waits in LDS but k, q and the heads' partial sums.
// Measured at 32 / 8 heads, d = 128: 512 rows, 0.55 GB, in 102 us, 5.4 TB/s (a
// copy of 2 GiB: 4.9); 8 rows 5.2 us, the time of a launch.
#include "common.h"
#include "linear.h"

namespace augtree {
namespace {

// x summed over the four 16-lane rows of the wavefront
__device__ __forceinline__ float sum_rows(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return pair_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

constexpr int kCols = 64;   // state columns of a workgroup
constexpr int kHeads = 4;   // query heads taken at a time

// A workgroup takes 64 columns of one state: 16 lanes with four columns each,
// 16 groups of lanes with D / 16 rows each.
template <int D>
__global__ __launch_bounds__(256) void lin_step_kernel(LinStepParams p) {
  constexpr int NR = D / 16;
  __shared__ float kq[1 + kHeads][D];
  __shared__ f32x4 part[4][kHeads][kCols / 4];
  const int slices = D / kCols;
  const int unit = blockIdx.x / slices, slice = blockIdx.x - unit * slices;
  const int row = unit / p.heads_kv, kvh = unit - row * p.heads_kv;
  const int tid = threadIdx.x, grp = tid >> 4, wave = tid >> 6;
  const int col = slice * kCols + (tid & 15) * 4;
  const float gamma = p.decay[kvh];
  const int64_t kv = ((int64_t)row * p.heads_kv + kvh) * D;

  const int src = p.src ? p.src[row] : row;
  f32x4 s[NR];
  if (src >= 0 && src < p.n_states) {
    const float* in = p.state_in + ((int64_t)src * p.heads_kv + kvh) * D * D + col;
#pragma unroll
    for (int i = 0; i < NR; ++i) s[i] = *reinterpret_cast<const f32x4*>(in + (grp + 16 * i) * D);
  } else {
#pragma unroll
    for (int i = 0; i < NR; ++i) s[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  f32x4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = __uint_as_float((uint32_t)p.v[kv + col + e] << 16);

  for (int h0 = 0; h0 < p.group; h0 += kHeads) {
    const int nh = min(kHeads, p.group - h0);
    const int64_t q0 = kv * p.group + (int64_t)h0 * D;
    for (int i = tid; i < (1 + nh) * D; i += 256) {
      const uint16_t b = i < D ? p.k[kv + i] : p.q[q0 + i - D];
      kq[i / D][i % D] = __uint_as_float((uint32_t)b << 16);
    }
    __syncthreads();
    if (h0 == 0) {
      float* out = p.state_out + ((int64_t)row * p.heads_kv + kvh) * D * D + col;
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        s[i] = s[i] * gamma + v * kq[0][grp + 16 * i];
        *reinterpret_cast<f32x4*>(out + (grp + 16 * i) * D) = s[i];
      }
    }
    for (int h = 0; h < nh; ++h) {
      f32x4 a = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < NR; ++i) a += s[i] * kq[1 + h][grp + 16 * i];
#pragma unroll
      for (int e = 0; e < 4; ++e) a[e] = sum_rows(a[e]);
      if ((tid & 63) < 16) part[wave][h][tid & 15] = a;
    }
    __syncthreads();
    if (tid < nh * kCols) {
      const int h = tid / kCols, c = tid % kCols;
      float a = 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) a += part[k][h][c >> 2][c & 3];
      const __bf16 o = (__bf16)(a * p.scale);
      *reinterpret_cast<__bf16*>(p.o + q0 + (int64_t)h * D + slice * kCols + c) = o;
    }
  }
}

}  // namespace

hipError_t launch_lin_step(const LinStepParams& p, int head_dim, hipStream_t stream) {
  const dim3 grid(p.rows * p.heads_kv * (head_dim / kCols));
  if (head_dim == 128) lin_step_kernel<128><<<grid, 256, 0, stream>>>(p);
  else lin_step_kernel<64><<<grid, 256, 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace augtree
