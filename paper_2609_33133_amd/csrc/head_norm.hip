// Group norm whose groups are the heads of a packed [rows, heads, d] tensor,
// with an activation or a gate. For one row and head:
//   n = (x - mean) / sqrt(var + eps),  a = n w + b,
//   y = act(a), or with a gate y = a act(gate);  act(u) = u / (1 + e^-u) or u.
// Backward, with da = dy act'(a) (gate: dy act(gate), dgate = dy a act'(gate)):
//   dn = da w,  dx = (dn - mean(dn) - n mean(dn n)) / sqrt(var + eps),
//   dw = sum_rows da n,  db = sum_rows da.
// Both are bound by HBM: every tensor is read or written once, the statistics
// are formed again in the backward. Arithmetic in fp32, one rounding at the end.
//
// A head is taken by T lanes (the power of two from d / 8 on, at most 64), each
// holding NC pieces of 8 channels, so its sums stay inside a wavefront.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "linear.h"

namespace augtree {
namespace {

template <int T>
__device__ __forceinline__ float lane_sum(float x) {
#pragma unroll
  for (int k = 1; k < T; k <<= 1) x += __shfl_xor(x, k);
  return x;
}

// the channels of this lane, as fp32; channels past the head are zero
template <int T, int NC>
__device__ __forceinline__ void load16(float* v, const uint16_t* base, int l, int pieces) {
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int k = l + c * T;
    raw16 r = {0u, 0u, 0u, 0u};
    if (k < pieces) r = *reinterpret_cast<const raw16*>(base + 8 * k);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[8 * c + 2 * i] = __uint_as_float(r[i] << 16);
      v[8 * c + 2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
    }
  }
}
template <int T, int NC>
__device__ __forceinline__ void store16(uint16_t* base, const float* v, int l, int pieces) {
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int k = l + c * T;
    bf16x8 r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = (__bf16)v[8 * c + i];
    if (k < pieces) *reinterpret_cast<bf16x8*>(base + 8 * k) = r;
  }
}
template <int T, int NC>
__device__ __forceinline__ void load32(float* v, const float* base, int l, int pieces, float none) {
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int k = l + c * T;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[8 * c + i] = base && k < pieces ? base[8 * k + i] : none;
  }
}

// x becomes n; returns 1 / sqrt(var + eps)
template <int T, int NC>
__device__ __forceinline__ float normalise(float* x, int l, int pieces, float inv_d, float eps) {
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < 8 * NC; ++i) sum += x[i];
  const float mean = lane_sum<T>(sum) * inv_d;
  float sq = 0.f;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const bool in = l + c * T < pieces;
#pragma unroll
    for (int i = 8 * c; i < 8 * c + 8; ++i) {
      x[i] = in ? x[i] - mean : 0.f;
      sq += x[i] * x[i];
    }
  }
  const float rstd = 1.f / sqrtf(lane_sum<T>(sq) * inv_d + eps);
#pragma unroll
  for (int i = 0; i < 8 * NC; ++i) x[i] *= rstd;
  return rstd;
}

__device__ __forceinline__ float sigmoid(float u) { return 1.f / (1.f + expf(-u)); }

template <int T, int NC, bool GATE, bool SILU>
__global__ __launch_bounds__(256) void head_norm_fwd_kernel(HeadNormParams p) {
  const int l = threadIdx.x & (T - 1), pieces = p.d / 8;
  const float inv_d = 1.f / (float)p.d;
  const int64_t units = p.rows * p.heads, step = (int64_t)gridDim.x * (256 / T);
  for (int64_t u = (int64_t)blockIdx.x * (256 / T) + threadIdx.x / T; u < units; u += step) {
    const int64_t at = u * p.d;
    const int head = (int)(u % p.heads);
    float x[8 * NC], w[8 * NC], b[8 * NC], gt[8 * NC];
    load16<T, NC>(x, p.x + at, l, pieces);
    if (GATE) load16<T, NC>(gt, p.gate + at, l, pieces);
    load32<T, NC>(w, p.weight ? p.weight + head * p.d : nullptr, l, pieces, 1.f);
    load32<T, NC>(b, p.bias ? p.bias + head * p.d : nullptr, l, pieces, 0.f);
    normalise<T, NC>(x, l, pieces, inv_d, p.eps);
#pragma unroll
    for (int i = 0; i < 8 * NC; ++i) {
      const float a = x[i] * w[i] + b[i], t = GATE ? gt[i] : a;
      const float act = SILU ? t * sigmoid(t) : t;
      x[i] = GATE ? a * act : act;
    }
    store16<T, NC>(p.y + at, x, l, pieces);
  }
}

// A workgroup takes the rows of one of `row_parts` parts and a run of `hpw`
// heads; 256 / T / hpw groups of lanes share the rows of a head. Each group
// leaves its sums of dweight and dbias as one of p.parts partial sums.
template <int T, int NC, bool GATE, bool SILU>
__global__ __launch_bounds__(256) void head_norm_bwd_kernel(HeadNormParams p, int hpw, int row_parts) {
  const int l = threadIdx.x & (T - 1), grp = threadIdx.x / T, pieces = p.d / 8;
  const int rl = 256 / T / hpw;  // groups that share a head
  const int head = blockIdx.y * hpw + grp % hpw, sub = grp / hpw;
  if (head >= p.heads || sub >= rl) return;
  const float inv_d = 1.f / (float)p.d;
  const int64_t r0 = p.rows * blockIdx.x / row_parts, r1 = p.rows * (blockIdx.x + 1) / row_parts;
  float w[8 * NC], b[8 * NC], dw[8 * NC], db[8 * NC];
  load32<T, NC>(w, p.weight ? p.weight + head * p.d : nullptr, l, pieces, 1.f);
  load32<T, NC>(b, p.bias ? p.bias + head * p.d : nullptr, l, pieces, 0.f);
#pragma unroll
  for (int i = 0; i < 8 * NC; ++i) dw[i] = db[i] = 0.f;
  for (int64_t r = r0 + sub; r < r1; r += rl) {
    const int64_t at = (r * p.heads + head) * p.d;
    float n[8 * NC], gt[8 * NC], dy[8 * NC];
    load16<T, NC>(n, p.x + at, l, pieces);
    load16<T, NC>(dy, p.dy + at, l, pieces);
    if (GATE) load16<T, NC>(gt, p.gate + at, l, pieces);
    const float rstd = normalise<T, NC>(n, l, pieces, inv_d, p.eps);
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int i = 0; i < 8 * NC; ++i) {
      const float a = n[i] * w[i] + b[i], t = GATE ? gt[i] : a;
      const float sg = SILU ? sigmoid(t) : 1.f;
      const float slope = SILU ? sg * (1.f + t * (1.f - sg)) : 1.f;
      if (GATE) gt[i] = dy[i] * a * slope;
      const float da = dy[i] * (GATE ? t * sg : slope);
      dw[i] += da * n[i];
      db[i] += da;
      dy[i] = da * w[i];
      s1 += dy[i];
      s2 += dy[i] * n[i];
    }
    s1 = lane_sum<T>(s1) * inv_d;
    s2 = lane_sum<T>(s2) * inv_d;
#pragma unroll
    for (int i = 0; i < 8 * NC; ++i) n[i] = rstd * (dy[i] - s1 - n[i] * s2);
    store16<T, NC>(p.dx + at, n, l, pieces);
    if (GATE) store16<T, NC>(p.dgate + at, gt, l, pieces);
  }
  if (!p.part) return;
  float* const out = p.part + ((int64_t)blockIdx.x * rl + sub) * 2 * p.heads * p.d + (int64_t)head * p.d;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int k = l + c * T;
    if (k >= pieces) continue;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      out[8 * k + i] = dw[8 * c + i];
      out[(int64_t)p.heads * p.d + 8 * k + i] = db[8 * c + i];
    }
  }
}

// dweight, dbias: the partial sums in order. 64 channels a workgroup, four
// wavefronts with every fourth part each.
__global__ __launch_bounds__(256) void head_norm_sum_kernel(const float* part, int parts, int width, float* dweight,
                                                            float* dbias) {
  __shared__ float s[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int i = blockIdx.x * 64 + lane;  // of 2 * width
  float a = 0.f;
  if (i < 2 * width)
    for (int k = wave; k < parts; k += 4) a += part[(int64_t)k * 2 * width + i];
  s[wave][lane] = a;
  __syncthreads();
  if (wave == 0 && i < 2 * width) {
    a = (s[0][lane] + s[1][lane]) + (s[2][lane] + s[3][lane]);
    if (i < width) {
      if (dweight) dweight[i] = a;
    } else if (dbias) {
      dbias[i - width] = a;
    }
  }
}

template <class F>
hipError_t with_shape(int d, F f) {
  const int pieces = d / 8;
  if (pieces <= 1) return f(std::integral_constant<int, 1>{}, std::integral_constant<int, 1>{});
  if (pieces <= 2) return f(std::integral_constant<int, 2>{}, std::integral_constant<int, 1>{});
  if (pieces <= 4) return f(std::integral_constant<int, 4>{}, std::integral_constant<int, 1>{});
  if (pieces <= 8) return f(std::integral_constant<int, 8>{}, std::integral_constant<int, 1>{});
  if (pieces <= 16) return f(std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{});
  if (pieces <= 32) return f(std::integral_constant<int, 32>{}, std::integral_constant<int, 1>{});
  if (pieces <= 64) return f(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
  return f(std::integral_constant<int, 64>{}, std::integral_constant<int, 2>{});
}

}  // namespace

hipError_t launch_head_norm_fwd(const HeadNormParams& p, hipStream_t stream) {
  return with_shape(p.d, [&](auto t, auto nc) {
    constexpr int T = decltype(t)::value, NC = decltype(nc)::value;
    const int64_t units = p.rows * p.heads, per = 256 / T;
    const dim3 grid((unsigned)std::min<int64_t>((units + per - 1) / per, 8192));
    if (p.gate && p.silu) head_norm_fwd_kernel<T, NC, true, true><<<grid, 256, 0, stream>>>(p);
    else if (p.gate) head_norm_fwd_kernel<T, NC, true, false><<<grid, 256, 0, stream>>>(p);
    else if (p.silu) head_norm_fwd_kernel<T, NC, false, true><<<grid, 256, 0, stream>>>(p);
    else head_norm_fwd_kernel<T, NC, false, false><<<grid, 256, 0, stream>>>(p);
    return hipGetLastError();
  });
}

hipError_t launch_head_norm_bwd(const HeadNormParams& p, hipStream_t stream) {
  const hipError_t e = with_shape(p.d, [&](auto t, auto nc) {
    constexpr int T = decltype(t)::value, NC = decltype(nc)::value;
    const HeadNormGrid g = head_norm_grid(p.rows, p.heads, p.d);
    const dim3 grid(g.row_parts, g.head_blocks);
    if (p.gate && p.silu) head_norm_bwd_kernel<T, NC, true, true><<<grid, 256, 0, stream>>>(p, g.heads, g.row_parts);
    else if (p.gate) head_norm_bwd_kernel<T, NC, true, false><<<grid, 256, 0, stream>>>(p, g.heads, g.row_parts);
    else if (p.silu) head_norm_bwd_kernel<T, NC, false, true><<<grid, 256, 0, stream>>>(p, g.heads, g.row_parts);
    else head_norm_bwd_kernel<T, NC, false, false><<<grid, 256, 0, stream>>>(p, g.heads, g.row_parts);
    return hipGetLastError();
  });
  if (e != hipSuccess || !p.part) return e;
  const int width = p.heads * p.d;
  head_norm_sum_kernel<<<(2 * width + 63) / 64, 256, 0, stream>>>(p.part, head_norm_grid(p.rows, p.heads, p.d).parts,
                                                                  width, p.dweight, p.dbias);
  return hipGetLastError();
}

}  // namespace augtree
