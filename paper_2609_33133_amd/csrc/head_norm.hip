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
// holding NC pieces of 8 channels, so its sums stay inside a wavefront: exchanges
// by DPP, no LDS. A lane stays with its channels and goes down the rows, so that
// weight and bias are read once and their gradients are summed in registers.
// What else costs here is the vector ALU: the exact expf and division of the
// activation alone kept the forward at 3.2 of the 4.9 TB/s that a copy reaches.
// 49152 rows of 32 heads of 128 with a gate: forward 245 us (4.9 TB/s), backward
// 417 us (4.8 TB/s).
#include <type_traits>

#include "common.h"
#include "linear.h"

namespace augtree {
namespace {

template <int CTRL>
__device__ __forceinline__ float dpp_add(float x) {
  return x + __uint_as_float(__builtin_amdgcn_mov_dpp((int)__float_as_uint(x), CTRL, 0xf, 0xf, true));
}

// the sum over T neighbouring lanes, in each of them
template <int T>
__device__ __forceinline__ float lane_sum(float x) {
  if constexpr (T >= 2) x = dpp_add<0xB1>(x);   // quad_perm 1, 0, 3, 2
  if constexpr (T >= 4) x = dpp_add<0x4E>(x);   // quad_perm 2, 3, 0, 1
  if constexpr (T >= 8) x = dpp_add<0x141>(x);  // row_half_mirror: the other four of eight
  if constexpr (T >= 16) x = dpp_add<0x140>(x); // row_mirror: the other eight of sixteen
  if constexpr (T >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  if constexpr (T >= 64) x = pair_sum(x);
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
  // 1 ulp; the instruction takes denormals for zero (both may be one), hence the power of two
  const float var = lane_sum<T>(sq) * inv_d + eps;
  const bool tiny = var < 0x1p-126f;
  const float rstd = __builtin_amdgcn_rsqf(tiny ? var * 0x1p64f : var) * (tiny ? 0x1p32f : 1.f);
#pragma unroll
  for (int i = 0; i < 8 * NC; ++i) x[i] *= rstd;
  return rstd;
}

// 1 / (1 + e^-u) by the hardware's exp2 and reciprocal, 1 ulp each. The product
// u log2(e) is rounded once, which is off by 2^-24 |u| in the exponent.
__device__ __forceinline__ float sigmoid(float u) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(u * -1.442695041f));
}

// The lanes' place: a workgroup takes a run of hpw heads and one of row_parts
// parts of the rows, which the 256 / T / hpw groups of lanes of a head share.
template <int T>
struct Place {
  int l, head, sub, sharing;
  bool idle;
  int64_t r0, r1;
  __device__ __forceinline__ Place(const HeadNormParams& p, int hpw, int row_parts) {
    const int grp = threadIdx.x / T;
    l = threadIdx.x & (T - 1);
    sharing = 256 / T / hpw;
    sub = grp / hpw;
    head = blockIdx.y * hpw + grp - sub * hpw;
    idle = head >= p.heads || sub >= sharing;
    r0 = p.rows * blockIdx.x / row_parts;
    r1 = p.rows * (blockIdx.x + 1) / row_parts;
  }
};

template <int T, int NC, bool GATE, bool SILU>
__global__ __launch_bounds__(256) void head_norm_fwd_kernel(HeadNormParams p, int hpw, int row_parts) {
  const Place<T> at(p, hpw, row_parts);
  if (at.idle) return;
  const int l = at.l, pieces = p.d / 8;
  const float inv_d = 1.f / (float)p.d;
  float w[8 * NC], b[8 * NC];
  load32<T, NC>(w, p.weight ? p.weight + at.head * p.d : nullptr, l, pieces, 1.f);
  load32<T, NC>(b, p.bias ? p.bias + at.head * p.d : nullptr, l, pieces, 0.f);
  for (int64_t r = at.r0 + at.sub; r < at.r1; r += at.sharing) {
    const int64_t o = (r * p.heads + at.head) * p.d;
    float x[8 * NC], gt[8 * NC];
    load16<T, NC>(x, p.x + o, l, pieces);
    if (GATE) load16<T, NC>(gt, p.gate + o, l, pieces);
    normalise<T, NC>(x, l, pieces, inv_d, p.eps);
#pragma unroll
    for (int i = 0; i < 8 * NC; ++i) {
      const float a = x[i] * w[i] + b[i], t = GATE ? gt[i] : a;
      const float act = SILU ? t * sigmoid(t) : t;
      x[i] = GATE ? a * act : act;
    }
    store16<T, NC>(p.y + o, x, l, pieces);
  }
}

// Every group of lanes leaves its sums of dweight and dbias as a partial sum.
template <int T, int NC, bool GATE, bool SILU>
__global__ __launch_bounds__(256) void head_norm_bwd_kernel(HeadNormParams p, int hpw, int row_parts) {
  const Place<T> place(p, hpw, row_parts);
  if (place.idle) return;
  const int l = place.l, head = place.head, pieces = p.d / 8;
  const float inv_d = 1.f / (float)p.d;
  float w[8 * NC], b[8 * NC], dw[8 * NC], db[8 * NC];
  load32<T, NC>(w, p.weight ? p.weight + head * p.d : nullptr, l, pieces, 1.f);
  load32<T, NC>(b, p.bias ? p.bias + head * p.d : nullptr, l, pieces, 0.f);
#pragma unroll
  for (int i = 0; i < 8 * NC; ++i) dw[i] = db[i] = 0.f;
  for (int64_t r = place.r0 + place.sub; r < place.r1; r += place.sharing) {
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
  float* const out = p.part + ((int64_t)blockIdx.x * place.sharing + place.sub) * 2 * p.heads * p.d + (int64_t)head * p.d;
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

// dweight, dbias: the partial sums. 64 channels a workgroup, 16 wavefronts with
// every 16th part each (4 wavefronts took 54 us for 512 parts of 2 x 4096
// where these take 6), then the 16 in order.
__global__ __launch_bounds__(1024) void head_norm_sum_kernel(const float* part, int parts, int width, float* dweight,
                                                             float* dbias) {
  __shared__ float s[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t i = (int64_t)blockIdx.x * 64 + lane, row = 2 * (int64_t)width;
  float a = 0.f;
  if (i < row) {
#pragma unroll 8
    for (int k = wave; k < parts; k += 16) a += part[k * row + i];
  }
  s[wave][lane] = a;
  __syncthreads();
  if (wave == 0 && i < row) {
    a = 0.f;
#pragma unroll
    for (int k = 0; k < 16; ++k) a += s[k][lane];
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
    const HeadNormGrid g = head_norm_grid(p.rows, p.heads, p.d, 4096);
    const dim3 grid(g.row_parts, g.head_blocks);
    if (p.gate && p.silu) head_norm_fwd_kernel<T, NC, true, true><<<grid, 256, 0, stream>>>(p, g.heads, g.row_parts);
    else if (p.gate) head_norm_fwd_kernel<T, NC, true, false><<<grid, 256, 0, stream>>>(p, g.heads, g.row_parts);
    else if (p.silu) head_norm_fwd_kernel<T, NC, false, true><<<grid, 256, 0, stream>>>(p, g.heads, g.row_parts);
    else head_norm_fwd_kernel<T, NC, false, false><<<grid, 256, 0, stream>>>(p, g.heads, g.row_parts);
    return hipGetLastError();
  });
}

hipError_t launch_head_norm_bwd(const HeadNormParams& p, hipStream_t stream) {
  if (p.sum) {
    const int width = p.heads * p.d;
    head_norm_sum_kernel<<<(2 * width + 63) / 64, 1024, 0, stream>>>(
        p.part, head_norm_bwd_grid(p.rows, p.heads, p.d).parts, width, p.dweight, p.dbias);
    return hipGetLastError();
  }
  return with_shape(p.d, [&](auto t, auto nc) {
    constexpr int T = decltype(t)::value, NC = decltype(nc)::value;
    const HeadNormGrid g = head_norm_bwd_grid(p.rows, p.heads, p.d);
    const dim3 grid(g.row_parts, g.head_blocks);
    if (p.gate && p.silu) head_norm_bwd_kernel<T, NC, true, true><<<grid, 256, 0, stream>>>(p, g.heads, g.row_parts);
    else if (p.gate) head_norm_bwd_kernel<T, NC, true, false><<<grid, 256, 0, stream>>>(p, g.heads, g.row_parts);
    else if (p.silu) head_norm_bwd_kernel<T, NC, false, true><<<grid, 256, 0, stream>>>(p, g.heads, g.row_parts);
    else head_norm_bwd_kernel<T, NC, false, false><<<grid, 256, 0, stream>>>(p, g.heads, g.row_parts);
    return hipGetLastError();
  });
}

}  // namespace augtree
