// The block step that the forward attention kernels share: 32 (query row, head)
// pairs of a wavefront, one per lane column, against blocks of 64 keys whose K
// and V lie in swizzled LDS tiles.
//
// Per block: 16 MFMAs for S^T = K Q^T (d = 128; K rows from LDS, Q^T in
// registers), the online-softmax update in fp32 with exp2 (the output is
// rescaled only when a row maximum grows), and 16 MFMAs for O^T += V^T P^T (V^T
// by transpose reads of the row-major V tile, P^T straight from the S^T
// accumulators rounded to bf16). The step of block b forms the scores of block
// b + 1: its S MFMAs are interleaved one by one with the exponentials of block b
// (explicit scheduling groups), so one wavefront keeps the matrix cores and the
// vector ALUs busy together. LDS addresses come from per-lane offset tables
// computed once, and operand reads run a few MFMAs ahead of their MFMA.
#pragma once

#include "common.h"

namespace augtree {

constexpr int FWD_DEPTH = 4;  // LDS operand reads run this many MFMAs ahead
constexpr int PV_DEPTH = 3;   // the same for the P V MFMAs (two reads each)
constexpr int FWD_VALU_PER_MFMA = 7;  // softmax instructions placed after each S MFMA
// The exponent reference of a row (its running maximum) moves only when a
// block's maximum exceeds it by more than this many powers of two. Exact: the
// reference cancels between numerator and denominator; P stays <= 2^8, far
// inside the fp32 and bf16 ranges.
constexpr float RESCALE_MARGIN_LOG2 = 8.f;

template <int D, class Max = MaxPlain>
struct FwdCore {
  static constexpr int BN = kFwdBlockN;  // keys per block

  bf16x8 qreg[D / 16];  // Q^T operand (B of S^T = K Q^T): lane holds its pair's query, d = 16*ks + 8*hf .. +7
  f32x16 oacc[D / 32];
  float c;      // scale in powers of two
  float m_run;  // running max of raw q.k over this lane's query
  float l_run;  // this half-wave's share of the running sum
  int hf;
  RowOffsets<D> k_off;    // K row l32; row 32 + l32 has the same swizzle, 32 rows further
  TrOffsets<D> vtr_off;  // V^T operands

  __device__ __forceinline__ void load_q(const uint16_t* q) {
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) qreg[ks] = as_bf16x8(ldg16(q + hf * 8 + ks * 16));
  }

  __device__ __forceinline__ void init(float scale_log2, int l32, int lane) {
    c = scale_log2;
    m_run = -INFINITY;
    l_run = 0.f;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) oacc[db][i] = 0.f;
    k_off.init(l32, hf);
    vtr_off.init(0, lane);
  }

  // S^T of one 64-key block (two 32-key halves), raw scores
  __device__ __forceinline__ void s_mfma(const __bf16* kl, f32x16& s0, f32x16& s1) const {
#pragma unroll
    for (int i = 0; i < 16; ++i) { s0[i] = 0.f; s1[i] = 0.f; }
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      s0 = mfma32(lds_row8_at<D>(kl, k_off.o[ks]), qreg[ks], s0);
      s1 = mfma32(lds_row8_at<D>(kl + 32 * D, k_off.o[ks]), qreg[ks], s1);
    }
  }

  // mask (keys of the block behind limit(), where masked(), which is uniform),
  // running max and (when it grew) rescale for a block; returns the exponent
  // offset of the block
  template <class Masked, class Limit>
  __device__ __forceinline__ float stats(Masked masked, Limit limit, f32x16& s0, f32x16& s1) {
    if (masked()) {
      const int lim = limit();
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        if (acc_row(i, hf) > lim) s0[i] = -INFINITY;
        if (acc_row(i, hf) + 32 > lim) s1[i] = -INFINITY;
      }
    }
    // four independent chains of three-input maxima (v_max3_f32, written
    // out: left to itself the compiler pairs the values with two-input maxima
    // first and needs about a third more instructions), and the half-wave
    // exchange without LDS
    auto max3 = [](float a, float b, float c) {
      float r;
      asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
      return r;
    };
    float m4[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float m = max3(s0[j], s1[j], s0[j + 4]);
      m = max3(m, s1[j + 4], s0[j + 8]);
      m = max3(m, s1[j + 8], s0[j + 12]);
      m4[j] = Max::of(m, s1[j + 12]);
    }
    const float mx = pair_max<Max>(Max::of(max3(m4[0], m4[1], m4[2]), m4[3]));
    const float mnew = Max::of(m_run, mx);
    // rescale only when some row maximum of this wavefront passed its
    // reference by more than the margin (always on a row's first visible key:
    // the reference starts at -inf)
    if (__any(mx * c > m_run * c + RESCALE_MARGIN_LOG2)) {
      const float alpha = (mnew == -INFINITY) ? 1.f : __builtin_amdgcn_exp2f((m_run - mnew) * c);
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) oacc[db][i] *= alpha;
      m_run = mnew;
    }
    return (m_run == -INFINITY) ? 0.f : m_run * c;
  }

  // One block step, first half: the softmax. Scores of the block arrive in s0/s1
  // (computed one step earlier); the S MFMAs of the next block (next(), s_mfma or
  // the like) are interleaved one by one with the exponentials, row sums and bf16
  // conversion (to pb) of this one, so the matrix cores and the vector ALUs of
  // the wavefront work at the same time. On the last block the extra S is
  // computed from a stale buffer and never used.
  template <class Masked, class Limit, class Next>
  __device__ __forceinline__ void softmax(Masked masked, Limit limit, f32x16& s0, f32x16& s1, Next next, bf16x8 (&pb)[4]) {
    const float ms = stats(masked, limit, s0, s1);
    __builtin_amdgcn_sched_barrier(0);
    next();
    float l4[4];  // four independent partial sums
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s0[i] = __builtin_amdgcn_exp2f(s0[i] * c - ms);
      s1[i] = __builtin_amdgcn_exp2f(s1[i] * c - ms);
      l4[i & 3] = i < 4 ? s0[i] + s1[i] : l4[i & 3] + (s0[i] + s1[i]);
    }
    l_run += (l4[0] + l4[1]) + (l4[2] + l4[3]);
    pb[0] = to_bf16x8(s0, 0);
    pb[1] = to_bf16x8(s0, 8);
    pb[2] = to_bf16x8(s1, 0);
    pb[3] = to_bf16x8(s1, 8);
    // 16 MFMAs with one K read each (reads run FWD_DEPTH ahead), the ~112
    // vector instructions of the softmax spread over them
    __builtin_amdgcn_sched_group_barrier(0x100, FWD_DEPTH, 0);
#pragma unroll
    for (int i = 0; i < D / 8; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      if (i < D / 8 - FWD_DEPTH) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x402, FWD_VALU_PER_MFMA, 0);
    }
  }

  // All of it: the softmax, then O += V^T P^T.
  template <class Masked, class Limit>
  __device__ __forceinline__ void step(Masked masked, Limit limit, f32x16& s0, f32x16& s1, const __bf16* kn,
                                       const __bf16* vl, f32x16& n0, f32x16& n1) {
    bf16x8 pb[4];
    softmax(masked, limit, s0, s1, [&] { s_mfma(kn, n0, n1); }, pb);
    set_wave_priority<1>();
    // k-step outer, output column block inner: consecutive MFMAs go to
    // different accumulators (each still sums its four k-steps in order)
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
#pragma unroll
      for (int db = 0; db < D / 32; ++db) oacc[db] = mfma32(vtr_off.read(vl, ks, db), pb[ks], oacc[db]);
    pace_lds_mfma<D / 8, 2, PV_DEPTH>();
    set_wave_priority<0>();
  }
};

}  // namespace augtree
