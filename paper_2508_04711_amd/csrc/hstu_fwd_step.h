// The software-pipelined step of the forward pass: of whole sequences (hstu_fwd.hip) and of many new rows over a paged cache
// (hstu_paged_many.hip).
#pragma once
#include "hstu_mfma.h"

namespace hstu {

namespace {

// =============================================================================================
// Forward: owners are query rows, keys and values are streamed.
//   S^T = K Q^T (A = K tile rows, B = Q registers)  ->  P^T in accumulator layout
//   O^T += V^T P^T (A = V tile transposed read, B = P^T registers)
// =============================================================================================

// The stream of keys is processed in blocks of 32, software-pipelined across blocks and tiles.
// Step i issues, interleaved and independent of each other,
//   the matrix instructions of S(i+1) = K(i+1) Q^T              (DQK/16 instructions),
//   the matrix instructions of O^T += V(i-1)^T P(i-1)^T          (DV/16 instructions),
//   the SiLU that turns S(i) into P(i)                           (vector instructions),
// so that every wave's instruction stream is an even mix of matrix and vector work: two waves
// of a SIMD then keep both pipes busy whatever their relative phase (a matrix instruction
// holds its own wave's issue for a while, the other wave's vector instructions fill that time).
// Two S accumulator sets and two P operand sets alternate by block parity.
//
// Causal mask: key r (accumulator element) of block i is visible to the lane's query iff
// 8*(r/4) + 4*hh + r%4 <= rel, rel = query position - block position; applied to the finished
// P under a wave-uniform branch, so the matrix instructions follow one path whether or not a
// block is masked.  A block none of whose keys is visible comes out as zeros.
template <int DQK, int DV, bool PV, class VAddr, class Init, class Vis>
__device__ __forceinline__ void fwd_step(const Init& init, const char* kn, int bn, const char* vp, int bp,
                                         const RowAddr<DQK>& ra, const VAddr& ca,
                                         const bf16x8 (&qreg)[DQK / 16], const f32x16& s_in,
                                         f32x16& s_out, const bf16x8 (&p_prev)[2],
                                         bf16x8 (&p_cur)[2], f32x16 (&oacc)[DV / 32], float c1,
                                         bool mask, const Vis& vis_of) {
  constexpr int KS = DQK / 16, NPV = DV / 16, NSL = KS > NPV ? KS : NPV;
  constexpr int AHEAD = 3;  // operand reads in flight ahead of their use
  bf16x8 ka[KS], va[NPV];
  auto fence = [] { __builtin_amdgcn_sched_barrier(0); };
  init(s_out);
#pragma unroll
  for (int m = 0; m < AHEAD; ++m) {
    if (m < KS) ka[m] = ra.read(kn, bn, m);
    if (PV && m < NPV) va[m] = ca.read(vp, bp * 2 + (m & 1), m >> 1);
  }
  fence();
  float p[16];
#pragma unroll
  for (int m = 0; m < NSL; ++m) {
    const int e0 = m * 16 / NSL, e1 = (m + 1) * 16 / NSL, em = (e0 + e1 + 1) / 2;
    if (m < KS) s_out = mfma(ka[m], qreg[m], s_out);
    if (m + AHEAD < KS) ka[m + AHEAD] = ra.read(kn, bn, m + AHEAD);
#pragma unroll
    for (int e = e0; e < em; ++e) p[e] = s_in[e] * sigmoid_scaled(s_in[e], c1);
    fence();
    if (PV && m < NPV) oacc[m >> 1] = mfma(va[m], p_prev[m & 1], oacc[m >> 1]);
    if (PV && m + AHEAD < NPV) va[m + AHEAD] = ca.read(vp, bp * 2 + ((m + AHEAD) & 1), (m + AHEAD) >> 1);
#pragma unroll
    for (int e = em; e < e1; ++e) p[e] = s_in[e] * sigmoid_scaled(s_in[e], c1);
    fence();
  }
  if (mask) {
    asm volatile("" ::: "memory");  // not speculable: keeps the selects off the unmasked path
    const auto vis = vis_of();      // (the block's position is worked out on this path only)
#pragma unroll
    for (int r = 0; r < 16; ++r) p[r] = vis(r) ? p[r] : 0.f;
  }
  p_cur[0] = pack8(p);
  p_cur[1] = pack8(p + 8);
  fence();
}

}  // namespace

}  // namespace hstu
