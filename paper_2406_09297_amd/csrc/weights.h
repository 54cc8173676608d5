// From the scores of a tile to the weights of an online softmax, shared by the
// attention kernels of the long-context operators.
#pragma once

#include <hip/hip_runtime.h>

#include "tile.h"

namespace mlkv {

// Maximum of eight multiply-add results: canonical numbers, of which the
// compiler forms three-input maxima without canonicalising each first.
__device__ __forceinline__ float max_of8(const float (&x)[8]) {
  return fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])),
               fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
}

// How far (log2) the reference lies above the row's maximum where it is set.
// With it weights stay <= 2^-24 = 2^(kLazyRescale - kLead): their sums over 2^24
// values of bf16's largest magnitude, and their products with a 4-bit block's
// power of two, stay finite, which weights up to 2^kLazyRescale did not.  At the
// other end weights and products below 2^-126 are lost, beside a denominator of
// 2^-kLead or more: 2^-94 max(1, |v|) of the result for each position.
constexpr float kLead = 32.f;

// A row that has attended nothing yet.
template <int D>
__device__ __forceinline__ void clear_rows(WaveState<D>& st) {
  st.m = 0.f;
  st.den = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int db = 0; db < Tile<D>::DB; ++db) st.acc[db] = f32x4{0.f, 0.f, 0.f, 0.f};
}

// x[c][e], the raw score of token 8 grp + e for this lane's row of block c (-inf
// where it is not attended), becomes its weight 2^(x scale - m), and pf the
// same rounded to bf16 (the matrix cores multiply values by 16-bit operands;
// half a step is 2^-8 of a weight, and as the denominator sums the same rounded
// weights, a row of ones times P^T, an error moves a result only by what its value
// differs from the result).  The reference m is kLead above the row's maximum in
// the first tile of which it attends something (until then the denominator is
// zero) and is moved only when a tile exceeds that maximum by more than
// kLazyRescale; one vote of the wave decides whether any row's is.  A score that
// is not a number, or a maximum of +-inf, makes the denominator NaN or leaves it
// zero, and the quotient NaN.
template <int D, int NB>
__device__ __forceinline__ void weigh_rows(WaveState<D> (&st)[NB], float (&x)[NB][8],
                                           float scale_log2, bf16x8 (&pf)[NB]) {
  bool move = false;
#pragma unroll
  for (int c = 0; c < NB; ++c) {
    const float neg_m = -st[c].m;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[c][e] = fmaf(x[c][e], scale_log2, neg_m);
    move |= max_of8(x[c]) > kLazyRescale - kLead || st[c].den[0] == 0.f;
  }
  if (__ballot(move)) {
#pragma unroll
    for (int c = 0; c < NB; ++c) {
      float top = max_of8(x[c]);
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const bool fresh = st[c].den[0] == 0.f;
      const bool raise = top > kLazyRescale - kLead || (fresh && top > -INFINITY);
      const float d = raise ? top + kLead : 0.f;
      const float alpha = fresh ? 1.f : fast_exp2(-d);
      st[c].m += d;
      st[c].den *= alpha;
#pragma unroll
      for (int db = 0; db < Tile<D>::DB; ++db) st[c].acc[db] *= alpha;
#pragma unroll
      for (int e = 0; e < 8; ++e) x[c][e] -= d;
    }
  }
  const u16x8 ones = {0x3F80, 0x3F80, 0x3F80, 0x3F80, 0x3F80, 0x3F80, 0x3F80, 0x3F80};
#pragma unroll
  for (int c = 0; c < NB; ++c) {
    u16x8 bits;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[c][e] = fast_exp2(x[c][e]);
      bits[e] = f32_to_bf16_bits(x[c][e]);
    }
    pf[c] = as_bf16(bits);
    st[c].den = mfma_bf16(as_bf16(ones), pf[c], st[c].den);
  }
}

}  // namespace mlkv
