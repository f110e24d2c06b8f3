// Rotation of 8 pairs held in fp32, rounded to bf16 once: shared by the read-back of packed keys and the norm of
// queries and keys.
#pragma once

#include <math.h>

#include "ct_internal.h"

namespace ct {

// The frequencies of fill_rope_table as products of theta^(-2 2^i / D): six powers instead of 64, because calls with few
// rows last as long as the host takes to launch them (0.45 us of 5).  Six roundings in fp64 at most: 1e-9 rad at position
// 2^20.
inline void fill_rope_products(const ct_layer_cfg* cfg, RopeTable* t) {
  double step[6];
  for (int i = 0; i < 6; ++i) step[i] = pow(cfg->rope_theta, -2.0 * (double)(1 << i) / (double)cfg->head_dim);
  t->turns[0] = 1.0 / 6.283185307179586476925286766559;
  for (int j = 1; j < 64; ++j) t->turns[j] = t->turns[j & (j - 1)] * step[__builtin_ctz(j)];
}

// A thread jg of the D / 16 of a head row owns the 16-byte pieces at elements 8 jg and D / 2 + 8 jg, neighbours next to
// each other in both rotation styles, so that a store fills whole lines (with STYLE 1 pieces of one thread side by
// side, streaming stores took up to 1.7 times as long).  Its pairs: STYLE 0 the elements (i, i + D / 2) of both pieces;
// STYLE 1 four pairs (2 j, 2 j + 1) in each.  pair_of: the rotation pair, and so the frequency, of its pair i.
template <int D>
__device__ __forceinline__ int piece_a(int jg) { return jg * 8; }
template <int D>
__device__ __forceinline__ int piece_b(int jg) { return jg * 8 + D / 2; }
template <int D, int STYLE>
__device__ __forceinline__ int pair_of(int jg, int i) {
  return STYLE == 0 ? jg * 8 + i : jg * 4 + i % 4 + i / 4 * (D / 4);
}

__device__ __forceinline__ void widen8(u32x4 x, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = bf16_lo(x[i]);
    f[2 * i + 1] = bf16_hi(x[i]);
  }
}

// STYLE 0: pair i is element i of `a` and of `b`; STYLE 1: elements 2i and 2i + 1 of the 16 in `a`, then `b`.
template <int STYLE>
__device__ __forceinline__ void rotate8(const float (&a)[8], const float (&b)[8], const float (&cs)[8], const float (&sn)[8],
                                        u32x4& ra, u32x4& rb) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int e = 2 * i, f = 2 * i + 1;
    if (STYLE == 0) {
      ra[i] = pack_bf16(a[e] * cs[e] - b[e] * sn[e], a[f] * cs[f] - b[f] * sn[f]);
      rb[i] = pack_bf16(a[e] * sn[e] + b[e] * cs[e], a[f] * sn[f] + b[f] * cs[f]);
    } else {
      ra[i] = pack_bf16(a[e] * cs[i] - a[f] * sn[i], a[e] * sn[i] + a[f] * cs[i]);
      rb[i] = pack_bf16(b[e] * cs[4 + i] - b[f] * sn[4 + i], b[e] * sn[4 + i] + b[f] * cs[4 + i]);
    }
  }
}

}  // namespace ct
