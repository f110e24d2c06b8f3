// Layout of a packed K/V cache and the conversions of its elements, shared by the kernels that write, read back and
// attend over it.
//
// Elements are held in 4 bits (e2m1) or 8 (e4m3) with one scale 2^e, a byte e + 127, for 32 consecutive elements of a
// head row: the element types that gfx950 converts to and from bf16 with the scale applied, two elements an
// instruction, at the rate of a multiply-add (54 lanes per cycle and compute unit measured for both; rounding to the
// nearest, ties to even, checked over all bf16 values).  A scale byte of 255 stands for NaN and makes its 32
// elements NaN.
//
// Rows lie in blocks of 32; a block holds, per KV head and in one piece, the codes of its 32 K rows, of its 32 V
// rows, and their scales: everything that one MFMA step of the attention (32 keys) needs of a head is contiguous and
// starts on a 128-byte line, and a run of whole blocks is contiguous for all heads.
//   K codes   [32 rows][D]: the A operand of S^T = K Q^T takes D / 4 elements of one row per lane
//   V codes   [4 key groups][16 lanes][8 rows][D / 16]: the A operand of O^T += V^T P^T wants 8 keys of one
//             dimension in a lane; a lane that holds 8 keys x D / 16 dimensions gets there with one v_perm per
//             pair of elements, and nothing goes through LDS
// Lanes load 16 bytes at a time; where a lane's share is longer, the first 16 bytes of all lanes lie together, then the
// second (so that streaming loads, which do not find the rest of a line in a cache, use it whole).
//   K scales  [D / 32][32], rows in the order in which a lane of the two 16-key MFMA tiles needs them
//   V scales  [D / 32][32 rows]
#pragma once

#include "ct_internal.h"

namespace ct {

constexpr int kPackRows = 32;      // rows per block
constexpr int kPackGroup = 32;     // elements per scale
constexpr int kScaleMin = 10;      // lowest scale byte: 2^-117, so that every non-zero element is a normal bf16 number
constexpr int kScaleNaN = 255;

template <int D, int BITS>
struct PackLayout {
  static constexpr int kRowBytes = D * BITS / 8;               // codes of one K row
  static constexpr int kCodeBytes = kPackRows * kRowBytes;     // of one tensor, head and block
  static constexpr int kScaleBytes = D;                        // D / 32 groups x 32 rows
  static constexpr int kVCodes = kCodeBytes, kKScales = 2 * kCodeBytes, kVScales = 2 * kCodeBytes + kScaleBytes;
  static constexpr int kBytes = 2 * (kCodeBytes + kScaleBytes);   // one head of one block
  static constexpr int kLaneDims = D / 16;                     // V dimensions per lane
  static constexpr int kLaneBytes = kLaneDims * BITS / 8;      // of one key

  // A lane's share of a K row or of V (16, 32 or 64 bytes, or 8) lies in quads of 16 bytes, the same quad of neighbouring
  // lanes side by side.
  static constexpr int kShareK = kRowBytes / 4;
  static __device__ __forceinline__ int k_code(int row, int dim) {
    const int byte = dim * BITS / 8, in = byte % kShareK;
    return row * kRowBytes + (kShareK <= 16 ? byte : in / 16 * 64 + byte / kShareK * 16 + in % 16);
  }
  static __device__ __forceinline__ int v_code(int row, int dim) {
    const int lane = (row >> 3) * 16 + dim / kLaneDims, in = (row & 7) * kLaneBytes + dim % kLaneDims * BITS / 8;
    return kVCodes + in / 16 * 1024 + lane * 16 + in % 16;
  }
  static __device__ __forceinline__ int k_scale(int row, int group) {
    return kKScales + group * kPackRows + (row & 24) + (row & 3) * 2 + ((row >> 2) & 1);
  }
  static __device__ __forceinline__ int v_scale(int row, int group) { return kVScales + group * kPackRows + row; }
};

inline size_t pack_block_bytes(const ct_layer_cfg* cfg, int bits) {
  return (size_t)cfg->n_kv_heads * 2 * (kPackRows * cfg->head_dim * bits / 8 + cfg->head_dim);
}

#if defined(__HIPCC__)
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }
// Scale byte I of a word.  The conversions look at the exponent of their scale alone (checked: all 256 bytes with 64
// patterns in sign and mantissa), so the other bytes may stay.
template <int I>
__device__ __forceinline__ float scale_in(uint32_t w) {
  return __uint_as_float(I == 3 ? w >> 1 : w << (23 - 8 * I));
}

// Byte (two elements, 4 bits each) or halfword (8 bits each) PART of a word of codes, scaled, as a pair of bf16.
template <int BITS, int PART>
__device__ __forceinline__ uint32_t unpack_pair(uint32_t w, float scale) {
  bf16x2 p;
  if constexpr (BITS == 4) p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, PART);
  else p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, PART != 0);
  return __builtin_bit_cast(uint32_t, p);
}
// Eight elements (one word of 4-bit codes, two of 8-bit ones) as four pairs of bf16.
template <int BITS>
__device__ __forceinline__ u32x4 unpack8(const uint32_t* w, float scale) {
  if constexpr (BITS == 4)
    return u32x4{unpack_pair<4, 0>(w[0], scale), unpack_pair<4, 1>(w[0], scale), unpack_pair<4, 2>(w[0], scale),
                 unpack_pair<4, 3>(w[0], scale)};
  else
    return u32x4{unpack_pair<8, 0>(w[0], scale), unpack_pair<8, 1>(w[0], scale), unpack_pair<8, 0>(w[1], scale),
                 unpack_pair<8, 1>(w[1], scale)};
}

// Scale byte of a group from its largest magnitude, given as the bf16 pattern without its sign: the smallest e >= -117
// with max <= 1.75 2^emax 2^e, emax = 2 for e2m1 (7, which rounds to 6: an error of half the step there; normal values are
// off by 11.2 % in relative 2-norm, by 11.5 % with a limit of 6 or 8) and 8 for e4m3 (448, its largest value).
template <int BITS>
__device__ __forceinline__ uint32_t scale_byte(uint32_t max_bits) {
  constexpr int EMAX = BITS == 4 ? 2 : 8;
  if (max_bits >= 0x7f80u) return kScaleNaN;
  const int b = (int)(max_bits >> 7) - EMAX + ((max_bits & 0x7fu) > 0x60u);
  return b < kScaleMin ? kScaleMin : b;
}
// Magnitudes above 1.75 * 2^127 are taken for that: rounded up they would come back as infinities, which not even a
// probability of zero silences.
constexpr uint32_t kMaxBits = 0x7f60u;
__device__ __forceinline__ uint32_t clamp_pair(uint32_t w) {
  const uint32_t lo = min(w & 0x7fffu, kMaxBits), hi = min((w >> 16) & 0x7fffu, kMaxBits);
  return (w & 0x80008000u) | hi << 16 | lo;
}
// Eight bf16 elements to codes: one word (4 bits) or two (8 bits).
template <int BITS>
__device__ __forceinline__ u32x2 pack8(u32x4 x, float scale) {
  auto pair = [&](int i) { return __builtin_bit_cast(bf16x2, (uint32_t)x[i]); };
  if constexpr (BITS == 4) {
    uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(0u, pair(0), scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, pair(1), scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, pair(2), scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, pair(3), scale, 3);
    return u32x2{w, 0u};
  } else {
    typedef __attribute__((ext_vector_type(2))) short s16x2;
    u32x2 r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      s16x2 w = {0, 0};
      w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, pair(2 * i), scale, false);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, pair(2 * i + 1), scale, true);
      r[i] = __builtin_bit_cast(uint32_t, w);
    }
    return r;
  }
}
#endif

}  // namespace ct
