// Attention of the newest tokens of each sequence over a packed K/V cache (ct_packed_attention): the steps that follow
// a partial prefill, one token (or a few drafted ones) per sequence at a time.
//
// Bound: the cache is read once and used for few queries, so memory decides as long as the conversion of the codes
// keeps up: an element costs one conversion instruction per two, and V one v_perm per two besides.  64 sequences of
// 4096 rows (32/8 heads of 128) 49 us in 4 bits, 5.8 TB/s; 2 of 131072 in 8 bits 85 us, 6.5 TB/s (a large copy moves
// 5.1); short calls are a launch of 5 us, and a merge of 4 behind it where the key range is divided.  With more than 16
// columns of queries the vector and matrix units decide: 16 sequences of 8192 rows with 64 columns 71 us in 4 bits.
//
// Formulation, as in the selected-row attention: S^T = K Q^T and O^T += V^T P^T on 16 x 16 x 32 matrix instructions,
// the columns being the G query heads of a KV head times the new tokens.  The cache's layout hands a lane its
// operands directly (ct_packed.h): nothing of K, V or P goes through LDS, and the waves of a workgroup walk
// alternate blocks of 32 keys without waiting for one another; they are joined once, at the end.  Key order within a
// block: lane row h takes keys 8h .. 8h + 7, in S^T as the rows 4h .. 4h + 3 of two 16-key tiles, which makes the
// scores of a lane the B operand of the PV step.
#include <algorithm>
#include <type_traits>
#include <utility>

#include "ct_packed.h"

namespace ct {

namespace {

constexpr int kWaves = 4;
constexpr int kMaxParts = 3 * kNumCUs;
constexpr int kOrdered = 256;      // sequences that are taken in the order of their lengths
// Probabilities are held as 2^-kLift of what they are, in reach of the largest values and of the smallest: sums over 2^19
// rows of up to 2^kLag * 1.75 * 2^127 stay below 2^128 (a sum that does not is an infinity, which no weight of zero
// silences when waves are joined), and a product with the smallest value of a cache, 2^-126, is still one of fp32's.
constexpr float kLift = 23.f;
constexpr float kLag = 4.f;        // binary orders by which a maximum may exceed the reference of the exponents

struct PackedAttnArgs {
  const uint16_t* q;              // [n_seq, n_new, Hq, D]
  const unsigned char* cache;
  const int32_t* seq_start;
  const int32_t* seq_len;
  uint16_t* out;
  float* lse;
  float* partial;                 // O of every part: [sequence, KV head][part][column][D]
  float* partial_ml;              // and its (m, l): [sequence, KV head][column][part]
  int32_t n_seq, n_new, n_rows, max_len;
  int32_t Hq, Hkv, group_shift;   // query heads per KV head: 1 << group_shift
  int32_t round;                  // sequences in the order of their lengths, so many to a round (see by_length); 0: as they come
  int32_t n_parts, part_blocks;   // most parts of a key range, and the blocks of 32 rows in each, about
  int32_t col_blocks;
  float scale_log2;               // softmax scale * log2(e)
};

// The rows of sequence b in the cache, and the parts its blocks are divided into.  Lengths and starts that do not
// fit the cache are cut to it.
struct Sequence {
  int32_t first, end;   // rows [first, end)
  int32_t b0, b1;       // blocks [b0, b1)
  int32_t n_parts;
};
__device__ __forceinline__ Sequence sequence_of(const PackedAttnArgs& a, int b) {
  Sequence s;
  const int32_t start = a.seq_start[b], len = min(a.seq_len[b], a.max_len);
  const bool some = start >= 0 && start < a.n_rows && len > 0;
  s.first = some ? start : 0;
  s.end = some ? start + min(len, a.n_rows - start) : 0;
  s.b0 = s.first / kPackRows;
  s.b1 = (s.end + kPackRows - 1) / kPackRows;
  s.n_parts = (s.b1 - s.b0 + a.part_blocks - 1) / a.part_blocks;
  return s;
}

// The sequence at place r of all, the longest first (of equal lengths in blocks the lower number), for up to 64 K of
// them: each wave finds it for itself, bit by bit from the top, counting lanes.
template <int K>
__device__ __forceinline__ int longest_but(const PackedAttnArgs& a, int r) {
  const int lane = threadIdx.x & 63;
  uint32_t key[K];      // blocks + 1; 0: no sequence
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int i = lane + 64 * k;
    key[k] = i < a.n_seq ? min(max(a.seq_len[i], 0), a.max_len) / kPackRows + 1 : 0;
  }
  uint32_t at = 0;      // the key at place r: the largest that more than r reach
  for (uint32_t bit = 1u << (31 - __clz(a.max_len / kPackRows + 1)); bit != 0; bit >>= 1) {
    int n = 0;
#pragma unroll
    for (int k = 0; k < K; ++k) n += __popcll(__ballot(key[k] >= (at | bit)));
    if (n > r) at |= bit;
  }
#pragma unroll
  for (int k = 0; k < K; ++k) r -= __popcll(__ballot(key[k] > at));
  int found = 0;        // the one behind r others with this key
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const uint64_t equal = __ballot(key[k] == at);
    const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(equal >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)equal, 0));
    const uint64_t it = __ballot(key[k] == at && before == r);
    if (it != 0) found = 64 * k + __ffsll((unsigned long long)it) - 1;
    r -= __popcll(equal);
  }
  return found;
}

// Which sequence a workgroup takes, of those that are not divided.  Workgroups go to the compute units in rounds; the
// first round takes the longest sequences, the longest ahead, the second the next ones from its shortest on, and so
// forth, so that units get about as much each.
__device__ __forceinline__ int by_length(const PackedAttnArgs& a, int place) {
  const int first = place / a.round * a.round;
  const int r = place / a.round % 2 == 0 ? place : first + min(first + a.round, a.n_seq) - 1 - place;
  return a.n_seq <= 64 ? longest_but<1>(a, r) : longest_but<kOrdered / 64>(a, r);
}

template <int N, typename F, int... I>
__device__ __forceinline__ void static_for_impl(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void static_for(F&& f) {
  static_for_impl<N>(f, std::make_integer_sequence<int, N>{});
}

// Over the four 16-lane rows of a wave.
template <typename Op>
__device__ __forceinline__ float reduce_rows_one(float x, Op op) {
  uint32_t u = __float_as_uint(x);
  auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  u = __float_as_uint(op(__uint_as_float(r[0]), __uint_as_float(r[1])));
  r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return op(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// What a lane holds of one block of 32 rows.
template <int D, int BITS>
struct Raw {
  static constexpr int KW = D / 4 * BITS / 32;    // words of one K row
  static constexpr int VW = D / 16 * BITS / 4;    // words of 8 keys x D / 16 dimensions of V
  uint32_t k[2][KW];
  uint32_t v[VW];
  uint32_t ks;      // two scale bytes
  uint32_t vs[2];   // eight
};

// (STRIDE: bytes between the 16-byte quads of a lane)
template <int STRIDE, bool STREAM, int W>
__device__ __forceinline__ void load_words(uint32_t (&dst)[W], const unsigned char* p) {
  if constexpr (W % 4 == 0) {
#pragma unroll
    for (int i = 0; i < W; i += 4) {
      const u32x4* q = reinterpret_cast<const u32x4*>(p + i / 4 * STRIDE);
      const u32x4 x = STREAM ? __builtin_nontemporal_load(q) : *q;
      dst[i] = x[0]; dst[i + 1] = x[1]; dst[i + 2] = x[2]; dst[i + 3] = x[3];
    }
  } else {
    static_assert(W == 2, "words per lane");
    const u32x2 x = *reinterpret_cast<const u32x2*>(p);
    dst[0] = x[0]; dst[1] = x[1];
  }
}

// Pair e2 (dimensions 2 e2, 2 e2 + 1 of the lane's) of key s.
template <int D, int BITS, int S, int E2>
__device__ __forceinline__ uint32_t v_pair(const uint32_t* v, float scale) {
  constexpr int byte = (S * (D / 16) + 2 * E2) * BITS / 8;
  return unpack_pair<BITS, BITS == 4 ? byte % 4 : byte % 4 / 2>(v[byte / 4], scale);
}

// STREAM: loads of codes that do not stay in the caches (see stream_loads).
// Registers for three waves per SIMD (16 columns) or two (32): left alone the compiler keeps the accumulators in
// registers of their own and two waves, or one, remain.
template <int D, int BITS, int NT, bool STREAM>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(NT == 1 ? 3 : 2))) void packed_attn_kernel(PackedAttnArgs a) {
  using L = PackLayout<D, BITS>;
  using R = Raw<D, BITS>;
  constexpr int KS = D / 32;
  constexpr int MT = L::kLaneDims;      // O^T tiles: row j of tile m is dimension j * MT + m
  const int lane = threadIdx.x & 63, l16 = lane & 15, h = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  uint32_t rest = blockIdx.x;
  auto next_of = [&](uint32_t n) __attribute__((always_inline)) {
    const uint32_t q = rest / n, r = rest - q * n;
    rest = q;
    return (int)r;
  };
  const int g = next_of(a.Hkv), cb = next_of(a.col_blocks), part = next_of(a.n_parts);
  const int b = a.round > 0 ? by_length(a, (int)rest) : (int)rest;
  const Sequence seq = sequence_of(a, b);
  if (part >= max(seq.n_parts, 1)) return;            // (an empty sequence still gets its zeros, from part 0)

  // ---- this lane's columns: column c is head c mod G of new token c / G --------------------------------
  const int G = 1 << a.group_shift;
  const int n_cols = a.n_new << a.group_shift;
  const int col0 = cb * 16 * NT;
  bf16x8 qf[NT][KS];
  int32_t last[NT];                                   // the last row that the column sees
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int c = min(col0 + 16 * n + l16, n_cols - 1);
    const int t = c >> a.group_shift;
    last[n] = seq.end - a.n_new + t;
    const uint16_t* qp = a.q + (((int64_t)b * a.n_new + t) * a.Hq + g * G + (c & (G - 1))) * D + h * (D / 4);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[n][ks] = *reinterpret_cast<const bf16x8*>(qp + 8 * ks);
  }
  const int32_t first_last = seq.end - a.n_new + (col0 >> a.group_shift);   // the lowest of `last`

  // ---- where a lane finds its share of a block -------------------------------------------------------
  const int k_row = 8 * (l16 >> 2) + (l16 & 3);       // row of 16-key tile 0; tile 1: 4 rows further on
  const uint32_t k_off = k_row * L::kRowBytes + h * (L::kShareK < 16 ? L::kShareK : 16);
  const int out_group = h * (D / 4) / kPackGroup;     // scale group of the K dimensions, and of the output dimensions
  const uint32_t ks_off = L::kKScales + out_group * kPackRows + 2 * l16;
  const uint32_t v_off = L::kVCodes + lane * 16;
  const uint32_t vs_off = L::kVScales + l16 * MT / kPackGroup * kPackRows + 8 * h;
  auto block_ptr = [&](int blk) __attribute__((always_inline)) {
    return a.cache + ((int64_t)blk * a.Hkv + g) * L::kBytes;
  };
  auto load = [&](R& r, int blk) __attribute__((always_inline)) {
    const unsigned char* p = block_ptr(blk);
    load_words<64, STREAM>(r.k[0], p + k_off);
    load_words<64, STREAM>(r.k[1], p + k_off + 4 * L::kRowBytes);
    r.ks = *reinterpret_cast<const uint16_t*>(p + ks_off);
    load_words<1024, STREAM>(r.v, p + v_off);
    load_words<0, false>(r.vs, p + vs_off);
  };

  // ---- state -----------------------------------------------------------------------------------------
  f32x4 o[MT][NT];
  float m_run[NT], m_limit[NT], l_run[NT];
  const float limit_step = kLag / a.scale_log2;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    m_run[n] = m_limit[n] = -INFINITY;
    l_run[n] = 0.f;
#pragma unroll
    for (int m = 0; m < MT; ++m) o[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  auto compute = [&](R& r, int blk) __attribute__((always_inline)) {
    // scores
    f32x4 s[2][NT];
    const float k_scale[2] = {scale_in<0>(r.ks), scale_in<1>(r.ks)};
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const u32x4 kw = unpack8<BITS>(&r.k[u][ks * BITS / 4], k_scale[u]);
        const bf16x8 kf = __builtin_bit_cast(bf16x8, kw);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
          s[u][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[n][ks], ks == 0 ? zero : s[u][n], 0, 0, 0);
        }
      }
    // Blocks that reach over an end of the sequence, or past the earliest of the new tokens: rows outside the
    // sequence may hold anything, rows that only some columns see may hold NaN.
    const int32_t row0 = blk * kPackRows;
    if (row0 < seq.first || row0 + kPackRows - 1 > first_last) {
      // Bit i of a mask stands for key 8h + i.  (Masks of bits in vector registers: comparisons key by key need more
      // scalar registers for their results than there are.)
      auto bits_below = [](int n) __attribute__((always_inline)) { return (1u << min(max(n, 0), 8)) - 1u; };
      auto spread = [](uint32_t bits, int i) __attribute__((always_inline)) { return (uint32_t)((int32_t)(bits << (31 - i)) >> 31); };
      const int base = row0 + 8 * h;
      const uint32_t from_first = ~bits_below(seq.first - base), in = from_first & bits_below(seq.end - base);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const uint32_t seen = from_first & bits_below(last[n] + 1 - base);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t m = spread(seen, i);
          s[i / 4][n][i % 4] = __uint_as_float((__float_as_uint(s[i / 4][n][i % 4]) & m) | (0xff800000u & ~m));
        }
      }
      // A probability of zero does not silence a NaN: such elements of V become zeros here, and NaN goes to the
      // columns that do see one.
      uint32_t nan = 0;      // scale bytes of 255
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const uint32_t top = ((r.vs[w] & 0x7f7f7f7fu) + 0x01010101u) & r.vs[w] & 0x80808080u;
        nan |= ((top >> 7) * 0x10204080u >> 28) << (4 * w);      // bits 0, 8, 16, 24 next to one another
      }
      const uint32_t keep = in & ~nan;
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const uint32_t bytes = ((keep >> (4 * w) & 15u) * 0x00204081u & 0x01010101u) * 255u;
        r.vs[w] = (r.vs[w] & bytes) | (0x7f7f7f7fu & ~bytes);
      }
#pragma unroll
      for (int w = 0; w < R::VW; ++w) {
        if constexpr (L::kLaneBytes == 2) r.v[w] &= (spread(keep, 2 * w) & 0xffffu) | spread(keep, 2 * w + 1) << 16;
        else r.v[w] &= spread(keep, 4 * w / L::kLaneBytes);
      }
      if (__any((in & nan) != 0)) {
        const unsigned char* vs = block_ptr(blk) + L::kVScales + out_group * kPackRows;
        bool sees[NT] = {};
#pragma unroll 1
        for (int i = 0; i < kPackRows; ++i) {
          const int32_t row = row0 + i;
#pragma unroll
          for (int n = 0; n < NT; ++n) sees[n] |= vs[i] == kScaleNaN && row >= seq.first && row <= last[n];
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
          if (sees[n])
#pragma unroll
            for (int m = 0; m < MT; ++m) o[m][n] = f32x4{NAN, NAN, NAN, NAN};
      }
    }
    // Online softmax.  The reference of the exponents follows the running maximum lazily: it moves when a score exceeds
    // it by more than 2^kLag, so rescaling is rare.  (2^8 instead of 2^4: within 0.5 %.)
    float mx[NT];
    bool moves = false;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      mx[n] = m_limit[n];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) mx[n] = fmaxf(mx[n], s[u][n][i]);
      mx[n] = reduce_rows_one(mx[n], [](float x, float y) { return fmaxf(x, y); });
      moves |= mx[n] > m_limit[n];
    }
    if (__any(moves)) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
        if (mx[n] > m_limit[n]) {
          const float m_new = mx[n] * a.scale_log2 + kLift;
          const float alpha = __builtin_amdgcn_exp2f(m_run[n] - m_new);   // (0 from the first reference on)
          m_run[n] = m_new;
          m_limit[n] = mx[n] + limit_step;
          l_run[n] *= alpha;
#pragma unroll
          for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[m][n][i] *= alpha;
        }
    }
    bf16x8 pf[NT], pl[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const float m_use = m_run[n] == -INFINITY ? 0.f : m_run[n];
      float p[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i / 4][n][i % 4], a.scale_log2, -m_use));
      l_run[n] += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
      // bf16 operands: a probability is the sum of two, its rounding and the rounding of what that leaves, which is off by
      // up to 2^-16 of it; the sum above is unrounded.  (The first alone is off by up to 2^-8: outputs 0.0023 from the exact
      // ones in relative 2-norm, where their own rounding makes 0.0017.  The second product, 32/8 heads of 128: one token in
      // 8 bits 0 to 1 %, in 4 bits 1 to 6 % (64 uneven sequences up to 4099 rows 32.9 -> 33.5 us, 64 of 4096 46.7 -> 49),
      // one sequence of 1024 rows with heads of 64 5.35 -> 5.7, 64 columns over 16 sequences of 8192 rows 58 -> 71, in 8 bits
      // 75.5 -> 81.  What the rounding leaves by a dot product of bf16 pairs instead of a shift and a difference: 2 % less of
      // the slowest of these, as much of the others.)
      const u32x4 w = {pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3]), pack_bf16(p[4], p[5]), pack_bf16(p[6], p[7])};
      pf[n] = __builtin_bit_cast(bf16x8, w);
      u32x4 rest;
#pragma unroll
      for (int i = 0; i < 4; ++i) rest[i] = pack_bf16(p[2 * i] - bf16_lo(w[i]), p[2 * i + 1] - bf16_hi(w[i]));
      pl[n] = __builtin_bit_cast(bf16x8, rest);
    }
    // O^T += V^T P^T
    float v_scale[8];
    static_for<8>([&](auto sc) __attribute__((always_inline)) {
      constexpr int S = decltype(sc)::value;
      v_scale[S] = scale_in<S % 4>(r.vs[S / 4]);
    });
    static_for<MT / 2>([&](auto ec) __attribute__((always_inline)) {
      constexpr int E2 = decltype(ec)::value;
      uint32_t c[8];
      static_for<8>([&](auto sc) __attribute__((always_inline)) {
        constexpr int S = decltype(sc)::value;
        c[S] = v_pair<D, BITS, S, E2>(r.v, v_scale[S]);
      });
      u32x4 even, odd;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        even[i] = __builtin_amdgcn_perm(c[2 * i + 1], c[2 * i], 0x05040100u);
        odd[i] = __builtin_amdgcn_perm(c[2 * i + 1], c[2 * i], 0x07060302u);
      }
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        o[2 * E2][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, even), pf[n], o[2 * E2][n], 0, 0, 0);
        o[2 * E2 + 1][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, odd), pf[n], o[2 * E2 + 1][n], 0, 0, 0);
      }
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        o[2 * E2][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, even), pl[n], o[2 * E2][n], 0, 0, 0);
        o[2 * E2 + 1][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, odd), pl[n], o[2 * E2 + 1][n], 0, 0, 0);
      }
    });
  };

  // ---- the blocks of this wave, the next one on its way while one is worked on ---------------------------------
  // The parts of a sequence take four blocks in turn and so walk through the same stretch of memory together (each a
  // range of its own: 2 sequences of 131072 rows in 8 bits 87.5 us instead of 85.4, one of 32768 13.6 instead of 13.3).
  const int step = kWaves * max(seq.n_parts, 1), blk1 = seq.b1;
  // (Two or three blocks ahead instead of one: within 3 % of this with 4-bit codes, registers spill with 8-bit ones.)
  const int blk0 = seq.b0 + part * kWaves + wave;
  if (blk0 < blk1) {
    R r[2];
    load(r[0], blk0);
    for (int blk = blk0; blk < blk1;) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        load(r[1 - i], min(blk + step, blk1 - 1));
        compute(r[i], blk);
        blk += step;
        if (blk >= blk1) break;
      }
    }
  }

  // ---- the four waves joined ---------------------------------------------------------------------------
  __shared__ __align__(16) float o_lds[kWaves][16][D + 4];
  __shared__ float m_lds[kWaves][16 * NT], l_lds[kWaves][16 * NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const float l_tot = reduce_rows_one(l_run[n], [](float x, float y) { return x + y; });
    if (h == 0) {
      m_lds[wave][16 * n + l16] = m_run[n];
      l_lds[wave][16 * n + l16] = l_tot;
    }
  }
  __syncthreads();
  const bool final = seq.n_parts <= 1;
  const int64_t pair = (int64_t)b * a.Hkv + g;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    // (0 where no wave has a maximum: no key seen, and zeros for sums and weights, or scores that are all NaN, which stay
    // NaN through a weight of zero)
    auto top_of = [&](int c) __attribute__((always_inline)) {
      float m = m_lds[0][c];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) m = fmaxf(m, m_lds[w][c]);
      return m == -INFINITY ? 0.f : m;
    };
    {
      const float f = __builtin_amdgcn_exp2f(m_run[n] - top_of(16 * n + l16));
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int m = 0; m < MT; m += 4)
          *reinterpret_cast<f32x4*>(&o_lds[wave][l16][(4 * h + i) * MT + m]) =
              f32x4{o[m][n][i], o[m + 1][n][i], o[m + 2][n][i], o[m + 3][n][i]} * f;
    }
    __syncthreads();
    constexpr int PER = D / 16;                        // 16 threads per column
    const int c_l = threadIdx.x >> 4, c = 16 * n + c_l, d0 = (threadIdx.x & 15) * PER;
    const int col = col0 + c;
    if (col < n_cols) {
      const float top = top_of(c);
      float total = 0.f;
      f32x4 acc[PER / 4];
#pragma unroll
      for (int e = 0; e < PER / 4; ++e) acc[e] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        total += l_lds[w][c] * __builtin_amdgcn_exp2f(m_lds[w][c] - top);
#pragma unroll
        for (int e = 0; e < PER / 4; ++e) acc[e] += *reinterpret_cast<const f32x4*>(&o_lds[w][c_l][d0 + 4 * e]);
      }
      if (final) {
        const int t = col >> a.group_shift;
        const int64_t row = ((int64_t)b * a.n_new + t) * a.Hq + g * G + (col & (G - 1));
        const float inv = total == 0.f ? 0.f : 1.0f / total;
        uint32_t w[PER / 2];
#pragma unroll
        for (int e = 0; e < PER / 2; ++e) w[e] = pack_bf16(acc[e / 2][e % 2 * 2] * inv, acc[e / 2][e % 2 * 2 + 1] * inv);
        uint16_t* op = a.out + row * D + d0;
        if constexpr (PER == 8) *reinterpret_cast<u32x4*>(op) = u32x4{w[0], w[1], w[2], w[3]};
        else *reinterpret_cast<u32x2*>(op) = u32x2{w[0], w[1]};
        if (a.lse != nullptr && d0 == 0)
          a.lse[row] = (top + __builtin_log2f(total)) * 0.69314718055994531f;      // (-inf where the sum is 0)
      } else {
        float* op = a.partial + ((pair * a.n_parts + part) * n_cols + col) * D + d0;
#pragma unroll
        for (int e = 0; e < PER / 4; ++e) *reinterpret_cast<f32x4*>(op + 4 * e) = acc[e];
        if (d0 == 0) reinterpret_cast<f32x2*>(a.partial_ml)[(pair * n_cols + col) * a.n_parts + part] = f32x2{total == 0.f ? -INFINITY : top, total};
      }
    }
    if (n + 1 < NT) __syncthreads();
  }
}

// The parts of a key range joined: out = sum_i w_i O_i / sum_i w_i l_i, w_i = 2^(m_i - max m).  One workgroup per query
// row: the weights first, a thread each, then D / 4 threads side by side over a part's row and 1024 / D parts at a time.
// (One wave per row and one part after the other took 44 us for 32 rows of 128 parts.)
constexpr int kMergeThreads = 256;
template <int D>
__global__ __launch_bounds__(kMergeThreads) void packed_merge_kernel(PackedAttnArgs a) {
  constexpr int LANES = D / 4, SLOTS = kMergeThreads / LANES;
  const int tid = threadIdx.x;
  const int G = 1 << a.group_shift, n_cols = a.n_new << a.group_shift;
  const int64_t row = blockIdx.x;                       // (sequence, new token, query head)
  const uint32_t bt = blockIdx.x / (uint32_t)a.Hq, n_new = a.n_new;   // (in 32 bits: a division in 64 is some 100 steps)
  const int hq = blockIdx.x - bt * (uint32_t)a.Hq, b = bt / n_new, t = bt - (uint32_t)b * n_new;
  const int np = sequence_of(a, b).n_parts;
  if (np <= 1) return;                                  // written by the attention kernel
  const int col = (t << a.group_shift) + (hq & (G - 1));
  const int64_t pair = (int64_t)b * a.Hkv + (hq >> a.group_shift);
  const f32x2* ml = reinterpret_cast<const f32x2*>(a.partial_ml) + (pair * n_cols + col) * a.n_parts;
  __shared__ float w_lds[kMaxParts], red[kMergeThreads / 64], red_l[kMergeThreads / 64];
  __shared__ __align__(16) float o_lds[SLOTS][D];
  float top = -INFINITY;
  for (int i = tid; i < np; i += kMergeThreads) top = fmaxf(top, ml[i][0]);
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
  if ((tid & 63) == 0) red[tid >> 6] = top;
  __syncthreads();
  top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  if (top == -INFINITY) top = 0.f;                      // (as in the attention kernel)
  float total = 0.f;
  for (int i = tid; i < np; i += kMergeThreads) {
    const f32x2 x = ml[i];
    const float w = __builtin_amdgcn_exp2f(x[0] - top);
    w_lds[i] = w;
    total += w * x[1];
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) total += __shfl_xor(total, off);
  if ((tid & 63) == 0) red_l[tid >> 6] = total;
  __syncthreads();
  total = (red_l[0] + red_l[1]) + (red_l[2] + red_l[3]);
  const int slot = tid / LANES, d0 = tid % LANES * 4;
  const float* base = a.partial + (pair * a.n_parts * n_cols + col) * D + d0;
  const int64_t stride = (int64_t)n_cols * D;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int i = slot; i < np; i += SLOTS) acc += w_lds[i] * *reinterpret_cast<const f32x4*>(base + i * stride);
  *reinterpret_cast<f32x4*>(&o_lds[slot][d0]) = acc;
  __syncthreads();
  if (tid >= LANES) return;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < SLOTS; ++i) sum += *reinterpret_cast<const f32x4*>(&o_lds[i][tid * 4]);
  const float inv = total == 0.f ? 0.f : 1.0f / total;
  *reinterpret_cast<u32x2*>(a.out + row * D + tid * 4) =
      u32x2{pack_bf16(sum[0] * inv, sum[1] * inv), pack_bf16(sum[2] * inv, sum[3] * inv)};
  if (a.lse != nullptr && tid == 0)
    a.lse[row] = (top + __builtin_log2f(total)) * 0.69314718055994531f;
}

// Codes that are read once stream past the caches: 64 sequences of 4096 rows 52.4 -> 49.3 us in 4 bits (5.8 TB/s), of 2048
// rows 48.3 -> 43.9 in 8, 2 of 131072 in 8 93.9 -> 84.9.  What several workgroups read suffers in 8 bits, not in 4: 16
// sequences of 8192 rows with 64 columns in two workgroups 81 -> 93 (71 -> 71), 64 sequences that are the same 32768 rows
// 308 -> 421 (243 -> 244).  So 8-bit codes stream where one workgroup holds all columns and the cache has rows enough for all
// sequences at their longest, so that none need share any.  (Uneven sequences that lie one close behind the other in a
// cache of no more rows than they have go through the caches too; where each lies is on the device.)
bool stream_loads(int bits, int col_blocks, int64_t n_seq, int64_t max_len, int64_t n_rows) {
  return bits == 4 || (col_blocks == 1 && n_seq * max_len <= n_rows);
}

// Sequences to a round of by_length, or 0: taken as they come.  32/8 heads of 128, uneven lengths up to max_len, as they come
// and by length: 64 sequences up to 4099 rows 38.2 -> 33.6 us in 4 bits (all of the mean length 33.3), 70.8 -> 62.2 in 8; 128
// up to 4099 71.2 -> 66.4, 200 up to 3000 in 8 bits 146.8 -> 138.5.  A wave needs 0.6 us more for it, with more than 64
// sequences 1.3, about as much as is gained up to 2048 rows (64 sequences 21.4 and 21.0 us, 256 66.4 and 64.8; up to 1024
// rows 128 sequences 22.8 and 23.6).
int round_of(int64_t workgroups, int64_t n_seq, int64_t max_len) {
  if (workgroups <= kNumCUs || n_seq > kOrdered || max_len <= 2048) return 0;
  return (int)std::max<int64_t>(kNumCUs * n_seq / workgroups, 1);
}

struct PackedPlan {
  int col_tiles;      // 16-column tiles per workgroup
  int col_blocks;
  int part_blocks;    // blocks of 32 rows per part
  int n_parts;
  size_t o_bytes, ws_bytes;
};

// How the key range is divided.  A wave alone takes about 0.64 us for a block of 32 rows (219 instructions with 4 bits, 211
// with 8, and the latency of its loads; 0.46 with heads of 64) and the merge's launch 4 us: sequences of up to 1024 rows stay
// whole (one token, 32/8 heads of 128, 1, 4 and 16 sequences of 1024 rows: 7.5, 8.2 and 8.5 us whole, 7.4, 8.4 and 10.3
// in parts; 8/2 heads of 64 5.6, 6.0 and 6.6, and 6.7 to 7.4, 7.1 to 7.5 and 7.7; of 2048 rows 12.6, 12.9 and 13.4, and 8.0, 8.5
// and 12.9; 9.2, 9.6 and 10.2, and 7.1, 7.4 and 7.8).  The lines cross between 1024 rows (one sequence of heads of 128), 1300
// to 1500 (heads of 64) and 1800 (16 sequences of heads of 128): up to there calls pay up to 1.8 us more than whole.
// Longer ones are divided until a workgroup stands on each compute unit, into parts of at least 128 rows; where
// parts would be longer than 4096 rows, until two do, because sequences of uneven length leave units idle for as long
// as a part takes.  256 / 512 workgroups, 32/8 heads of 128, 4 bits, one token: one sequence of 8192 rows 10.0 / 10.1 us,
// of 32768 12.9 / 14.6, of 65536 18.0 / 19.7; four of 8192 12.6 / 13.4, of 32768 28.7 / 28.7, two of 131072 in 8 bits
// 83.4 / 84.7; but eight of 4096 to 16384 rows with four tokens 29.0 / 26.8.  Never a few more than fit, and two or three to
// a unit where fewer would leave places empty (as many parts as reach 256 or 512 workgroups / this rule: 5 sequences of
// 65536 rows 76 / 61 us, 9 of up to 4099 15.3 / 13.1, 12 18.5 / 14.4, in 8 bits 26.2 / 21.2, 24 of up to 8192 37.9 / 33.1;
// the worst, 13 of up to 16384, 33.5 / 36.9).  Three to a unit are slower where two fill it (32 sequences of 8192 rows 51 us
// with 512 workgroups, 52.3 with 768), and more are not planned for, though a unit holds four with heads of 64.
// More whole sequences than units are not divided in two: taken by length they share the units well, and no merge is needed
// (uneven lengths, divided / whole: 36 sequences up to 4099 rows 31.3 / 25.8 us, 48 up to 16384 102.8 / 97.6, in 8 bits 192 /
// 190), except long ones that leave more than half of the units with one workgroup alone (33 up to 16384 rows 91.6 / 94.7,
// in 8 bits 162 / 163 and 219 / 265 where all are as long).
PackedPlan plan_packed(const ct_layer_cfg* cfg, int64_t n_seq, int64_t n_new, int64_t max_len) {
  PackedPlan p;
  const int64_t n_cols = n_new * (cfg->n_q_heads / cfg->n_kv_heads);
  p.col_tiles = n_cols > 16 ? 2 : 1;
  p.col_blocks = (int)((n_cols + 16 * p.col_tiles - 1) / (16 * p.col_tiles));
  const int64_t blocks = (max_len + kPackRows - 1) / kPackRows + 1;   // a sequence may start inside a block
  const int64_t groups = n_seq * cfg->n_kv_heads * p.col_blocks;
  int64_t parts[4], used[4];      // where k workgroups stand on a unit: parts of a sequence, sixteenths of the places that are taken
  const int fit = p.col_tiles == 1 ? 3 : 2;      // what a unit holds with heads of 128
  for (int k = 1; k <= fit; ++k) {
    parts[k] = std::max<int64_t>(k * kNumCUs / groups, 1);
    used[k] = std::min<int64_t>(16 * groups * parts[k] / (k * kNumCUs), 16);
  }
  auto blocks_per = [&](int k) { return (blocks + parts[k] - 1) / parts[k]; };
  int64_t per = blocks_per(1);
  if (groups <= kNumCUs || (blocks > 257 && 2 * groups < 3 * kNumCUs)) {
    int k = per > 128 ? 2 : 1;
    const int64_t most = *std::max_element(used + 1, used + fit + 1);
    while (k < fit && used[k] < most - 1) ++k;
    per = blocks_per(k);
  }
  if (per < 4) per = 4;
  if (blocks * p.col_tiles <= 33) per = blocks;
  p.part_blocks = (int)per;
  p.n_parts = (int)((blocks + per - 1) / per);
  p.o_bytes = (size_t)(n_seq * cfg->n_kv_heads * p.n_parts) * n_cols * cfg->head_dim * sizeof(float);
  p.ws_bytes = p.n_parts > 1 ? p.o_bytes + p.o_bytes / cfg->head_dim * 2 : 0;
  return p;
}

ct_status check_attn_sizes(const ct_layer_cfg* cfg, int32_t n_seq, int32_t n_new, int32_t max_len) {
  if (n_seq < 0 || max_len < 0) return fail(CT_ERR_SHAPE, "negative size (n_seq %d, max_len %d)", n_seq, max_len);
  if (n_new < 1) return fail(CT_ERR_SHAPE, "n_new %d must be at least 1", n_new);
  if (n_new > 64) return fail(CT_ERR_UNSUPPORTED, "n_new %d: at most 64 new tokens per sequence", n_new);
  if ((int64_t)n_seq * n_new * cfg->n_q_heads > kMaxWorkgroups)      // (of the merge, one per row)
    return fail(CT_ERR_UNSUPPORTED, "n_seq %d x n_new %d x %d heads are too many rows for one launch", n_seq, n_new, cfg->n_q_heads);
  return CT_OK;
}

}  // namespace

}  // namespace ct

using namespace ct;

extern "C" {

size_t ct_packed_attention_workspace_bytes(const ct_layer_cfg* cfg, int32_t n_seq, int32_t n_new, int32_t max_len) {
  if (check_cfg(cfg) != CT_OK || check_attn_sizes(cfg, n_seq, n_new, max_len) != CT_OK || n_seq == 0) return 0;
  return plan_packed(cfg, n_seq, n_new, max_len).ws_bytes;
}

ct_status ct_packed_attention(const ct_layer_cfg* cfg, const void* q, int32_t n_seq, int32_t n_new, const void* cache,
                              int32_t n_rows, int32_t bits, const int32_t* seq_start, const int32_t* seq_len, int32_t max_len,
                              void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  ct_status st = check_packed(cfg, n_rows, bits);
  if (st != CT_OK) return st;
  if ((st = check_attn_sizes(cfg, n_seq, n_new, max_len)) != CT_OK) return st;
  if (max_len > n_rows) return fail(CT_ERR_SHAPE, "max_len %d exceeds the cache's %d rows", max_len, n_rows);
  if (n_seq == 0) return CT_OK;
  if (!q || !cache || !seq_start || !seq_len || !out)
    return fail(CT_ERR_NULL, "q, cache, seq_start, seq_len and out must be non-NULL");
  if ((((uintptr_t)q | (uintptr_t)cache | (uintptr_t)out) & 15) != 0)
    return fail(CT_ERR_UNSUPPORTED, "q, cache and out must be 16-byte aligned");
  const PackedPlan p = plan_packed(cfg, n_seq, n_new, max_len);
  const int64_t groups = (int64_t)n_seq * cfg->n_kv_heads * p.col_blocks * p.n_parts;
  if (groups > kMaxWorkgroups) return fail(CT_ERR_UNSUPPORTED, "n_seq %d with max_len %d: too many workgroups", n_seq, max_len);
  if (p.ws_bytes > 0) {
    if (workspace == nullptr) return fail(CT_ERR_WORKSPACE, "workspace is NULL but %zu bytes are needed", p.ws_bytes);
    if (workspace_bytes < p.ws_bytes)
      return fail(CT_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, p.ws_bytes);
    if (((uintptr_t)workspace & 255) != 0) return fail(CT_ERR_WORKSPACE, "workspace is not 256-byte aligned");
  }
  PackedAttnArgs a;
  a.q = static_cast<const uint16_t*>(q);
  a.cache = static_cast<const unsigned char*>(cache);
  a.seq_start = seq_start;
  a.seq_len = seq_len;
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse;
  a.partial = static_cast<float*>(workspace);
  a.partial_ml = reinterpret_cast<float*>(static_cast<char*>(workspace) + p.o_bytes);
  a.n_seq = n_seq;
  a.n_new = n_new;
  a.n_rows = n_rows;
  a.max_len = max_len;
  a.Hq = cfg->n_q_heads;
  a.Hkv = cfg->n_kv_heads;
  a.group_shift = 0;
  while ((a.Hkv << a.group_shift) < a.Hq) ++a.group_shift;
  a.n_parts = p.n_parts;
  a.part_blocks = p.part_blocks;
  a.col_blocks = p.col_blocks;
  a.round = p.n_parts == 1 ? round_of(groups, n_seq, max_len) : 0;
  const float scale = cfg->softmax_scale > 0.f ? cfg->softmax_scale : 1.0f / sqrtf((float)cfg->head_dim);
  a.scale_log2 = scale * 1.4426950408889634f;
  hipStream_t s = static_cast<hipStream_t>(stream);
  auto launch = [&](auto kernel) {
    launch_kernel(KC_PACKED_ATTN, kernel, dim3((unsigned)groups), dim3(64 * kWaves), 0, s, a);
  };
  auto by_cols = [&](auto one, auto two) { p.col_tiles == 1 ? launch(one) : launch(two); };
  const bool stream_in = stream_loads(bits, p.col_blocks, n_seq, max_len, n_rows);
  if (cfg->head_dim == 128) {
    if (bits == 4) by_cols(packed_attn_kernel<128, 4, 1, true>, packed_attn_kernel<128, 4, 2, true>);
    else if (stream_in) by_cols(packed_attn_kernel<128, 8, 1, true>, packed_attn_kernel<128, 8, 2, true>);
    else by_cols(packed_attn_kernel<128, 8, 1, false>, packed_attn_kernel<128, 8, 2, false>);
  } else {
    if (bits == 4) by_cols(packed_attn_kernel<64, 4, 1, true>, packed_attn_kernel<64, 4, 2, true>);
    else if (stream_in) by_cols(packed_attn_kernel<64, 8, 1, true>, packed_attn_kernel<64, 8, 2, true>);
    else by_cols(packed_attn_kernel<64, 8, 1, false>, packed_attn_kernel<64, 8, 2, false>);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return hip_fail(e, "packed attention kernel launch");
  if (p.n_parts > 1) {
    const dim3 grid((unsigned)((int64_t)n_seq * n_new * cfg->n_q_heads));
    if (cfg->head_dim == 128) launch_kernel(KC_MERGE, packed_merge_kernel<128>, grid, dim3(kMergeThreads), 0, s, a);
    else launch_kernel(KC_MERGE, packed_merge_kernel<64>, grid, dim3(kMergeThreads), 0, s, a);
    e = hipGetLastError();
    if (e != hipSuccess) return hip_fail(e, "packed attention merge kernel launch");
  }
  return CT_OK;
}

}  // extern "C"
