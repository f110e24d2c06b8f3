// Packed K/V cache: rows written in 4 or 8 bits (ct_pack_kv) and read back into layer buffers with the keys rotated to
// their new positions (ct_unpack_kv; Eq. 8 in delta form, as for chunks cached in bf16).
//
// Bound: memory.  Both move every byte once: a token of 8 heads of 128 is 4096 bytes in bf16 (K and V) and 1088 in 4
// bits, 2112 in 8.  32768 tokens to 4 bits and back: 61 us for 340 MB, 5.6 TB/s.  Tokens that lie anywhere in the cache cost
// more than their bytes: a row of one head is part of one line of K codes, two of V codes and two of scales in 4 bits.
#include "ct_packed.h"
#include "ct_rotate.h"

namespace ct {

namespace {

constexpr int kThreads = 256;

struct PackArgs {
  const uint16_t* k;
  const uint16_t* v;
  int64_t k_stride, v_stride;   // elements between rows
  const int32_t* rows;          // cache row of token t, or NULL: first_row + t
  int32_t first_row;
  int32_t n_tokens;
  unsigned char* cache;
  int32_t n_rows;
  int32_t Hkv;
};

// A workgroup takes 32 tokens of one head (those of one block of the cache, where the rows are a run), so that every
// line of codes is written by one workgroup in whole (a thread per 8 elements in the order of the rows, whose lines
// several dies write in parts: 32768 tokens and back 80 us instead of 71).  A thread takes 8 elements at a time; threads
// lie along the row for K and along the tokens for V, which is the order of their codes; the threads that share a scale
// are 1, 2 and 3 (K) or 8, 16 and 24 (V) apart.  A row's number comes before its elements are sent for (both at once:
// 0.3 us less for 48 tokens, but 63 us instead of 59 for 32768 and back).
template <int D, int BITS>
__global__ __launch_bounds__(kThreads) void pack_kernel(PackArgs a) {
  using L = PackLayout<D, BITS>;
  constexpr int PIECES = D / 8, STEP = kThreads / PIECES;      // pieces of a row, rows per step
  const int head = blockIdx.x % a.Hkv;
  const int skip = a.rows != nullptr ? 0 : a.first_row % kPackRows;      // rows of the first block ahead of the run
  const int64_t t0 = (int64_t)(blockIdx.x / a.Hkv) * kPackRows - skip;
  const int tid = threadIdx.x;
  u32x4 x[2][kPackRows / STEP];
  int32_t row[2][kPackRows / STEP];
  auto place = [&](bool is_v, int i, int& tok, int& piece) __attribute__((always_inline)) {
    if (is_v) {
      tok = i * STEP + (tid / (8 * PIECES)) * 8 + tid % 8;
      piece = tid / 8 % PIECES;
    } else {
      tok = i * STEP + tid / PIECES;
      piece = tid % PIECES;
    }
  };
#pragma unroll
  for (int v = 0; v < 2; ++v)
#pragma unroll
    for (int i = 0; i < kPackRows / STEP; ++i) {
      int tok, piece;
      place(v != 0, i, tok, piece);
      const int64_t t = t0 + tok;
      row[v][i] = t < 0 || t >= a.n_tokens ? -1 : a.rows != nullptr ? a.rows[t] : a.first_row + (int32_t)t;
      if (row[v][i] >= 0) x[v][i] = *reinterpret_cast<const u32x4*>((v ? a.v + t * a.v_stride : a.k + t * a.k_stride) + head * D + piece * 8);
    }
#pragma unroll
  for (int v = 0; v < 2; ++v)
#pragma unroll
    for (int i = 0; i < kPackRows / STEP; ++i) {
      if (row[v][i] < 0 || row[v][i] >= a.n_rows) continue;     // (the same for the four threads of a scale)
      int tok, piece;
      place(v != 0, i, tok, piece);
      uint32_t top = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) top = max(top, max(x[v][i][e] & 0x7fffu, (x[v][i][e] >> 16) & 0x7fffu));
      top = max(top, (uint32_t)__shfl_xor((int)top, v ? 8 : 1));
      top = max(top, (uint32_t)__shfl_xor((int)top, v ? 16 : 2));
      if (top > kMaxBits && top < 0x7f80u) {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[v][i][e] = clamp_pair(x[v][i][e]);
        top = kMaxBits;
      }
      const uint32_t sb = scale_byte<BITS>(top);
      // (a group that holds infinities or NaN reads back as NaN whatever its codes are: they are cleared)
      u32x2 w = pack8<BITS>(x[v][i], scale_of(sb));
      if (sb == kScaleNaN) w = u32x2{0u, 0u};
      unsigned char* block = a.cache + ((int64_t)(row[v][i] / kPackRows) * a.Hkv + head) * L::kBytes;
      const int r = row[v][i] % kPackRows, group = piece / 4;
      unsigned char* p = block + (v ? L::v_code(r, piece * 8) : L::k_code(r, piece * 8));
      if (v == 0 || D == 128) {
        if (BITS == 4) *reinterpret_cast<uint32_t*>(p) = w[0];
        else *reinterpret_cast<u32x2*>(p) = w;
      } else {   // two lanes of the attention hold four of the elements each
        unsigned char* p2 = block + L::v_code(r, piece * 8 + 4);
        if (BITS == 4) {
          *reinterpret_cast<uint16_t*>(p) = (uint16_t)w[0];
          *reinterpret_cast<uint16_t*>(p2) = (uint16_t)(w[0] >> 16);
        } else {
          *reinterpret_cast<uint32_t*>(p) = w[0];
          *reinterpret_cast<uint32_t*>(p2) = w[1];
        }
      }
      if (piece % 4 == 0) block[v ? L::v_scale(r, group) : L::k_scale(r, group)] = (unsigned char)sb;
    }
}

struct UnpackArgs {
  const unsigned char* cache;
  int32_t n_rows;
  int32_t Hkv;
  const int32_t* rows;          // cache row of token t (outside [0, n_rows): left out), or NULL: first_row + t
  int32_t first_row;
  const int32_t* old_pos;       // NULL: 0
  const int32_t* new_pos;       // NULL: no rotation
  int32_t n_tokens;
  uint16_t* k;
  uint16_t* v;
};

// Codes and scale byte of eight elements, as they lie in the cache.
template <int D, int BITS>
struct Packed8 {
  uint32_t w[2];
  uint32_t scale;
  __device__ __forceinline__ void load_k(const unsigned char* block, int r, int dim) {
    using L = PackLayout<D, BITS>;
    const unsigned char* p = block + L::k_code(r, dim);
    if constexpr (BITS == 4) {
      w[0] = *reinterpret_cast<const uint32_t*>(p);
    } else {
      const u32x2 x = *reinterpret_cast<const u32x2*>(p);
      w[0] = x[0];
      w[1] = x[1];
    }
    scale = block[L::k_scale(r, dim / kPackGroup)];
  }
  __device__ __forceinline__ void load_v(const unsigned char* block, int r, int dim) {
    using L = PackLayout<D, BITS>;
    const unsigned char* p = block + L::v_code(r, dim);
    if constexpr (D == 64) {      // two lanes of the attention hold four of the elements each
      const unsigned char* p2 = block + L::v_code(r, dim + 4);
      if constexpr (BITS == 4) {
        w[0] = *reinterpret_cast<const uint16_t*>(p) | (uint32_t) * reinterpret_cast<const uint16_t*>(p2) << 16;
      } else {
        w[0] = *reinterpret_cast<const uint32_t*>(p);
        w[1] = *reinterpret_cast<const uint32_t*>(p2);
      }
    } else if constexpr (BITS == 4) {
      w[0] = *reinterpret_cast<const uint32_t*>(p);
    } else {
      const u32x2 x = *reinterpret_cast<const u32x2*>(p);
      w[0] = x[0];
      w[1] = x[1];
    }
    scale = block[L::v_scale(r, dim / kPackGroup)];
  }
  __device__ __forceinline__ u32x4 value() const { return unpack8<BITS>(w, scale_of(scale)); }
};

// A workgroup takes a tile of tokens (32, or 64 with heads of 64) and two heads.  K: a thread owns 8 rotation pairs of one
// token, its sines and cosines serve both heads.  V: a thread takes 8 elements, threads along the tokens, the order of
// the codes; both write whole lines.  One, two, four or eight heads per workgroup: 8192 tokens in 4 bits 9.5 / 8.0 / 8.2 /
// 10.3 us (36 MB), 31901 in 8 bits 37 / 31.5 / 36 / 37 when that was measured (now
// 28.2 for 169 MB in turn over three inputs, 6.0 TB/s, 30.3 over four, 37.9 over six; a large copy moves 5.1).
// The stores do not stay in the caches: 8.0 against 9.7 us, and 33.9 against 42.1 when that was measured; what follows in
// a partial prefill takes about as much longer as the call gains (unpack, projection, scatter and attention of 15 % of
// 31901 rows 1281 us with either, of 5 % 500 against 497; of 15 % of 8192 186.6 against 186.0).
constexpr int kUnpackHeads = 2;
template <int D, int BITS, int STYLE>
__global__ __launch_bounds__(kThreads) void unpack_kernel(UnpackArgs a, RopeTable table) {
  using L = PackLayout<D, BITS>;
  constexpr int PER_TOKEN = D / 16, TILE = kThreads / PER_TOKEN, PIECES = D / 8, STEP = kThreads / PIECES;
  const int tid = threadIdx.x;
  const int64_t t0 = (int64_t)blockIdx.x * TILE;
  const int head0 = blockIdx.y * kUnpackHeads;
  auto row_of = [&](int64_t t) __attribute__((always_inline)) {
    int32_t row = -1;
    if (t < a.n_tokens) row = a.rows != nullptr ? a.rows[t] : a.first_row + (int32_t)t;
    return row < a.n_rows ? row : -1;
  };
  const int64_t t_k = t0 + tid / PER_TOKEN;
  const int jg = tid % PER_TOKEN;
  const int32_t row_k = row_of(t_k);
  int32_t row_v[2];
  int64_t t_v[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    t_v[i] = t0 + i * STEP + tid / (8 * PIECES) * 8 + tid % 8;
    row_v[i] = row_of(t_v[i]);
  }
  const int d_a = piece_a<D>(jg), d_b = piece_b<D>(jg), d_v = tid / 8 % PIECES * 8;
  // both heads are on their way while the angles are worked out
  struct Head {
    Packed8<D, BITS> ka, kb, v[2];
  };
  auto load = [&](Head& x, int head) __attribute__((always_inline)) {
    if (row_k >= 0) {
      const unsigned char* block = a.cache + ((int64_t)(row_k / kPackRows) * a.Hkv + head) * L::kBytes;
      x.ka.load_k(block, row_k % kPackRows, d_a);
      x.kb.load_k(block, row_k % kPackRows, d_b);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (row_v[i] >= 0) x.v[i].load_v(a.cache + ((int64_t)(row_v[i] / kPackRows) * a.Hkv + head) * L::kBytes, row_v[i] % kPackRows, d_v);
  };
  Head x[kUnpackHeads];
#pragma unroll
  for (int i = 0; i < kUnpackHeads; ++i)
    if (head0 + i < a.Hkv) load(x[i], head0 + i);
  const bool turns = a.new_pos != nullptr;
  float cs[8], sn[8];
  if (turns && row_k >= 0) {
    const int32_t delta = a.new_pos[t_k] - (a.old_pos != nullptr ? a.old_pos[t_k] : 0);
#pragma unroll
    for (int i = 0; i < 8; ++i) sincos_turns(delta, table.turns[pair_of<D, STYLE>(jg, i)], cs[i], sn[i]);
  }
  auto finish = [&](const Head& x, int head) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (row_v[i] >= 0) __builtin_nontemporal_store(x.v[i].value(), reinterpret_cast<u32x4*>(a.v + (t_v[i] * a.Hkv + head) * D + d_v));
    if (row_k >= 0) {
      u32x4 ka = x.ka.value(), kb = x.kb.value();
      if (turns) {
        float fa[8], fb[8];
        widen8(ka, fa);
        widen8(kb, fb);
        rotate8<STYLE>(fa, fb, cs, sn, ka, kb);
      }
      uint16_t* kd = a.k + (t_k * a.Hkv + head) * D;
      __builtin_nontemporal_store(ka, reinterpret_cast<u32x4*>(kd + d_a));
      __builtin_nontemporal_store(kb, reinterpret_cast<u32x4*>(kd + d_b));
    }
  };
#pragma unroll
  for (int i = 0; i < kUnpackHeads; ++i)
    if (head0 + i < a.Hkv) finish(x[i], head0 + i);
}

}  // namespace

ct_status check_packed(const ct_layer_cfg* cfg, int32_t n_rows, int32_t bits) {
  ct_status st = check_cfg(cfg);
  if (st != CT_OK) return st;
  if (bits != 4 && bits != 8) return fail(CT_ERR_UNSUPPORTED, "bits %d: a packed cache holds 4 or 8", bits);
  if (n_rows <= 0 || n_rows % kPackRows != 0)
    return fail(CT_ERR_SHAPE, "n_rows %d must be a positive multiple of %d", n_rows, kPackRows);
  return CT_OK;
}

namespace {

ct_status check_rows(const int32_t* rows, int32_t first_row, int32_t n_tokens, int32_t n_rows) {
  if (rows == nullptr && (first_row < 0 || (int64_t)first_row + n_tokens > n_rows))
    return fail(CT_ERR_INDEX, "rows %d to %lld do not lie in the cache's %d", first_row, (long long)first_row + n_tokens - 1, n_rows);
  return CT_OK;
}

}  // namespace

}  // namespace ct

using namespace ct;

extern "C" {

size_t ct_packed_kv_bytes(const ct_layer_cfg* cfg, int32_t n_rows, int32_t bits) {
  if (check_packed(cfg, n_rows, bits) != CT_OK) return 0;
  return (size_t)(n_rows / kPackRows) * pack_block_bytes(cfg, bits);
}

ct_status ct_pack_kv(const ct_layer_cfg* cfg, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                     int32_t n_tokens, const int32_t* rows, int32_t first_row, void* cache, int32_t n_rows, int32_t bits,
                     void* stream) {
  ct_status st = check_packed(cfg, n_rows, bits);
  if (st != CT_OK) return st;
  if (n_tokens < 0) return fail(CT_ERR_SHAPE, "n_tokens %d is negative", n_tokens);
  const int64_t row_elems = (int64_t)cfg->n_kv_heads * cfg->head_dim;
  if (k_stride < row_elems || v_stride < row_elems)
    return fail(CT_ERR_SHAPE, "strides %lld and %lld must be at least a row's %lld elements", (long long)k_stride,
                (long long)v_stride, (long long)row_elems);
  if (n_tokens == 0) return CT_OK;
  if (!k || !v || !cache) return fail(CT_ERR_NULL, "k, v and cache must be non-NULL");
  if ((st = check_rows(rows, first_row, n_tokens, n_rows)) != CT_OK) return st;
  if (((((uintptr_t)k | (uintptr_t)v | (uintptr_t)cache) & 15) | ((k_stride | v_stride) & 7)) != 0)
    return fail(CT_ERR_UNSUPPORTED, "k, v and cache must be 16-byte aligned and the strides multiples of 8");
  PackArgs a = {static_cast<const uint16_t*>(k), static_cast<const uint16_t*>(v), k_stride, v_stride, rows, first_row, n_tokens,
                static_cast<unsigned char*>(cache), n_rows, cfg->n_kv_heads};
  const int64_t tiles = ((rows != nullptr ? 0 : first_row % kPackRows) + (int64_t)n_tokens + kPackRows - 1) / kPackRows;
  if (tiles * cfg->n_kv_heads > kMaxWorkgroups)
    return fail(CT_ERR_UNSUPPORTED, "n_tokens %d x %d heads are too many for one launch", n_tokens, cfg->n_kv_heads);
  const dim3 grid((unsigned)(tiles * cfg->n_kv_heads));
  hipStream_t s = static_cast<hipStream_t>(stream);
  auto launch = [&](auto kernel) { launch_kernel(KC_PACK, kernel, grid, dim3(kThreads), 0, s, a); };
  if (cfg->head_dim == 128) bits == 4 ? launch(pack_kernel<128, 4>) : launch(pack_kernel<128, 8>);
  else bits == 4 ? launch(pack_kernel<64, 4>) : launch(pack_kernel<64, 8>);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return hip_fail(e, "pack kernel launch");
  return CT_OK;
}

ct_status ct_unpack_kv(const ct_layer_cfg* cfg, const void* cache, int32_t n_rows, int32_t bits, const int32_t* rows,
                       int32_t first_row, const int32_t* old_pos, const int32_t* new_pos, int32_t n_tokens, void* k_dst,
                       void* v_dst, void* stream) {
  ct_status st = check_packed(cfg, n_rows, bits);
  if (st != CT_OK) return st;
  if (n_tokens < 0) return fail(CT_ERR_SHAPE, "n_tokens %d is negative", n_tokens);
  if (n_tokens == 0) return CT_OK;
  if (!cache || !k_dst || !v_dst) return fail(CT_ERR_NULL, "cache, k_dst and v_dst must be non-NULL");
  if (old_pos != nullptr && new_pos == nullptr) return fail(CT_ERR_NULL, "old_pos is given but new_pos is NULL");
  if ((st = check_rows(rows, first_row, n_tokens, n_rows)) != CT_OK) return st;
  if ((((uintptr_t)cache | (uintptr_t)k_dst | (uintptr_t)v_dst) & 15) != 0)
    return fail(CT_ERR_UNSUPPORTED, "cache, k_dst and v_dst must be 16-byte aligned");
  UnpackArgs a = {static_cast<const unsigned char*>(cache), n_rows, cfg->n_kv_heads, rows, first_row, old_pos, new_pos, n_tokens,
                  static_cast<uint16_t*>(k_dst), static_cast<uint16_t*>(v_dst)};
  const int tile = kThreads / (cfg->head_dim / 16);
  const int64_t tiles = ((int64_t)n_tokens + tile - 1) / tile, head_tiles = (cfg->n_kv_heads + kUnpackHeads - 1) / kUnpackHeads;
  if (tiles > kMaxWorkgroups || head_tiles > 0xffff)
    return fail(CT_ERR_UNSUPPORTED, "n_tokens %d x %d heads are too many for one launch", n_tokens, cfg->n_kv_heads);
  const dim3 grid((unsigned)tiles, (unsigned)head_tiles);
  RopeTable table = {};
  if (new_pos != nullptr) fill_rope_products(cfg, &table);
  hipStream_t s = static_cast<hipStream_t>(stream);
  auto launch = [&](auto kernel) { launch_kernel(KC_PACK, kernel, grid, dim3(kThreads), 0, s, a, table); };
  auto by_style = [&](auto k0, auto k1) { cfg->rope_style == 0 ? launch(k0) : launch(k1); };
  if (cfg->head_dim == 128)
    bits == 4 ? by_style(unpack_kernel<128, 4, 0>, unpack_kernel<128, 4, 1>) : by_style(unpack_kernel<128, 8, 0>, unpack_kernel<128, 8, 1>);
  else
    bits == 4 ? by_style(unpack_kernel<64, 4, 0>, unpack_kernel<64, 4, 1>) : by_style(unpack_kernel<64, 8, 0>, unpack_kernel<64, 8, 1>);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return hip_fail(e, "unpack kernel launch");
  return CT_OK;
}

}  // extern "C"
