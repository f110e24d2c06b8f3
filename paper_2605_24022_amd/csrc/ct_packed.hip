// Packed K/V cache: rows written in 4 or 8 bits (ct_pack_kv) and read back into layer buffers with the keys rotated to
// their new positions (ct_unpack_kv; Eq. 8 in delta form, as for chunks cached in bf16).
//
// Both move every byte once.  A token of 8 heads of 128 is 4096 bytes in bf16 (K and V) and 1088 in 4 bits, 2112 in 8.
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

// One thread per 8 elements of a row of K or V (blockIdx.y), four neighbours share a scale.
template <int D, int BITS>
__global__ __launch_bounds__(kThreads) void pack_kernel(PackArgs a) {
  using L = PackLayout<D, BITS>;
  constexpr int PIECES = D / 8;
  const int64_t gid = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int piece = (int)(gid % PIECES);
  const int64_t rest = gid / PIECES;
  const int head = (int)(rest % a.Hkv);
  const int64_t t = rest / a.Hkv;
  if (t >= a.n_tokens) return;
  const int32_t row = a.rows != nullptr ? a.rows[t] : a.first_row + (int32_t)t;
  if (row < 0 || row >= a.n_rows) return;   // (the same for the four lanes of a group)
  const bool is_v = blockIdx.y != 0;
  u32x4 x = *reinterpret_cast<const u32x4*>((is_v ? a.v + t * a.v_stride : a.k + t * a.k_stride) + head * D + piece * 8);
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = x[i] & 0x7fffu, hi = (x[i] >> 16) & 0x7fffu;
    top = max(top, max(lo, hi));
  }
  top = max(top, (uint32_t)__shfl_xor((int)top, 1));
  top = max(top, (uint32_t)__shfl_xor((int)top, 2));
  if (top > kMaxBits && top < 0x7f80u) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = clamp_pair(x[i]);
    top = kMaxBits;
  }
  const uint32_t sb = scale_byte<BITS>(top);
  // (a group that holds infinities or NaN reads back as NaN whatever its codes are: they are cleared)
  u32x2 w = pack8<BITS>(x, scale_of(sb));
  if (sb == kScaleNaN) w = u32x2{0u, 0u};
  unsigned char* block = a.cache + ((int64_t)(row / kPackRows) * a.Hkv + head) * L::kBytes;
  const int r = row % kPackRows, group = piece / 4;
  if (!is_v) {
    unsigned char* p = block + L::k_code(r, piece * 8);
    if (BITS == 4) *reinterpret_cast<uint32_t*>(p) = w[0];
    else *reinterpret_cast<u32x2*>(p) = w;
    if (piece % 4 == 0) block[L::k_scale(r, group)] = (unsigned char)sb;
  } else {
    unsigned char* p = block + L::v_code(r, piece * 8);
    if (D == 128) {
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
    if (piece % 4 == 0) block[L::v_scale(r, group)] = (unsigned char)sb;
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

template <int D, int BITS>
__device__ __forceinline__ u32x4 load_k8(const unsigned char* block, int r, int dim) {
  using L = PackLayout<D, BITS>;
  const float scale = scale_of(block[L::k_scale(r, dim / kPackGroup)]);
  const uint32_t* p = reinterpret_cast<const uint32_t*>(block + L::k_code(r, dim));
  uint32_t w[2] = {p[0], BITS == 8 ? p[1] : 0u};
  return unpack8<BITS>(w, scale);
}
template <int D, int BITS>
__device__ __forceinline__ u32x4 load_v8(const unsigned char* block, int r, int dim) {
  using L = PackLayout<D, BITS>;
  const float scale = scale_of(block[L::v_scale(r, dim / kPackGroup)]);
  const unsigned char* p = block + L::v_code(r, dim);
  uint32_t w[2] = {0u, 0u};
  if (D == 128) {
    w[0] = reinterpret_cast<const uint32_t*>(p)[0];
    if (BITS == 8) w[1] = reinterpret_cast<const uint32_t*>(p)[1];
  } else {
    const unsigned char* p2 = block + L::v_code(r, dim + 4);
    if (BITS == 4) {
      w[0] = *reinterpret_cast<const uint16_t*>(p) | (uint32_t) * reinterpret_cast<const uint16_t*>(p2) << 16;
    } else {
      w[0] = *reinterpret_cast<const uint32_t*>(p);
      w[1] = *reinterpret_cast<const uint32_t*>(p2);
    }
  }
  return unpack8<BITS>(w, scale);
}

// One thread per 8 rotation pairs of a token's head: cos and sin once per thread and head.
template <int D, int BITS, int STYLE>
__global__ __launch_bounds__(kThreads) void unpack_kernel(UnpackArgs a, RopeTable table) {
  using L = PackLayout<D, BITS>;
  constexpr int THREADS = D / 16;
  const int64_t gid = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int jg = (int)(gid % THREADS);
  const int64_t rest = gid / THREADS;
  const int head = (int)(rest % a.Hkv);
  const int64_t t = rest / a.Hkv;
  if (t >= a.n_tokens) return;
  const int32_t row = a.rows != nullptr ? a.rows[t] : a.first_row + (int32_t)t;
  if (row < 0 || row >= a.n_rows) return;
  const unsigned char* block = a.cache + ((int64_t)(row / kPackRows) * a.Hkv + head) * L::kBytes;
  const int r = row % kPackRows;
  const int d_a = piece_a<D, STYLE>(jg), d_b = piece_b<D, STYLE>(jg);
  u32x4 ka = load_k8<D, BITS>(block, r, d_a), kb = load_k8<D, BITS>(block, r, d_b);
  const u32x4 va = load_v8<D, BITS>(block, r, d_a), vb = load_v8<D, BITS>(block, r, d_b);
  if (a.new_pos != nullptr) {
    const int32_t delta = a.new_pos[t] - (a.old_pos != nullptr ? a.old_pos[t] : 0);
    float cs[8], sn[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sincos_turns(delta, table.turns[jg * 8 + i], cs[i], sn[i]);
    float fa[8], fb[8];
    widen8(ka, fa);
    widen8(kb, fb);
    rotate8<STYLE>(fa, fb, cs, sn, ka, kb);
  }
  uint16_t* kd = a.k + (t * a.Hkv + head) * D;
  uint16_t* vd = a.v + (t * a.Hkv + head) * D;
  *reinterpret_cast<u32x4*>(kd + d_a) = ka;
  *reinterpret_cast<u32x4*>(kd + d_b) = kb;
  *reinterpret_cast<u32x4*>(vd + d_a) = va;
  *reinterpret_cast<u32x4*>(vd + d_b) = vb;
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

// Workgroups of kThreads for n_tokens x Hkv x per_head threads; false where the grid would not hold them.
bool grid_for(int64_t n_tokens, int64_t Hkv, int64_t per_head, unsigned* blocks) {
  const int64_t b = (n_tokens * Hkv * per_head + kThreads - 1) / kThreads;
  *blocks = (unsigned)b;
  return b <= 0x7fffffff;
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
  unsigned blocks;
  if (!grid_for(n_tokens, cfg->n_kv_heads, cfg->head_dim / 8, &blocks))
    return fail(CT_ERR_UNSUPPORTED, "n_tokens %d x %d heads are too many for one launch", n_tokens, cfg->n_kv_heads);
  hipStream_t s = static_cast<hipStream_t>(stream);
  auto launch = [&](auto kernel) { launch_kernel(KC_PACK, kernel, dim3(blocks, 2), dim3(kThreads), 0, s, a); };
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
  unsigned blocks;
  if (!grid_for(n_tokens, cfg->n_kv_heads, cfg->head_dim / 16, &blocks))
    return fail(CT_ERR_UNSUPPORTED, "n_tokens %d x %d heads are too many for one launch", n_tokens, cfg->n_kv_heads);
  RopeTable table;
  fill_rope_table(cfg, &table);
  hipStream_t s = static_cast<hipStream_t>(stream);
  auto launch = [&](auto kernel) { launch_kernel(KC_PACK, kernel, dim3(blocks), dim3(kThreads), 0, s, a, table); };
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
