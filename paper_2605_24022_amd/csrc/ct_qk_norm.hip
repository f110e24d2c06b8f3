// Queries and keys of projected rows normed head by head and rotated in one pass (ct_qk_norm_rope), for models that
// norm q and k per head before RoPE, where the rotation cannot ride on the projection's epilogue (ct_qkv_selected).
//
//   y = x / sqrt(mean(x^2) + eps) * w over the D elements of a head, then RoPE at the token's position; v is copied.
// fp32 from the bf16 input to the one rounding of the result.  Bound: memory, each element read and written once: 4915
// rows of 32 + 8 + 8 heads of 128, 121 MB, 22.4 us (5.4 TB/s; a large copy reaches 5.1) in turn over six inputs, 19.0 over
// four or fewer; 7 rows 4.5 to 5.2 us, the launch.
#include <math.h>

#include "ct_internal.h"
#include "ct_rotate.h"

namespace ct {

namespace {

constexpr int kThreads = 256;

struct QkNormArgs {
  const uint16_t* qkv;      // [n_tokens, (Hq + 2 Hkv) D]
  const int32_t* pos;
  const uint16_t* q_weight;
  const uint16_t* k_weight;
  uint16_t* q;
  uint16_t* k;
  uint16_t* v;              // NULL: the values stay where they are
  int32_t n_tokens, Hq, Hkv, heads;   // heads: of a row that are worked on
  float eps;
};

// One thread per 8 rotation pairs of a head.  (Two, four or eight heads per thread share the sines and cosines but
// leave fewer threads: 4915 rows 25.7, 25.1 and 49.6 us.)  The stores bypass the caches: 26.5 us without, and the
// packing of the keys that follows is no slower for it (both 34.2 -> 32.9 us; norm, scatter and attention of 1228 rows
// 126.3 -> 125.3, of 4915 1143 -> 1147).
template <int D, int STYLE>
__global__ __launch_bounds__(kThreads) void qk_norm_rope_kernel(QkNormArgs a, RopeTable table) {
  constexpr int THREADS = D / 16;
  const uint32_t gid = blockIdx.x * kThreads + threadIdx.x, rest = gid / THREADS, n_heads = a.heads;   // (below 2^32 threads)
  const int jg = gid % THREADS;
  const int64_t t = rest / n_heads;
  const int head = rest - (uint32_t)t * n_heads;
  if (t >= a.n_tokens) return;
  const int d_a = piece_a<D>(jg), d_b = piece_b<D>(jg);
  const uint16_t* src = a.qkv + (t * (a.Hq + 2 * a.Hkv) + head) * D;
  // everything that is read is sent for at once: with few rows the latency counts
  const u32x4 xa = *reinterpret_cast<const u32x4*>(src + d_a), xb = *reinterpret_cast<const u32x4*>(src + d_b);
  const bool is_q = head < a.Hq;
  const uint16_t* w = is_q ? a.q_weight : a.k_weight;
  const u32x4 wa = *reinterpret_cast<const u32x4*>(w + d_a), wb = *reinterpret_cast<const u32x4*>(w + d_b);
  const int32_t pos = a.pos[t];
  if (head >= a.Hq + a.Hkv) {
    uint16_t* dst = a.v + (t * a.Hkv + head - a.Hq - a.Hkv) * D;
    __builtin_nontemporal_store(xa, reinterpret_cast<u32x4*>(dst + d_a));
    __builtin_nontemporal_store(xb, reinterpret_cast<u32x4*>(dst + d_b));
    return;
  }
  float fa[8], fb[8];
  widen8(xa, fa);
  widen8(xb, fb);
  auto sum_squares = [&]() __attribute__((always_inline)) {
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) t += fa[i] * fa[i] + fb[i] * fb[i];
#pragma unroll
    for (int off = THREADS / 2; off >= 1; off >>= 1) t += __shfl_xor(t, off);   // (the lanes of a head leave together)
    return t;
  };
  float ss = sum_squares(), ms = ss / (float)D + a.eps;
  if (!(ss <= 0x1p120f) || ms < 0x1p-80f) {   // squares that leave fp32: the same with elements and root scaled by 2^k
    const float up = ss <= 0x1p120f ? 0x1p96f : 0x1p-70f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      fa[i] *= up;
      fb[i] *= up;
    }
    ms = sum_squares() / (float)D + a.eps * up * up;
  }
  const float inv = 1.0f / sqrtf(ms);
  // (the element by the root first, then by the weight: no size of a head leaves fp32 beside any weight)
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    fa[2 * i] = fa[2 * i] * inv * bf16_lo(wa[i]);
    fa[2 * i + 1] = fa[2 * i + 1] * inv * bf16_hi(wa[i]);
    fb[2 * i] = fb[2 * i] * inv * bf16_lo(wb[i]);
    fb[2 * i + 1] = fb[2 * i + 1] * inv * bf16_hi(wb[i]);
  }
  float cs[8], sn[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) sincos_turns(pos, table.turns[pair_of<D, STYLE>(jg, i)], cs[i], sn[i]);
  u32x4 ra, rb;
  rotate8<STYLE>(fa, fb, cs, sn, ra, rb);
  uint16_t* dst = is_q ? a.q + (t * a.Hq + head) * D : a.k + (t * a.Hkv + head - a.Hq) * D;
  __builtin_nontemporal_store(ra, reinterpret_cast<u32x4*>(dst + d_a));
  __builtin_nontemporal_store(rb, reinterpret_cast<u32x4*>(dst + d_b));
}

}  // namespace

}  // namespace ct

using namespace ct;

extern "C" {

ct_status ct_qk_norm_rope(const ct_layer_cfg* cfg, const void* qkv, const int32_t* pos, int32_t n_tokens,
                          const void* q_weight, const void* k_weight, float eps, void* q_out, void* k_out, void* v_out,
                          void* stream) {
  ct_status st = check_cfg(cfg);
  if (st != CT_OK) return st;
  if (n_tokens < 0) return fail(CT_ERR_SHAPE, "n_tokens %d is negative", n_tokens);
  if (!(eps >= 0.f) || !isfinite(eps)) return fail(CT_ERR_SHAPE, "eps must be >= 0 and finite");
  if (n_tokens == 0) return CT_OK;
  if (!qkv || !pos || !q_weight || !k_weight || !q_out || !k_out)
    return fail(CT_ERR_NULL, "qkv, pos, q_weight, k_weight, q_out and k_out must be non-NULL");
  if ((((uintptr_t)qkv | (uintptr_t)q_weight | (uintptr_t)k_weight | (uintptr_t)q_out | (uintptr_t)k_out | (uintptr_t)v_out) & 15) != 0)
    return fail(CT_ERR_UNSUPPORTED, "qkv, the weights and the outputs must be 16-byte aligned");
  QkNormArgs a = {static_cast<const uint16_t*>(qkv), pos, static_cast<const uint16_t*>(q_weight),
                  static_cast<const uint16_t*>(k_weight), static_cast<uint16_t*>(q_out), static_cast<uint16_t*>(k_out),
                  static_cast<uint16_t*>(v_out), n_tokens, cfg->n_q_heads, cfg->n_kv_heads,
                  cfg->n_q_heads + (v_out != nullptr ? 2 : 1) * cfg->n_kv_heads, eps};
  const int64_t blocks = ((int64_t)n_tokens * a.heads * (cfg->head_dim / 16) + kThreads - 1) / kThreads;
  if (blocks > kMaxWorkgroups) return fail(CT_ERR_UNSUPPORTED, "n_tokens %d x %d heads are too many for one launch", n_tokens, a.heads);
  RopeTable table;
  fill_rope_products(cfg, &table);
  hipStream_t s = static_cast<hipStream_t>(stream);
  auto launch = [&](auto kernel) { launch_kernel(KC_NORM, kernel, dim3((unsigned)blocks), dim3(kThreads), 0, s, a, table); };
  if (cfg->head_dim == 128) cfg->rope_style == 0 ? launch(qk_norm_rope_kernel<128, 0>) : launch(qk_norm_rope_kernel<128, 1>);
  else cfg->rope_style == 0 ? launch(qk_norm_rope_kernel<64, 0>) : launch(qk_norm_rope_kernel<64, 1>);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return hip_fail(e, "query/key norm kernel launch");
  return CT_OK;
}

}  // extern "C"
