// Attention of each sequence's newest tokens over its 8-bit paged cache.
#include <cmath>

#include "kv8.cuh"

namespace szo {
namespace kv8 {

namespace {

// One block of four warps per (new token, query head): lanes split the head dimension, warp w takes the
// positions w, w + 4, ...; online softmax per warp, the four states are merged in warp order.
template <typename T, int HD>
__global__ void __launch_bounds__(128)
kv8_attention_kernel(View V, const T* __restrict__ q, int64_t q_stride, T* __restrict__ o, int64_t o_stride, int H, float scale) {
  constexpr int E = HD / 32;
  __shared__ float part_acc[4][HD];
  __shared__ float part_m[4], part_l[4];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const unsigned item = blockIdx.x;
  const int hq = item % H, t = item / H % V.max_new, b = item / H / V.max_new;
  const Seq seq = load_seq(V, b);
  if (t >= seq.n) return;
  const int hk = hq / (H / V.hkv), pos = seq.len - seq.n + t;
  const T* qp = q + (seq.row0 + t) * q_stride + hq * HD;
  float qr[E], acc[E], mx = -INFINITY, l = 0.f;
#pragma unroll
  for (int j = 0; j < E; ++j) {
    qr[j] = widen<T>(qp[lane * E + j]) * scale;
    acc[j] = 0.f;
  }
  for (int n = w; n <= pos; n += 4) {
    const int page = load_page(V, b, n >> V.page_shift);
    if (page < 0) continue;
    const float2 sc = V.scales[static_cast<int64_t>(page) * V.hkv + hk];
    const int64_t at = page_offset(V, page, hk, HD) + (n & ((1 << V.page_shift) - 1)) * HD + lane * E;
    const float ks = exp2_int(scale_exponent(sc.x)), vs = exp2_int(scale_exponent(sc.y));
    float dot = 0.f;
    float2 vv[E / 2];
#pragma unroll
    for (int j = 0; j < E; j += 2) {
      const float2 kk = decode2f(*reinterpret_cast<const uint16_t*>(V.k + at + j));
      vv[j / 2] = decode2f(*reinterpret_cast<const uint16_t*>(V.v + at + j));
      dot = fmaf(qr[j], kk.x, fmaf(qr[j + 1], kk.y, dot));
    }
#pragma unroll
    for (int off = 16; off; off >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, off);
    dot *= ks;
    const float mn = fmaxf(mx, dot);
    const float corr = mx == -INFINITY ? 0.f : expf(mx - mn), p = expf(dot - mn);
    l = l * corr + p;
#pragma unroll
    for (int j = 0; j < E; j += 2) {
      acc[j] = fmaf(p, vv[j / 2].x * vs, acc[j] * corr);
      acc[j + 1] = fmaf(p, vv[j / 2].y * vs, acc[j + 1] * corr);
    }
    mx = mn;
  }
#pragma unroll
  for (int j = 0; j < E; ++j) part_acc[w][lane * E + j] = acc[j];
  if (lane == 0) {
    part_m[w] = mx;
    part_l[w] = l;
  }
  __syncthreads();
  if (w != 0) return;
  float M = -INFINITY, L = 0.f, out[E];
#pragma unroll
  for (int i = 0; i < 4; ++i) M = fmaxf(M, part_m[i]);
#pragma unroll
  for (int j = 0; j < E; ++j) out[j] = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float f = part_m[i] == -INFINITY ? 0.f : expf(part_m[i] - M);
    L += part_l[i] * f;
#pragma unroll
    for (int j = 0; j < E; ++j) out[j] = fmaf(part_acc[i][lane * E + j], f, out[j]);
  }
  const float inv = M == -INFINITY && L == 0.f ? 0.f : 1.0f / L;      // nothing attended to: zeros
  T* op = o + (seq.row0 + t) * o_stride + hq * HD;
#pragma unroll
  for (int j = 0; j < E; ++j) op[lane * E + j] = narrow<T>(out[j] * inv);
}

}  // namespace
}  // namespace kv8
}  // namespace szo

using namespace szo;

extern "C" szo_status szo_attention_kv8(const szo_kv8_cache* cache, const szo_kv8_batch* batch, const void* q, int64_t q_stride,
                                        void* o, int64_t o_stride, szo_dtype dtype, int32_t n_heads, float scale, void* stream) {
  kv8::View V;
  SZO_TRY(kv8::make_view(cache, batch, &V));
  SZO_REQUIRE(q && o, SZO_ERR_INVALID_ARG, "NULL q or o");
  SZO_REQUIRE(dtype == SZO_F32 || dtype == SZO_BF16 || dtype == SZO_F16, SZO_ERR_UNSUPPORTED, "dtype must be f32, bf16 or f16");
  SZO_REQUIRE(n_heads > 0 && n_heads % cache->n_kv_heads == 0, SZO_ERR_SHAPE, "n_heads must be a multiple of n_kv_heads");
  SZO_REQUIRE(std::isfinite(scale), SZO_ERR_INVALID_ARG, "scale must be finite");
  const int64_t width = static_cast<int64_t>(n_heads) * cache->head_dim, vec = dtype == SZO_F32 ? 4 : 8;
  SZO_REQUIRE(q_stride >= width && o_stride >= width, SZO_ERR_SHAPE, "row strides must be at least n_heads * head_dim");
  SZO_REQUIRE(aligned16(q) && aligned16(o) && q_stride % vec == 0 && o_stride % vec == 0, SZO_ERR_ALIGNMENT,
              "row buffers and rows must be 16-byte aligned");
  if (V.batch == 0 || V.max_new == 0 || V.rows == 0) return SZO_OK;
  SZO_REQUIRE(static_cast<int64_t>(V.max_new) * V.batch <= 0x7fffffff / n_heads, SZO_ERR_SHAPE, "too many rows and heads for one launch");
  SZO_TRY(kv8::set_status_word(&V));
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const unsigned blocks = static_cast<unsigned>(V.max_new) * V.batch * n_heads;
#define SZO_KV8_ATTN(T, HD) \
  kv8::kv8_attention_kernel<T, HD><<<blocks, 128, 0, st>>>(V, static_cast<const T*>(q), q_stride, static_cast<T*>(o), o_stride, n_heads, scale)
  const bool wide = cache->head_dim == 128;
  if (dtype == SZO_F32) { if (wide) SZO_KV8_ATTN(float, 128); else SZO_KV8_ATTN(float, 64); }
  else if (dtype == SZO_BF16) { if (wide) SZO_KV8_ATTN(__nv_bfloat16, 128); else SZO_KV8_ATTN(__nv_bfloat16, 64); }
  else { if (wide) SZO_KV8_ATTN(__half, 128); else SZO_KV8_ATTN(__half, 64); }
#undef SZO_KV8_ATTN
  count_launch();
  SZO_CHECK_LAUNCH("kv8_attention_kernel");
  return SZO_OK;
}
