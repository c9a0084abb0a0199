// Attention over the 8-bit paged cache for sequences that continue shared prompts.
//
// A row's softmax over its positions is joined from two parts with their own maxima and sums: the whole pages that its group
// shares, and the rest of its sequence's positions.
#include <cmath>

#include "kv8_prefix.cuh"

namespace szo {
namespace kv8 {

namespace {

// One warp per (row, head): lanes split the head dimension
template <typename T, int HD>
__global__ void __launch_bounds__(128) kv8_prefix_row_kernel(View V, Prefix P, const T* __restrict__ q, int64_t q_stride, T* __restrict__ o,
                                                             int64_t o_stride, int H, float scale_log2e) {
  constexpr int kPer = HD / 32;
  const int lane = threadIdx.x & 31;
  const int64_t item = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 5);
  const int head = static_cast<int>(item % H);
  const int64_t bi = item / H;
  const int b = static_cast<int>(bi / V.max_new), i = static_cast<int>(bi % V.max_new);
  if (b >= V.batch) return;
  if (item == 0)
    for (int g = lane; g < P.n_groups; g += 32) load_shared(V, P, g, true);
  const Seq s = load_seq(V, b);
  if (i >= s.n) return;
  const Shared sh = load_shared(V, P, group_of(P, b), false);
  const int h = head / (H / V.hkv), pos = s.len - s.n + i;
  const int64_t row = s.row0 + i;
  float x[kPer], m = -INFINITY, l = 0.f, acc[kPer];
  bool fine = true;
  for (int k = 0; k < kPer; ++k) {
    x[k] = widen<T>(q[row * q_stride + static_cast<int64_t>(head) * HD + lane * kPer + k]);
    fine = fine && isfinite(x[k]);
    acc[k] = 0.f;
  }
  fine = __all_sync(0xffffffffu, fine);
  for (int p = 0; p <= pos; ++p) {
    const int page = load_page(V, p < sh.len ? sh.first : b, p >> V.page_shift);
    if (page < 0) continue;
    const int64_t at = page_offset(V, page, h, HD) + static_cast<int64_t>(p & ((1 << V.page_shift) - 1)) * HD + lane * kPer;
    const float2 sc = V.scales[static_cast<int64_t>(page) * V.hkv + h];
    float dot = 0.f, v[kPer];
    for (int k = 0; k < kPer; ++k) {
      dot = fmaf(x[k], decode2f(V.k[at + k]).x, dot);
      v[k] = decode2f(V.v[at + k]).x * exp2_int(scale_exponent(sc.y));
    }
    for (int off = 16; off; off >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, off);
    const float t = dot * exp2_int(scale_exponent(sc.x)) * scale_log2e, mn = fmaxf(m, t), ref = mn == -INFINITY ? 0.f : mn;
    const float c = exp2f(m - ref), w = exp2f(t - ref);
    m = mn;
    l = fmaf(l, c, w);
    for (int k = 0; k < kPer; ++k) acc[k] = fmaf(acc[k], c, w * v[k]);
  }
  for (int k = 0; k < kPer; ++k) {
    float y = l == 0.f ? 0.f : acc[k] / l;
    if (!fine && pos >= 0) y = __int_as_float(0x7fffffff);
    o[row * o_stride + static_cast<int64_t>(head) * HD + lane * kPer + k] = narrow<T>(y);
  }
}

template <typename T, int HD> szo_status launch_prefix(const View& V, const Prefix& P, const Rows& A, float* ws, cudaStream_t st) {
  const int64_t items = static_cast<int64_t>(V.batch) * V.max_new * A.H;
  SZO_REQUIRE(items <= 0x7fffffff, SZO_ERR_SHAPE, "too many rows and heads for one launch");
  kv8_prefix_row_kernel<T, HD><<<static_cast<unsigned>(ceil_div(items, 4)), 128, 0, st>>>(V, P, static_cast<const T*>(A.q), A.q_stride, static_cast<T*>(A.o),
                                                                                          A.o_stride, A.H, A.scale * 1.4426950408889634f);
  count_launch();
  SZO_CHECK_LAUNCH("kv8_prefix_row_kernel");
  return SZO_OK;
}

szo_status make_prefix(const szo_kv8_prefix* p, const View& V, Prefix* out) {
  SZO_REQUIRE(p != nullptr, SZO_ERR_INVALID_ARG, "NULL prefix");
  SZO_REQUIRE(p->n_groups >= 0 && p->max_seqs >= 0, SZO_ERR_SHAPE, "negative n_groups or max_seqs");
  SZO_REQUIRE(p->n_groups == 0 || p->len != nullptr, SZO_ERR_INVALID_ARG, "NULL len");
  SZO_REQUIRE(p->seqs != nullptr || p->n_groups <= 1, SZO_ERR_SHAPE, "without seqs there is one group");
  SZO_REQUIRE(aligned16(p->len) && aligned16(p->seqs), SZO_ERR_ALIGNMENT, "buffers must be 16-byte aligned");
  *out = Prefix{p->len, p->seqs, p->n_groups, p->seqs == nullptr ? V.batch : p->max_seqs};
  return SZO_OK;
}

size_t workspace_bytes(const View&, const Prefix&, int, int) { return 0; }

}  // namespace
}  // namespace kv8
}  // namespace szo

using namespace szo;

extern "C" {

size_t szo_attention_kv8_prefix_workspace_bytes(const szo_kv8_cache* cache, const szo_kv8_batch* batch, const szo_kv8_prefix* prefix, int32_t n_heads) {
  kv8::View V;
  kv8::Prefix P;
  if (kv8::make_view(cache, batch, &V) != SZO_OK || kv8::make_prefix(prefix, V, &P) != SZO_OK || n_heads <= 0 || n_heads % cache->n_kv_heads != 0) return 0;
  return kv8::workspace_bytes(V, P, n_heads, cache->head_dim);
}

szo_status szo_attention_kv8_prefix(const szo_kv8_cache* cache, const szo_kv8_batch* batch, const szo_kv8_prefix* prefix, const void* q, int64_t q_stride,
                                    void* o, int64_t o_stride, szo_dtype dtype, int32_t n_heads, float scale, void* workspace, size_t workspace_bytes,
                                    void* stream) {
  kv8::View V;
  kv8::Prefix P;
  SZO_TRY(kv8::make_view(cache, batch, &V));
  SZO_TRY(kv8::make_prefix(prefix, V, &P));
  SZO_TRY(kv8::check_rows(cache, q, q_stride, o, o_stride, dtype, n_heads, scale, workspace));
  if (V.batch == 0 || V.max_new == 0 || V.rows == 0) return SZO_OK;
  SZO_TRY(kv8::check_sizes(cache, V, n_heads));
  const size_t need = kv8::workspace_bytes(V, P, n_heads, cache->head_dim);
  SZO_REQUIRE(need == 0 || (workspace && workspace_bytes >= need), SZO_ERR_WORKSPACE, "workspace: %zu bytes needed, %zu given", need,
              workspace ? workspace_bytes : size_t(0));
  SZO_TRY(kv8::set_status_word(&V));
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const kv8::Rows A{q, o, q_stride, o_stride, n_heads, scale};
  float* ws = static_cast<float*>(workspace);
  const bool wide = cache->head_dim == 128;
  if (dtype == SZO_F32) return wide ? kv8::launch_prefix<float, 128>(V, P, A, ws, st) : kv8::launch_prefix<float, 64>(V, P, A, ws, st);
  if (dtype == SZO_BF16) return wide ? kv8::launch_prefix<__nv_bfloat16, 128>(V, P, A, ws, st) : kv8::launch_prefix<__nv_bfloat16, 64>(V, P, A, ws, st);
  return wide ? kv8::launch_prefix<__half, 128>(V, P, A, ws, st) : kv8::launch_prefix<__half, 64>(V, P, A, ws, st);
}

}  // extern "C"
