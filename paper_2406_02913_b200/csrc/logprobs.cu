// Log probabilities of given tokens under softmax(scale * logits), with entropy and the best alternatives,
// and the gradient with respect to the logits.
#include <cmath>

#include "common.cuh"

namespace szo {
namespace {

constexpr int kMaxTop = 32, kMaxTargets = 64;

template <typename T> __device__ __forceinline__ float widen(T x);
template <> __device__ __forceinline__ float widen<float>(float x) { return x; }
template <> __device__ __forceinline__ float widen<__half>(__half x) { return __half2float(x); }
template <> __device__ __forceinline__ float widen<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T narrow(float x);
template <> __device__ __forceinline__ float narrow<float>(float x) { return x; }
template <> __device__ __forceinline__ __half narrow<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// Running softmax statistics of a part of a row: maximum m, s = sum e^(x-m), t = sum e^(x-m) (x-m).
// Terms with e^(x-m) = 0 count nothing in t (their x - m may be -inf).
struct Stat {
  float m, s, t;
};
__device__ __forceinline__ void add(Stat& a, float x) {
  if (x > a.m) {
    const float d = a.m - x, f = a.m == -INFINITY ? 0.f : expf(d);      // every earlier term by e^d, its (x-m) by + d
    a.t = f == 0.f ? 0.f : f * fmaf(d, a.s, a.t);
    a.s *= f;
    a.m = x;
  }
  const float y = x - a.m, e = x == -INFINITY ? 0.f : expf(y);
  a.s += e;
  if (e != 0.f) a.t = fmaf(e, y, a.t);
}
__device__ __forceinline__ Stat merge(const Stat& a, const Stat& b) {
  Stat r;
  r.m = fmaxf(a.m, b.m);
  const float da = a.m - r.m, db = b.m - r.m;
  const float fa = a.m == -INFINITY ? 0.f : expf(da), fb = b.m == -INFINITY ? 0.f : expf(db);
  r.s = fa * a.s + fb * b.s;
  r.t = (fa == 0.f ? 0.f : fa * fmaf(da, a.s, a.t)) + (fb == 0.f ? 0.f : fb * fmaf(db, b.s, b.t));
  if (isnan(a.s) || isnan(b.s)) r.s = r.t = __int_as_float(0x7fffffff);
  return r;
}
// Order of alternatives: larger logit first, then lower index; NaN before everything, -0 = +0.
__device__ __forceinline__ uint64_t order_key(float x, uint32_t idx) {
  uint32_t u = isnan(x) ? 0x7fffffffu : __float_as_uint(x + 0.0f);
  u = u & 0x80000000u ? ~u : u | 0x80000000u;
  return static_cast<uint64_t>(u) << 32 | (0xffffffffu - idx);
}
__device__ __forceinline__ uint32_t key_index(uint64_t k) { return 0xffffffffu - static_cast<uint32_t>(k); }

// One block per row: statistics, then n_top passes that each find the largest key below the previous one.
template <typename T>
__global__ void __launch_bounds__(256)
token_logprobs_kernel(const T* __restrict__ logits, int64_t ld, int vocab, float scale, const int32_t* __restrict__ targets,
                      int n_targets, int n_top, float* __restrict__ logp, float* __restrict__ entropy, float* __restrict__ lse_out,
                      int32_t* __restrict__ top_ids, float* __restrict__ top_logp, int32_t* status) {
  __shared__ Stat part[8];
  __shared__ uint64_t best[8];
  const int64_t row = blockIdx.x;
  const T* x = logits + row * ld;
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  Stat st{-INFINITY, 0.f, 0.f};
  for (int j = threadIdx.x; j < vocab; j += 256) add(st, widen<T>(x[j]) * scale);
#pragma unroll
  for (int o = 16; o; o >>= 1)
    st = merge(st, Stat{__shfl_xor_sync(~0u, st.m, o), __shfl_xor_sync(~0u, st.s, o), __shfl_xor_sync(~0u, st.t, o)});
  if (lane == 0) part[w] = st;
  __syncthreads();
  st = part[0];
  for (int i = 1; i < 8; ++i) st = merge(st, part[i]);
  const float lse = st.m == -INFINITY && st.s == 0.f ? -INFINITY : st.m + logf(st.s);
  auto value = [&](float v) {                                     // log probability of a logit
    const float y = v * scale;
    return y == -INFINITY && !isnan(lse) ? -INFINITY : y - lse;
  };
  if (threadIdx.x == 0) {
    if (lse_out) lse_out[row] = lse;
    if (entropy) entropy[row] = lse == -INFINITY ? 0.f : logf(st.s) - st.t / st.s;
  }
  for (int i = threadIdx.x; i < n_targets; i += 256) {
    const int t = targets[row * n_targets + i];
    if (t >= vocab) atomicExch(status, static_cast<int32_t>(SZO_ERR_INVALID_ARG));
    logp[row * n_targets + i] = t < 0 ? 0.f : t >= vocab ? __int_as_float(0x7fffffff) : value(widen<T>(x[t]));
  }
  uint64_t last = ~0ull;
  for (int r = 0; r < n_top; ++r) {
    uint64_t k = 0;
    for (int j = threadIdx.x; j < vocab; j += 256) {
      const uint64_t c = order_key(widen<T>(x[j]), j);
      if (c < last && c > k) k = c;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      const uint64_t c = __shfl_xor_sync(~0u, k, o);
      if (c > k) k = c;
    }
    __syncthreads();
    if (lane == 0) best[w] = k;
    __syncthreads();
    for (int i = 0; i < 8; ++i)
      if (best[i] > k) k = best[i];
    last = k;
    if (threadIdx.x == 0) {
      top_ids[row * n_top + r] = key_index(k);
      top_logp[row * n_top + r] = value(widen<T>(x[key_index(k)]));
    }
  }
}

// d_logits[j] = scale * ( sum_i d_logp[i] (1[j = t_i] - p_j) - d_entropy p_j (log p_j + H) )
template <typename T>
__global__ void __launch_bounds__(256)
token_logprobs_bwd_kernel(const T* logits, int64_t ld, int vocab, float scale, const int32_t* __restrict__ targets, int n_targets,
                          const float* __restrict__ lse_in, const float* __restrict__ entropy, const float* __restrict__ d_logp,
                          const float* __restrict__ d_entropy, T* d_logits, int64_t dld) {
  const int64_t row = blockIdx.x;
  const T* x = logits + row * ld;
  T* d = d_logits + row * dld;
  const float lse = lse_in[row], gh = d_entropy ? d_entropy[row] : 0.f, ent = d_entropy ? entropy[row] : 0.f;
  float sum = 0.f;
  for (int i = 0; i < n_targets; ++i) {
    const int t = targets[row * n_targets + i];
    if (t >= 0 && t < vocab) sum += d_logp[row * n_targets + i];
  }
  for (int j = threadIdx.x; j < vocab; j += 256) {
    const float lp = widen<T>(x[j]) * scale - lse, p = expf(lp);
    float g = lse == -INFINITY ? 0.f : -p * sum - (p == 0.f || gh == 0.f ? 0.f : gh * p * (lp + ent));
    if (lse != -INFINITY)
      for (int i = 0; i < n_targets; ++i)
        if (targets[row * n_targets + i] == j) g += d_logp[row * n_targets + i];
    d[j] = narrow<T>(g * scale);
  }
}

szo_status check_logits(const void* logits, szo_dtype dt, int64_t rows, int64_t vocab, int64_t ld, float scale, const void* targets,
                        int32_t n_targets) {
  SZO_REQUIRE(dt == SZO_F32 || dt == SZO_BF16 || dt == SZO_F16, SZO_ERR_UNSUPPORTED, "dtype must be f32, bf16 or f16");
  SZO_REQUIRE(rows >= 0 && rows <= 0x7fffffff && vocab >= 1 && vocab <= (1 << 30), SZO_ERR_SHAPE, "need 0 <= rows < 2^31 and 1 <= vocab <= 2^30");
  SZO_REQUIRE(ld >= vocab, SZO_ERR_SHAPE, "row_stride must be at least vocab");
  SZO_REQUIRE(std::isfinite(scale) && scale > 0.f, SZO_ERR_INVALID_ARG, "scale must be positive and finite");
  SZO_REQUIRE(n_targets >= 0 && n_targets <= kMaxTargets, SZO_ERR_UNSUPPORTED, "n_targets must be in [0, %d]", kMaxTargets);
  SZO_REQUIRE(rows == 0 || logits, SZO_ERR_INVALID_ARG, "logits is NULL");
  SZO_REQUIRE(rows == 0 || n_targets == 0 || targets, SZO_ERR_INVALID_ARG, "targets is NULL");
  SZO_REQUIRE(aligned16(logits) && aligned16(targets), SZO_ERR_ALIGNMENT, "buffers must be 16-byte aligned");
  return SZO_OK;
}

}  // namespace
}  // namespace szo

using namespace szo;

extern "C" {

szo_status szo_token_logprobs(const void* logits, szo_dtype dtype, int64_t rows, int64_t vocab, int64_t row_stride, float scale,
                              const int32_t* targets, int32_t n_targets, int32_t n_top, float* logp, float* entropy, float* lse,
                              int32_t* top_ids, float* top_logp, void* stream) {
  SZO_TRY(check_logits(logits, dtype, rows, vocab, row_stride, scale, targets, n_targets));
  SZO_REQUIRE(n_top >= 0 && n_top <= kMaxTop && n_top <= vocab, SZO_ERR_UNSUPPORTED, "n_top must be in [0, min(%d, vocab)]", kMaxTop);
  SZO_REQUIRE(rows == 0 || n_targets == 0 || logp, SZO_ERR_INVALID_ARG, "logp is NULL");
  SZO_REQUIRE(rows == 0 || n_top == 0 || (top_ids && top_logp), SZO_ERR_INVALID_ARG, "top_ids or top_logp is NULL");
  SZO_REQUIRE(aligned16(logp) && aligned16(entropy) && aligned16(lse) && aligned16(top_ids) && aligned16(top_logp), SZO_ERR_ALIGNMENT,
              "buffers must be 16-byte aligned");
  if (rows == 0) return SZO_OK;
  int32_t* status = device_status_word();
  SZO_REQUIRE(status != nullptr, SZO_ERR_CUDA, "no device status word (no CUDA device?)");
  cudaStream_t st = static_cast<cudaStream_t>(stream);
#define SZO_LOGP(T)                                                                                                         \
  token_logprobs_kernel<T><<<static_cast<unsigned>(rows), 256, 0, st>>>(static_cast<const T*>(logits), row_stride,              \
      static_cast<int>(vocab), scale, targets, n_targets, n_top, logp, entropy, lse, top_ids, top_logp, status)
  if (dtype == SZO_F32) SZO_LOGP(float);
  else if (dtype == SZO_BF16) SZO_LOGP(__nv_bfloat16);
  else SZO_LOGP(__half);
#undef SZO_LOGP
  count_launch();
  SZO_CHECK_LAUNCH("token_logprobs_kernel");
  return SZO_OK;
}

szo_status szo_token_logprobs_bwd(const void* logits, szo_dtype dtype, int64_t rows, int64_t vocab, int64_t row_stride, float scale,
                                  const int32_t* targets, int32_t n_targets, const float* lse, const float* entropy,
                                  const float* d_logp, const float* d_entropy, void* d_logits, int64_t d_row_stride, void* stream) {
  SZO_TRY(check_logits(logits, dtype, rows, vocab, row_stride, scale, targets, n_targets));
  SZO_REQUIRE(d_row_stride >= vocab, SZO_ERR_SHAPE, "d_row_stride must be at least vocab");
  SZO_REQUIRE(rows == 0 || (lse && d_logits), SZO_ERR_INVALID_ARG, "lse or d_logits is NULL");
  SZO_REQUIRE(rows == 0 || n_targets == 0 || d_logp, SZO_ERR_INVALID_ARG, "d_logp is NULL");
  SZO_REQUIRE(d_entropy == nullptr || entropy, SZO_ERR_INVALID_ARG, "d_entropy needs entropy");
  SZO_REQUIRE(d_logits != logits || d_row_stride == row_stride, SZO_ERR_INVALID_ARG, "in place needs equal row strides");
  SZO_REQUIRE(aligned16(lse) && aligned16(entropy) && aligned16(d_logp) && aligned16(d_entropy) && aligned16(d_logits), SZO_ERR_ALIGNMENT,
              "buffers must be 16-byte aligned");
  if (rows == 0) return SZO_OK;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
#define SZO_LOGP_BWD(T)                                                                                                     \
  token_logprobs_bwd_kernel<T><<<static_cast<unsigned>(rows), 256, 0, st>>>(static_cast<const T*>(logits), row_stride,          \
      static_cast<int>(vocab), scale, targets, n_targets, lse, entropy, d_logp, d_entropy, static_cast<T*>(d_logits), d_row_stride)
  if (dtype == SZO_F32) SZO_LOGP_BWD(float);
  else if (dtype == SZO_BF16) SZO_LOGP_BWD(__nv_bfloat16);
  else SZO_LOGP_BWD(__half);
#undef SZO_LOGP_BWD
  count_launch();
  SZO_CHECK_LAUNCH("token_logprobs_bwd_kernel");
  return SZO_OK;
}

}  // extern "C"
