// Next-token cross entropy straight from hidden states, and its gradient: the logits x = scale * h W^T of a tile are
// formed, used and dropped.
//
// Forward: every (row, tile of the vocabulary) leaves (m, s): m the tile's largest logit and s = sum 2^(x - m) over it in base 2,
// WITHOUT the target's own term, which is kept apart.  Joined over the tiles with S and M,
//   lse = M + log2(S + 2^(x_t - M)),   loss = log(1 + S 2^(M - x_t)):
// loss does not come from the difference of two numbers of the size of lse, so a confident row's keeps its relative precision.
// Backward: G = scale ((a + b) p - a 1[t]) (a = d_loss, b = d_lse), p = 2^(x - lse), for a piece of the vocabulary at a time, in the
// 16-bit type of the products that follow; p - 1 of the target is formed before the rounding (expm1).
#include <cmath>

#include "head_ce.cuh"

namespace szo {
namespace head {

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kSide = 64, kDepthK = 16, kThreads = 256;

template <typename T> __device__ __forceinline__ float widen(T x);
template <> __device__ __forceinline__ float widen<__half>(__half x) { return __half2float(x); }
template <> __device__ __forceinline__ float widen<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T narrow(float x);
template <> __device__ __forceinline__ __half narrow<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// A product of two 16-bit matrices by strides: sum_k A(m, k) B(n, k), 64 x 64 per block, 4 x 4 per thread.
template <typename T> struct Operand {
  const T* p;
  int64_t s_row, s_k, rows;
};
template <typename T>
__device__ __forceinline__ void tile_product(const Operand<T>& A, const Operand<T>& B, int64_t m0, int64_t n0, int64_t K, float (&acc)[4][4]) {
  __shared__ float as[kDepthK][kSide + 4], bs[kDepthK][kSide + 4];
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = 0.f;
  for (int64_t k0 = 0; k0 < K; k0 += kDepthK) {
    for (int i = threadIdx.x; i < kSide * kDepthK; i += kThreads) {
      const int r = i / kDepthK, k = i % kDepthK;
      as[k][r] = m0 + r < A.rows && k0 + k < K ? widen<T>(A.p[(m0 + r) * A.s_row + (k0 + k) * A.s_k]) : 0.f;
      bs[k][r] = n0 + r < B.rows && k0 + k < K ? widen<T>(B.p[(n0 + r) * B.s_row + (k0 + k) * B.s_k]) : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kDepthK; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(as[k][ty * 4 + i], bs[k][tx * 4 + j], acc[i][j]);
    __syncthreads();
  }
}

// Statistics of 64 x 64 logits: grid (row tiles, vocabulary tiles)
template <typename T>
__global__ void __launch_bounds__(kThreads) head_stats_kernel(Operand<T> h, Operand<T> W, int64_t d, float c, const int32_t* __restrict__ targets,
                                                              float2* __restrict__ part, float* __restrict__ xt) {
  float acc[4][4];
  const int64_t m0 = static_cast<int64_t>(blockIdx.x) * kSide, n0 = static_cast<int64_t>(blockIdx.y) * kSide;
  tile_product(h, W, m0, n0, d, acc);
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  for (int i = 0; i < 4; ++i) {
    const int64_t r = m0 + ty * 4 + i;
    const int64_t t = r < h.rows ? targets[r] : -1;
    float m = -INFINITY, s = 0.f;
    for (int j = 0; j < 4; ++j) {
      const int64_t col = n0 + tx * 4 + j;
      acc[i][j] *= c;
      if (col == t && t < W.rows) xt[r] = acc[i][j];
      if (col == t || col >= W.rows) acc[i][j] = -INFINITY;
      m = fmaxf(m, acc[i][j]);
    }
    for (int o = 8; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    const float ref = m == -INFINITY ? 0.f : m;
    for (int j = 0; j < 4; ++j) s += exp2f(acc[i][j] - ref);
    for (int o = 8; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (tx == 0 && r < h.rows) part[blockIdx.y * h.rows + r] = make_float2(m, s);
  }
}

// Joins a row's parts: 32 rows per block, eight warps of parts, joined in warp order
__global__ void __launch_bounds__(256) head_join_kernel(const float2* __restrict__ part, const float* __restrict__ xt, const int32_t* __restrict__ targets,
                                                        int64_t rows, int64_t vocab, int parts, float* __restrict__ loss, float* __restrict__ lse,
                                                        int32_t* status) {
  __shared__ float ms[8][32], ss[8][32];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int64_t r = static_cast<int64_t>(blockIdx.x) * 32 + lane;
  float m = -INFINITY, s = 0.f;
  if (r < rows)
    for (int i = w; i < parts; i += 8) {
      const float2 p = part[i * rows + r];
      const float mn = fmaxf(m, p.x), ref = mn == -INFINITY ? 0.f : mn;
      s = s * exp2f(m - ref) + p.y * exp2f(p.x - ref);
      m = mn;
    }
  ms[w][lane] = m;
  ss[w][lane] = s;
  __syncthreads();
  if (w != 0 || r >= rows) return;
  for (int i = 0; i < 8; ++i) m = fmaxf(m, ms[i][lane]);
  const float ref = m == -INFINITY ? 0.f : m;
  s = 0.f;
  for (int i = 0; i < 8; ++i) s += ss[i][lane] * exp2f(ms[i][lane] - ref);
  const int32_t t = targets[r];
  float out = 0.f, total;
  if (t < 0 || t >= vocab) {
    total = s == 0.f ? -INFINITY : kLn2 * (m + log2f(s));
    if (t >= vocab) {
      out = __int_as_float(0x7fffffff);
      atomicExch(status, static_cast<int32_t>(SZO_ERR_INVALID_ARG));
    }
  } else {
    const float x = xt[r], top = fmaxf(m, x), tref = top == -INFINITY ? 0.f : top;
    const float all = s * exp2f(m - tref) + exp2f(x - tref);
    total = all == 0.f ? -INFINITY : kLn2 * (tref + log2f(all));
    out = m - x > 64.f ? total - kLn2 * x : s == 0.f ? 0.f : log1pf(s * exp2f(m - x));
    if (isnan(total)) out = total;
  }
  if (isnan(total) || total == INFINITY) total = out = __int_as_float(0x7fffffff);
  loss[r] = out;
  if (lse != nullptr) lse[r] = total;
}

// What the gradient needs of a row: x = lse in base 2, y = weight of p, z = weight of the target (both times scale and, for fp16, a
// power of two that brings the larger to [2^13, 2^14)), w = that power's inverse.  Rows that weigh nothing have y = z = 0.
__global__ void head_rows_kernel(const int32_t* __restrict__ targets, const float* __restrict__ lse, const float* __restrict__ d_loss,
                                 const float* __restrict__ d_lse, int64_t rows, int64_t vocab, float scale, bool half, float4* __restrict__ info,
                                 int32_t* __restrict__ exponent) {
  const int64_t r = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
  if (r >= rows) return;
  const int32_t t = targets[r];
  const float a = t >= 0 && t < vocab ? d_loss[r] : 0.f, b = d_lse != nullptr ? d_lse[r] : 0.f, l = lse[r];
  float y = scale * (a + b), z = scale * a, inv = 1.f;
  if (l == -INFINITY) y = z = 0.f;
  if (half && (y != 0.f || z != 0.f)) {
    const float top = fmaxf(fmaxf(fabsf(y), fabsf(z)), fabsf(scale * b));
    const int e = min(max(((__float_as_int(top) >> 23) & 255) - 127, -100), 100);      // (rows beyond: as near as it goes)
    const float f = __int_as_float((13 - e + 127) << 23);
    y *= f;
    z *= f;
    inv = __int_as_float((e - 13 + 127) << 23);
    atomicMax(exponent, e);
  }
  info[r] = make_float4(l * kLog2e, y, z, inv);
}

// h for dW: rows that weigh nothing become zeros; fp16 rows are brought to the largest weight (exactly but for what falls below fp16's range)
template <typename T>
__global__ void head_copy_kernel(const T* __restrict__ h, int64_t h_stride, int64_t rows, int64_t d, const float4* __restrict__ info,
                                 const int32_t* __restrict__ exponent, T* __restrict__ out) {
  const int64_t per = d / 8, i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
  if (i >= rows * per) return;
  const int64_t r = i / per, c = i % per * 8;
  const float4 f = info[r];
  uint4 x = make_uint4(0u, 0u, 0u, 0u);
  if (f.y != 0.f || f.z != 0.f) {
    x = *reinterpret_cast<const uint4*>(h + r * h_stride + c);
    if constexpr (sizeof(T) == 2 && !std::is_same<T, __nv_bfloat16>::value) {
      const float to = f.w * __int_as_float((13 - *exponent + 127) << 23);
      T* e = reinterpret_cast<T*>(&x);
#pragma unroll
      for (int k = 0; k < 8; ++k) e[k] = narrow<T>(widen<T>(e[k]) * to);
    }
  }
  *reinterpret_cast<uint4*>(out + r * d + c) = x;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) head_grad_kernel(Operand<T> h, Operand<T> W, int64_t d, int64_t j0, float c, const int32_t* __restrict__ targets,
                                                             const float4* __restrict__ info, T* __restrict__ G, int64_t g_stride) {
  float acc[4][4];
  const int64_t m0 = static_cast<int64_t>(blockIdx.x) * kSide, n0 = static_cast<int64_t>(blockIdx.y) * kSide;
  tile_product(h, W, m0, n0, d, acc);
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  for (int i = 0; i < 4; ++i) {
    const int64_t r = m0 + ty * 4 + i;
    if (r >= h.rows) continue;
    const float4 f = info[r];
    const int64_t t = static_cast<int64_t>(targets[r]) - j0;
    for (int j = 0; j < 4; ++j) {
      const int64_t col = n0 + tx * 4 + j;
      if (col >= W.rows) continue;
      const float x = fmaf(acc[i][j], c, -f.x), p = exp2f(x);
      float g = f.y * p;
      if (col == t) g = fmaf(f.y - f.z, p, f.z * expm1f(x * kLn2));
      if (f.y == 0.f && f.z == 0.f) g = 0.f;
      G[r * g_stride + col] = narrow<T>(g);
    }
  }
}

// acc = or += A B^T in fp32
template <typename T>
__global__ void __launch_bounds__(kThreads) head_sum_kernel(Operand<T> A, Operand<T> B, int64_t K, float* __restrict__ out, int64_t stride, bool add) {
  float acc[4][4];
  const int64_t m0 = static_cast<int64_t>(blockIdx.x) * kSide, n0 = static_cast<int64_t>(blockIdx.y) * kSide;
  tile_product(A, B, m0, n0, K, acc);
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int64_t r = m0 + ty * 4 + i, col = n0 + tx * 4 + j;
      if (r >= A.rows || col >= B.rows) continue;
      float* p = out + r * stride + col;
      *p = add ? *p + acc[i][j] : acc[i][j];
    }
}
// out = A B^T times the power of two that the rows were brought to, rounded
template <typename T>
__global__ void __launch_bounds__(kThreads) head_out_kernel(Operand<T> A, Operand<T> B, int64_t K, T* __restrict__ out, int64_t stride,
                                                            const int32_t* __restrict__ exponent) {
  float acc[4][4];
  const int64_t m0 = static_cast<int64_t>(blockIdx.x) * kSide, n0 = static_cast<int64_t>(blockIdx.y) * kSide;
  tile_product(A, B, m0, n0, K, acc);
  const float f = weight_of<T>(exponent);
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int64_t r = m0 + ty * 4 + i, col = n0 + tx * 4 + j;
      if (r < A.rows && col < B.rows) out[r * stride + col] = narrow<T>(acc[i][j] * f);
    }
}

// dh: the sums of a row times its power of two, rounded
template <typename T>
__global__ void head_round_kernel(const float* __restrict__ acc, int64_t rows, int64_t d, const float4* __restrict__ info, T* __restrict__ out,
                                  int64_t stride) {
  const int64_t per = d / 8, i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
  if (i >= rows * per) return;
  const int64_t r = i / per, c = i % per * 8;
  const float f = info[r].w;
  alignas(16) T y[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) y[k] = narrow<T>(acc[r * d + c + k] * f);
  *reinterpret_cast<uint4*>(out + r * stride + c) = *reinterpret_cast<const uint4*>(y);
}

// ------------------------------------------------------------------------------ host side
struct Shape {
  int64_t rows, vocab, d;
};
struct Parts {                                                    // of a workspace, in bytes from its start
  size_t part, xt, info, exponent, copy, G, acc, total;
  int64_t piece;                                                  // vocabulary rows of a piece
};
Parts forward_parts(const Shape& s) {
  Parts p = {};
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t from = at;
    at += round_up(bytes, 256);
    return from;
  };
  p.part = take(static_cast<size_t>(ceil_div(s.vocab, kSide)) * s.rows * sizeof(float2));
  p.xt = take(static_cast<size_t>(s.rows) * sizeof(float));
  p.total = at;
  return p;
}
Parts backward_parts(const Shape& s, bool dh, bool dw) {
  Parts p = {};
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t from = at;
    at += round_up(bytes, 256);
    return from;
  };
  p.piece = s.vocab < 8192 ? static_cast<int64_t>(round_up(s.vocab, 64)) : 8192;
  p.info = take(static_cast<size_t>(s.rows) * sizeof(float4));
  p.exponent = take(sizeof(int32_t));
  if (dw) p.copy = take(static_cast<size_t>(s.rows) * s.d * 2);
  p.G = take(static_cast<size_t>(s.rows) * p.piece * 2);
  if (dh) p.acc = take(static_cast<size_t>(s.rows) * s.d * sizeof(float));
  p.total = at;
  return p;
}
bool fits(int64_t rows, int64_t vocab, int64_t d) {
  constexpr int64_t kMost = 0x7fffff00;
  return rows >= 0 && vocab > 0 && d > 0 && d % 8 == 0 && rows <= kMost && vocab <= kMost && d <= kMost;
}
szo_status check(const void* h, int64_t h_stride, const void* W, int64_t w_stride, szo_dtype dtype, int64_t rows, int64_t vocab, int64_t d,
                 float scale, const int32_t* targets) {
  SZO_REQUIRE(dtype == SZO_BF16 || dtype == SZO_F16, SZO_ERR_UNSUPPORTED, "dtype must be bf16 or f16");
  SZO_REQUIRE(fits(rows, vocab, d), SZO_ERR_SHAPE, "rows >= 0, vocab > 0 and d a positive multiple of 8, each below 2^31 - 256");
  SZO_REQUIRE(std::isfinite(scale) && scale >= 1e-30f && scale <= 1e30f, SZO_ERR_INVALID_ARG, "scale must be in [1e-30, 1e30]");
  SZO_REQUIRE(W != nullptr && (rows == 0 || (h != nullptr && targets != nullptr)), SZO_ERR_INVALID_ARG, "NULL h, W or targets");
  SZO_REQUIRE(h_stride >= d && w_stride >= d, SZO_ERR_SHAPE, "row strides must be at least d");
  SZO_REQUIRE(aligned16(h) && aligned16(W) && aligned16(targets) && h_stride % 8 == 0 && w_stride % 8 == 0, SZO_ERR_ALIGNMENT,
              "buffers and rows must be 16-byte aligned");
  return SZO_OK;
}
unsigned blocks_of(int64_t n, int per) { return static_cast<unsigned>(ceil_div(n, per)); }

template <typename T>
szo_status forward(const Shape& s, const T* h, int64_t hs, const T* W, int64_t ws_, float scale, const int32_t* targets, float* loss, float* lse,
                   unsigned char* ws, int32_t* status, cudaStream_t st) {
  const Parts p = forward_parts(s);
  float2* part = reinterpret_cast<float2*>(ws + p.part);
  float* xt = reinterpret_cast<float*>(ws + p.xt);
  const int parts = static_cast<int>(ceil_div(s.vocab, kSide));
  head_stats_kernel<T><<<dim3(blocks_of(s.rows, kSide), parts), kThreads, 0, st>>>(Operand<T>{h, hs, 1, s.rows}, Operand<T>{W, ws_, 1, s.vocab}, s.d,
                                                                                 scale * kLog2e, targets, part, xt);
  count_launch();
  SZO_CHECK_LAUNCH("head_stats_kernel");
  head_join_kernel<<<blocks_of(s.rows, 32), 256, 0, st>>>(part, xt, targets, s.rows, s.vocab, parts, loss, lse, status);
  count_launch();
  SZO_CHECK_LAUNCH("head_join_kernel");
  return SZO_OK;
}

template <typename T>
szo_status backward(const Shape& s, const T* h, int64_t hs, const T* W, int64_t ws_, float scale, const int32_t* targets, const float* lse,
                    const float* d_loss, const float* d_lse, T* dh, int64_t dhs, T* dw, int64_t dws, unsigned char* ws, cudaStream_t st) {
  const Parts p = backward_parts(s, dh != nullptr, dw != nullptr);
  float4* info = reinterpret_cast<float4*>(ws + p.info);
  int32_t* exponent = reinterpret_cast<int32_t*>(ws + p.exponent);
  T* copy = reinterpret_cast<T*>(ws + p.copy);
  T* G = reinterpret_cast<T*>(ws + p.G);
  float* acc = reinterpret_cast<float*>(ws + p.acc);
  SZO_CHECK_CUDA(cudaMemsetAsync(exponent, 0x80, sizeof(int32_t), st));      // (below every exponent)
  head_rows_kernel<<<blocks_of(s.rows, 256), 256, 0, st>>>(targets, lse, d_loss, d_lse, s.rows, s.vocab, scale, !std::is_same<T, __nv_bfloat16>::value,
                                                         info, exponent);
  count_launch();
  if (dw != nullptr) {
    head_copy_kernel<T><<<blocks_of(s.rows * (s.d / 8), 256), 256, 0, st>>>(h, hs, s.rows, s.d, info, exponent, copy);
    count_launch();
  }
  for (int64_t j0 = 0; j0 < s.vocab; j0 += p.piece) {
    const int64_t n = s.vocab - j0 < p.piece ? s.vocab - j0 : p.piece;
    head_grad_kernel<T><<<dim3(blocks_of(s.rows, kSide), blocks_of(n, kSide)), kThreads, 0, st>>>(
        Operand<T>{h, hs, 1, s.rows}, Operand<T>{W + j0 * ws_, ws_, 1, n}, s.d, j0, scale * kLog2e, targets, info, G, p.piece);
    count_launch();
    if (dh != nullptr) {
      head_sum_kernel<T><<<dim3(blocks_of(s.rows, kSide), blocks_of(s.d, kSide)), kThreads, 0, st>>>(
          Operand<T>{G, p.piece, 1, s.rows}, Operand<T>{W + j0 * ws_, 1, ws_, s.d}, n, acc, s.d, j0 > 0);
      count_launch();
    }
    if (dw != nullptr) {
      head_out_kernel<T><<<dim3(blocks_of(n, kSide), blocks_of(s.d, kSide)), kThreads, 0, st>>>(
          Operand<T>{G, 1, p.piece, n}, Operand<T>{copy, 1, s.d, s.d}, s.rows, dw + j0 * dws, dws, exponent);
      count_launch();
    }
  }
  if (dh != nullptr) {
    head_round_kernel<T><<<blocks_of(s.rows * (s.d / 8), 256), 256, 0, st>>>(acc, s.rows, s.d, info, dh, dhs);
    count_launch();
  }
  SZO_CHECK_LAUNCH("the kernels of szo_head_ce_bwd");
  return SZO_OK;
}

}  // namespace
}  // namespace head
}  // namespace szo

using namespace szo;

extern "C" {

size_t szo_head_ce_workspace_bytes(int64_t rows, int64_t vocab, int64_t d) {
  return head::fits(rows, vocab, d) && rows > 0 ? head::forward_parts({rows, vocab, d}).total : 0;
}

szo_status szo_head_ce(const void* h, int64_t h_stride, const void* W, int64_t w_stride, szo_dtype dtype, int64_t rows, int64_t vocab, int64_t d,
                       float scale, const int32_t* targets, float* loss, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  SZO_TRY(head::check(h, h_stride, W, w_stride, dtype, rows, vocab, d, scale, targets));
  SZO_REQUIRE(rows == 0 || loss != nullptr, SZO_ERR_INVALID_ARG, "NULL loss");
  SZO_REQUIRE(aligned16(loss) && aligned16(lse) && aligned16(workspace), SZO_ERR_ALIGNMENT, "buffers must be 16-byte aligned");
  if (rows == 0) return SZO_OK;
  const size_t need = szo_head_ce_workspace_bytes(rows, vocab, d);
  SZO_REQUIRE(workspace && workspace_bytes >= need, SZO_ERR_WORKSPACE, "workspace: %zu bytes needed, %zu given", need,
              workspace ? workspace_bytes : size_t(0));
  int32_t* status = device_status_word();
  SZO_REQUIRE(status != nullptr, SZO_ERR_CUDA, "no device status word (no CUDA device?)");
  const head::Shape s{rows, vocab, d};
  auto* ws = static_cast<unsigned char*>(workspace);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (dtype == SZO_BF16)
    return head::forward(s, static_cast<const __nv_bfloat16*>(h), h_stride, static_cast<const __nv_bfloat16*>(W), w_stride, scale, targets, loss, lse, ws,
                         status, st);
  return head::forward(s, static_cast<const __half*>(h), h_stride, static_cast<const __half*>(W), w_stride, scale, targets, loss, lse, ws, status, st);
}

size_t szo_head_ce_bwd_workspace_bytes(int64_t rows, int64_t vocab, int64_t d, int32_t want_dh, int32_t want_dw) {
  if (!head::fits(rows, vocab, d) || rows == 0 || (!want_dh && !want_dw)) return 0;
  return head::backward_parts({rows, vocab, d}, want_dh != 0, want_dw != 0).total;
}

szo_status szo_head_ce_bwd(const void* h, int64_t h_stride, const void* W, int64_t w_stride, szo_dtype dtype, int64_t rows, int64_t vocab, int64_t d,
                           float scale, const int32_t* targets, const float* lse, const float* d_loss, const float* d_lse, void* dh, int64_t dh_stride,
                           void* dW, int64_t dw_stride, void* workspace, size_t workspace_bytes, void* stream) {
  SZO_TRY(head::check(h, h_stride, W, w_stride, dtype, rows, vocab, d, scale, targets));
  SZO_REQUIRE(rows == 0 || (lse != nullptr && d_loss != nullptr), SZO_ERR_INVALID_ARG, "NULL lse or d_loss");
  SZO_REQUIRE((dh == nullptr || dh_stride >= d) && (dW == nullptr || dw_stride >= d), SZO_ERR_SHAPE, "row strides must be at least d");
  SZO_REQUIRE(aligned16(lse) && aligned16(d_loss) && aligned16(d_lse) && aligned16(dh) && aligned16(dW) && aligned16(workspace) &&
                  (dh == nullptr || dh_stride % 8 == 0) && (dW == nullptr || dw_stride % 8 == 0),
              SZO_ERR_ALIGNMENT, "buffers and rows must be 16-byte aligned");
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (rows == 0) {
    if (dW != nullptr) SZO_CHECK_CUDA(cudaMemset2DAsync(dW, dw_stride * 2, 0, d * 2, vocab, st));
    return SZO_OK;
  }
  if (dh == nullptr && dW == nullptr) return SZO_OK;
  const size_t need = szo_head_ce_bwd_workspace_bytes(rows, vocab, d, dh != nullptr, dW != nullptr);
  SZO_REQUIRE(workspace && workspace_bytes >= need, SZO_ERR_WORKSPACE, "workspace: %zu bytes needed, %zu given", need,
              workspace ? workspace_bytes : size_t(0));
  const head::Shape s{rows, vocab, d};
  auto* ws = static_cast<unsigned char*>(workspace);
  if (dtype == SZO_BF16)
    return head::backward(s, static_cast<const __nv_bfloat16*>(h), h_stride, static_cast<const __nv_bfloat16*>(W), w_stride, scale, targets, lse, d_loss,
                          d_lse, static_cast<__nv_bfloat16*>(dh), dh_stride, static_cast<__nv_bfloat16*>(dW), dw_stride, ws, st);
  return head::backward(s, static_cast<const __half*>(h), h_stride, static_cast<const __half*>(W), w_stride, scale, targets, lse, d_loss, d_lse,
                        static_cast<__half*>(dh), dh_stride, static_cast<__half*>(dW), dw_stride, ws, st);
}

}  // extern "C"
