// Log probabilities of given tokens under softmax(scale * logits), with entropy and the best alternatives,
// and the gradient with respect to the logits.
//
// Forward: one pass over a row.  Every thread keeps a reference maximum m, s = sum e^(x-m), t = sum e^(x-m) (x-m) and
// its best (logit, index); what bounds it is reading the logits, next to it the exponentials (16 per cycle and SM: 0.72 of
// the time that 16-bit logits take to arrive), so sums run as packed pairs and m moves only when it is exceeded by e^8.
// lse = m + log s and H = log s - t / s come out of the same pass.  Few rows are cut over the blocks of a cluster and
// joined through distributed shared memory.
//
// Best alternatives: the n-th largest of the threads' best keys is a lower bound of the row's n-th largest key, and
// only the (at most n) threads whose best reaches it can hold a candidate: those alone read their part again, from L2.
// Keys are (logit, index) in one 64-bit number, all different, so ties need no care and the result no order of arrival.
#include <cooperative_groups.h>

#include <cmath>

#include "common.cuh"

namespace cg = cooperative_groups;

namespace szo {
namespace {

constexpr int kMaxTop = 32, kMaxTargets = 64, kThreads = 256, kMaxCand = 2048, kMaxCluster = 8;
constexpr float kLog2e = 1.4426950408889634f, kSlack = 8.0f;

template <typename T> __device__ __forceinline__ float widen(T x);
template <> __device__ __forceinline__ float widen<float>(float x) { return x; }
template <> __device__ __forceinline__ float widen<__half>(__half x) { return __half2float(x); }
template <> __device__ __forceinline__ float widen<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T narrow(float x);
template <> __device__ __forceinline__ float narrow<float>(float x) { return x; }
template <> __device__ __forceinline__ __half narrow<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

template <typename T> struct alignas(16) Vec {
  static constexpr int kN = 16 / static_cast<int>(sizeof(T));
  T x[kN];
};
// A row as 16-byte vectors on 16-byte addresses: vector v holds elements v * kN - off + [0, kN), of which the first and
// the last vector may have some outside the row (those are neither read nor written).
template <typename T> struct Row {
  T* base;
  int off, n, vecs;
  __device__ __forceinline__ Row(T* row, int vocab) {
    off = static_cast<int>((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(T));
    base = row - off;
    n = vocab;
    vecs = (off + vocab + Vec<T>::kN - 1) / Vec<T>::kN;
  }
  __device__ __forceinline__ bool whole(int v) const { return v * Vec<T>::kN >= off && (v + 1) * Vec<T>::kN <= off + n; }
  __device__ __forceinline__ bool inside(int v, int i) const { return v * Vec<T>::kN + i >= off && v * Vec<T>::kN + i < off + n; }
  __device__ __forceinline__ int index(int v, int i) const { return v * Vec<T>::kN + i - off; }
  template <typename U> __device__ __forceinline__ void load(int v, U (&x)[Vec<T>::kN], float outside) const {
    if (whole(v)) {
      const Vec<T> r = *reinterpret_cast<const Vec<T>*>(base + static_cast<int64_t>(v) * Vec<T>::kN);
#pragma unroll
      for (int i = 0; i < Vec<T>::kN; ++i) x[i] = widen<typename std::remove_const<T>::type>(r.x[i]);
    } else {
#pragma unroll
      for (int i = 0; i < Vec<T>::kN; ++i)
        x[i] = inside(v, i) ? widen<typename std::remove_const<T>::type>(base[static_cast<int64_t>(v) * Vec<T>::kN + i]) : outside;
    }
  }
};

__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// pairs of fp32 in one register pair
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ float2 unpair(uint64_t p) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(p));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// Softmax statistics of a part of a row relative to m; a part that holds NaN or +inf has s = NaN.
struct Stat {
  float m, s, t;
};
__device__ __forceinline__ Stat merge(const Stat& a, const Stat& b) {
  Stat r;
  r.m = fmaxf(a.m, b.m);
  const float da = a.m - r.m, db = b.m - r.m;
  const float fa = a.m == -INFINITY ? 0.f : expf(da), fb = b.m == -INFINITY ? 0.f : expf(db);
  r.s = fa * a.s + fb * b.s;
  r.t = (fa == 0.f ? 0.f : fa * fmaf(da, a.s, a.t)) + (fb == 0.f ? 0.f : fb * fmaf(db, b.s, b.t));
  return r;
}
// Order of alternatives: larger logit first, then lower index; NaN before everything, -0 = +0.  Never 0.
__device__ __forceinline__ uint64_t order_key(float x, uint32_t idx) {
  uint32_t u = isnan(x) ? 0x7fffffffu : __float_as_uint(x + 0.0f);
  u = u & 0x80000000u ? ~u : u | 0x80000000u;
  return static_cast<uint64_t>(u) << 32 | (0xffffffffu - idx);
}
__device__ __forceinline__ uint32_t key_index(uint64_t k) { return 0xffffffffu - static_cast<uint32_t>(k); }

struct Out {
  float *logp, *entropy, *lse, *top_logp;
  int32_t* top_ids;
};

// Block = a row, or the rank-th of `parts` shares of its vectors; a cluster = a row.
template <typename T>
__global__ void __launch_bounds__(kThreads, 4)
token_logprobs_kernel(const T* __restrict__ logits, int64_t ld, int vocab, float scale, const int32_t* __restrict__ targets,
                      int n_targets, int n_top, Out out, int32_t* status, int parts) {
  constexpr int kN = Vec<T>::kN, kW = kThreads / 32, kUnroll = 4;
  __shared__ Stat part[kW];
  __shared__ Stat mine;
  __shared__ uint64_t keys[kThreads];                             // best of every thread; later the cluster's lists
  __shared__ uint64_t cand[kMaxCand];
  __shared__ uint64_t top[kMaxTop];
  __shared__ uint64_t bound;
  __shared__ int n_cand;
  const int64_t row = blockIdx.x / parts;
  const int rank = blockIdx.x % parts, tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  const Row<const T> R(logits + row * ld, vocab);
  const int v_lo = static_cast<int>(static_cast<int64_t>(R.vecs) * rank / parts), v_hi = static_cast<int>(static_cast<int64_t>(R.vecs) * (rank + 1) / parts);

  float m = -INFINITY, best = -INFINITY;
  uint64_t s2 = 0, t2 = 0, key = 0;
  bool bad = false;
  const uint64_t log2e2 = pair(kLog2e, kLog2e);
  auto take = [&](const float (&x)[kN], int v) {
    float top_x = x[0];
#pragma unroll
    for (int i = 1; i < kN; ++i) top_x = max_nan(top_x, x[i]);
    if (n_top > 0 && (key == 0 || !(top_x <= best))) {            // (vectors come in rising order: equal logits keep the earlier key)
#pragma unroll
      for (int i = 0; i < kN; ++i) {
        if (!R.inside(v, i)) continue;
        const uint64_t k = order_key(x[i], R.index(v, i));
        if (k > key) key = k;
      }
      best = top_x;
    }
    const float z = __fmul_rn(top_x, scale);
    if (!(z < INFINITY)) bad = true;
    if (!(z > -INFINITY)) return;                                 // nothing but masked tokens (or NaN)
    if (z > m + kSlack || m == -INFINITY) {
      const float d = fmaxf(m - z, -120.f), f = ex2(d * kLog2e);       // every earlier term by e^d, its (x-m) by + d
      const uint64_t f2 = pair(f, f), d2 = pair(d, d);
      t2 = mul2(f2, fma2(d2, s2, t2));
      s2 = mul2(f2, s2);
      m = z;
    }
    const uint64_t ref = pair(-m, -m);
#pragma unroll
    for (int i = 0; i < kN; i += 2) {
      // x * scale is rounded as in m (a product fused with the subtraction would leave its rounding error, which is huge
      // near the end of fp32's range), by single products: the assembler fuses a packed product with a packed sum
      const float2 a = unpair(add2(pair(__fmul_rn(x[i], scale), __fmul_rn(x[i + 1], scale)), ref));
      const uint64_t y = pair(fmaxf(a.x, -120.f), fmaxf(a.y, -120.f));         // e^-120 is 0 in fp32, and 0 * -120 too
      const float2 b = unpair(mul2(y, log2e2));
      const uint64_t e = pair(ex2(b.x), ex2(b.y));
      s2 = add2(s2, e);
      t2 = fma2(e, y, t2);
    }
  };
  int v = v_lo + tid;
  auto take_one = [&]() {
    float x[kN];
    R.load(v, x, -INFINITY);
    take(x, v);
    v += kThreads;
  };
  if (v < v_hi && !R.whole(v)) take_one();
  for (; v + (kUnroll - 1) * kThreads < v_hi && R.whole(v + (kUnroll - 1) * kThreads); v += kUnroll * kThreads) {      // all loads first
    Vec<T> r[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) r[u] = *reinterpret_cast<const Vec<T>*>(R.base + static_cast<int64_t>(v + u * kThreads) * kN);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      float x[kN];
#pragma unroll
      for (int i = 0; i < kN; ++i) x[i] = widen<T>(r[u].x[i]);
      take(x, v + u * kThreads);
    }
  }
  while (v < v_hi) take_one();
  const float2 sp = unpair(s2), tp = unpair(t2);
  Stat st{m, bad ? __int_as_float(0x7fffffff) : sp.x + sp.y, tp.x + tp.y};
#pragma unroll
  for (int o = 16; o; o >>= 1)
    st = merge(st, Stat{__shfl_xor_sync(~0u, st.m, o), __shfl_xor_sync(~0u, st.s, o), __shfl_xor_sync(~0u, st.t, o)});
  if (lane == 0) part[w] = st;
  if (tid == 0) {
    n_cand = 0;
    bound = 1;
  }
  if (tid < kMaxTop) top[tid] = 0;
  keys[tid] = key;
  __syncthreads();
  st = part[0];
  for (int i = 1; i < kW; ++i) st = merge(st, part[i]);

  if (n_top > 0) {
    if (key != 0) {
      int above = 0;
#pragma unroll 8
      for (int i = 0; i < kThreads; ++i) above += keys[i] > key;
      if (above == n_top - 1) bound = key;
    }
    __syncthreads();
    if (key >= bound) {
#pragma unroll 4
      for (v = v_lo + tid; v < v_hi; v += kThreads) {
        float x[kN];
        R.load(v, x, -INFINITY);
#pragma unroll
        for (int i = 0; i < kN; ++i) {
          const uint64_t k = R.inside(v, i) ? order_key(x[i], R.index(v, i)) : 0;
          if (k >= bound) {
            const int at = atomicAdd(&n_cand, 1);
            if (at < kMaxCand) cand[at] = k;
          }
        }
      }
    }
    __syncthreads();
    if (n_cand <= kMaxCand) {
      for (int c = tid; c < n_cand; c += kThreads) {
        const uint64_t k = cand[c];
        int above = 0;
        for (int i = 0; i < n_cand; ++i) above += cand[i] > k;
        if (above < n_top) top[above] = k;
      }
    } else {                                                      // the largest logits crowd in few threads: one pass for each
      uint64_t last = ~0ull;
      for (int r = 0; r < n_top; ++r) {
        uint64_t k = 0;
        for (v = v_lo + tid; v < v_hi; v += kThreads) {
          float x[kN];
          R.load(v, x, -INFINITY);
#pragma unroll
          for (int i = 0; i < kN; ++i) {
            const uint64_t c = R.inside(v, i) ? order_key(x[i], R.index(v, i)) : 0;
            if (c < last && c > k) k = c;
          }
        }
        __syncthreads();
        keys[tid] = k;
        __syncthreads();
        for (int i = 0; i < kThreads; ++i) k = keys[i] > k ? keys[i] : k;
        if (tid == 0) top[r] = k;
        last = k;
      }
    }
    __syncthreads();
  }

  if (parts > 1) {                                                // the shares joined in order, by the first block
    if (tid == 0) mine = st;
    cg::cluster_group cluster = cg::this_cluster();
    cluster.sync();
    if (rank == 0) {
      for (int i = 1; i < parts; ++i) st = merge(st, *cluster.map_shared_rank(&mine, i));
      if (n_top > 0) {
        const int n = parts * n_top;                              // at most kThreads
        uint64_t k = 0;
        if (tid < n) k = *cluster.map_shared_rank(&top[tid % n_top], tid / n_top);
        __syncthreads();                                          // (nobody reads keys or top any more)
        if (tid < n) keys[tid] = k;
        __syncthreads();
        int above = 0;
        for (int i = 0; i < n; ++i) above += keys[i] > k;
        if (k != 0 && above < n_top) top[above] = k;
        __syncthreads();
      }
    }
    cluster.sync();
    if (rank != 0) return;
  }

  const float lse = st.m == -INFINITY && st.s == 0.f ? -INFINITY : st.m + logf(st.s);
  auto value = [&](float x) {                                     // log probability of a logit
    const float z = __fmul_rn(x, scale);
    return z == -INFINITY && !isnan(lse) ? -INFINITY : z - lse;
  };
  const T* x = logits + row * ld;
  if (tid == 0) {
    if (out.lse) out.lse[row] = lse;
    if (out.entropy) out.entropy[row] = lse == -INFINITY ? 0.f : logf(st.s) - st.t / st.s;
  }
  for (int i = tid; i < n_targets; i += kThreads) {
    const int t = targets[row * n_targets + i];
    if (t >= vocab) atomicExch(status, static_cast<int32_t>(SZO_ERR_INVALID_ARG));
    out.logp[row * n_targets + i] = t < 0 ? 0.f : t >= vocab ? __int_as_float(0x7fffffff) : value(widen<T>(x[t]));
  }
  if (tid < n_top) {
    const uint32_t id = key_index(top[tid]);
    out.top_ids[row * n_top + tid] = id;
    out.top_logp[row * n_top + tid] = value(widen<T>(x[id]));
  }
}

// d_logits[j] = scale * ( sum_i d_logp[i] (1[j = t_i] - p_j) - d_entropy p_j (log p_j + H) ): a stream of one read and one
// write.  Block = kChunk vectors of a row, all loads first; the block's own targets, mostly none, are picked out before.
constexpr int kBwdUnroll = 4, kChunk = kThreads * kBwdUnroll;
template <typename T>
__global__ void __launch_bounds__(kThreads, 4)
token_logprobs_bwd_kernel(const T* logits, int64_t ld, int vocab, float scale, const int32_t* __restrict__ targets, int n_targets,
                          const float* __restrict__ lse_in, const float* __restrict__ entropy, const float* __restrict__ d_logp,
                          const float* __restrict__ d_entropy, T* d_logits, int64_t dld, int chunks) {
  constexpr int kN = Vec<T>::kN;
  __shared__ int own_t[kMaxTargets];
  __shared__ float own_g[kMaxTargets];
  __shared__ int n_own;
  const int64_t row = blockIdx.x / chunks;
  const int v0 = blockIdx.x % chunks * kChunk, tid = threadIdx.x;
  const Row<const T> X(logits + row * ld, vocab);
  const Row<T> D(d_logits + row * dld, vocab);
  Vec<T> r[kBwdUnroll];
  const bool same = X.off == D.off;                               // else element by element (row strides that differ modulo 16 bytes)
#pragma unroll
  for (int u = 0; u < kBwdUnroll; ++u) {
    const int v = v0 + u * kThreads + tid;
    if (v < X.vecs && X.whole(v)) r[u] = *reinterpret_cast<const Vec<T>*>(X.base + static_cast<int64_t>(v) * kN);
  }
  const float lse = lse_in[row], gh = d_entropy ? d_entropy[row] : 0.f, ent = d_entropy ? entropy[row] : 0.f;
  float sum = 0.f;
  for (int i = 0; i < n_targets; ++i) {
    const int t = targets[row * n_targets + i];
    if (t >= 0 && t < vocab) sum += d_logp[row * n_targets + i];
  }
  if (tid == 0) {                                                 // in order: the same target twice adds up the same way every time
    n_own = 0;
    for (int i = 0; i < n_targets; ++i) {
      const int t = targets[row * n_targets + i];
      if (t < 0 || t >= vocab || t + X.off < v0 * kN || t + X.off >= (v0 + kChunk) * kN) continue;
      int at = 0;
      while (at < n_own && own_t[at] != t) ++at;
      own_g[at] = at < n_own ? own_g[at] + d_logp[row * n_targets + i] : d_logp[row * n_targets + i];
      own_t[at] = t;
      if (at == n_own) ++n_own;
    }
  }
  __syncthreads();
  const float poison = isnan(lse) ? lse : 0.f;
  const bool empty = lse == -INFINITY;
  const float a = -sum - gh * ent;                                // -p (sum + gh H) - gh p log p
#pragma unroll
  for (int u = 0; u < kBwdUnroll; ++u) {
    const int v = v0 + u * kThreads + tid;
    if (v >= X.vecs) continue;
    const bool whole = X.whole(v);
    float g[kN];
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const float x = whole ? widen<T>(r[u].x[i]) : X.inside(v, i) ? widen<T>(X.base[static_cast<int64_t>(v) * kN + i]) : 0.f;
      const float lp = fmaxf(__fmul_rn(x, scale) - lse, -120.f), p = ex2(lp * kLog2e);        // e^-120 is 0 in fp32
      g[i] = fmaf(p, fmaf(-gh, lp, a), poison);
    }
    for (int k = 0; k < n_own; ++k) {
      const int at = own_t[k] + X.off - v * kN;
#pragma unroll
      for (int i = 0; i < kN; ++i)
        if (at == i) g[i] += own_g[k];
    }
    Vec<T> o;
#pragma unroll
    for (int i = 0; i < kN; ++i) o.x[i] = narrow<T>(empty ? 0.f : g[i] * scale);
    if (whole && same) {
      *reinterpret_cast<Vec<T>*>(D.base + static_cast<int64_t>(v) * kN) = o;
    } else {
#pragma unroll
      for (int i = 0; i < kN; ++i)
        if (X.inside(v, i)) d_logits[row * dld + X.index(v, i)] = o.x[i];
    }
  }
}

szo_status check_logits(const void* logits, szo_dtype dt, int64_t rows, int64_t vocab, int64_t ld, float scale, const void* targets,
                        int32_t n_targets) {
  SZO_REQUIRE(dt == SZO_F32 || dt == SZO_BF16 || dt == SZO_F16, SZO_ERR_UNSUPPORTED, "dtype must be f32, bf16 or f16");
  SZO_REQUIRE(rows >= 0 && rows <= 0x7fffffff && vocab >= 1 && vocab <= (1 << 30), SZO_ERR_SHAPE, "need 0 <= rows < 2^31 and 1 <= vocab <= 2^30");
  SZO_REQUIRE(ld >= vocab, SZO_ERR_SHAPE, "row_stride must be at least vocab");
  SZO_REQUIRE(scale >= 1e-30f && scale <= 1e30f, SZO_ERR_INVALID_ARG, "scale must be in [1e-30, 1e30]");
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
  // A row is cut over the blocks of a cluster while that leaves SMs idle and each thread two vectors
  const int64_t vecs = ceil_div(vocab, 16 / static_cast<int64_t>(dtype_size(dtype)));
  int parts = 1;
  while (parts < kMaxCluster && rows * parts < 148 * 2 && vecs >= static_cast<int64_t>(parts) * 2 * kThreads * 2) parts *= 2;
  SZO_REQUIRE(rows * parts <= 0x7fffffff, SZO_ERR_SHAPE, "too many rows for one launch");
  const Out out{logp, entropy, lse, top_logp, top_ids};
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(rows * parts));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = parts;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = parts > 1 ? 1 : 0;
#define SZO_LOGP(T)                                                                                                              \
  SZO_CHECK_CUDA(cudaLaunchKernelEx(&cfg, token_logprobs_kernel<T>, static_cast<const T*>(logits), row_stride, static_cast<int>(vocab), \
                                    scale, targets, n_targets, n_top, out, status, parts))
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
  // vectors of a row, one more for a row that does not start on 16 bytes
  const int64_t chunks = ceil_div(ceil_div(vocab, 16 / static_cast<int64_t>(dtype_size(dtype))) + 1, kChunk);
  SZO_REQUIRE(rows * chunks <= 0x7fffffff, SZO_ERR_SHAPE, "too many rows for one launch");
#define SZO_LOGP_BWD(T)                                                                                                     \
  token_logprobs_bwd_kernel<T><<<static_cast<unsigned>(rows * chunks), kThreads, 0, st>>>(static_cast<const T*>(logits), row_stride, \
      static_cast<int>(vocab), scale, targets, n_targets, lse, entropy, d_logp, d_entropy, static_cast<T*>(d_logits), d_row_stride,  \
      static_cast<int>(chunks))
  if (dtype == SZO_F32) SZO_LOGP_BWD(float);
  else if (dtype == SZO_BF16) SZO_LOGP_BWD(__nv_bfloat16);
  else SZO_LOGP_BWD(__half);
#undef SZO_LOGP_BWD
  count_launch();
  SZO_CHECK_LAUNCH("token_logprobs_bwd_kernel");
  return SZO_OK;
}

}  // extern "C"
