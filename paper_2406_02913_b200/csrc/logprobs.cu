// Log probabilities of given tokens under softmax(scale * logits), with entropy and the best alternatives,
// and the gradient with respect to the logits.
//
// Forward: one pass over a row.  Every thread keeps a reference maximum m, s = sum e^(x-m), t = sum e^(x-m) (x-m) and
// its best (logit, index); what bounds it is reading the logits, next to it the exponentials (16 per cycle and SM: 0.72 of
// the time that 16-bit logits take to arrive) and the instructions around them (4.5 per logit), so maxima and sums run
// as packed pairs, the scale and log2 e are one factor of one packed fma, and m moves only when it is exceeded by e^8.
// lse = m + log s and H = log s - t / s come out of the same pass.  Few rows are cut over the blocks of a cluster and
// joined through distributed shared memory.  Measured: 4096 x 50272 bf16, two targets each, 76 us (5.4 TB/s, 0.84 of the
// measured copy bandwidth); 2048 x 32000 bf16 with 5 best tokens 43 us (without 30); 8 x 32000 with 5 best 7 us in bf16 and 7.9 in fp32 (20
// best: 8.9), which is the chain of a launch, two trips to memory, the ranking and the join.  Five blocks per SM without best tokens (48 registers; four: 89 us
// for the first), four with (five: 0.9 of the time for 2048 x 32000, 1.1 for 494 x 63388 in fp32).
//
// Best alternatives: the n-th largest of 64 groups' largest logits is a lower bound of the row's n-th largest, and only
// the threads whose largest reaches it can hold a candidate: their parts alone are read again, from L2, by the whole
// block.  Candidates are ranked as (logit, index) in one 64-bit number, all different, so ties need no care and the result no order of arrival.
// Only where too many logits or threads reach the bound (masked rows, whose logits are equal) every thread looks for its
// best such number first, and the n-th largest of those leaves few.
#include <cooperative_groups.h>

#include <cmath>
#include <type_traits>

#include "common.cuh"

namespace cg = cooperative_groups;

namespace szo {
namespace {

// (a thread per target and per entry of the cluster's joined list: kThreads >= kMaxTargets, kMaxCluster * kMaxTop)
constexpr int kMaxTop = 32, kMaxTargets = 64, kThreads = 256, kMaxCand = 512, kMaxCluster = 8, kUnroll = 4;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f, kSlack = 8.0f, kBigRef = 65536.0f;

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
  using E = typename std::remove_const<T>::type;
  __device__ __forceinline__ Vec<E> vec(int v) const { return *reinterpret_cast<const Vec<E>*>(base + static_cast<int64_t>(v) * Vec<T>::kN); }
  __device__ __forceinline__ Vec<E> edge(int v) const {           // element by element, -inf outside
    Vec<E> r;
#pragma unroll
    for (int i = 0; i < Vec<T>::kN; ++i) r.x[i] = inside(v, i) ? base[static_cast<int64_t>(v) * Vec<T>::kN + i] : narrow<E>(-INFINITY);
    return r;
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

// Elements 2 i and 2 i + 1 of a vector as a pair of fp32, and two fp32 rounded into them
__device__ __forceinline__ uint64_t widen2(const Vec<float>& v, int i) { return pair(v.x[2 * i], v.x[2 * i + 1]); }
__device__ __forceinline__ uint64_t widen2(const Vec<__nv_bfloat16>& v, int i) {
  const uint32_t w = reinterpret_cast<const uint32_t*>(v.x)[i];
  return pair(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
__device__ __forceinline__ uint64_t widen2(const Vec<__half>& v, int i) {
  const float2 f = __half22float2(reinterpret_cast<const __half2*>(v.x)[i]);
  return pair(f.x, f.y);
}
__device__ __forceinline__ void narrow2(Vec<float>& v, int i, float2 f) {
  v.x[2 * i] = f.x;
  v.x[2 * i + 1] = f.y;
}
__device__ __forceinline__ void narrow2(Vec<__nv_bfloat16>& v, int i, float2 f) { reinterpret_cast<__nv_bfloat162*>(v.x)[i] = __floats2bfloat162_rn(f.x, f.y); }
__device__ __forceinline__ void narrow2(Vec<__half>& v, int i, float2 f) { reinterpret_cast<__half2*>(v.x)[i] = __floats2half2_rn(f.x, f.y); }

// Softmax statistics of a part of a row relative to m; a part that holds NaN or +inf has s = NaN.
struct Stat {
  float m, s, t;
};
// Joins the statistics of 2^k neighbouring lanes, in every one of them: one exponential per lane
template <int kLanes> __device__ __forceinline__ Stat join_lanes(Stat a) {
  float m = a.m;
#pragma unroll
  for (int o = kLanes / 2; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (a.m != -INFINITY) {                                         // (else s is 0, or NaN where only NaN was seen)
    const float d = fmaxf(a.m - m, -120.f), f = expf(d);
    a.t = f * fmaf(d, a.s, a.t);
    a.s *= f;
  }
#pragma unroll
  for (int o = kLanes / 2; o; o >>= 1) {
    a.s += __shfl_xor_sync(0xffffffffu, a.s, o);
    a.t += __shfl_xor_sync(0xffffffffu, a.t, o);
  }
  a.m = m;
  return a;
}
// Order of alternatives: larger logit first, then lower index; NaN before everything, -0 = +0.  Never 0 nor ~0.
__device__ __forceinline__ uint64_t order_key(float x, uint32_t idx) {
  uint32_t u = isnan(x) ? 0x7fffffffu : __float_as_uint(x + 0.0f);
  u = u & 0x80000000u ? ~u : u | 0x80000000u;
  return static_cast<uint64_t>(u) << 32 | (0xfffffffeu - idx);
}
// The same order of logits alone, as signed numbers
__device__ __forceinline__ int order_of(float x) {
  const int u = isnan(x) ? 0x7fffffff : __float_as_int(x + 0.0f);
  return u >= 0 ? u : u ^ 0x7fffffff;
}
__device__ __forceinline__ uint32_t key_index(uint64_t k) { return 0xfffffffeu - static_cast<uint32_t>(k); }

struct Out {
  float *logp, *entropy, *lse, *top_logp;
  int32_t* top_ids;
};

// Largest element (NaN if there is one) and the elements kept at or above `low`, packed for 16-bit types
__device__ __forceinline__ float largest(const Vec<float>& r) { return max_nan(max_nan(r.x[0], r.x[1]), max_nan(r.x[2], r.x[3])); }
__device__ __forceinline__ Vec<float> at_least(const Vec<float>& r, float low) {
  Vec<float> o;
#pragma unroll
  for (int i = 0; i < 4; ++i) o.x[i] = fmaxf(r.x[i], low);
  return o;
}
template <typename T2, typename T> __device__ __forceinline__ float largest16(const Vec<T>& r) {
  const T2* p = reinterpret_cast<const T2*>(r.x);
  const T2 hi = __hmax2_nan(__hmax2_nan(p[0], p[1]), __hmax2_nan(p[2], p[3]));
  return max_nan(widen<T>(hi.x), widen<T>(hi.y));
}
template <typename T2, typename T> __device__ __forceinline__ Vec<T> at_least16(const Vec<T>& r, T low) {
  Vec<T> o;
  T2 l;
  l.x = l.y = low;
#pragma unroll
  for (int i = 0; i < 4; ++i) reinterpret_cast<T2*>(o.x)[i] = __hmax2(reinterpret_cast<const T2*>(r.x)[i], l);
  return o;
}
__device__ __forceinline__ float largest(const Vec<__nv_bfloat16>& r) { return largest16<__nv_bfloat162>(r); }
__device__ __forceinline__ float largest(const Vec<__half>& r) { return largest16<__half2>(r); }
__device__ __forceinline__ Vec<__nv_bfloat16> at_least(const Vec<__nv_bfloat16>& r, __nv_bfloat16 low) { return at_least16<__nv_bfloat162>(r, low); }
__device__ __forceinline__ Vec<__half> at_least(const Vec<__half>& r, __half low) { return at_least16<__half2>(r, low); }
// A logit that stands for -inf: its product with c is about -2^20, far below every reference that is used with it (those are
// above -kBigRef), so 2^y is 0, and small enough to stay finite itself for every c >= 1e-30 log2 e and in the products with y
constexpr float kFloor = -1048576.0f;
template <typename T> __device__ __forceinline__ T floor_of(float c) { return narrow<T>(kFloor / c); }
template <> __device__ __forceinline__ __half floor_of<__half>(float c) { return narrow<__half>(fmaxf(kFloor / c, -65504.f)); }

// One thread's statistics.  With c = scale log2 e, the reference logit g and ref = RN(g c):
//   s = sum 2^y, t = sum 2^y y,  y = x c - ref = (x - g) c + eps,  eps = g c - ref (the rounding of ref, known exactly)
// one fma per element and free of rounding in the exponent.  Masked tokens are raised to a floor first (2^y is 0 all the
// same, and y stays finite).  Where the floor is too near (fp16) or ref so large that its rounding counts, y is formed as
// (RN(x scale) - RN(g scale)) log2 e + eps, kept above -160 (2^-160 is 0).
template <typename T> struct Running {
  float ref = 0.f, eps = 0.f, z = -INFINITY;                      // z = RN(g scale); -inf: nothing yet
  uint64_t s2 = 0, t2 = 0;
  bool bad = false;                                               // NaN or +inf seen
  template <int kU> __device__ __forceinline__ void take(const Vec<T> (&r)[kU], float mx, float scale, float c, T low, float low_y) {
    constexpr int kN = Vec<T>::kN;
    const float top = __fmul_rn(mx, scale);
    if (!(top < INFINITY)) bad = true;
    if (!(top > -INFINITY)) return;                               // nothing but masked tokens (or NaN)
    if (top > z + kSlack) {
      const float ref_n = __fmul_rn(mx, c), eps_n = fabsf(ref_n) < kBigRef ? fmaf(mx, c, -ref_n) : 0.f;
      // every earlier term by 2^d, its y by + d
      const float d = z == -INFINITY ? 0.f : fmaxf((z - top) * kLog2e + (eps_n - eps), -160.f), f = ex2(d);
      t2 = mul2(pair(f, f), fma2(pair(d, d), s2, t2));
      s2 = mul2(pair(f, f), s2);
      ref = ref_n;
      eps = eps_n;
      z = top;
    }
    if (fabsf(ref) < kBigRef && ref > low_y) {
      const uint64_t c2 = pair(c, c), r2 = pair(-ref, -ref);
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const Vec<T> q = at_least(r[u], low);
#pragma unroll
        for (int i = 0; i < kN; i += 2) {
          const uint64_t y = fma2(widen2(q, i / 2), c2, r2);
          const float2 b = unpair(y);
          const uint64_t e = pair(ex2(b.x), ex2(b.y));
          s2 = add2(s2, e);
          t2 = fma2(e, y, t2);
        }
      }
    } else {
#pragma unroll
      for (int u = 0; u < kU; ++u) {
#pragma unroll
        for (int i = 0; i < kN; i += 2) {
          float y[2];
#pragma unroll
          for (int k = 0; k < 2; ++k) y[k] = fmaxf(fmaf(__fmul_rn(widen<T>(r[u].x[i + k]), scale) - z, kLog2e, eps), -160.f);
          const uint64_t e = pair(ex2(y[0]), ex2(y[1]));
          s2 = add2(s2, e);
          t2 = fma2(e, pair(y[0], y[1]), t2);
        }
      }
    }
  }
  __device__ __forceinline__ Stat stat() const {                  // relative to z, in natural units
    const float2 s = unpair(s2), t = unpair(t2);
    const float f = ex2(-eps), sum = s.x + s.y, ts = fmaf(-eps, sum, t.x + t.y);
    return Stat{z, bad ? __int_as_float(0x7fffffff) : f * sum, f * ts * kLn2};
  }
};

// Block = a row, or the rank-th of `parts` shares of its vectors; a cluster = a row.
template <typename T, bool kTop>
__global__ void __launch_bounds__(kThreads, kTop ? 4 : 5)
token_logprobs_kernel(const T* __restrict__ logits, int64_t ld, int vocab, float scale, const int32_t* __restrict__ targets,
                      int n_targets, int n_top, Out out, int32_t* status, int parts) {
  constexpr int kN = Vec<T>::kN, kW = kThreads / 32;
  __shared__ Stat part[kW];
  __shared__ Stat mine;
  __shared__ uint64_t keys[kThreads];                             // best of every thread; the cluster's lists
  __shared__ __align__(16) int groups[kThreads / 4];              // largest of every four threads
  __shared__ uint64_t cand[kTop ? kMaxCand : 1];
  __shared__ uint64_t top[kMaxTop];
  __shared__ uint64_t bound;
  __shared__ int n_cand, n_who, low_bound;
  __shared__ unsigned char who[kTop ? kThreads : 1];              // threads whose largest reaches the bound
  const int64_t row = blockIdx.x / parts;
  const int rank = blockIdx.x % parts, tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  const Row<const T> R(logits + row * ld, vocab);
  const int v_lo = static_cast<int>(static_cast<int64_t>(R.vecs) * rank / parts), v_hi = static_cast<int>(static_cast<int64_t>(R.vecs) * (rank + 1) / parts);

  // the targets' logits (one per thread) are fetched with the first vectors
  int target = -1;
  float target_x = 0.f;
  if (rank == 0 && tid < n_targets) {
    target = targets[row * n_targets + tid];
    if (target >= 0 && target < vocab) target_x = widen<T>(logits[row * ld + target]);
  }
  Running<T> run;
  float best = -INFINITY;
  const float c = scale * kLog2e;
  const T low = floor_of<T>(c);
  const float low_y = fmaf(widen<T>(low), c, 200.f);              // the floor counts as -inf for references above this
  auto take = [&](const auto& r) {
    float mx = largest(r[0]);
#pragma unroll
    for (int u = 1; u < static_cast<int>(sizeof(r) / sizeof(r[0])); ++u) mx = max_nan(mx, largest(r[u]));
    if (kTop) best = max_nan(best, mx);
    run.take(r, mx, scale, c, low, low_y);
  };
  int v = v_lo + tid;
  {
    Vec<T> r[kUnroll];
    Vec<T> one[1];
    if (v == 0 && v < v_hi && !R.whole(0)) {                      // a row that starts inside a vector (or a single partial one)
      one[0] = R.edge(0);
      take(one);
      v = kThreads;
    }
    const int v_whole = v_hi - (rank == parts - 1 && !R.whole(R.vecs - 1));
    for (; v + (kUnroll - 1) * kThreads < v_whole; v += kUnroll * kThreads) {        // all loads first
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) r[u] = R.vec(v + u * kThreads);
      take(r);
    }
    for (; v < v_hi; v += kThreads) {                             // what is left
      one[0] = v < v_whole ? R.vec(v) : R.edge(v);
      take(one);
    }
  }
  Stat st = join_lanes<32>(run.stat());
  if (lane == 0) part[w] = st;
  if (tid == 0) {
    n_cand = n_who = 0;
    bound = 1;
  }
  if constexpr (kTop) {
    if (tid < kMaxTop) top[tid] = 0;
    int g = order_of(best);
    g = max(g, __shfl_xor_sync(0xffffffffu, g, 1));
    g = max(g, __shfl_xor_sync(0xffffffffu, g, 2));
    if (tid % 4 == 0) groups[tid / 4] = g;
  }
  __syncthreads();
  st = join_lanes<kW>(part[lane % kW]);                           // (every warp: all threads know the row's)

  if constexpr (kTop) {
    // this thread's vectors, in the order of their indexes
    auto each = [&](auto f) {
#pragma unroll 4
      for (int v = v_lo + tid; v < v_hi; v += kThreads) {
        const Vec<T> x = R.whole(v) ? R.vec(v) : R.edge(v);
        f(x, v);
      }
    };
    auto key_at = [&](const Vec<T>& x, int v, int i) { return R.inside(v, i) ? order_key(widen<T>(x.x[i]), R.index(v, i)) : 0; };
    auto at_most = [&](const Vec<T>& x, int v) { return order_key(largest(x), max(R.index(v, 0), 0)); };      // a vector's keys are not above this
    if (w < 2) {                                                  // the n-th largest group (equal ones: in order)
      static_assert(kThreads / 4 == 64 && kMaxTop <= 64, "");
      const int g = groups[tid];
      int above = 0;
#pragma unroll 4
      for (int i = 0; i < 16; ++i) {
        const int4 x = reinterpret_cast<const int4*>(groups)[i];
        above += x.x > g || (x.x == g && 4 * i < tid);
        above += x.y > g || (x.y == g && 4 * i + 1 < tid);
        above += x.z > g || (x.z == g && 4 * i + 2 < tid);
        above += x.w > g || (x.w == g && 4 * i + 3 < tid);
      }
      if (above == n_top - 1) low_bound = g;
    }
    __syncthreads();
    const int lb = low_bound;
    if (order_of(best) >= lb) who[atomicAdd(&n_who, 1)] = tid;
    __syncthreads();
    const int threads = n_who, rounds = (v_hi - v_lo + kThreads - 1) / kThreads;
    const int work = threads > kThreads / 2 ? 0 : threads * rounds;
#pragma unroll 4
    for (int i = tid; i < work; i += kThreads) {                  // their vectors, by all threads: few loads one after the other
      const int v = v_lo + who[i % threads] + i / threads * kThreads;
      if (v >= v_hi) continue;
      const Vec<T> x = R.whole(v) ? R.vec(v) : R.edge(v);
      if (order_of(largest(x)) < lb) continue;
#pragma unroll
      for (int k = 0; k < kN; ++k)
        if (order_of(widen<T>(x.x[k])) >= lb && R.inside(v, k) && *const_cast<volatile int*>(&n_cand) <= kMaxCand) {
          const int at = atomicAdd(&n_cand, 1);
          if (at < kMaxCand) cand[at] = order_key(widen<T>(x.x[k]), R.index(v, k));
        }
    }
    __syncthreads();
    if (n_cand > kMaxCand || threads > kThreads / 2) {            // (the block)
      uint64_t key = 0;
      each([&](const Vec<T>& x, int v) {
        if (at_most(x, v) <= key) return;
#pragma unroll
        for (int i = 0; i < kN; ++i) key = max(key, key_at(x, v, i));
      });
      __syncthreads();                                            // (all have seen n_cand)
      keys[tid] = key;
      if (tid == 0) n_cand = 0;
      __syncthreads();
      if (key != 0) {
        int above = 0;
#pragma unroll 8
        for (int i = 0; i < kThreads; ++i) above += keys[i] > key;
        if (above == n_top - 1) bound = key;
      }
      __syncthreads();
      if (key >= bound)
        each([&](const Vec<T>& x, int v) {
          if (at_most(x, v) < bound) return;
#pragma unroll
          for (int i = 0; i < kN; ++i) {
            const uint64_t k = key_at(x, v, i);
            if (k >= bound) {
              const int at = atomicAdd(&n_cand, 1);
              if (at < kMaxCand) cand[at] = k;
            }
          }
        });
      __syncthreads();
    }
    if (n_cand <= kMaxCand) {
      for (int j = tid; j < n_cand; j += kThreads) {
        const uint64_t k = cand[j];
        int above = 0;
        for (int i = 0; i < n_cand; ++i) above += cand[i] > k;
        if (above < n_top) top[above] = k;
      }
    } else {                                                      // the largest logits crowd in few threads: one pass for each
      uint64_t last = ~0ull;
      for (int r = 0; r < n_top; ++r) {
        uint64_t k = 0;
        each([&](const Vec<T>& x, int v) {
          if (at_most(x, v) <= k) return;
#pragma unroll
          for (int i = 0; i < kN; ++i) {
            const uint64_t ck = key_at(x, v, i);
            if (ck < last && ck > k) k = ck;
          }
        });
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
      st = join_lanes<kMaxCluster>(lane % kMaxCluster < parts ? *cluster.map_shared_rank(&mine, lane % kMaxCluster) : Stat{-INFINITY, 0.f, 0.f});
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
  if (tid < n_targets) {
    if (target >= vocab) atomicExch(status, static_cast<int32_t>(SZO_ERR_INVALID_ARG));
    out.logp[row * n_targets + tid] = target < 0 ? 0.f : target >= vocab ? __int_as_float(0x7fffffff) : value(target_x);
  }
  if (tid < n_top) {
    const uint32_t id = key_index(top[tid]);
    out.top_ids[row * n_top + tid] = id;
    out.top_logp[row * n_top + tid] = value(widen<T>(x[id]));
  }
}

// d_logits[j] = scale * ( sum_i d_logp[i] (1[j = t_i] - p_j) - d_entropy p_j (log p_j + H) ): a stream of one read and one
// write, which bounds it.  Block = one of `parts` shares of a row's vectors: four vectors per thread are on their way while four
// are worked on; the row's targets are sorted out once, while the first are.  Measured: 2048 x 32000 bf16 48.7 us (5.4 TB/s, 0.84
// of the measured copy bandwidth), 24 x 50271 fp32 5.4 us.
template <typename T>
__global__ void __launch_bounds__(kThreads, 4)
token_logprobs_bwd_kernel(const T* logits, int64_t ld, int vocab, float scale, const int32_t* __restrict__ targets, int n_targets,
                          const float* __restrict__ lse_in, const float* __restrict__ entropy, const float* __restrict__ d_logp,
                          const float* __restrict__ d_entropy, T* d_logits, int64_t dld, int parts) {
  constexpr int kN = Vec<T>::kN;
  __shared__ int own_t[kMaxTargets];
  __shared__ float own_g[kMaxTargets];
  __shared__ float sum_s;
  __shared__ int n_own;
  const int64_t row = blockIdx.x / parts;
  const int rank = blockIdx.x % parts, tid = threadIdx.x;
  const Row<const T> X(logits + row * ld, vocab);
  const Row<T> D(d_logits + row * dld, vocab);
  const int v_lo = static_cast<int>(static_cast<int64_t>(X.vecs) * rank / parts), v_hi = static_cast<int>(static_cast<int64_t>(X.vecs) * (rank + 1) / parts);
  const bool same = X.off == D.off;                               // else element by element (row strides that differ modulo 16 bytes)
  Vec<T> r[kUnroll], next[kUnroll];
  auto load4 = [&](Vec<T>(&x)[kUnroll], int v) {
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (v + u * kThreads < v_hi && X.whole(v + u * kThreads)) x[u] = X.vec(v + u * kThreads);
  };
  int v = v_lo + tid;
  load4(r, v);
  const float lse = lse_in[row], gh = d_entropy ? d_entropy[row] : 0.f, ent = d_entropy ? entropy[row] : 0.f;
  if (tid < 32) {                                                 // in order: the same target twice adds up the same way every time
    int n = 0;
    float sum = 0.f;
    for (int i0 = 0; i0 < n_targets; i0 += 32) {
      const int i = i0 + tid;
      const int t = i < n_targets ? targets[row * n_targets + i] : -1;
      const float g = i < n_targets ? d_logp[row * n_targets + i] : 0.f;
      for (int k = 0; k < min(32, n_targets - i0); ++k) {
        const int tk = __shfl_sync(0xffffffffu, t, k);
        const float gk = __shfl_sync(0xffffffffu, g, k);
        if (tk < 0 || tk >= vocab) continue;
        sum += gk;
        const int at = tk + X.off;
        if (at < v_lo * kN || at >= v_hi * kN) continue;
        if (tid == 0) {
          int j = 0;
          while (j < n && own_t[j] != tk) ++j;
          own_g[j] = j < n ? own_g[j] + gk : gk;
          own_t[j] = tk;
          n = j < n ? n : n + 1;
        }
      }
    }
    if (tid == 0) {
      n_own = n;
      sum_s = sum;
    }
  }
  __syncthreads();
  const int n = n_own;
  // With c = scale log2 e, ref = RN(lse log2 e) and y = x c - ref, one fma: p = 2^(y + delta), log p = (y + delta) ln 2 with
  // delta = ref - lse log2 e, so that scale times the formula without its targets is 2^y (A + B y).  Masked logits are raised
  // to a floor as in the forward pass; where the floor is too near (fp16), ref too large, or A or B so large that a product with the
  // floor (2^20) may overflow, the plain form.
  const float c = scale * kLog2e, ref = lse * kLog2e, delta = -fmaf(lse, kLog2e, -ref), F = exp2f(delta);
  const float a = -sum_s - gh * ent;                              // p (a - gh log p)
  const float B = -gh * kLn2 * F * scale, A = fmaf(B, delta, a * F * scale);
  const T low = floor_of<T>(c);
  const bool fast = fabsf(lse) < kBigRef && ref > fmaf(widen<T>(low), c, 200.f) && fmaf(fabsf(B), 4e6f, fabsf(A)) < 1e37f;
  const uint64_t c2 = pair(c, c), r2 = pair(-ref, -ref), A2 = pair(A, A), B2 = pair(B, B);
  for (; v < v_hi; v += kUnroll * kThreads) {
    load4(next, v + kUnroll * kThreads);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int at = v + u * kThreads;
      if (at >= v_hi) break;
      const bool whole = X.whole(at);
      if (!whole) r[u] = X.edge(at);
      float2 g[kN / 2];
      if (fast) {
        const Vec<T> q = at_least(r[u], low);
#pragma unroll
        for (int i = 0; i < kN / 2; ++i) {
          const uint64_t y = fma2(widen2(q, i), c2, r2);
          const float2 f = unpair(y);
          g[i] = unpair(mul2(pair(ex2(f.x), ex2(f.y)), fma2(B2, y, A2)));
        }
      } else {
        auto plain = [&](float x) {                               // (p times each factor first: nothing overflows that the result does not)
          const float lp = fmaxf(__fmul_rn(x, scale) - lse, -120.f), p = ex2(lp * kLog2e);
          return lse == -INFINITY ? 0.f : isnan(lse) ? lse : scale * fmaf(-(p * gh), lp, p * a);
        };
#pragma unroll
        for (int i = 0; i < kN / 2; ++i) g[i] = make_float2(plain(widen<T>(r[u].x[2 * i])), plain(widen<T>(r[u].x[2 * i + 1])));
      }
      for (int k = 0; k < n; ++k) {
        const int j = own_t[k] + X.off - at * kN;
        if (j >= 0 && j < kN && lse != -INFINITY) {
#pragma unroll
          for (int i = 0; i < kN / 2; ++i) {
            if (j == 2 * i) g[i].x = fmaf(scale, own_g[k], g[i].x);
            if (j == 2 * i + 1) g[i].y = fmaf(scale, own_g[k], g[i].y);
          }
        }
      }
      Vec<T> o;
#pragma unroll
      for (int i = 0; i < kN / 2; ++i) narrow2(o, i, g[i]);
      if (whole && same) {
        *reinterpret_cast<Vec<T>*>(D.base + static_cast<int64_t>(at) * kN) = o;
      } else {
#pragma unroll
        for (int i = 0; i < kN; ++i)
          if (X.inside(at, i)) d_logits[row * dld + X.index(at, i)] = o.x[i];
      }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) r[u] = next[u];
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

szo_status check_token_logprobs(const void* logits, szo_dtype dtype, int64_t rows, int64_t vocab, int64_t row_stride, float scale,
                                const int32_t* targets, int32_t n_targets, int32_t n_top, const float* logp, const float* entropy,
                                const float* lse, const int32_t* top_ids, const float* top_logp) {
  SZO_TRY(check_logits(logits, dtype, rows, vocab, row_stride, scale, targets, n_targets));
  SZO_REQUIRE(n_top >= 0 && n_top <= kMaxTop && n_top <= vocab, SZO_ERR_UNSUPPORTED, "n_top must be in [0, min(%d, vocab)]", kMaxTop);
  SZO_REQUIRE(rows == 0 || n_targets == 0 || logp, SZO_ERR_INVALID_ARG, "logp is NULL");
  SZO_REQUIRE(rows == 0 || n_top == 0 || (top_ids && top_logp), SZO_ERR_INVALID_ARG, "top_ids or top_logp is NULL");
  SZO_REQUIRE(aligned16(logp) && aligned16(entropy) && aligned16(lse) && aligned16(top_ids) && aligned16(top_logp), SZO_ERR_ALIGNMENT,
              "buffers must be 16-byte aligned");
  return SZO_OK;
}

}  // namespace szo

using namespace szo;

extern "C" {

szo_status szo_token_logprobs(const void* logits, szo_dtype dtype, int64_t rows, int64_t vocab, int64_t row_stride, float scale,
                              const int32_t* targets, int32_t n_targets, int32_t n_top, float* logp, float* entropy, float* lse,
                              int32_t* top_ids, float* top_logp, void* stream) {
  SZO_TRY(check_token_logprobs(logits, dtype, rows, vocab, row_stride, scale, targets, n_targets, n_top, logp, entropy, lse, top_ids, top_logp));
  if (rows == 0) return SZO_OK;
  int32_t* status = device_status_word();
  SZO_REQUIRE(status != nullptr, SZO_ERR_CUDA, "no device status word (no CUDA device?)");
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  // A row is cut over the blocks of a cluster while that leaves SMs idle and each thread eight vectors, below which the join
  // costs more than the cut saves (bf16, cut down to two vectors / to eight, us: 8 x 32000 with 5 best 7.8 / 7.0, 128 x 32000
  // 7.0 / 5.5, 1 x 9789 4.1 / 3.3, but 8 x 63388 5.5 / 6.6; 200 x 128256 in two 13.7, uncut 15.2).
  const int64_t vecs = ceil_div(vocab, 16 / static_cast<int64_t>(dtype_size(dtype)));
  int parts = 1;
  while (parts < kMaxCluster && rows * parts < 148 * 2 && vecs >= static_cast<int64_t>(parts) * 2 * kThreads * 8) parts *= 2;
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
  SZO_CHECK_CUDA(cudaLaunchKernelEx(&cfg, n_top > 0 ? token_logprobs_kernel<T, true> : token_logprobs_kernel<T, false>,              \
                                    static_cast<const T*>(logits), row_stride, static_cast<int>(vocab), scale, targets, n_targets, n_top, \
                                    out, status, parts))
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
  // A row is cut while that leaves SMs without their four blocks and each thread its four vectors (bf16, cut / uncut, us:
  // 24 x 50272 4.9 / 12.9, 128 x 32000 6.1 / 9.1, 500 x 128256 48.7 / 51.6)
  const int64_t vecs = ceil_div(vocab, 16 / static_cast<int64_t>(dtype_size(dtype)));
  int parts = 1;
  while (rows * parts < 148 * 4 && vecs >= static_cast<int64_t>(parts) * 2 * kThreads * kUnroll) parts *= 2;
  SZO_REQUIRE(rows * parts <= 0x7fffffff, SZO_ERR_SHAPE, "too many rows for one launch");
#define SZO_LOGP_BWD(T)                                                                                                     \
  token_logprobs_bwd_kernel<T><<<static_cast<unsigned>(rows * parts), kThreads, 0, st>>>(static_cast<const T*>(logits), row_stride, \
      static_cast<int>(vocab), scale, targets, n_targets, lse, entropy, d_logp, d_entropy, static_cast<T*>(d_logits), d_row_stride,  \
      parts)
  if (dtype == SZO_F32) SZO_LOGP_BWD(float);
  else if (dtype == SZO_BF16) SZO_LOGP_BWD(__nv_bfloat16);
  else SZO_LOGP_BWD(__half);
#undef SZO_LOGP_BWD
  count_launch();
  SZO_CHECK_LAUNCH("token_logprobs_bwd_kernel");
  return SZO_OK;
}

}  // extern "C"
