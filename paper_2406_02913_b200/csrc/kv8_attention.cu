// Attention of each sequence's newest tokens over its 8-bit paged cache: a few query rows per key/value head.
//
// The query rows of a sequence that share a key/value head (new tokens x query heads of the group) are taken
// together, so a cached element is read once for up to 8 kNT rows.  What bounds it is reading the cache, one byte per
// element; everything else is arranged around keeping enough loads in flight:
//   * tokens are the M dimension of the products (16 per mma.sync m16n8k16), the query rows its N dimension: scores
//     S^T = K q^T and outputs O^T = V^T P^T.  Both cache operands then are A fragments, which a thread can load
//     straight from global memory in 16-byte pieces (the order of the contracted head dimension, and of the output's
//     rows, is free), with no shared memory and no barrier in the loop; the next step's 4 KB per warp (head_dim 128)
//     are in flight while this one is multiplied.  tcgen05 would need the converted operands in shared memory and
//     128 rows of queries to be worth it: the arithmetic here is a fraction of the tensor pipe either way.
//   * a sequence's positions are divided among the warps of a block and among the blocks of a cluster (up to 16),
//     whose partial results are joined through distributed shared memory in a fixed order: no workspace, no second
//     launch, and the same bits every time.
//
// Numbers.  Codes become fp16 exactly (one cvt per two).  A query row is divided by the power of two of its largest
// element and is then exact in fp16 for bf16 and fp16 input (elements below 2^-14 of the largest lose bits that fp32
// sums would drop too); fp32 rows are split into two fp16 parts, as are the weights.  With t_j = s_j + e_j (logit in base 2,
// plus the exponent of the page's value scale) and m' the running maximum of t, the weights w_j = 2^(t_j - m' + 14) and
//   acc = sum w_j code_j,   l = sum 2^-e_j w_j,   o = acc / l
// never multiply a code by its scale: what limits w is each token's CONTRIBUTION, so that w fits fp16 (largest 2^14,
// smallest 2^-24: 38 binary orders) whatever the scales of the pages are.  m', l and acc are fp32; w is rounded to
// fp16's 11 bits for the product (22 bits for fp32 queries).
#include <cooperative_groups.h>

#include <cmath>

#include "kv8.cuh"

namespace cg = cooperative_groups;

namespace szo {
namespace kv8 {

namespace {

constexpr int kWarps = 4, kStep = 16;
constexpr float kOffset = 14.0f;

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// what pack_f16 lost of (lo, hi), again as fp16
__device__ __forceinline__ uint32_t pack_rest(uint32_t packed, float lo, float hi) {
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&packed));
  return pack_f16(lo - f.x, hi - f.y);
}
__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ uint4 load_stream16(const uint8_t* p) {
  uint4 r;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
  return r;
}
__device__ __forceinline__ uint2 load_stream8(const uint8_t* p) {
  uint2 r;
  asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(r.x), "=r"(r.y) : "l"(p));
  return r;
}
__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t b, uint32_t sel) {
  uint32_t d;
  asm("prmt.b32 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(sel));
  return d;
}

// One step (16 tokens) of a page and head as the thread (g, t) = (lane / 4, lane % 4) of a warp holds it.
//   keys    tokens g and g + 8, dims [16 t, 16 t + 16) and, for 128, [64 + 16 t, ...): word i of a row feeds k-step i
//   values  tokens 2 t, 2 t + 1, 2 t + 8, 2 t + 9, dims [kPiece g, kPiece (g + 1)), kPiece = HD / 8
template <int HD> struct Raw {
  uint32_t k[2][HD / 16];
  uint32_t v[4][HD / 32];
};
template <int HD>
__device__ __forceinline__ void load_step(Raw<HD>& r, const uint8_t* k, const uint8_t* v, int g, int t) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
#pragma unroll
    for (int j = 0; j < HD / 64; ++j) {
      const uint4 x = load_stream16(k + (g + 8 * i) * HD + 64 * j + 16 * t);
      r.k[i][4 * j] = x.x;
      r.k[i][4 * j + 1] = x.y;
      r.k[i][4 * j + 2] = x.z;
      r.k[i][4 * j + 3] = x.w;
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint8_t* p = v + (2 * t + (i & 1) + 8 * (i >> 1)) * HD + HD / 8 * g;
    if constexpr (HD == 128) {
      const uint4 x = load_stream16(p);
      r.v[i][0] = x.x;
      r.v[i][1] = x.y;
      r.v[i][2] = x.z;
      r.v[i][3] = x.w;
    } else {
      const uint2 x = load_stream8(p);
      r.v[i][0] = x.x;
      r.v[i][1] = x.y;
    }
  }
}

template <typename T, int HD, int NT>
__global__ void __launch_bounds__(kWarps * 32)
kv8_attention_kernel(View V, const T* __restrict__ q, int64_t q_stride, T* __restrict__ o, int64_t o_stride, int H, float scale_log2e,
                     int row_tiles, int nsplit) {
  constexpr int R = 8 * NT, kK = HD / 16;
  constexpr bool kSplit = sizeof(T) == 4;
  extern __shared__ __align__(16) unsigned char smem_kv8[];
  float* part = reinterpret_cast<float*>(smem_kv8);               // [kWarps][R][HD]; the block's own sum ends up in [0]
  float* wm = part + kWarps * R * HD;                             // [kWarps][R] maxima, then [R] the block's
  float* wl = wm + kWarps * R;                                    // the same for sums of weights
  int* nan_at = reinterpret_cast<int*>(wl + kWarps * R);          // [HD]: first position in the masked steps whose value is NaN

  chain_release();
  chain_wait();
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  unsigned item = blockIdx.x;
  const int split = item % nsplit;
  item /= nsplit;
  const int rt = item % row_tiles;
  item /= row_tiles;
  const int h = item % V.hkv, b = item / V.hkv, G = H / V.hkv;
  const Seq seq = load_seq(V, b);
  const int r0 = rt * R, n_rows = static_cast<int>(min(static_cast<int64_t>(seq.n) * G - r0, static_cast<int64_t>(R)));
  if (n_rows <= 0) return;                                        // (the same in every block of a cluster)
  for (int i = threadIdx.x; i < HD; i += kWarps * 32) nan_at[i] = 0x7fffffff;
  const int first = seq.len - seq.n;                              // position of the sequence's row 0; negative: padding
  const int pos_lo = first + r0 / G, pos_hi = first + (r0 + n_rows - 1) / G;

  // queries: B fragments of k-step i are row g's dims dim(i, t) .. + 3
  uint32_t qa[NT][kK][2], qb[kSplit ? NT : 1][kK][2];
  float rs[NT][2];
  int rpos[NT][2];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int r = 8 * n + g;
    float x[kK][4], amax = 0.f;
    bool fine = true;
    const T* qp = q + (seq.row0 + (r0 + r) / G) * q_stride + (h * G + (r0 + r) % G) * static_cast<int64_t>(HD) + 16 * t;
#pragma unroll
    for (int j = 0; j < HD / 64; ++j) {
#pragma unroll
      for (int i = 0; i < 16; i += Vec<T>::kN) {
        Vec<T> v = {};
        if (r < n_rows) v = *reinterpret_cast<const Vec<T>*>(qp + 64 * j + i);
#pragma unroll
        for (int u = 0; u < Vec<T>::kN; ++u) {
          const float y = widen<T>(v.x[u]);
          x[4 * j + (i + u) / 4][(i + u) % 4] = y;
          amax = fmaxf(amax, fabsf(y));
          fine = fine && isfinite(y);
        }
      }
    }
#pragma unroll
    for (int off = 1; off <= 2; off <<= 1) {
      amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, off));
      fine = __shfl_xor_sync(0xffffffffu, static_cast<int>(fine), off) && fine;
    }
    const int e = min(max((__float_as_int(amax) >> 23) - 127, -126), 126);
    const float inv = exp2_int(-e);
#pragma unroll
    for (int i = 0; i < kK; ++i) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const float lo = x[i][2 * u] * inv, hi = x[i][2 * u + 1] * inv;
        qa[n][i][u] = pack_f16(lo, hi);
        if constexpr (kSplit) qb[n][i][u] = pack_rest(qa[n][i][u], lo, hi);
      }
    }
    // a row that holds NaN or an infinity has NaN logits throughout
    const float mine = fine ? exp2_int(e) * scale_log2e : __int_as_float(0x7fffffff);
#pragma unroll
    for (int u = 0; u < 2; ++u) {                                 // this thread's scores are those of rows 2 t, 2 t + 1
      rs[n][u] = __shfl_sync(0xffffffffu, mine, (2 * t + u) * 4);
      const int rr = 8 * n + 2 * t + u;
      rpos[n][u] = rr < n_rows ? first + (r0 + rr) / G : pos_hi;
    }
  }
  __syncthreads();

  // this warp's steps
  const int total = pos_hi < 0 ? 0 : pos_hi / kStep + 1;
  int s_lo = static_cast<int>(static_cast<int64_t>(total) * split / nsplit), s_hi = static_cast<int>(static_cast<int64_t>(total) * (split + 1) / nsplit);
  {
    const int span = s_hi - s_lo, base = s_lo;
    s_lo = base + span * w / kWarps;
    s_hi = base + span * (w + 1) / kWarps;
  }
  float acc[NT][HD / 16][4], m[NT][2], l[NT][2];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    m[n][0] = m[n][1] = -INFINITY;
    l[n][0] = l[n][1] = 0.f;
#pragma unroll
    for (int i = 0; i < HD / 16; ++i) acc[n][i][0] = acc[n][i][1] = acc[n][i][2] = acc[n][i][3] = 0.f;
  }
  // Page ids and scales of 32 steps at a time, one step per lane, loaded a chunk ahead
  const int per_page = V.page_shift - 4;
  int page_c = -1, page_n = -1;
  float2 sc_c = make_float2(0.f, 0.f), sc_n = sc_c;
  auto load_meta = [&](int s, int& page, float2& sc) {
    page = -1;
    if (s + lane < s_hi) {
      page = load_page(V, b, (s + lane) >> per_page);
      if (page >= 0) sc = V.scales[static_cast<int64_t>(page) * V.hkv + h];
    }
  };
  auto fetch = [&](Raw<HD>& r, int page, int s) {
    if (page < 0) return;
    const int64_t at = page_offset(V, page, h, HD) + ((s << 4) & ((1 << V.page_shift) - 1)) * HD;
    load_step<HD>(r, V.k + at, V.v + at, g, t);
  };
  load_meta(s_lo, page_c, sc_c);
  load_meta(s_lo + 32, page_n, sc_n);
  Raw<HD> cur;
  int page = __shfl_sync(0xffffffffu, page_c, 0);
  fetch(cur, page, s_lo);
#pragma unroll 2
  for (int s = s_lo; s < s_hi; ++s) {
    const int i = (s - s_lo) & 31, i1 = (i + 1) & 31;
    const int ek = scale_exponent(__shfl_sync(0xffffffffu, sc_c.x, i)), ev = scale_exponent(__shfl_sync(0xffffffffu, sc_c.y, i));
    const bool have = page >= 0;
    page = __shfl_sync(0xffffffffu, i1 ? page_c : page_n, i1);
    Raw<HD> next;
    if (s + 1 < s_hi) fetch(next, page, s + 1);
    if (i1 == 0) {
      page_c = page_n;
      sc_c = sc_n;
      load_meta(s + 33, page_n, sc_n);
    }
    if (have) {
      float c[NT][4];
#pragma unroll
      for (int n = 0; n < NT; ++n) c[n][0] = c[n][1] = c[n][2] = c[n][3] = 0.f;
#pragma unroll
      for (int k = 0; k < kK; ++k) {
        const uint32_t a0 = decode2(cur.k[0][k]), a1 = decode2(cur.k[1][k]), a2 = decode2(cur.k[0][k] >> 16), a3 = decode2(cur.k[1][k] >> 16);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          mma_f16(c[n], a0, a1, a2, a3, qa[n][k][0], qa[n][k][1]);
          if constexpr (kSplit) mma_f16(c[n], a0, a1, a2, a3, qb[n][k][0], qb[n][k][1]);
        }
      }
      const bool masked = s * kStep + kStep - 1 > pos_lo;         // some row does not see the whole step
      const float ks = exp2_int(ek), fe = static_cast<float>(ev), el = exp2_int(-ev);
      uint32_t pa[NT][2], pb[kSplit ? NT : 1][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float x[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          x[u] = fmaf(c[n][u], rs[n][u & 1] * ks, fe);
          if (masked && s * kStep + g + 8 * (u >> 1) > rpos[n][u & 1]) x[u] = -INFINITY;
        }
        float mx[2] = {fmaxf(x[0], x[2]), fmaxf(x[1], x[3])};
#pragma unroll
        for (int off = 4; off <= 16; off <<= 1) {
          mx[0] = fmaxf(mx[0], __shfl_xor_sync(0xffffffffu, mx[0], off));
          mx[1] = fmaxf(mx[1], __shfl_xor_sync(0xffffffffu, mx[1], off));
        }
        const bool grew = mx[0] > m[n][0] || mx[1] > m[n][1];
        if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const float mn = fmaxf(m[n][u], mx[u]), corr = mn == -INFINITY ? 1.f : ex2(m[n][u] - mn);
            m[n][u] = mn;
            l[n][u] *= corr;
#pragma unroll
            for (int j = 0; j < HD / 16; ++j) {
              acc[n][j][u] *= corr;
              acc[n][j][u + 2] *= corr;
            }
          }
        }
        float y[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) y[u] = ex2(x[u] - (m[n][u & 1] == -INFINITY ? 0.f : m[n][u & 1] - kOffset));
        l[n][0] = fmaf(el, y[0] + y[2], l[n][0]);
        l[n][1] = fmaf(el, y[1] + y[3], l[n][1]);
        const uint32_t h0 = pack_f16(y[0], y[1]), h1 = pack_f16(y[2], y[3]);
        pa[n][0] = transpose8x8(h0);
        pa[n][1] = transpose8x8(h1);
        if constexpr (kSplit) {
          pb[n][0] = transpose8x8(pack_rest(h0, y[0], y[1]));
          pb[n][1] = transpose8x8(pack_rest(h1, y[2], y[3]));
        }
      }
      if (masked) {
        // 0 * NaN: a NaN value must not reach rows that do not see its token.  It is taken out here, and the rows that do
        // see it are set to NaN when the block's sums are joined.
#pragma unroll
        for (int i2 = 0; i2 < 4; ++i2) {
#pragma unroll
          for (int j = 0; j < HD / 32; ++j) {
            uint32_t bad = ((cur.v[i2][j] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
            cur.v[i2][j] &= ~((bad >> 7) * 0xffu);
            while (bad) {
              const int byte = (__ffs(bad) - 1) >> 3;
              bad &= bad - 1;
              atomicMin(nan_at + HD / 8 * g + 4 * j + byte, s * kStep + 2 * t + (i2 & 1) + 8 * (i2 >> 1));
            }
          }
        }
      }
#pragma unroll
      for (int j = 0; j < HD / 32; ++j) {
        const uint32_t lo0 = prmt(cur.v[0][j], cur.v[1][j], 0x5140), hi0 = prmt(cur.v[0][j], cur.v[1][j], 0x7362);
        const uint32_t lo1 = prmt(cur.v[2][j], cur.v[3][j], 0x5140), hi1 = prmt(cur.v[2][j], cur.v[3][j], 0x7362);
#pragma unroll
        for (int u = 0; u < 2; ++u) {                             // dims kPiece g + 4 j + 2 u and + 1 are rows g and g + 8 of tile 2 j + u
          const uint32_t x0 = u ? hi0 : lo0, x1 = u ? hi1 : lo1;
          const uint32_t a0 = decode2(x0), a1 = decode2(x0 >> 16), a2 = decode2(x1), a3 = decode2(x1 >> 16);
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            mma_f16(acc[n][2 * j + u], a0, a1, a2, a3, pa[n][0], pa[n][1]);
            if constexpr (kSplit) mma_f16(acc[n][2 * j + u], a0, a1, a2, a3, pb[n][0], pb[n][1]);
          }
        }
      }
    }
    cur = next;
  }

  // the block's warps joined in warp order
#pragma unroll
  for (int n = 0; n < NT; ++n) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int off = 4; off <= 16; off <<= 1) l[n][u] += __shfl_xor_sync(0xffffffffu, l[n][u], off);
      const int r = 8 * n + 2 * t + u;
      if (g == 0) {
        wm[w * R + r] = m[n][u];
        wl[w * R + r] = l[n][u];
      }
#pragma unroll
      for (int j = 0; j < HD / 16; ++j) {
        float* p = part + (w * R + r) * HD + HD / 8 * g + 2 * j;
        *reinterpret_cast<float2*>(p) = make_float2(acc[n][j][u], acc[n][j][u + 2]);
      }
    }
  }
  __syncthreads();
  float bm[R * HD / (kWarps * 32)];                               // values of this thread: one dim, every (128 / HD)-th row
  constexpr int kPer = R * HD / (kWarps * 32), kRowStep = kWarps * 32 / HD;
  const int dim = threadIdx.x % HD, row_a = threadIdx.x / HD;
  const int nan_pos = nan_at[dim];
  float rm[kPer], rl[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int r = row_a + i * kRowStep;
    float mm = -INFINITY, sum = 0.f, ll = 0.f;
#pragma unroll
    for (int x = 0; x < kWarps; ++x) mm = fmaxf(mm, wm[x * R + r]);
#pragma unroll
    for (int x = 0; x < kWarps; ++x) {
      const float f = mm == -INFINITY ? 1.f : ex2(wm[x * R + r] - mm);
      sum = fmaf(f, part[(x * R + r) * HD + dim], sum);
      ll = fmaf(f, wl[x * R + r], ll);
    }
    if (first + (r0 + r) / G >= nan_pos) sum = __int_as_float(0x7fffffff);
    bm[i] = sum;
    rm[i] = mm;
    rl[i] = ll;
  }
  auto store = [&](int r, int d, float sum, float ll) {
    o[(seq.row0 + (r0 + r) / G) * o_stride + (h * G + (r0 + r) % G) * static_cast<int64_t>(HD) + d] =
        narrow<T>(ll == 0.f ? (sum == 0.f ? 0.f : sum) : sum / ll);                // nothing attended to: zeros
  };
  if (nsplit == 1) {
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (row_a + i * kRowStep < n_rows) store(row_a + i * kRowStep, dim, bm[i], rl[i]);
    return;
  }
  // the cluster's blocks joined in block order; block i writes the i-th share of the results
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int r = row_a + i * kRowStep;
    part[r * HD + dim] = bm[i];
    if (dim == 0) {
      wm[r] = rm[i];
      wl[r] = rl[i];
    }
  }
  cg::cluster_group cluster = cg::this_cluster();
  cluster.sync();
  const int share = R * HD / nsplit;
  for (int i = threadIdx.x; i < share; i += kWarps * 32) {
    const int at = split * share + i, r = at / HD;
    if (r >= n_rows) continue;
    float mm = -INFINITY, sum = 0.f, ll = 0.f;
    for (int x = 0; x < nsplit; ++x) mm = fmaxf(mm, cluster.map_shared_rank(wm, x)[r]);
    for (int x = 0; x < nsplit; ++x) {
      const float f = mm == -INFINITY ? 1.f : ex2(cluster.map_shared_rank(wm, x)[r] - mm);
      sum = fmaf(f, cluster.map_shared_rank(part, x)[at], sum);
      ll = fmaf(f, cluster.map_shared_rank(wl, x)[r], ll);
    }
    store(r, at % HD, sum, ll);
  }
  cluster.sync();                                                 // nobody leaves while its sums are being read
}

template <typename T, int HD, int NT>
szo_status launch_rows(const View& V, const void* q, int64_t q_stride, void* o, int64_t o_stride, int H, float scale, cudaStream_t st) {
  constexpr int R = 8 * NT;
  const size_t smem = static_cast<size_t>(kWarps) * R * (HD + 2) * 4 + HD * 4;
  const int64_t tiles = ceil_div(static_cast<int64_t>(V.max_new) * (H / V.hkv), R);
  const int64_t capacity = static_cast<int64_t>(V.max_pages) << V.page_shift;
  // Blocks per sequence and head: enough for eight per SM, as long as a warp keeps two steps
  int nsplit = 1;
  while (nsplit < 16 && tiles * V.batch * V.hkv * nsplit < 148 * 8 && capacity >= static_cast<int64_t>(nsplit) * 2 * kWarps * kStep * 2) nsplit *= 2;
  unsigned blocks;
  SZO_TRY(grid_items(tiles * nsplit, V, &blocks));
  auto kern = kv8_attention_kernel<T, HD, NT>;
  SZO_CHECK_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)));
  SZO_CHECK_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3(kWarps * 32);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = nsplit;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = nsplit > 1 ? 1 : 0;
  SZO_CHECK_CUDA(cudaLaunchKernelEx(&cfg, kern, V, static_cast<const T*>(q), q_stride, static_cast<T*>(o), o_stride, H,
                                    scale * 1.4426950408889634f, static_cast<int>(tiles), nsplit));
  count_launch();
  return SZO_OK;
}

template <typename T, int HD>
szo_status launch_attention(const View& V, const void* q, int64_t q_stride, void* o, int64_t o_stride, int H, float scale, cudaStream_t st) {
  const int64_t rows = static_cast<int64_t>(V.max_new) * (H / V.hkv);
  if (rows <= 8) return launch_rows<T, HD, 1>(V, q, q_stride, o, o_stride, H, scale, st);
  return launch_rows<T, HD, 2>(V, q, q_stride, o, o_stride, H, scale, st);
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
  SZO_REQUIRE(static_cast<int64_t>(V.max_new) * n_heads <= 0x7fffffff, SZO_ERR_SHAPE, "too many rows and heads");
  SZO_TRY(kv8::set_status_word(&V));
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool wide = cache->head_dim == 128;
  if (dtype == SZO_F32)
    return wide ? kv8::launch_attention<float, 128>(V, q, q_stride, o, o_stride, n_heads, scale, st)
                : kv8::launch_attention<float, 64>(V, q, q_stride, o, o_stride, n_heads, scale, st);
  if (dtype == SZO_BF16)
    return wide ? kv8::launch_attention<__nv_bfloat16, 128>(V, q, q_stride, o, o_stride, n_heads, scale, st)
                : kv8::launch_attention<__nv_bfloat16, 64>(V, q, q_stride, o, o_stride, n_heads, scale, st);
  return wide ? kv8::launch_attention<__half, 128>(V, q, q_stride, o, o_stride, n_heads, scale, st)
              : kv8::launch_attention<__half, 64>(V, q, q_stride, o, o_stride, n_heads, scale, st);
}
