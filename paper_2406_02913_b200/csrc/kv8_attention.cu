// Attention of each sequence's newest tokens over its 8-bit paged cache: a few query rows per key/value head.
//
// The query rows of a sequence that share a key/value head (new tokens x query heads of the group) are taken
// together, so a cached element is read once for up to 8 kNT rows.  What bounds it is reading the cache, one byte per
// element; everything else is arranged around keeping enough loads in flight:
//   * tokens are the M dimension of the products (16 per mma.sync m16n8k16), the query rows its N dimension: scores
//     S^T = K q^T and outputs O^T = V^T P^T.  Both cache operands then are A fragments that a thread takes in
//     16-byte pieces (the order of the contracted head dimension, and of the output's rows, is free).  tcgen05 would
//     need the converted operands in shared memory and 128 rows of queries to be worth it: the arithmetic here is a
//     fraction of the tensor pipe either way;
//   * every warp runs on its own: its share of the positions arrives 32 tokens (8 KB for head_dim 128) at a time by TMA
//     in a private ring, two units deep, so that 16 KB per warp are in flight whatever the registers hold; no block
//     barrier in the loop.  The TMA swizzle makes both fragment reads free of bank conflicts;
//   * a sequence's positions are divided among the warps of a block and among the blocks of a cluster, whose
//     partial results are joined through distributed shared memory: no workspace and no second launch.  Where one
//     cluster per sequence and head leaves SMs idle (few sequences and heads, long contexts: seven clusters of 16 such
//     blocks fit this GPU), blocks of 12 warps, one per SM, write their partial results to a workspace and a second,
//     chained launch joins them.  Both join in a fixed order: the same bits every time.
// Measured (16-bit, 32 heads over 8 of 128): one sequence of 131071 positions 50.1 to 51.5 us (5.2 to 5.4 TB/s, 0.81 to 0.83 of the
// measured copy bandwidth), 32 of 513 to 8192, the longest first, 57.2 to 57.9 us (4.9 to 5.0 TB/s; the longest
// last 59.5, three shuffled orders 61 to 66), 64 of 2048 with 40 heads over 40
// 195 us (6.9 TB/s: reads alone, faster than the copy), one of 1024 6.9 us (launch, two trips to memory, join).
//
// Numbers.  Codes become fp16 exactly (one cvt per two).  A query row is divided by the power of two of its largest
// element and is then exact in fp16 for bf16 and fp16 input (elements below 2^-14 of the largest lose bits that fp32
// sums would drop too); fp32 rows are split into two fp16 parts, as are the weights.  With t_j = s_j + e_j (logit in base 2,
// plus the exponent of the page's value scale) and m' the running maximum of t, the weights w_j = 2^(t_j - m' + 12) and
//   acc = sum w_j code_j,   l = sum 2^-e_j w_j,   o = acc / l
// never multiply a code by its scale: what limits w is each token's CONTRIBUTION, so that w fits fp16 (below 2^15, m'
// being up to 2^3 behind, and down to 2^-24) whatever the scales of the pages are.  m', l and acc are fp32; w is rounded to
// fp16's 11 bits for the product (22 bits for fp32 queries).
#include <cooperative_groups.h>

#include <cmath>
#include <type_traits>

#include "kv8_attention.cuh"

namespace cg = cooperative_groups;

namespace szo {
namespace kv8 {

namespace {

constexpr int kUnit = 32, kDepth = 2;     // kDepth: units of a warp's ring
// The largest weight is 2^kOffset when the reference maximum m is set; m follows the running maximum only once that
// is more than 2^kSlack above it (weights then stay below 2^15), so the outputs are rescaled a few times per sequence.
constexpr float kOffset = 12.0f, kSlack = 3.0f;
constexpr int kWideUnits = 12 * 16 * 2;        // see plan()

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
// what pack_f16 lost of (lo, hi), again as fp16
__device__ __forceinline__ uint32_t pack_rest(uint32_t packed, float lo, float hi) {
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&packed));
  return pack_f16(lo - f.x, hi - f.y);
}
__device__ __forceinline__ uint4 lds16(uint32_t a) {
  uint4 r;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(a));
  return r;
}
__device__ __forceinline__ uint2 lds8(uint32_t a) {
  uint2 r;
  asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(r.x), "=r"(r.y) : "r"(a));
  return r;
}

// Shared-memory image of 16 tokens (a TMA box): rows of HD bytes, 16-byte chunks permuted by the TMA swizzle.
template <int HD> __device__ __forceinline__ uint32_t chunk_at(uint32_t base, int row, int chunk) {
  return base + row * HD + ((chunk ^ (HD == 128 ? row & 7 : (row >> 1) & 3)) << 4);
}
// Keys of 16 tokens as the thread (g, t) = (lane / 4, lane % 4) holds them: tokens g and g + 8, dims [kDims t, kDims (t + 1)),
// kDims = HD / 4: word i of a row feeds k-step i.  (Chunks 2 t and 2 t + 1 and not t and t + 4: with the swizzle eight
// neighbouring lanes then read eight different bank groups.)
template <int HD> __device__ __forceinline__ void load_keys(uint32_t (&k)[2][HD / 16], uint32_t base, int g, int t) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
#pragma unroll
    for (int j = 0; j < HD / 64; ++j) {
      const uint4 x = lds16(chunk_at<HD>(base, g + 8 * i, HD / 64 * t + j));
      k[i][4 * j] = x.x;
      k[i][4 * j + 1] = x.y;
      k[i][4 * j + 2] = x.z;
      k[i][4 * j + 3] = x.w;
    }
  }
}
// Values of 16 tokens: tokens 2 t, 2 t + 1, 2 t + 8, 2 t + 9, dims [kPiece g, kPiece (g + 1)), kPiece = HD / 8
template <int HD> __device__ __forceinline__ void load_values(uint32_t (&v)[4][HD / 32], uint32_t base, int g, int t) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = 2 * t + (i & 1) + 8 * (i >> 1);
    if constexpr (HD == 128) {
      const uint4 x = lds16(chunk_at<HD>(base, row, g));
      v[i][0] = x.x;
      v[i][1] = x.y;
      v[i][2] = x.z;
      v[i][3] = x.w;
    } else {
      const uint2 x = lds8(chunk_at<HD>(base, row, g >> 1) + 8 * (g & 1));
      v[i][0] = x.x;
      v[i][1] = x.y;
    }
  }
}

__host__ __device__ __forceinline__ int box_tokens(const View& V) { return V.page_shift < 5 ? kStep : kUnit; }

template <int HD> constexpr int kRingBytes = kDepth * kUnit * HD * 2;       // per warp

// Four dims of a row of a pass's share: the block's warps joined in warp order, NaN where the row sees one, stored
template <int HD, int R, int kWarps, int kRing>
__device__ __forceinline__ void store_share(int i, const unsigned char* ring0, const float* wm, const float* wl, const int* nan_at, int last,
                                            int64_t row_head, const Part& part) {
  const int r = i / (HD / 4), d = i % (HD / 4) * 4;
  float top = -INFINITY, l = 0.f;
#pragma unroll
  for (int x = 0; x < kWarps; ++x) top = fmaxf(top, wm[x * R + r]);
  float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int x = 0; x < kWarps; ++x) {
    const float f = top == -INFINITY ? 1.f : ex2(wm[x * R + r] - top);
    const float4 y = *reinterpret_cast<const float4*>(ring0 + x * kRing + (r * HD + d) * 4);
    sum = make_float4(fmaf(f, y.x, sum.x), fmaf(f, y.y, sum.y), fmaf(f, y.z, sum.z), fmaf(f, y.w, sum.w));
    l = fmaf(f, wl[x * R + r], l);
  }
  const float nan = __int_as_float(0x7fffffff);
  if (last >= nan_at[d]) sum.x = nan;
  if (last >= nan_at[d + 1]) sum.y = nan;
  if (last >= nan_at[d + 2]) sum.z = nan;
  if (last >= nan_at[d + 3]) sum.w = nan;
  *reinterpret_cast<float4*>(part.sums + row_head * HD + d) = sum;
  if (d == 0) part.stats[row_head] = make_float2(top - kOffset, l);
}

template <typename T, int HD, int NT, int kWarps, bool kPart = false>
__global__ void __launch_bounds__(kWarps * 32, NT == 1 ? (kWarps == 4 ? 3 : 1) : 1)
kv8_attention_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, View V, const T* __restrict__ q,
                     int64_t q_stride, T* __restrict__ o, int64_t o_stride, int H, float scale_log2e, int row_tiles, int nsplit, float* __restrict__ ws, const Part part_of) {
  constexpr int R = 8 * NT, kK = HD / 16, kRing = kRingBytes<HD>;
  constexpr bool kSplit = sizeof(T) == 4;
  static_assert(R * HD * 4 <= kRing, "a warp's partial result takes the place of its ring");
  extern __shared__ __align__(1024) unsigned char smem_kv8[];
  __shared__ float wm[kWarps * R], wl[kWarps * R];                // per warp: row maxima, sums of weights; [0, R): the block's
  __shared__ int nan_at[HD];                                      // first position in the masked steps whose value is NaN
  __shared__ __align__(8) uint64_t full[kWarps][kDepth];
  __shared__ int abort_flag;
  unsigned char* ring0 = smem_kv8 + ((1024u - (tc::smem_u32(smem_kv8) & 1023u)) & 1023u);
  auto part = [&](int warp) { return reinterpret_cast<float*>(ring0 + warp * kRing); };     // [R][HD]; the block's sum ends up in part(0)

  if constexpr (kPart) {
    // a pass over shared positions waits for the groups' description before it lets the sequences' pass begin, which so has it too and runs
    // beside it; its first block alone waits for the other pass to end (waiting blocks would keep the rest of their launch from the SMs), so
    // that what is launched behind it finds both done
    if (part_of.prefix) chain_wait();
    chain_release();
  } else {
    chain_release();
    chain_wait();
  }
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  unsigned item = blockIdx.x;
  const int split = item % nsplit;
  item /= nsplit;
  const int rt = item % row_tiles;
  item /= row_tiles;
  const int h = item % V.hkv, b = item / V.hkv, G = H / V.hkv;
  const Work work = kPart ? load_work(V, part_of, b) : Work{load_seq(V, b), 0, b};
  const Seq seq = work.seq;
  const bool prefix = kPart && part_of.prefix;
  const int r0 = rt * R, n_rows = static_cast<int>(min(static_cast<int64_t>(seq.n) * G - r0, static_cast<int64_t>(R)));
  if (n_rows <= 0) {                                              // (the same in every block of a cluster)
    if (kPart && !part_of.prefix && blockIdx.x == 0) chain_wait();
    return;
  }
  for (int i = threadIdx.x; i < HD; i += kWarps * 32) nan_at[i] = 0x7fffffff;
  if (threadIdx.x == 0) abort_flag = 0;
  const uint32_t ring = tc::smem_u32(ring0) + w * kRing, bars = tc::smem_u32(&full[w][0]);
  if (lane == 0) {
    for (int i = 0; i < kDepth; ++i) tc::mbar_init(bars + 8 * i, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncwarp();
  const int first = seq.len - seq.n;                              // position of the sequence's row 0; negative: padding
  auto last_of = [&](int r) {                                     // the last position that row r of the tile sees
    if (prefix) return min(__ldg(part_of.pos + seq.row0 + (r0 + r) / G), seq.len - 1);
    return first + (r0 + r) / G;
  };
  int pos_lo = first + r0 / G;
  const int pos_hi = prefix ? seq.len - 1 : first + (r0 + n_rows - 1) / G;

  // this warp's units of two steps; a last unit may have one
  const int steps = pos_hi < 0 ? 0 : pos_hi / kStep + 1, units = (steps + 1) / 2;
  int u_lo = static_cast<int>(static_cast<int64_t>(units) * split / nsplit), u_hi = static_cast<int>(static_cast<int64_t>(units) * (split + 1) / nsplit);
  {
    const int span = u_hi - u_lo, base = u_lo;
    u_lo = base + span * w / kWarps;
    u_hi = base + span * (w + 1) / kWarps;
  }
  float acc[NT][HD / 16][4], m[NT][2], l[NT][2];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    m[n][0] = m[n][1] = -INFINITY;
    l[n][0] = l[n][1] = 0.f;
#pragma unroll
    for (int i = 0; i < HD / 16; ++i) acc[n][i][0] = acc[n][i][1] = acc[n][i][2] = acc[n][i][3] = 0.f;
  }
  // Rows (of the tensor maps) and scales of 32 steps (16 units) at a time, one step per lane: table entries are loaded two
  // chunks ahead, scales one, so that nothing waits for either
  struct Meta {
    int row;                                                      // -1: no page, or behind this warp's share
    float2 sc;                                                    // as stored
  };
  const int32_t* table = V.table + static_cast<int64_t>(work.owner) * V.max_pages + (work.skip >> V.page_shift);
  const int s_end = min(2 * u_hi, steps);
  auto load_entry = [&](int s) { return s + lane < s_end ? __ldg(table + ((s + lane) >> (V.page_shift - 4))) : -1; };
  auto load_meta = [&](int entry, int s) {                        // (whether an entry is needed goes by its place: any value may stand in the table)
    Meta r{-1, make_float2(0.f, 0.f)};
    if (static_cast<uint32_t>(entry) < static_cast<uint64_t>(V.n_pages)) {
      r.row = ((entry * V.hkv + h) << V.page_shift) + (((s + lane) << 4) & ((1 << V.page_shift) - 1));
      r.sc = __ldg(V.scales + static_cast<int64_t>(entry) * V.hkv + h);
    } else if (s + lane < s_end) {
      report_page(V);
    }
    return r;
  };
  // A unit into ring slot `slot`: lanes 0 and 1 copy its keys and its values where a page holds a unit, lanes 0-3 16 tokens
  // each (keys, keys, values, values) where not (pages of 32, either way: 8 sequences of 8192 20.8 / 22.0 us, 131071 50.1 / 50.4).  A copy without a page is left out.  Called by the whole warp; row: of the
  // lane's first token.
  const int box = box_tokens(V), nb = kUnit / box;
  auto issue = [&](int slot, int row) {
    const uint32_t bar = bars + 8 * slot;
    const unsigned live = __ballot_sync(0xffffffffu, lane < 2 * nb && row >= 0);
    if (lane == 0) tc::mbar_expect_tx(bar, __popc(live) * box * HD);
    __syncwarp();
    if (lane < 2 * nb && row >= 0)
      tc::tma_load_2d(ring + slot * kUnit * HD * 2 + lane * box * HD, lane < nb ? &map_k : &map_v, 0, row, bar);
  };
  int entry = load_entry(2 * u_lo), entry_n = load_entry(2 * u_lo + 32);
  Meta mc = load_meta(entry, 2 * u_lo);
#pragma unroll
  for (int i = 0; i < kDepth; ++i) {
    const int row = __shfl_sync(0xffffffffu, mc.row, 2 * i + (lane & (nb - 1)));
    if (u_lo + i < u_hi) issue(i, row);
  }
  Meta mn = load_meta(entry_n, 2 * u_lo + 32);
  entry_n = load_entry(2 * u_lo + 64);
  float ks_c, fe_c;                                               // this chunk's: 2^(keys' exponent), the values' exponent; no page: -inf
  auto take_scales = [&]() {
    ks_c = exp2_int(scale_exponent(mc.sc.x));
    fe_c = mc.row >= 0 ? static_cast<float>(scale_exponent(mc.sc.y)) : -INFINITY;
  };
  // queries: the B fragments of k-step i are row g's dims (HD / 4) t + 4 i .. + 3
  uint32_t qa[NT][kK][2], qb[kSplit ? NT : 1][kK][2];
  float rs[NT][2];
  int rpos[NT][2];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int r = 8 * n + g;
    float x[kK][4], amax = 0.f;
    bool fine = true;
    const T* qp = q + (seq.row0 + (r0 + r) / G) * q_stride + (h * G + (r0 + r) % G) * static_cast<int64_t>(HD) + HD / 4 * t;
#pragma unroll
    for (int i = 0; i < HD / 4; i += Vec<T>::kN) {
      Vec<T> v = {};
      if (r < n_rows) v = *reinterpret_cast<const Vec<T>*>(qp + i);
#pragma unroll
      for (int u = 0; u < Vec<T>::kN; ++u) {
        const float y = widen<T>(v.x[u]);
        x[(i + u) / 4][(i + u) % 4] = y;
        amax = fmaxf(amax, fabsf(y));
        fine = fine && isfinite(y);
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
      rpos[n][u] = rr < n_rows ? last_of(rr) : pos_hi;
    }
  }
  if (kPart && prefix) {                                          // every row sees all of it, or each unit is masked
    const int r = threadIdx.x;
    pos_lo = __syncthreads_and(r >= n_rows || last_of(r) == pos_hi) ? pos_hi : -1;
  } else {
    __syncthreads();
  }

  take_scales();
  int slot = 0;
  uint32_t phase = 0;
  for (int u = u_lo; u < u_hi; ++u) {
    const int i = 2 * (u - u_lo) & 31;
    bool have[2];
    float ks[2], fe[2], el[2];
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      ks[a] = __shfl_sync(0xffffffffu, ks_c, i + a);
      fe[a] = __shfl_sync(0xffffffffu, fe_c, i + a);
      have[a] = fe[a] != -INFINITY;
      el[a] = have[a] ? exp2_int(-static_cast<int>(fe[a])) : 0.f;
    }
    if (!__all_sync(0xffffffffu, tc::mbar_wait(bars + 8 * slot, phase, &abort_flag, V.status, 0))) break;
    const uint32_t at = ring + slot * kUnit * HD * 2;
    float c[2][NT][4];
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      uint32_t kk[2][kK];
      load_keys<HD>(kk, at + a * kStep * HD, g, t);
      // (with one tile of rows even and odd k-steps are summed apart: four chains of products instead of two)
      float odd[NT][4];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        c[a][n][0] = c[a][n][1] = c[a][n][2] = c[a][n][3] = 0.f;
        odd[n][0] = odd[n][1] = odd[n][2] = odd[n][3] = 0.f;
      }
#pragma unroll
      for (int k = 0; k < kK; ++k) {
        const uint32_t a0 = decode2(kk[0][k]), a1 = decode2(kk[1][k]), a2 = decode2(kk[0][k] >> 16), a3 = decode2(kk[1][k] >> 16);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float(&to)[4] = NT == 1 && (k & 1) ? odd[n] : c[a][n];
          mma_f16(to, a0, a1, a2, a3, qa[n][k][0], qa[n][k][1]);
          if constexpr (kSplit) mma_f16(to, a0, a1, a2, a3, qb[n][k][0], qb[n][k][1]);
        }
      }
      if constexpr (NT == 1) {
#pragma unroll
        for (int j = 0; j < 4; ++j) c[a][0][j] += odd[0][j];
      }
    }
    uint32_t vv[2][4][HD / 32];
    load_values<HD>(vv[0], at + 2 * kStep * HD, g, t);
    load_values<HD>(vv[1], at + 3 * kStep * HD, g, t);
    const bool masked = u * kUnit + kUnit - 1 > pos_lo || !have[0] || !have[1];      // some row does not see the whole unit
    uint32_t pa[NT][4], pb[kSplit ? NT : 1][4];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float x[2][4];
#pragma unroll
      for (int a = 0; a < 2; ++a) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          x[a][j] = fmaf(c[a][n][j], rs[n][j & 1] * ks[a], fe[a]);
          if (masked && (!have[a] || u * kUnit + a * kStep + g + 8 * (j >> 1) > rpos[n][j & 1])) x[a][j] = -INFINITY;
        }
      }
      float mx[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) mx[j] = fmaxf(fmaxf(x[0][j], x[0][j + 2]), fmaxf(x[1][j], x[1][j + 2]));
      if (__any_sync(0xffffffffu, mx[0] > m[n][0] + kSlack || mx[1] > m[n][1] + kSlack)) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
          for (int off = 4; off <= 16; off <<= 1) mx[j] = fmaxf(mx[j], __shfl_xor_sync(0xffffffffu, mx[j], off));
          const float mn = fmaxf(m[n][j], mx[j]), corr = mn == -INFINITY ? 1.f : ex2(m[n][j] - mn);
          m[n][j] = mn;
          l[n][j] *= corr;
#pragma unroll
          for (int k = 0; k < HD / 16; ++k) {
            acc[n][k][j] *= corr;
            acc[n][k][j + 2] *= corr;
          }
        }
      }
#pragma unroll
      for (int a = 0; a < 2; ++a) {
        float y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = ex2(x[a][j] - (m[n][j & 1] == -INFINITY ? 0.f : m[n][j & 1] - kOffset));
        l[n][0] = fmaf(el[a], y[0] + y[2], l[n][0]);
        l[n][1] = fmaf(el[a], y[1] + y[3], l[n][1]);
        const uint32_t h0 = pack_f16(y[0], y[1]), h1 = pack_f16(y[2], y[3]);
        pa[n][2 * a] = transpose8x8(h0);
        pa[n][2 * a + 1] = transpose8x8(h1);
        if constexpr (kSplit) {
          pb[n][2 * a] = transpose8x8(pack_rest(h0, y[0], y[1]));
          pb[n][2 * a + 1] = transpose8x8(pack_rest(h1, y[2], y[3]));
        }
      }
    }
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      if (masked) {
        // 0 * NaN: a NaN value must not reach rows that do not see its token.  It is taken out here, and the rows that do
        // see it are set to NaN when the block's sums are joined.  (Without a page the slot holds leftovers: zeros.)
#pragma unroll
        for (int i2 = 0; i2 < 4; ++i2) {
#pragma unroll
          for (int j = 0; j < HD / 32; ++j) {
            if (!have[a]) vv[a][i2][j] = 0;
            uint32_t bad = ((vv[a][i2][j] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
            vv[a][i2][j] &= ~((bad >> 7) * 0xffu);
            while (bad) {
              const int byte = (__ffs(bad) - 1) >> 3;
              bad &= bad - 1;
              atomicMin(nan_at + HD / 8 * g + 4 * j + byte, u * kUnit + a * kStep + 2 * t + (i2 & 1) + 8 * (i2 >> 1));
            }
          }
        }
      }
#pragma unroll
      for (int j = 0; j < HD / 32; ++j) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {                             // dims kPiece g + 4 j + 2 x and + 1 are rows g and g + 8 of tile 2 j + x
          const uint32_t x0 = tc::prmt(vv[a][0][j], vv[a][1][j], x ? 0x7362 : 0x5140), x1 = tc::prmt(vv[a][2][j], vv[a][3][j], x ? 0x7362 : 0x5140);
          const uint32_t a0 = decode2(x0), a1 = decode2(x0 >> 16), a2 = decode2(x1), a3 = decode2(x1 >> 16);
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            mma_f16(acc[n][2 * j + x], a0, a1, a2, a3, pa[n][2 * a], pa[n][2 * a + 1]);
            if constexpr (kSplit) mma_f16(acc[n][2 * j + x], a0, a1, a2, a3, pb[n][2 * a], pb[n][2 * a + 1]);
          }
        }
      }
    }
    // the slot's next unit (its rows are in this chunk of metadata or the next one)
    const int i3 = i + 2 * kDepth, src = (i3 & 31) + (lane & (nb - 1));
    const int rc = __shfl_sync(0xffffffffu, mc.row, src), rn = __shfl_sync(0xffffffffu, mn.row, src);
    if (u + kDepth < u_hi) issue(slot, i3 < 32 ? rc : rn);
    if (i == 30) {
      mc = mn;
      take_scales();
      mn = load_meta(entry_n, 2 * u + 34);
      entry_n = load_entry(2 * u + 66);
    }
    if (++slot == kDepth) {
      slot = 0;
      phase ^= 1;
    }
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
        float* p = part(w) + r * HD + HD / 8 * g + 2 * j;
        *reinterpret_cast<float2*>(p) = make_float2(acc[n][j][u], acc[n][j][u + 2]);
      }
    }
  }
  __syncthreads();
  constexpr int kThreads = kWarps * 32, kPer = (R * HD + kThreads - 1) / kThreads;      // results of this thread: threadIdx.x + i * kThreads
  if constexpr (kPart) {
    // (a short loop: as straight code, an element at a time, this took 4 us of a block that has little else to do)
#pragma unroll 1
    for (int i = threadIdx.x; i < n_rows * (HD / 4); i += kThreads) store_share<HD, R, kWarps, kRing>(i, ring0, wm, wl, nan_at, last_of(i / (HD / 4)),
                                                                                                 split * part_of.row_heads + (seq.row0 + (r0 + i / (HD / 4)) / G) * H +
                                                                                                     h * G + (r0 + i / (HD / 4)) % G, part_of);
    if (!prefix && blockIdx.x == 0) chain_wait();
    return;
  }
  float bm[kPer], rm[kPer], rl[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int at = threadIdx.x + i * kThreads, r = at / HD, d = at % HD;
    bm[i] = rl[i] = 0.f;
    rm[i] = -INFINITY;
    if (at >= R * HD) continue;
#pragma unroll
    for (int x = 0; x < kWarps; ++x) rm[i] = fmaxf(rm[i], wm[x * R + r]);
#pragma unroll
    for (int x = 0; x < kWarps; ++x) {
      const float f = rm[i] == -INFINITY ? 1.f : ex2(wm[x * R + r] - rm[i]);
      bm[i] = fmaf(f, part(x)[at], bm[i]);
      rl[i] = fmaf(f, wl[x * R + r], rl[i]);
    }
    if (first + (r0 + r) / G >= nan_at[d]) bm[i] = __int_as_float(0x7fffffff);
  }
  auto store = [&](int r, int d, float sum, float ll) {
    o[(seq.row0 + (r0 + r) / G) * o_stride + (h * G + (r0 + r) % G) * static_cast<int64_t>(HD) + d] =
        narrow<T>(ll == 0.f ? sum : sum / ll);                    // nothing attended to: sum = 0
  };
  if (nsplit == 1) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int at = threadIdx.x + i * kThreads;
      if (at < n_rows * HD) store(at / HD, at % HD, bm[i], rl[i]);
    }
    return;
  }
  if (ws != nullptr) {                                            // [item][split]: R * HD sums, R maxima, R sums of weights
    float* mine = ws + static_cast<int64_t>(blockIdx.x) * (R * (HD + 2));
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int at = threadIdx.x + i * kThreads;
      if (at >= n_rows * HD) continue;
      mine[at] = bm[i];
      if (at % HD == 0) {
        mine[R * HD + at / HD] = rm[i];
        mine[R * (HD + 1) + at / HD] = rl[i];
      }
    }
    return;
  }
  // the cluster's blocks joined in block order; block i writes the i-th share of the results
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int at = threadIdx.x + i * kThreads;
    if (at >= R * HD) continue;
    part(0)[at] = bm[i];
    if (at % HD == 0) {
      wm[at / HD] = rm[i];
      wl[at / HD] = rl[i];
    }
  }
  cg::cluster_group cluster = cg::this_cluster();
  cluster.sync();
  const int from = R * HD * split / nsplit, share = R * HD * (split + 1) / nsplit - from;
  for (int i = threadIdx.x; i < share; i += kWarps * 32) {
    const int at = from + i, r = at / HD;
    if (r >= n_rows) continue;
    float mm = -INFINITY, sum = 0.f, ll = 0.f;
    for (int x = 0; x < nsplit; ++x) mm = fmaxf(mm, cluster.map_shared_rank(wm, x)[r]);
    for (int x = 0; x < nsplit; ++x) {
      const float f = mm == -INFINITY ? 1.f : ex2(cluster.map_shared_rank(wm, x)[r] - mm);
      sum = fmaf(f, cluster.map_shared_rank(part(0), x)[at], sum);
      ll = fmaf(f, cluster.map_shared_rank(wl, x)[r], ll);
    }
    store(r, at % HD, sum, ll);
  }
  cluster.sync();                                                 // nobody leaves while its sums are being read
}

// The same for up to 32 rows of a group over its shared positions, 16-bit types: every code is turned into fp16 once for all of them
// (two tiles of 16 rows do so twice: 8 sequences of 4 rows on 65536 shared positions, 8 heads of 128, 65 us, here 60).  What
// bounds it is the latency of the chain in each of its 8 warps per SM (issue 35 %): 254 registers leave no room for more.  The queries' fragments do not fit the registers beside 32 rows of sums: they stay in shared
// memory, and 16 positions are taken at a time.
template <typename T, int HD>
__global__ void __launch_bounds__(128, 2)
kv8_prefix_rows_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, View V, const T* __restrict__ q,
                       int64_t q_stride, int H, float scale_log2e, int nsplit, const Part part_of) {
  constexpr int NT = 4, R = 8 * NT, kWarps = 4, kThreads = kWarps * 32, kK = HD / 16, kRing = kRingBytes<HD>;
  static_assert(R * HD * 4 <= kRing, "a warp's partial result takes the place of its ring");
  extern __shared__ __align__(1024) unsigned char smem_kv8[];
  __shared__ uint2 q_frag[NT][kK][32];
  __shared__ float row_scale[R], wm[kWarps * R], wl[kWarps * R];
  __shared__ int row_last[R], nan_at[HD];
  __shared__ __align__(8) uint64_t full[kWarps][kDepth];
  __shared__ int abort_flag;
  unsigned char* ring0 = smem_kv8 + ((1024u - (tc::smem_u32(smem_kv8) & 1023u)) & 1023u);
  chain_wait();
  chain_release();
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  unsigned item = blockIdx.x;
  const int split = item % nsplit;
  item /= nsplit;
  const int h = item % V.hkv, b = item / V.hkv, G = H / V.hkv;
  const Work work = load_work(V, part_of, b);
  const Seq seq = work.seq;
  const int n_rows = static_cast<int>(min(static_cast<int64_t>(seq.n) * G, static_cast<int64_t>(R)));
  if (n_rows <= 0) return;
  for (int i = threadIdx.x; i < HD; i += kThreads) nan_at[i] = 0x7fffffff;
  if (threadIdx.x == 0) abort_flag = 0;
  const uint32_t ring = tc::smem_u32(ring0) + w * kRing, bars = tc::smem_u32(&full[w][0]);
  if (lane == 0) {
    for (int i = 0; i < kDepth; ++i) tc::mbar_init(bars + 8 * i, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncwarp();
  // this warp's units of two steps; a last unit may have one
  const int pos_hi = seq.len - 1, steps = pos_hi / kStep + 1, units = (steps + 1) / 2;
  int u_lo = static_cast<int>(static_cast<int64_t>(units) * split / nsplit), u_hi = static_cast<int>(static_cast<int64_t>(units) * (split + 1) / nsplit);
  {
    const int span = u_hi - u_lo, base = u_lo;
    u_lo = base + span * w / kWarps;
    u_hi = base + span * (w + 1) / kWarps;
  }
  struct Meta {
    int row;                                                      // -1: no page, or behind this warp's share
    float2 sc;
  };
  const int32_t* table = V.table + static_cast<int64_t>(work.owner) * V.max_pages;
  const int s_end = min(2 * u_hi, steps);
  auto load_entry = [&](int s) { return s + lane < s_end ? __ldg(table + ((s + lane) >> (V.page_shift - 4))) : -1; };
  auto load_meta = [&](int entry, int s) {
    Meta r{-1, make_float2(0.f, 0.f)};
    if (static_cast<uint32_t>(entry) < static_cast<uint64_t>(V.n_pages)) {
      r.row = ((entry * V.hkv + h) << V.page_shift) + (((s + lane) << 4) & ((1 << V.page_shift) - 1));
      r.sc = __ldg(V.scales + static_cast<int64_t>(entry) * V.hkv + h);
    } else if (s + lane < s_end) {
      report_page(V);
    }
    return r;
  };
  const int box = box_tokens(V), nb = kUnit / box;
  auto issue = [&](int slot, int row) {
    const uint32_t bar = bars + 8 * slot;
    const unsigned live = __ballot_sync(0xffffffffu, lane < 2 * nb && row >= 0);
    if (lane == 0) tc::mbar_expect_tx(bar, __popc(live) * box * HD);
    __syncwarp();
    if (lane < 2 * nb && row >= 0)
      tc::tma_load_2d(ring + slot * kUnit * HD * 2 + lane * box * HD, lane < nb ? &map_k : &map_v, 0, row, bar);
  };
  int entry = load_entry(2 * u_lo), entry_n = load_entry(2 * u_lo + 32);
  Meta mc = load_meta(entry, 2 * u_lo);
#pragma unroll
  for (int i = 0; i < kDepth; ++i) {
    const int row = __shfl_sync(0xffffffffu, mc.row, 2 * i + (lane & (nb - 1)));
    if (u_lo + i < u_hi) issue(i, row);
  }
  Meta mn = load_meta(entry_n, 2 * u_lo + 32);
  entry_n = load_entry(2 * u_lo + 64);
  float ks_c, fe_c;
  auto take_scales = [&]() {
    ks_c = exp2_int(scale_exponent(mc.sc.x));
    fe_c = mc.row >= 0 ? static_cast<float>(scale_exponent(mc.sc.y)) : -INFINITY;
  };
  {
    // queries: warp w prepares the fragments of rows 8 w .. 8 w + 7 (see the kernel above)
    const int r = 8 * w + g;
    float x[kK][4], amax = 0.f;
    bool fine = true;
    const T* qp = q + (seq.row0 + r / G) * q_stride + (h * G + r % G) * static_cast<int64_t>(HD) + HD / 4 * t;
#pragma unroll
    for (int i = 0; i < HD / 4; i += Vec<T>::kN) {
      Vec<T> v = {};
      if (r < n_rows) v = *reinterpret_cast<const Vec<T>*>(qp + i);
#pragma unroll
      for (int u = 0; u < Vec<T>::kN; ++u) {
        const float y = widen<T>(v.x[u]);
        x[(i + u) / 4][(i + u) % 4] = y;
        amax = fmaxf(amax, fabsf(y));
        fine = fine && isfinite(y);
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
    for (int i = 0; i < kK; ++i) q_frag[w][i][lane] = make_uint2(pack_f16(x[i][0] * inv, x[i][1] * inv), pack_f16(x[i][2] * inv, x[i][3] * inv));
    if (t == 0) {
      row_scale[r] = fine ? exp2_int(e) * scale_log2e : __int_as_float(0x7fffffff);
      row_last[r] = r < n_rows ? min(__ldg(part_of.pos + seq.row0 + r / G), pos_hi) : pos_hi;
    }
  }
  __syncthreads();
  const bool all = __syncthreads_and(row_last[lane] == pos_hi);   // every row sees all of it, or each step is masked
  float acc[NT][HD / 16][4], m[NT][2], l[NT][2], rs[NT][2];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      m[n][u] = -INFINITY;
      l[n][u] = 0.f;
      rs[n][u] = row_scale[8 * n + 2 * t + u];                    // this thread's scores are those of rows 2 t, 2 t + 1
    }
#pragma unroll
    for (int i = 0; i < HD / 16; ++i) acc[n][i][0] = acc[n][i][1] = acc[n][i][2] = acc[n][i][3] = 0.f;
  }
  take_scales();
  int slot = 0;
  uint32_t phase = 0;
  for (int u = u_lo; u < u_hi; ++u) {
    const int i = 2 * (u - u_lo) & 31;
    if (!__all_sync(0xffffffffu, tc::mbar_wait(bars + 8 * slot, phase, &abort_flag, V.status, 0))) break;
    const uint32_t at = ring + slot * kUnit * HD * 2;
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      const float ks = __shfl_sync(0xffffffffu, ks_c, i + a), fe = __shfl_sync(0xffffffffu, fe_c, i + a);
      const bool have = fe != -INFINITY, masked = !all || !have;
      const float el = have ? exp2_int(-static_cast<int>(fe)) : 0.f;
      float c[NT][4];
#pragma unroll
      for (int n = 0; n < NT; ++n) c[n][0] = c[n][1] = c[n][2] = c[n][3] = 0.f;
      {
        uint32_t kk[2][kK];
        load_keys<HD>(kk, at + a * kStep * HD, g, t);
#pragma unroll
        for (int k = 0; k < kK; ++k) {
          const uint32_t a0 = decode2(kk[0][k]), a1 = decode2(kk[1][k]), a2 = decode2(kk[0][k] >> 16), a3 = decode2(kk[1][k] >> 16);
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            const uint2 f = q_frag[n][k][lane];
            mma_f16(c[n], a0, a1, a2, a3, f.x, f.y);
          }
        }
      }
      uint32_t vv[4][HD / 32];
      load_values<HD>(vv, at + (2 + a) * kStep * HD, g, t);
      uint32_t pa[NT][2];
      bool grows = false;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          c[n][j] = fmaf(c[n][j], rs[n][j & 1] * ks, fe);
          if (masked && (!have || u * kUnit + a * kStep + g + 8 * (j >> 1) > row_last[8 * n + 2 * t + (j & 1)])) c[n][j] = -INFINITY;
        }
        grows = grows || fmaxf(c[n][0], c[n][2]) > m[n][0] + kSlack || fmaxf(c[n][1], c[n][3]) > m[n][1] + kSlack;
      }
      if (__any_sync(0xffffffffu, grows)) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            float mx = fmaxf(c[n][j], c[n][j + 2]);
#pragma unroll
            for (int off = 4; off <= 16; off <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
            const float top = fmaxf(m[n][j], mx), corr = top == -INFINITY ? 1.f : ex2(m[n][j] - top);
            m[n][j] = top;
            l[n][j] *= corr;
#pragma unroll
            for (int k = 0; k < HD / 16; ++k) {
              acc[n][k][j] *= corr;
              acc[n][k][j + 2] *= corr;
            }
          }
        }
      }
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const float r0 = m[n][0] == -INFINITY ? 0.f : m[n][0] - kOffset, r1 = m[n][1] == -INFINITY ? 0.f : m[n][1] - kOffset;
        const float y0 = ex2(c[n][0] - r0), y1 = ex2(c[n][1] - r1), y2 = ex2(c[n][2] - r0), y3 = ex2(c[n][3] - r1);
        l[n][0] = fmaf(el, y0 + y2, l[n][0]);
        l[n][1] = fmaf(el, y1 + y3, l[n][1]);
        pa[n][0] = transpose8x8(pack_f16(y0, y1));
        pa[n][1] = transpose8x8(pack_f16(y2, y3));
      }
      if (masked) {                                               // (0 * NaN: see the kernel above)
#pragma unroll
        for (int i2 = 0; i2 < 4; ++i2) {
#pragma unroll
          for (int j = 0; j < HD / 32; ++j) {
            if (!have) vv[i2][j] = 0;
            uint32_t bad = ((vv[i2][j] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
            vv[i2][j] &= ~((bad >> 7) * 0xffu);
            while (bad) {
              const int byte = (__ffs(bad) - 1) >> 3;
              bad &= bad - 1;
              atomicMin(nan_at + HD / 8 * g + 4 * j + byte, u * kUnit + a * kStep + 2 * t + (i2 & 1) + 8 * (i2 >> 1));
            }
          }
        }
      }
#pragma unroll
      for (int j = 0; j < HD / 32; ++j) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const uint32_t x0 = tc::prmt(vv[0][j], vv[1][j], x ? 0x7362 : 0x5140), x1 = tc::prmt(vv[2][j], vv[3][j], x ? 0x7362 : 0x5140);
          const uint32_t a0 = decode2(x0), a1 = decode2(x0 >> 16), a2 = decode2(x1), a3 = decode2(x1 >> 16);
#pragma unroll
          for (int n = 0; n < NT; ++n) mma_f16(acc[n][2 * j + x], a0, a1, a2, a3, pa[n][0], pa[n][1]);
        }
      }
    }
    const int i3 = i + 2 * kDepth, src = (i3 & 31) + (lane & (nb - 1));
    const int rc = __shfl_sync(0xffffffffu, mc.row, src), rn = __shfl_sync(0xffffffffu, mn.row, src);
    if (u + kDepth < u_hi) issue(slot, i3 < 32 ? rc : rn);
    if (i == 30) {
      mc = mn;
      take_scales();
      mn = load_meta(entry_n, 2 * u + 34);
      entry_n = load_entry(2 * u + 66);
    }
    if (++slot == kDepth) {
      slot = 0;
      phase ^= 1;
    }
  }
  // the block's warps joined in warp order, four dims per thread
  float* mine = reinterpret_cast<float*>(ring0 + w * kRing);
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
      for (int j = 0; j < HD / 16; ++j) *reinterpret_cast<float2*>(mine + r * HD + HD / 8 * g + 2 * j) = make_float2(acc[n][j][u], acc[n][j][u + 2]);
    }
  }
  __syncthreads();
#pragma unroll 1
  for (int i = threadIdx.x; i < n_rows * (HD / 4); i += kThreads) {
    const int r = i / (HD / 4);
    store_share<HD, R, kWarps, kRing>(i, ring0, wm, wl, nan_at, row_last[r], split * part_of.row_heads + (seq.row0 + r / G) * H + h * G + r % G, part_of);
  }
}

// Joins the shares' partial results in the workspace: HD / 4 threads per row, four dims each.  With many shares (kGroups =
// 16) a block is one row, every group of threads taking every 16th share, and the groups' results are joined in order;
// with few, a block is four rows, since what it waits for is its chain of loads (64 row tiles of
// 256 in 2 shares of 512 positions: 35 us with the launch before it, with a thread per dim and a row per block 59).  `rows`: rows of
// a tile that can be there.
template <int kGroups> constexpr int kJoinRows = kGroups == 1 ? 4 : 1;
template <typename T, int HD, int kGroups>
__global__ void __launch_bounds__(HD / 4 * kGroups * kJoinRows<kGroups>)
kv8_join_kernel(View V, const float* __restrict__ ws, T* __restrict__ o, int64_t o_stride, int H, int R, int rows, int row_tiles, int nsplit,
                bool long_first, unsigned item0) {
  constexpr int kLanes = HD / 4;
  __shared__ float4 sums[kGroups][kLanes];
  __shared__ float ms[kGroups], ls[kGroups];
  chain_release();
  const int groups = (rows + kJoinRows<kGroups> - 1) / kJoinRows<kGroups>, part = threadIdx.x / kLanes, lane = threadIdx.x % kLanes;
  const int grp = kGroups > 1 ? part : 0, r = static_cast<int>(blockIdx.x % groups) * kJoinRows<kGroups> + (kGroups > 1 ? 0 : part), G = H / V.hkv;
  const unsigned item = item0 + blockIdx.x / groups, others = static_cast<unsigned>(V.batch) * V.hkv;
  const int rt = long_first ? row_tiles - 1 - static_cast<int>(item / others) : item % row_tiles;
  const unsigned bh = long_first ? item % others : item / row_tiles;
  const int h = bh % V.hkv, b = bh / V.hkv;
  const Seq seq = load_seq(V, b);                                 // (before the wait: the launch before this one was not chained to its own predecessor)
  const int64_t row = static_cast<int64_t>(rt) * R + r;
  chain_wait();
  if (r >= rows || row >= static_cast<int64_t>(seq.n) * G) return;      // (with groups: the whole block)
  const int64_t step = static_cast<int64_t>(R) * (HD + 2);
  const float* p = ws + static_cast<int64_t>(blockIdx.x / groups) * nsplit * step;
  float mm = -INFINITY, ll = 0.f;
  float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](float f, const float4& x, float l) {
    sum = make_float4(fmaf(f, x.x, sum.x), fmaf(f, x.y, sum.y), fmaf(f, x.z, sum.z), fmaf(f, x.w, sum.w));
    ll = fmaf(f, l, ll);
  };
#pragma unroll 8
  for (int x = grp; x < nsplit; x += kGroups) mm = fmaxf(mm, p[x * step + R * HD + r]);
#pragma unroll 4
  for (int x = grp; x < nsplit; x += kGroups)
    add(mm == -INFINITY ? 1.f : ex2(p[x * step + R * HD + r] - mm), *reinterpret_cast<const float4*>(p + x * step + r * HD + 4 * lane),
        p[x * step + R * (HD + 1) + r]);
  if constexpr (kGroups > 1) {
    sums[grp][lane] = sum;
    if (lane == 0) {
      ms[grp] = mm;
      ls[grp] = ll;
    }
    __syncthreads();
    if (grp != 0) return;
    mm = -INFINITY;
#pragma unroll
    for (int k = 0; k < kGroups; ++k) mm = fmaxf(mm, ms[k]);
    sum = make_float4(0.f, 0.f, 0.f, 0.f);
    ll = 0.f;
#pragma unroll
    for (int k = 0; k < kGroups; ++k) add(mm == -INFINITY ? 1.f : ex2(ms[k] - mm), sums[k][lane], ls[k]);
  }
  T y[4];
  y[0] = narrow<T>(ll == 0.f ? sum.x : sum.x / ll);
  y[1] = narrow<T>(ll == 0.f ? sum.y : sum.y / ll);
  y[2] = narrow<T>(ll == 0.f ? sum.z : sum.z / ll);
  y[3] = narrow<T>(ll == 0.f ? sum.w : sum.w / ll);
  struct alignas(4 * sizeof(T)) Four { T x[4]; };
  *reinterpret_cast<Four*>(o + (seq.row0 + row / G) * o_stride + (h * G + row % G) * HD + 4 * lane) = Four{{y[0], y[1], y[2], y[3]}};
}

// Keys or values as one matrix of bytes, a token and head per row; boxes of `rows` tokens, swizzled over the row
szo_status codes_map(const uint8_t* codes, const View& V, int hd, int rows, CUtensorMap* map) {
  return encode_map_2d(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, codes, (V.n_pages * V.hkv) << V.page_shift, hd, 1, rows, hd,
                       hd == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B);
}

template <typename T, int HD, int NT, int kWarps, bool kPart = false>
szo_status launch_rows(const View& V, const Rows& A, int nsplit, float* ws, cudaStream_t st, const Part& part = Part{}) {
  constexpr int R = 8 * NT;
  const size_t smem = static_cast<size_t>(kWarps) * kRingBytes<HD> + 1024;
  const int64_t tiles = ceil_div(static_cast<int64_t>(kPart ? part.max_rows : V.max_new) * (A.H / V.hkv), R);
  unsigned blocks;
  if (kPart) {
    const int64_t n = tiles * nsplit * part.items * V.hkv;
    SZO_REQUIRE(n <= 0x7fffffff, SZO_ERR_SHAPE, "too many rows, heads and sequences for one launch");
    blocks = static_cast<unsigned>(n);
  } else {
    SZO_TRY(grid_items(tiles * nsplit, V, &blocks));
  }
  CUtensorMap map_k, map_v;
  SZO_TRY(codes_map(V.k, V, HD, box_tokens(V), &map_k));
  SZO_TRY(codes_map(V.v, V, HD, box_tokens(V), &map_v));
  auto kern = kv8_attention_kernel<T, HD, NT, kWarps, kPart>;
  SZO_CHECK_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)));
  SZO_CHECK_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3(kWarps * 32);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  int attrs = 0;
  if (nsplit > 1 && ws == nullptr && !kPart) {
    attr[attrs].id = cudaLaunchAttributeClusterDimension;
    attr[attrs].val.clusterDim.x = nsplit;
    attr[attrs].val.clusterDim.y = attr[attrs].val.clusterDim.z = 1;
    ++attrs;
  }
  if (kPart) {
    attr[attrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[attrs].val.programmaticStreamSerializationAllowed = 1;
    ++attrs;
  }
  cfg.attrs = attr;
  cfg.numAttrs = attrs;
  SZO_CHECK_CUDA(cudaLaunchKernelEx(&cfg, kern, map_k, map_v, V, static_cast<const T*>(A.q), A.q_stride, static_cast<T*>(A.o), A.o_stride, A.H,
                                    A.scale * 1.4426950408889634f, static_cast<int>(tiles), nsplit, ws, part));
  count_launch();
  if (ws == nullptr) return SZO_OK;
  return launch_join<T, HD>(V, A, ws, R, static_cast<int>(tiles), nsplit, false, 0, tiles * V.batch * V.hkv, st);
}

// How the positions are cut: blocks of 4 warps, three per SM, joined in clusters of up to 16, or (`wide`) of 12, one per SM,
// joined by the second launch.  The lengths are on the device, so the rule goes by the number of (sequence, head, row tile)
// items alone: as many blocks as stay at two per SM; a second, partial round of blocks costs more than the idle third (8
// sequences of 4096 positions and 8 heads: clusters of 4 / 8 16.5 / 22.6 us; 16 sequences: 2 / 4 30.6 / 40.1).  Between one
// and two items per SM one block per item is best for equal lengths and worst for unequal ones, clusters of 3 near the best
// for both (32 sequences, 8 heads, 1 / 2 / 3 blocks: 4096 positions each 48 / 69 / 57 us, 513 to 8192 67 / 56 / 59 us).
// Blocks of 16 rows hold more registers and fewer clusters of 16 fit at once: beyond 8 items they go in clusters of 8 (32 rows,
// 8 heads, one sequence of 2048 / 8192 positions: 12.6 / 21.1 us, in clusters of 16 21.5 / 30.6; 8 items of 12 rows at 8192
// positions in 16 / 8: 15.7 / 17.8).  A cut stops at one unit per warp of what the page table could hold.
struct Plan {
  int rows, nsplit;
  bool wide;
};
Plan plan(const View& V, int H) {
  const int64_t rows = static_cast<int64_t>(V.max_new) * (H / V.hkv);
  Plan p{rows <= 8 ? 8 : 16, 1, false};
  const int64_t items = ceil_div(rows, p.rows) * V.batch * V.hkv;
  const int64_t units = ceil_div(static_cast<int64_t>(V.max_pages) << V.page_shift, kUnit);
  if (p.rows == 8 && items * 16 <= 148 * 2 && units >= kWideUnits) {
    p.wide = true;
    p.nsplit = static_cast<int>(148 / items);
    return p;
  }
  const int most = p.rows == 8 || items <= 8 ? 16 : 8;
  while (p.nsplit < most && items * p.nsplit * 2 <= 148 * 2 && units >= 2 * p.nsplit * 4) p.nsplit *= 2;
  if (p.nsplit == 1 && items > 148 && items <= 148 * 2 && units >= 3 * 4) p.nsplit = 3;
  return p;
}

// Whether a call of 16-bit type goes to the kernel for many rows.  That one takes 256 rows at a time and waits longer before
// its first product, this one reads the cache again for every 16 rows.  Measured with 8 key/value heads of 128 (this kernel /
// that one, us; the cut of the positions included): 32 rows per head, 1 sequence of 1024 / 8 of 4096 / 32 of 4096 positions
// 10.9 / 18.7, 37 / 49, 109 / 157; 64 rows, 1 of 1024 / 1 of 8192 / 1 of 65536 12 / 20, 22 / 25, 99 / 89 and, where the 16-row
// tiles fill the SMs, 8 of 4096 / 32 of 4096 / 64 of 513 86 / 51, 196 / 161, 117 / 88; 96 rows, 1 of 1024 / 1 of 65536 14 / 20,
// 184 / 92.
bool many_rows(const View& V, int H) {
  const int64_t rows = static_cast<int64_t>(V.max_new) * (H / V.hkv);
  return rows > 32 && ceil_div(rows, 16) * V.batch * V.hkv > 32;
}

template <typename T, int HD>
szo_status launch_attention(const View& V, const Rows& A, float* ws, cudaStream_t st) {
  if constexpr (sizeof(T) == 2)
    if (many_rows(V, A.H)) return launch_attention_tc<T, HD>(V, A, ws, st);
  const Plan p = plan(V, A.H);
  if (p.wide) return launch_rows<T, HD, 1, 12>(V, A, p.nsplit, ws, st);
  return p.rows == 8 ? launch_rows<T, HD, 1, 4>(V, A, p.nsplit, nullptr, st) : launch_rows<T, HD, 2, 4>(V, A, p.nsplit, nullptr, st);
}

size_t workspace_bytes(const View& V, int H, int hd) {
  if (V.batch == 0 || V.max_new == 0 || V.rows == 0) return 0;
  if (many_rows(V, H)) return workspace_bytes_tc(V, H, hd);         // (fp32 needs none then)
  const Plan p = plan(V, H);
  return p.wide ? static_cast<size_t>(148) * p.rows * (hd + 2) * sizeof(float) : 0;
}

}  // namespace

template <typename T, int HD> szo_status launch_prefix_rows(const View& V, const Rows& A, int nsplit, cudaStream_t st, const Part& part) {
  const size_t smem = static_cast<size_t>(4) * kRingBytes<HD> + 1024;
  const int64_t blocks = static_cast<int64_t>(nsplit) * part.items * V.hkv;
  SZO_REQUIRE(blocks <= 0x7fffffff, SZO_ERR_SHAPE, "too many rows, heads and sequences for one launch");
  CUtensorMap map_k, map_v;
  SZO_TRY(codes_map(V.k, V, HD, box_tokens(V), &map_k));
  SZO_TRY(codes_map(V.v, V, HD, box_tokens(V), &map_v));
  auto kern = kv8_prefix_rows_kernel<T, HD>;
  SZO_CHECK_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)));
  SZO_CHECK_CUDA(launch_maybe_chained(kern, dim3(static_cast<unsigned>(blocks)), dim3(128), smem, st, true, map_k, map_v, V, static_cast<const T*>(A.q),
                                      A.q_stride, A.H, A.scale * 1.4426950408889634f, nsplit, part));
  count_launch();
  return SZO_OK;
}
template <typename T, int HD> szo_status launch_part(const View& V, const Rows& A, const Part& part, int nsplit, cudaStream_t st) {
  const int64_t rows = static_cast<int64_t>(part.max_rows) * (A.H / V.hkv);
  if constexpr (sizeof(T) == 2)
    if (part.prefix && rows > 16 && rows <= kPrefixRows) return launch_prefix_rows<T, HD>(V, A, nsplit, st, part);
  return rows <= 8 ? launch_rows<T, HD, 1, 4, true>(V, A, nsplit, nullptr, st, part) : launch_rows<T, HD, 2, 4, true>(V, A, nsplit, nullptr, st, part);
}
#define SZO_KV8_PART(T, HD) template szo_status launch_part<T, HD>(const View&, const Rows&, const Part&, int, cudaStream_t)
SZO_KV8_PART(float, 64);
SZO_KV8_PART(float, 128);
SZO_KV8_PART(__nv_bfloat16, 64);
SZO_KV8_PART(__nv_bfloat16, 128);
SZO_KV8_PART(__half, 64);
SZO_KV8_PART(__half, 128);
#undef SZO_KV8_PART

szo_status check_rows(const szo_kv8_cache* cache, const void* q, int64_t q_stride, const void* o, int64_t o_stride, szo_dtype dtype,
                      int32_t n_heads, float scale, const void* workspace) {
  SZO_REQUIRE(q && o, SZO_ERR_INVALID_ARG, "NULL q or o");
  SZO_REQUIRE(dtype == SZO_F32 || dtype == SZO_BF16 || dtype == SZO_F16, SZO_ERR_UNSUPPORTED, "dtype must be f32, bf16 or f16");
  SZO_REQUIRE(n_heads > 0 && n_heads % cache->n_kv_heads == 0, SZO_ERR_SHAPE, "n_heads must be a multiple of n_kv_heads");
  SZO_REQUIRE(std::isfinite(scale), SZO_ERR_INVALID_ARG, "scale must be finite");
  const int64_t width = static_cast<int64_t>(n_heads) * cache->head_dim, vec = dtype == SZO_F32 ? 4 : 8;
  SZO_REQUIRE(q_stride >= width && o_stride >= width, SZO_ERR_SHAPE, "row strides must be at least n_heads * head_dim");
  SZO_REQUIRE(aligned16(q) && aligned16(o) && aligned16(workspace) && q_stride % vec == 0 && o_stride % vec == 0, SZO_ERR_ALIGNMENT,
              "buffers and rows must be 16-byte aligned");
  return SZO_OK;
}
szo_status check_sizes(const szo_kv8_cache* cache, const View& V, int32_t n_heads) {
  SZO_REQUIRE(static_cast<int64_t>(V.max_new) * n_heads <= 0x7fffffff, SZO_ERR_SHAPE, "too many rows and heads");
  SZO_REQUIRE(cache->n_pages <= 0x7fffffff / cache->n_kv_heads / cache->page_tokens, SZO_ERR_SHAPE,
              "n_pages * n_kv_heads * page_tokens must be below 2^31");
  return SZO_OK;
}

template <typename T, int HD>
szo_status launch_join(const View& V, const Rows& A, const float* ws, int R, int row_tiles, int nsplit, bool long_first, int64_t item0,
                       int64_t n_items, cudaStream_t st) {
  SZO_REQUIRE(n_items * R <= 0x7fffffff, SZO_ERR_SHAPE, "too many rows for one launch");
  const int rows = row_tiles > 1 ? R : static_cast<int>(static_cast<int64_t>(V.max_new) * (A.H / V.hkv));
  auto run = [&](auto kern, auto groups) {
    constexpr int kG = decltype(groups)::value, kRows = kJoinRows<kG>;
    return launch_maybe_chained(kern, dim3(static_cast<unsigned>(n_items * ceil_div(rows, kRows))), dim3(HD / 4 * kG * kRows), 0, st, true, V, ws,
                                static_cast<T*>(A.o), A.o_stride, A.H, R, rows, row_tiles, nsplit, long_first, static_cast<unsigned>(item0));
  };
  SZO_CHECK_CUDA(nsplit > 16 ? run(kv8_join_kernel<T, HD, 16>, std::integral_constant<int, 16>{})
                             : run(kv8_join_kernel<T, HD, 1>, std::integral_constant<int, 1>{}));
  count_launch();
  return SZO_OK;
}
#define SZO_KV8_JOIN(T, HD) \
  template szo_status launch_join<T, HD>(const View&, const Rows&, const float*, int, int, int, bool, int64_t, int64_t, cudaStream_t)
SZO_KV8_JOIN(float, 64);
SZO_KV8_JOIN(float, 128);
SZO_KV8_JOIN(__nv_bfloat16, 64);
SZO_KV8_JOIN(__nv_bfloat16, 128);
SZO_KV8_JOIN(__half, 64);
SZO_KV8_JOIN(__half, 128);
#undef SZO_KV8_JOIN

}  // namespace kv8
}  // namespace szo

using namespace szo;

extern "C" {

size_t szo_attention_kv8_workspace_bytes(const szo_kv8_cache* cache, const szo_kv8_batch* batch, int32_t n_heads) {
  kv8::View V;
  if (kv8::make_view(cache, batch, &V) != SZO_OK || n_heads <= 0 || n_heads % cache->n_kv_heads != 0) return 0;
  return kv8::workspace_bytes(V, n_heads, cache->head_dim);
}

szo_status szo_attention_kv8(const szo_kv8_cache* cache, const szo_kv8_batch* batch, const void* q, int64_t q_stride, void* o,
                             int64_t o_stride, szo_dtype dtype, int32_t n_heads, float scale, void* workspace, size_t workspace_bytes,
                             void* stream) {
  kv8::View V;
  SZO_TRY(kv8::make_view(cache, batch, &V));
  SZO_TRY(kv8::check_rows(cache, q, q_stride, o, o_stride, dtype, n_heads, scale, workspace));
  if (V.batch == 0 || V.max_new == 0 || V.rows == 0) return SZO_OK;
  SZO_TRY(kv8::check_sizes(cache, V, n_heads));
  const size_t need = kv8::workspace_bytes(V, n_heads, cache->head_dim);
  SZO_REQUIRE(need == 0 || (workspace && workspace_bytes >= need), SZO_ERR_WORKSPACE, "workspace: %zu bytes needed, %zu given", need,
              workspace ? workspace_bytes : size_t(0));
  SZO_TRY(kv8::set_status_word(&V));
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const kv8::Rows A{q, o, q_stride, o_stride, n_heads, scale};
  float* ws = static_cast<float*>(workspace);
  const bool wide = cache->head_dim == 128;
  if (dtype == SZO_F32) return wide ? kv8::launch_attention<float, 128>(V, A, ws, st) : kv8::launch_attention<float, 64>(V, A, ws, st);
  if (dtype == SZO_BF16) return wide ? kv8::launch_attention<__nv_bfloat16, 128>(V, A, ws, st) : kv8::launch_attention<__nv_bfloat16, 64>(V, A, ws, st);
  return wide ? kv8::launch_attention<__half, 128>(V, A, ws, st) : kv8::launch_attention<__half, 64>(V, A, ws, st);
}

}  // extern "C"
