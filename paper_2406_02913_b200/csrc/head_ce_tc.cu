// The products of the cross entropy from hidden states, and of its gradient, on the 5th-generation tensor cores: one persistent
// kernel for all of them, a launch takes up to three products (jobs) at once.
//
// A cluster of two CTAs computes 256 x 256 of a product (tcgen05.mma.cta_group::2): each CTA brings 128 rows of A and
// 128 of B per stage by TMA and keeps 128 rows x 256 columns of fp32 sums in TMEM, twice, so that a tile's epilogue runs
// beside the next tile's products.  An operand is read as it lies in memory, whichever of its dimensions is contracted:
//   logits   h [rows][d],  W [vocab][d]             both along their rows
//   dh       G [rows][vocab],  W [vocab][d]         W's rows are contracted
//   dW       G [rows][vocab],  h [rows][d]          both operands' rows are contracted
// With at most 128 rows of hidden states these are the columns of D (N = 32 to 128) and the vocabulary (for dh: d) its rows, so that
// the products take a fraction of the time in which W arrives; tiles are then as high as makes the clusters' shares equal.
// Roles of a CTA's 12 warps: 0 brings the operands (both CTAs' copies arrive on the leader's barriers), 1 issues the products
// (leader only), 2 has the TMEM, 4-11 the epilogue: two warps per 32 rows, 128 columns each, a thread per row.
// Tiles are written through 4 KB of shared memory per warp by TMA, which leaves out what lies outside.
#include <algorithm>
#include <mutex>

#include "head_ce.cuh"
#include "tc_common.cuh"

namespace szo {
namespace head {

namespace {

using namespace tc;

constexpr int kHalf = 128, kMostStages = 12, kRingBytes = 6 * 2 * kHalf * kBlockK * 2;
constexpr int kEpiWarp0 = 4, kEpiWarps = 8, kWarps = kEpiWarp0 + kEpiWarps, kOutBytes = 4096;
constexpr int kSmem = kRingBytes + kEpiWarps * kOutBytes + 1024;
constexpr int kMaxDevices = 64;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ uint32_t cluster_ctarank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync_all() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The address, in the cluster's shared memory, of the leader's variable at this CTA's address
__device__ __forceinline__ uint32_t of_leader(uint32_t local) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(local), "r"(0));
  return r;
}
__device__ __forceinline__ bool elect() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r != 0;
}
// A box into this CTA's shared memory, its bytes counted on the leader's barrier
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t leader_bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(leader_bar)
      : "memory");
}
__device__ __forceinline__ void store_box(const CUtensorMap* map, uint32_t src, int x, int y) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];" ::"l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y),
               "r"(src)
               : "memory");
}
__device__ __forceinline__ void store_box3(const CUtensorMap* map, uint32_t src, int x, int y, int z) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y),
               "r"(z), "r"(src)
               : "memory");
}
__device__ __forceinline__ void add_box3(const CUtensorMap* map, uint32_t src, int x, int y, int z) {
  asm volatile("cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(reinterpret_cast<uint64_t>(map)),
               "r"(x), "r"(y), "r"(z), "r"(src)
               : "memory");
}
__device__ __forceinline__ void store_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void store_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void store_wait() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void alloc_tmem(uint32_t result_smem) {
  asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(result_smem) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void free_tmem(uint32_t taddr) { asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(taddr) : "memory"); }
__device__ __forceinline__ void mma_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
// When the products issued so far are done: one arrival on the barrier at this offset in both CTAs
__device__ __forceinline__ void commit_both(uint32_t bar) {
  const uint16_t both = 3;
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"(both) : "memory");
}
__device__ __forceinline__ void arrive_at(uint32_t cluster_bar) { asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory"); }
__device__ __forceinline__ void put16(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float min_nan(float a, float b) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
template <typename T> __device__ __forceinline__ uint32_t pack(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack<__nv_bfloat16>(float lo, float hi) { return pack_bf16x2(lo, hi); }
template <> __device__ __forceinline__ uint32_t pack<__half>(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

template <typename T> __device__ __forceinline__ T round_to(float x);
template <> __device__ __forceinline__ __nv_bfloat16 round_to<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half round_to<__half>(float x) { return __float2half_rn(x); }
__device__ __forceinline__ void load16(uint32_t taddr, float (&f)[16]) {
  uint32_t v[16];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]),
        "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(taddr)
      : "memory");
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]), "+r"(v[10]),
                 "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15])::"memory");
#pragma unroll
  for (int i = 0; i < 16; ++i) f[i] = __uint_as_float(v[i]);
}
// Reduces 16 columns held by 32 lanes (one row each): lane l gets column lane_column(l), in 16 exchanges
__device__ __forceinline__ int lane_column(int lane) { return lane >> 1; }
__device__ __forceinline__ int column_lane(int column) { return column << 1; }
template <typename F> __device__ __forceinline__ float columns_reduce(float (&x)[16], int lane, F f) {
#pragma unroll
  for (int n = 8, o = 16; n >= 1; n >>= 1, o >>= 1) {             // columns [0, n) stay where bit o of the lane is 0, [n, 2 n) where it is 1
    const bool up = (lane & o) != 0;
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const float keep = up ? x[n + i] : x[i], give = up ? x[i] : x[n + i];
      x[i] = f(keep, __shfl_xor_sync(0xffffffffu, give, o));
    }
  }
  return f(x[0], __shfl_xor_sync(0xffffffffu, x[0], 1));
}

// Operand tiles (128-byte swizzle).  Contracted along its rows: 128 rows of 64 elements.  Rows contracted: two blocks of 64 rows (k) of 64
// elements, 8192 bytes apart.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, int mn) {
  return static_cast<uint64_t>((addr & 0x3FFFFu) >> 4) | (static_cast<uint64_t>(mn ? 8192 >> 4 : 1) << 16) | (static_cast<uint64_t>(1024 >> 4) << 32) |
         (1ull << 46) | (2ull << 61);
}

struct Unit {
  int j, m, n, part, kb0, kb1;
};
__device__ __forceinline__ Unit unit_of(const Jobs& P, int u) {
  Unit r;
  r.j = 0;
  while (r.j + 1 < P.n_jobs && u >= P.job[r.j].units) u -= P.job[r.j++].units;
  const Job& J = P.job[r.j];
  const int tiles = J.m_tiles * J.n_tiles;
  r.part = u / tiles;
  int t = u - r.part * tiles;
  int m0 = 0, width = J.m_tiles;
  if (J.m_band > 0) {
    const int band = t / (J.n_tiles * J.m_band);
    t -= band * J.n_tiles * J.m_band;
    m0 = band * J.m_band;
    width = min(J.m_band, J.m_tiles - m0);
  }
  r.n = t / width;
  r.m = m0 + t - r.n * width;
  r.kb0 = static_cast<int>(static_cast<int64_t>(J.nkb) * r.part / J.parts);
  r.kb1 = static_cast<int>(static_cast<int64_t>(J.nkb) * (r.part + 1) / J.parts);
  return r;
}

template <typename T>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kWarps * 32, 1) head_jobs_kernel(const __grid_constant__ Jobs P) {
  extern __shared__ unsigned char smem_raw[];
  __shared__ __align__(8) unsigned long long bars[2 * kMostStages + 4];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag_s;
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = static_cast<int>(cluster_ctarank());
  volatile int* abort_flag = &abort_flag_s;
  auto full = [&](int s) { return smem_u32(&bars[s]); };                          // leader: both CTAs' operands landed
  auto empty = [&](int s) { return smem_u32(&bars[kMostStages + s]); };               // the products that read the stage are done
  auto acc_full = [&](int a) { return smem_u32(&bars[2 * kMostStages + a]); };
  auto acc_empty = [&](int a) { return smem_u32(&bars[2 * kMostStages + 2 + a]); };   // leader: both CTAs' epilogues have read the sums
  if (threadIdx.x == 0) {
    abort_flag_s = 0;
    for (int s = 0; s < kMostStages; ++s) {
      mbar_init(full(s), 1);
      mbar_init(empty(s), 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(acc_full(a), 1);
      mbar_init(acc_empty(a), 2 * kEpiWarps);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  chain_release();
  if (warp == 2) alloc_tmem(smem_u32(&tmem_slot));
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();          // the peer's barriers exist before anyone arrives on them
  tc_fence_after();
  chain_wait();
  const uint32_t tmem = tmem_slot;
  const int pair = static_cast<int>(blockIdx.x >> 1), n_pairs = static_cast<int>(gridDim.x >> 1);

  if (warp == 0) {
    // ---------------------------------------------------------------- operands
    if (elect()) {
      RingPos x{0, 0};
      bool ok = true;
      for (int u = pair; u < P.units && ok; u += n_pairs) {
        const Unit t = unit_of(P, u);
        const Job& J = P.job[t.j];
        const CUtensorMap *ma = &J.a, *mb = &J.b;
        const int a0 = J.a_m0 + t.m * J.m_step + rank * (J.m_step / 2), b0 = J.b_n0 + t.n * J.n_step + rank * (J.n_step / 2);
        const uint32_t bytes = 2u * (J.a_bytes + J.b_bytes);
        const int a_mn = J.a_mn, b_mn = J.b_mn, a_k0 = J.a_k0, b_k0 = J.b_k0;
        for (int kb = t.kb0; kb < t.kb1; ++kb) {
          if (!mbar_wait(empty(x.idx), x.phase ^ 1u, abort_flag, P.status)) {
            ok = false;
            break;
          }
          if (rank == 0) mbar_expect_tx(full(x.idx), bytes);
          const uint32_t bar = of_leader(full(x.idx)), sa = base + x.idx * P.stage_bytes, sb = sa + P.b_at;
          const int k = kb * kBlockK;
          if (a_mn) {
            load_box(sa, ma, a0, a_k0 + k, bar);
            load_box(sa + 8192, ma, a0 + 64, a_k0 + k, bar);
          } else {
            load_box(sa, ma, k, a0, bar);
          }
          if (b_mn) {
            load_box(sb, mb, b0, b_k0 + k, bar);
            load_box(sb + 8192, mb, b0 + 64, b_k0 + k, bar);
          } else {
            load_box(sb, mb, k, b0, bar);
          }
          x.advance(P.stages);
        }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    // ---------------------------------------------------------------- products (leader only)
    if (rank == 0 && elect()) {
      RingPos x{0, 0};
      bool ok = true;
      int lt = 0;
      // kind::f16: fp32 sums, both operands of type T, M = 256; bits 15 / 16: rows of A / B are contracted
      constexpr uint32_t kType = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
      constexpr uint32_t kIdesc = (1u << 4) | (kType << 7) | (kType << 10) | (static_cast<uint32_t>(kTile >> 4) << 24);
      for (int u = pair; u < P.units && ok; u += n_pairs, ++lt) {
        const Unit t = unit_of(P, u);
        const int a_mn = P.job[t.j].a_mn, b_mn = P.job[t.j].b_mn;
        const uint32_t idesc = kIdesc | (static_cast<uint32_t>(P.job[t.j].n_step >> 3) << 17) | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u);
        const int step_a = a_mn ? 2048 >> 4 : 32 >> 4, step_b = b_mn ? 2048 >> 4 : 32 >> 4, as = lt & 1;
        if (!mbar_wait(acc_empty(as), static_cast<uint32_t>((lt >> 1) & 1) ^ 1u, abort_flag, P.status)) break;
        tc_fence_after();
        const uint32_t d = tmem + as * kTile;
        for (int kb = t.kb0; kb < t.kb1; ++kb) {
          if (!mbar_wait(full(x.idx), x.phase, abort_flag, P.status, 0)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint32_t sa = base + x.idx * P.stage_bytes;
          const uint64_t da = operand_desc(sa, a_mn), db = operand_desc(sa + P.b_at, b_mn);
#pragma unroll
          for (int k = 0; k < kBlockK / 16; ++k) mma_pair(d, da + k * step_a, db + k * step_b, idesc, kb > t.kb0 || k > 0);
          commit_both(empty(x.idx));
          x.advance(P.stages);
        }
        commit_both(acc_full(as));
      }
    }
    __syncwarp();
  } else if (warp >= kEpiWarp0) {
    // ---------------------------------------------------------------- epilogue: 32 rows, 128 columns
    const int w = warp - kEpiWarp0, quarter = warp & 3, half = w >> 2;
    const uint32_t stage = base + kRingBytes + w * kOutBytes;
    auto place = [&](int chunk) { return stage + lane * 128 + ((chunk ^ (lane & 7)) << 4); };
    auto reuse = [&]() {                                          // the warp's 4 KB may be written again
      if (lane == 0) store_wait_read();
      __syncwarp();
    };
    auto written = [&]() {
      fence_async_smem();
      __syncwarp();
    };
    int lt = 0;
    for (int u = pair; u < P.units; u += n_pairs, ++lt) {
      const Unit t = unit_of(P, u);
      const Job& J = P.job[t.j];
      const int as = lt & 1, mine = quarter * 32 + lane;           // (its place in this CTA's half of the tile)
      const int row0 = t.m * J.m_step + rank * (J.m_step / 2) + quarter * 32, row = row0 + lane, col0 = t.n * J.n_step + half * (J.n_step / 2);
      const bool there = row < J.m_limit && mine < J.m_step / 2;
      int target = -1;
      float4 info = make_float4(0.f, 0.f, 0.f, 0.f);
      float factor = 1.f;
      if (J.kind <= kGrad && there) target = P.targets[row];
      if (J.kind == kGrad && there) info = P.info[row];
      if (J.kind == kOut) factor = weight_of<T>(P.exponent);
      target = target >= 0 ? target - P.target0 - col0 : -1;      // (its place in these columns, or outside of [0, 128))
      if (target >= P.n_end - col0) target = -1;
      if (!mbar_wait(acc_full(as), static_cast<uint32_t>((lt >> 1) & 1), abort_flag, P.status, 128)) break;
      tc_fence_after();
      const uint32_t acc = tmem + (static_cast<uint32_t>(quarter * 32) << 16) + as * kTile + half * (J.n_step / 2);
      // some row of this warp is there (kStatsT: might be, its part is written all the same)
      const bool live = (row0 < J.m_limit || J.kind == kStatsT) && quarter * 32 < J.m_step / 2;
      if (!live) {
      } else if (J.kind == kStats) {
        float m = -INFINITY, s = 0.f;
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
          uint32_t v[32];
          tmem_ld32(acc + 32 * c, v);
          const int left = P.n_end - (col0 + 32 * c), hit = target - 32 * c;
          if (left < 32) {
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (i >= left) v[i] = 0xff800000u;
          }
          if (__any_sync(0xffffffffu, hit >= 0 && hit < 32)) {
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (i == hit) {
                P.xt[row] = __uint_as_float(v[i]) * P.c;
                v[i] = 0xff800000u;
              }
          }
          float top = -INFINITY;
#pragma unroll
          for (int i = 0; i < 32; ++i) top = fmaxf(top, __uint_as_float(v[i]));
          // (the difference before the factor: no exponent is above 0, whatever the scale)
          const float mn = fmaxf(m, top), ref = mn == -INFINITY ? 0.f : mn;
          float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = 0; i < 32; ++i) sum[i & 3] += ex2((__uint_as_float(v[i]) - ref) * P.c);
          s = fmaf(s, ex2((m - ref) * P.c), (sum[0] + sum[1]) + (sum[2] + sum[3]));
          m = mn;
        }
        if (there) P.part[static_cast<int64_t>(2 * t.n + half) * P.rows + row] = make_float2(m * P.c, s);
      } else if (J.kind == kGrad) {
        const bool weighs = info.y != 0.f || info.z != 0.f;
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
          uint32_t v[32];
          tmem_ld32(acc + 32 * c, v);
          if ((c & 1) == 0) reuse();
          const int hit = target - 32 * c;
          const bool any = __any_sync(0xffffffffu, hit >= 0 && hit < 32);
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            const float x = min_nan(fmaf(__uint_as_float(v[i]), P.c, -info.x), 0.f), p = ex2(x);      // (rounding may put x above lse)
            float g = info.y * p;
            if (any && i == hit) g = fmaf(info.y - info.z, p, info.z * expm1f(x * kLn2));
            v[i] = weighs ? __float_as_uint(g) : 0u;
          }
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            uint32_t o[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = pack<T>(__uint_as_float(v[8 * q + 2 * i]), __uint_as_float(v[8 * q + 2 * i + 1]));
            put16(place((c & 1) * 4 + q), o[0], o[1], o[2], o[3]);
          }
          if (c & 1) {
            written();
            if (lane == 0) {
              store_box(&J.out, stage, col0 + 32 * (c - 1), J.out_row0 + row0);
              store_commit();
            }
          }
        }
      } else if (J.kind == kSum) {
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
          uint32_t v[32];
          tmem_ld32(acc + 32 * c, v);
          reuse();
#pragma unroll
          for (int q = 0; q < 8; ++q) put16(place(q), v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
          written();
          if (lane == 0) {
            if (J.add) add_box3(&J.out, stage, col0 + 32 * c, row0, t.part);
            else store_box3(&J.out, stage, col0 + 32 * c, row0, t.part);
            store_commit();
          }
        }
      } else if (J.kind >= kStatsT) {
        // a thread is a vocabulary entry (kSumT: an element of d), the columns are rows of hidden states, 16 at a time
        const int last = static_cast<int>(P.rows), n_half = J.n_step / 2;
#pragma unroll 1
        for (int c = 0; c < n_half; c += 16) {
          const int r0 = col0 + c;
          if (r0 >= last) break;
          float v[16];
          load16(acc + c, v);
          if (J.kind == kSumT) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (there && r0 + i < last) {
                float* to = P.sums + (t.part * P.rows + r0 + i) * P.d + row;
                *to = J.add ? *to + v[i] : v[i];
              }
          } else if (J.kind == kGradT) {
            float4 f[16];
            int hit[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int r = min(r0 + i, last - 1);
              f[i] = __ldg(P.info + r);
              hit[i] = __ldg(P.targets + r);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float x = min_nan(fmaf(v[i], P.c, -f[i].x), 0.f), p = ex2(x);
              float g = f[i].y * p;
              if (hit[i] == P.target0 + row) g = fmaf(f[i].y - f[i].z, p, f[i].z * expm1f(x * kLn2));
              if (f[i].y == 0.f && f[i].z == 0.f) g = 0.f;
              if (there && r0 + i < last) static_cast<T*>(P.G)[(r0 + i) * P.g_stride + row] = round_to<T>(g);
            }
          } else {
            float top[16];
            int hit[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) hit[i] = __ldg(P.targets + min(r0 + i, last - 1));
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              if (!there) v[i] = -INFINITY;
              if (r0 + i < last && there && hit[i] == row) {
                P.xt[r0 + i] = v[i] * P.c;
                v[i] = -INFINITY;
              }
              top[i] = v[i];
            }
            const float mx = columns_reduce(top, lane, [](float a, float b) { return fmaxf(a, b); });
            float sum[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float m = __shfl_sync(0xffffffffu, mx, column_lane(i)), ref = m == -INFINITY ? 0.f : m;
              sum[i] = ex2((v[i] - ref) * P.c);
            }
            const float s = columns_reduce(sum, lane, [](float a, float b) { return a + b; });
            const int col = lane_column(lane);
            if ((lane & 1) == 0 && r0 + col < last)
              P.part[static_cast<int64_t>((t.m * 2 + rank) * ((J.m_step / 2 + 31) / 32) + quarter) * P.rows + r0 + col] = make_float2(mx * P.c, s);
          }
        }
      } else {
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
          uint32_t v[32];
          tmem_ld32(acc + 32 * c, v);
          if ((c & 1) == 0) reuse();
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            uint32_t o[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = pack<T>(__uint_as_float(v[8 * q + 2 * i]) * factor, __uint_as_float(v[8 * q + 2 * i + 1]) * factor);
            put16(place((c & 1) * 4 + q), o[0], o[1], o[2], o[3]);
          }
          if (c & 1) {
            written();
            if (lane == 0) {
              store_box(&J.out, stage, col0 + 32 * (c - 1), J.out_row0 + row0);
              store_commit();
            }
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) arrive_at(of_leader(acc_empty(as)));
    }
    if (lane == 0) store_wait();
    __syncwarp();
  }

  if (*abort_flag) {
    for (int i = 0; i < 200; ++i) __nanosleep(1000);              // (copies in flight land)
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();          // no CTA leaves while its peer may still signal it or read its operands
  tc_fence_after();
  if (warp == 2) free_tmem(tmem);
}

}  // namespace

template <typename T> szo_status launch_jobs(Jobs& P, bool chained, cudaStream_t st) {
  auto kern = head_jobs_kernel<T>;
  // per device: the function's attribute and the number of SM pairs, looked up once
  static std::mutex mu;
  static int pairs_of[kMaxDevices] = {};
  int dev = 0;
  SZO_CHECK_CUDA(cudaGetDevice(&dev));
  SZO_REQUIRE(dev >= 0 && dev < kMaxDevices, SZO_ERR_UNSUPPORTED, "device ordinal %d out of range", dev);
  int pairs;
  {
    std::lock_guard<std::mutex> lock(mu);
    if (pairs_of[dev] == 0) {
      int sms = 0;
      SZO_CHECK_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
      SZO_CHECK_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem));
      pairs_of[dev] = sms / 2;
    }
    pairs = pairs_of[dev];
  }
  if (P.units < pairs) pairs = P.units;
  // the ring: as many stages as fit of what the jobs' operands need, so that a few rows (a small B) keep as many bytes of W on their
  // way (8 rows: 53 us with 6 stages)
  P.b_at = P.stage_bytes = 0;
  for (int i = 0; i < P.n_jobs; ++i) P.b_at = std::max(P.b_at, static_cast<int>(round_up(P.job[i].a_bytes, 1024)));
  for (int i = 0; i < P.n_jobs; ++i) P.stage_bytes = std::max(P.stage_bytes, P.b_at + static_cast<int>(round_up(P.job[i].b_bytes, 1024)));
  P.stages = std::min(kMostStages, kRingBytes / P.stage_bytes);
  SZO_CHECK_CUDA(launch_maybe_chained(kern, dim3(static_cast<unsigned>(2 * pairs)), dim3(kWarps * 32), kSmem, st, chained, P));
  count_launch();
  return SZO_OK;
}
template szo_status launch_jobs<__nv_bfloat16>(Jobs&, bool, cudaStream_t);
template szo_status launch_jobs<__half>(Jobs&, bool, cudaStream_t);

}  // namespace head
}  // namespace szo
