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
// What bounds it: many rows, the tensor cores (their pipe 94 % busy, issue slots 10 %; 4096 rows of 32000 x 4096, bf16: loss 652 us, 1.65
// PFLOP/s, gradient down to h 1.40 ms; 128 x 256 tiles of single CTAs read each operand tile twice as often); at most 128 rows, the reads of W
// (8 rows of 32000 x 4096: 262 MB in 49.5 us, 5.3 TB/s; with the rows as rows of D, 71 us); small matrices, the chain of one tile (256 rows of
// 1024 x 256, 10 us: setup 0.7, first operands 1.5, products 1.4, epilogue 3, end 0.7, join).
#include <algorithm>
#include <mutex>

#include "head_ce.cuh"
#include "tc_common.cuh"

namespace szo {
namespace head {

namespace {

using namespace tc;

constexpr int kHalf = 128, kMostStages = 12;
// (with few rows their columns' data take 4 KB of shared memory)
template <bool kFew> constexpr int kRingBytes = 6 * 2 * kHalf * kBlockK * 2 - (kFew ? 4096 : 0);
constexpr int kEpiWarp0 = 4, kEpiWarps = 8, kWarps = kEpiWarp0 + kEpiWarps, kOutBytes = 4096;
template <bool kFew> constexpr int kSmem = kRingBytes<kFew> + kEpiWarps * kOutBytes + 1024;
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
__device__ __forceinline__ void load_box_hint(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t leader_bar, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3}], [%4], %5;" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(leader_bar), "l"(policy)
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
// p - 1 for p = e^t, t <= 0, to fp32's precision: the exponential's series where they cancel (nine terms: 2^-26 at t = -1/2).  (A few instructions:
// the function of the library, unrolled over a tile's columns, made a launch of a few rows wait for instructions.)
__device__ __forceinline__ float below_one(float t, float p) {
  float s = 1.f / 362880.f;
  s = fmaf(s, t, 1.f / 40320.f);
  s = fmaf(s, t, 1.f / 5040.f);
  s = fmaf(s, t, 1.f / 720.f);
  s = fmaf(s, t, 1.f / 120.f);
  s = fmaf(s, t, 1.f / 24.f);
  s = fmaf(s, t, 1.f / 6.f);
  s = fmaf(s, t, 0.5f);
  s = fmaf(s, t, 1.f);
  return t > -0.5f ? s * t : p - 1.f;
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

// ---- The order of the units
__device__ __forceinline__ int piece_len(const Jobs& P, int i) { return min(P.piece, P.vocab - i * P.piece); }
__device__ __forceinline__ const Extent& extent_of(const Jobs& P, int j, int i) { return i == P.pieces - 1 ? P.job[j].last : P.job[j].full; }
__device__ __forceinline__ int units_of(const Jobs& P, int j, int i) { return P.job[j].kind < 0 || i < 0 || i >= P.pieces ? 0 : extent_of(P, j, i).units; }
struct Unit {
  int j, i, m, n, part, kb0, kb1;
  int from_end, stride;                        // kSumT: the kb-th of its blocks is from_end - kb * stride
};
// Walks along the units: a role asks for rising ones only
template <bool kFew> struct Walk {
  int s, j = 0, first = 0;
  __device__ __forceinline__ Unit seek(const Jobs& P, int u) {
    Unit r;
    while (true) {
      r.i = j == 0 ? s : s - 1;
      const int n = units_of(P, j, r.i);
      if (u < first + n) break;
      first += n;
      if (++j == 3) {
        j = 0;
        ++s;
      }
    }
    const Extent& e = extent_of(P, j, r.i);
    r.j = j;
    const int tiles = e.m_tiles * e.n_tiles;
    u -= first;
    r.part = e.parts > 1 ? u / tiles : 0;
    int t = u - r.part * tiles, m0 = 0, width = e.m_tiles;
    const int in_band = P.job[j].m_band;
    if (in_band > 0) {
      const int band = t / (e.n_tiles * in_band);
      t -= band * e.n_tiles * in_band;
      m0 = band * in_band;
      width = min(in_band, e.m_tiles - m0);
    }
    r.n = t / width;
    r.m = m0 + t - r.n * width;
    r.kb0 = 0;
    r.kb1 = e.nkb;
    if (kFew && P.job[j].vocab_dim == 2) {
      // dh of few rows: all shares walk together from the vocabulary's end, which the logits' launch has left in L2, to its start
      r.from_end = e.nkb - 1 - r.part;
      r.stride = e.parts;
      r.kb1 = r.from_end / e.parts + 1;
    } else if (e.parts > 1) {                                     // (parts are few: no overflow below 2^31 / 16 blocks)
      r.kb0 = e.nkb * r.part / e.parts;
      r.kb1 = e.nkb * (r.part + 1) / e.parts;
    }
    return r;
  }
};
// Arrivals that mean that job 0 (done 0) or jobs 1 and 2 (done 1) of piece i are finished: every epilogue warp of both CTAs, once per unit
__device__ __forceinline__ int arrivals_of(const Jobs& P, int i, int done) {
  return 2 * kEpiWarps * (done == 0 ? units_of(P, 0, i) : units_of(P, 1, i) + units_of(P, 2, i));
}
__device__ __forceinline__ int32_t* counter_of(const Jobs& P, int i, int done) { return P.counters + 1 + 2 * i + done; }
// Waits, with a limit, until they are; what the counted epilogues wrote may then be read, by TMA too.  Units are handed out in their order
// and wait for earlier ones only, so what is waited for runs already, on whatever SMs this launch has.
__device__ __forceinline__ bool await_piece(const Jobs& P, int i, int done, volatile int* abort_flag) {
  const int32_t* at = counter_of(P, i, done);
  const int want = arrivals_of(P, i, done);
  const long long t0 = clock64();
  for (int polls = 0;; ++polls) {
    int32_t v;
    asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(at) : "memory");
    if (v >= want) break;
    __nanosleep(64);
    if ((polls & 255) == 255) {
      if (*abort_flag) return false;
      if (clock64() - t0 > kWaitLimitCycles) {
        *abort_flag = 1;
        atomicExch(P.status, static_cast<int32_t>(SZO_ERR_TIMEOUT));
        return false;
      }
    }
  }
  asm volatile("fence.proxy.async;" ::: "memory");
  return true;
}
__device__ __forceinline__ void arrive_piece(const Jobs& P, int i, int done) {
  asm volatile("red.release.gpu.global.add.s32 [%0], %1;" ::"l"(counter_of(P, i, done)), "r"(1) : "memory");
}

// ---- Units on their way through a cluster: the leader's warp 3 takes the next one from the counter and gives it to every role of both CTAs
constexpr int kFeedSlots = 2, kFeedReaders = 2 * kEpiWarps + 3;   // epilogues, both operand warps, the products' thread
__device__ __forceinline__ bool wait_cluster(uint32_t bar, uint32_t parity, volatile int* abort_flag, int32_t* status) {
  const long long t0 = clock64();
  for (int polls = 0;; ++polls) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    if (ok) return true;
    __nanosleep(32);
    if ((polls & 1023) == 1023) {
      if (*abort_flag) return false;
      if (clock64() - t0 > kWaitLimitCycles) {
        *abort_flag = 1;
        atomicExch(status, static_cast<int32_t>(SZO_ERR_TIMEOUT));
        return false;
      }
    }
  }
}
__device__ __forceinline__ uint32_t of_peer(uint32_t local) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(local), "r"(1));
  return r;
}

// kFew: few rows of hidden states, launches of one step (a kernel of its own: a launch of a few microseconds waits for instructions)
template <typename T, bool kFew>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kWarps * 32, 1) head_jobs_kernel(const __grid_constant__ Jobs P) {
  extern __shared__ unsigned char smem_raw[];
  __shared__ __align__(8) unsigned long long bars[2 * kMostStages + 4 + 2 * kFeedSlots];
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int feed[kFeedSlots];
  constexpr int kMostColumns = 128;
  __shared__ float4 columns_info[kFew ? kMostColumns : 1];
  __shared__ int columns_target[kFew ? kMostColumns : 1];
  __shared__ int abort_flag_s;
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = static_cast<int>(cluster_ctarank());
  volatile int* abort_flag = &abort_flag_s;
  auto full = [&](int s) { return smem_u32(&bars[s]); };                          // leader: both CTAs' operands landed
  auto empty = [&](int s) { return smem_u32(&bars[kMostStages + s]); };               // the products that read the stage are done
  auto acc_full = [&](int a) { return smem_u32(&bars[2 * kMostStages + a]); };
  auto acc_empty = [&](int a) { return smem_u32(&bars[2 * kMostStages + 2 + a]); };   // leader: both CTAs' epilogues have read the sums
  auto feed_full = [&](int s) { return smem_u32(&bars[2 * kMostStages + 4 + s]); };
  auto feed_empty = [&](int s) { return smem_u32(&bars[2 * kMostStages + 4 + kFeedSlots + s]); };      // leader
  if (threadIdx.x == 0) {
    abort_flag_s = 0;
    for (int s = 0; s < kFeedSlots; ++s) {
      mbar_init(feed_full(s), 1);
      mbar_init(feed_empty(s), kFeedReaders);
    }
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
  // The next unit for a role, or -1.  `one`: the role is a single thread, else a warp
  int next_static = pair;
  RingPos fed{0, 0};
  auto next_unit = [&](bool one) {
    if (kFew || P.counters == nullptr) {
      const int u = next_static;
      next_static += n_pairs;
      return u < P.units ? u : -1;
    }
    if (!wait_cluster(feed_full(fed.idx), fed.phase, abort_flag, P.status)) return -1;
    const int u = feed[fed.idx];
    if (u >= P.units) return -1;
    if (!one) __syncwarp();
    if (u >= 0 && (one || lane == 0)) arrive_at(of_leader(feed_empty(fed.idx)));      // (u has been read: the arrival depends on it)
    fed.advance(kFeedSlots);
    return u;
  };

  if (warp == 0) {
    // ---------------------------------------------------------------- operands
    if (elect()) {
      RingPos x{0, 0};
      Walk<kFew> walk{P.step};
      bool ok = true;
      int written = -1;                                           // G of this piece is complete
      const uint64_t keep = l2_policy_evict_last(), drop = l2_policy_evict_first();
      for (int u; ok && (u = next_unit(true)) >= 0;) {
        const Unit t = walk.seek(P, u);
        const Job& J = P.job[t.j];
        if (!kFew && t.j > 0 && t.i != written && P.counters != nullptr) {
          if (!await_piece(P, t.i, 0, abort_flag)) break;
          written = t.i;
        }
        const CUtensorMap *ma = &J.a, *mb = &J.b;
        const int in_vocab = t.i * P.piece, in_buffers = P.buffers > 1 ? t.i % P.buffers * P.piece : 0;
        const int ao = J.a_from == kVocab ? in_vocab : J.a_from == kBuffer ? in_buffers : 0;
        const int bo = J.b_from == kVocab ? in_vocab : J.b_from == kBuffer ? in_buffers : 0;
        const bool along_k = J.vocab_dim == 2;
        const int a0 = (along_k ? 0 : ao) + t.m * J.m_step + rank * (J.m_step / 2), b0 = (along_k ? 0 : bo) + t.n * J.n_step + rank * (J.n_step / 2);
        const uint32_t bytes = 2u * (J.a_bytes + J.b_bytes);
        const int a_mn = J.a_mn, b_mn = J.b_mn, a_k0 = along_k ? ao : 0, b_k0 = along_k ? bo : 0;
        for (int kb = t.kb0; kb < t.kb1; ++kb) {
          if (!mbar_wait(empty(x.idx), x.phase ^ 1u, abort_flag, P.status)) {
            ok = false;
            break;
          }
          if (rank == 0) mbar_expect_tx(full(x.idx), bytes);
          const uint32_t bar = of_leader(full(x.idx)), sa = base + x.idx * P.stage_bytes, sb = sa + P.b_at;
          const int k = (kFew && along_k ? t.from_end - kb * t.stride : kb) * kBlockK;
          if (kFew && J.keep_from >= 0) {
            // W of few rows' gradient: what the logits read last stays for dh, which reads it first and for the last time
            const uint64_t policy = !a_mn && a0 >= J.keep_from ? keep : drop;
            if (a_mn) {
              load_box_hint(sa, ma, a0, a_k0 + k, bar, policy);
              load_box_hint(sa + 8192, ma, a0 + 64, a_k0 + k, bar, policy);
            } else {
              load_box_hint(sa, ma, a_k0 + k, a0, bar, policy);
            }
          } else if (a_mn) {
            load_box(sa, ma, a0, a_k0 + k, bar);
            load_box(sa + 8192, ma, a0 + 64, a_k0 + k, bar);
          } else {
            load_box(sa, ma, a_k0 + k, a0, bar);
          }
          if (b_mn) {
            load_box(sb, mb, b0, b_k0 + k, bar);
            load_box(sb + 8192, mb, b0 + 64, b_k0 + k, bar);
          } else {
            load_box(sb, mb, b_k0 + k, b0, bar);
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
      Walk<kFew> walk{P.step};
      for (int u; ok && (u = next_unit(true)) >= 0; ++lt) {
        const Unit t = walk.seek(P, u);
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
  } else if (warp == 3) {
    // ---------------------------------------------------------------- units (leader only)
    if (!kFew && rank == 0 && P.counters != nullptr && elect()) {
      RingPos f{0, 0};
      for (int u = 0; u < P.units;) {
        if (!wait_cluster(feed_empty(f.idx), f.phase ^ 1u, abort_flag, P.status)) break;
        u = atomicAdd(P.counters, 1);
        feed[f.idx] = u;
        const uint32_t there = of_peer(smem_u32(const_cast<int*>(&feed[f.idx])));
        asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(there), "r"(u) : "memory");
        mbar_arrive(feed_full(f.idx));
        asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(of_peer(feed_full(f.idx))) : "memory");
        f.advance(kFeedSlots);
      }
    }
    __syncwarp();
  } else if (warp >= kEpiWarp0) {
    // ---------------------------------------------------------------- epilogue: 32 rows, 128 columns
    const int w = warp - kEpiWarp0, quarter = warp & 3, half = w >> 2;
    const uint32_t stage = base + kRingBytes<kFew> + w * kOutBytes;
    auto place = [&](int chunk) { return stage + lane * 128 + ((chunk ^ (lane & 7)) << 4); };
    auto reuse = [&]() {                                          // the warp's 4 KB may be written again
      if (lane == 0) store_wait_read();
      __syncwarp();
    };
    auto written = [&]() {
      fence_async_smem();
      __syncwarp();
    };
    if constexpr (kFew) {
      // what the columns need: their targets and, for the gradient, infos (at most 128)
      const int i = threadIdx.x - kEpiWarp0 * 32;
      if (i < kMostColumns && P.job[0].kind >= 0) {
        const int64_t r = i < P.rows ? i : P.rows - 1;
        columns_target[i] = P.targets[r];
        if (P.job[0].kind == kGradT) columns_info[i] = P.info[r];
      }
      asm volatile("bar.sync 1, %0;" ::"r"(kEpiWarps * 32) : "memory");
    }
    int lt = 0, free_before = P.buffers, added = -1;             // pieces below free_before have a buffer of G to write to; sums of piece `added` are there
    Walk<kFew> walk{P.step};
    bool ok = true;
    for (int u; ok && (u = next_unit(false)) >= 0; ++lt) {
      const Unit t = walk.seek(P, u);
      const Job& J = P.job[t.j];
      const int as = lt & 1, mine = quarter * 32 + lane;           // (its place in this CTA's half of the tile)
      const int row0 = t.m * J.m_step + rank * (J.m_step / 2) + quarter * 32, row = row0 + lane, col0 = t.n * J.n_step + half * (J.n_step / 2);
      const int n_end = piece_len(P, t.i), m_limit = J.vocab_dim == 0 ? n_end : J.m_limit, target0 = t.i * P.piece, buffer0 = P.buffers > 1 ? t.i % P.buffers * P.piece : 0;
      const bool there = row < m_limit && mine < J.m_step / 2;
      int target = -1;
      float4 info = make_float4(0.f, 0.f, 0.f, 0.f);
      float factor = 1.f;
      if (!kFew && J.kind <= kGrad && there) target = P.targets[row];
      if (!kFew && J.kind == kGrad && there) info = P.info[row];
      if (J.kind == kOut) factor = weight_of<T>(P.exponent);
      target = target >= 0 ? target - target0 - col0 : -1;        // (its place in these columns, or outside of [0, 128))
      if (target >= n_end - col0) target = -1;
      if (!mbar_wait(acc_full(as), static_cast<uint32_t>((lt >> 1) & 1), abort_flag, P.status, 128)) break;
      tc_fence_after();
      const uint32_t acc = tmem + (static_cast<uint32_t>(quarter * 32) << 16) + as * kTile + half * (J.n_step / 2);
      // some row of this warp is there (the vocabulary along m: might be, its part is written all the same)
      const bool live = (row0 < m_limit || J.kind == kStatsT || J.kind == kGradT) && quarter * 32 < J.m_step / 2;
      if (kFew) {
      } else if (J.kind == kGrad) {
        // the buffer of G was that of an earlier piece: its readers have to be through
        if (t.i >= free_before && P.counters != nullptr) {
          ok = __all_sync(0xffffffffu, await_piece(P, t.i - P.buffers, 1, abort_flag));
          free_before = t.i + 1;
        }
      } else if (J.kind == kSum && t.i > 0 && t.i - 1 != added && P.counters != nullptr) {
        ok = __all_sync(0xffffffffu, await_piece(P, t.i - 1, 1, abort_flag));      // (what this piece's sums are added to)
        added = t.i - 1;
      }
      if (!live || !ok) {
      } else if (!kFew && J.kind == kStats) {
        float m = -INFINITY, s = 0.f;
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
          uint32_t v[32];
          tmem_ld32(acc + 32 * c, v);
          const int left = n_end - (col0 + 32 * c), hit = target - 32 * c;
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
      } else if (!kFew && J.kind == kGrad) {
        const bool weighs = info.y != 0.f || info.z != 0.f;
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
          uint32_t v[32];
          tmem_ld32(acc + 32 * c, v);
          if ((c & 1) == 0) reuse();
          const int hit = target - 32 * c, left = n_end - (col0 + 32 * c);
          const bool any = __any_sync(0xffffffffu, hit >= 0 && hit < 32);
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            const float x = min_nan(fmaf(__uint_as_float(v[i]), P.c, -info.x), 0.f), p = ex2(x);      // (rounding may put x above lse)
            float g = info.y * p;
            if (any && i == hit) g = fmaf(info.y - info.z, p, info.z * below_one(x * kLn2, p));
            v[i] = weighs && i < left ? __float_as_uint(g) : 0u;  // (columns behind the vocabulary are contracted with zeros: they must be finite)
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
              store_box(&J.out, stage, buffer0 + col0 + 32 * (c - 1), row0);
              store_commit();
            }
          }
        }
      } else if (!kFew && J.kind == kSum) {
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
          uint32_t v[32];
          tmem_ld32(acc + 32 * c, v);
          reuse();
#pragma unroll
          for (int q = 0; q < 8; ++q) put16(place(q), v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
          written();
          if (lane == 0) {
            if (t.i > 0) add_box3(&J.out, stage, col0 + 32 * c, row0, t.part);
            else store_box3(&J.out, stage, col0 + 32 * c, row0, t.part);
            store_commit();
          }
        }
      } else if (kFew && J.kind >= kStatsT) {
        // a thread is a vocabulary entry (kSumT: an element of d), the columns are rows of hidden states, 16 at a time
        const int last = static_cast<int>(P.rows), n_half = J.n_step / 2, padded = (n_end + kBlockK - 1) / kBlockK * kBlockK;
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
                P.sums[((static_cast<int64_t>(t.i) * J.full.parts + t.part) * P.rows + r0 + i) * P.d + row] = v[i];
              }
          } else if (J.kind == kGradT) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float4 f = columns_info[r0 + i];
              const float x = min_nan(fmaf(v[i], P.c, -f.x), 0.f), p = ex2(x);
              float g = f.y * p;
              if (columns_target[r0 + i] == target0 + row) g = fmaf(f.y - f.z, p, f.z * below_one(x * kLn2, p));
              if (!there || (f.y == 0.f && f.z == 0.f)) g = 0.f;
              if (mine < J.m_step / 2 && row < padded && r0 + i < last) static_cast<T*>(P.G)[(r0 + i) * P.g_stride + buffer0 + row] = round_to<T>(g);
            }
          } else {
            float top[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              if (!there) v[i] = -INFINITY;
              if (r0 + i < last && there && columns_target[r0 + i] == row) {
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
              store_box(&J.out, stage, col0 + 32 * (c - 1), target0 + row0);
              store_commit();
            }
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) arrive_at(of_leader(acc_empty(as)));
      if (!kFew && P.counters != nullptr && lane == 0) {
        store_wait();                                             // this warp's part of the unit is written
        if (ok) arrive_piece(P, t.i, t.j > 0);
      }
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

template <typename T, bool kFew> szo_status launch(Jobs& P, bool chained, cudaStream_t st) {
  auto kern = head_jobs_kernel<T, kFew>;
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
      SZO_CHECK_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem<kFew>));
      pairs_of[dev] = sms / 2;
    }
    pairs = pairs_of[dev];
  }
  if (P.units < pairs) pairs = P.units;
  // the ring: as many stages as fit of what the jobs' operands need, so that a few rows (a small B) keep as many bytes of W on their
  // way (8 rows: 53 us with 6 stages, 51 with 12)
  P.b_at = P.stage_bytes = 0;
  auto used = [&](int j) { return P.job[j].kind >= 0 && !(P.idle >> j & 1); };
  for (int j = 0; j < 3; ++j)
    if (used(j)) P.b_at = std::max(P.b_at, static_cast<int>(round_up(P.job[j].a_bytes, 1024)));
  for (int j = 0; j < 3; ++j)
    if (used(j)) P.stage_bytes = std::max(P.stage_bytes, P.b_at + static_cast<int>(round_up(P.job[j].b_bytes, 1024)));
  P.stages = std::min(kMostStages, kRingBytes<kFew> / P.stage_bytes);
  SZO_CHECK_CUDA(launch_maybe_chained(kern, dim3(static_cast<unsigned>(2 * pairs)), dim3(kWarps * 32), kSmem<kFew>, st, chained, P));
  count_launch();
  return SZO_OK;
}
template <typename T> szo_status launch_jobs(Jobs& P, bool few, bool chained, cudaStream_t st) {
  return few ? launch<T, true>(P, chained, st) : launch<T, false>(P, chained, st);
}
template szo_status launch_jobs<__nv_bfloat16>(Jobs&, bool, bool, cudaStream_t);
template szo_status launch_jobs<__half>(Jobs&, bool, bool, cudaStream_t);

}  // namespace head
}  // namespace szo
