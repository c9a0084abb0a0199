// Attention over the 8-bit paged cache for many query rows per key/value head (prompts, chunks of prompts) on the
// 5th-generation tensor cores.
//
// A block takes 256 query rows (new tokens x heads of one key/value head) of a sequence as two row tiles of 128 and
// walks over the cached positions 128 at a time.  Per step and row tile: S = Q K^T (128 x 128), softmax weights P,
// O += P V, all accumulated in TMEM (S and O of both row tiles fill its 512 columns; P, fp16, takes the place of S and
// is the A operand of the second product from there).  The bound is the tensor pipe (2 x 2 x 128 x 128 x 128 multiply-
// adds per step), with three more close behind it: the exponentials (16 per cycle and SM: as long as the products),
// shared memory (operands of the products and the converted tiles, 128 bytes per cycle) and the issue slots of the
// softmax.  Hence the split into warps that only meet at mbarriers:
//   warps 0-7, 8-15  softmax of row tile 0 and 1, two threads per row (a TMEM lane), 64 columns each: no shuffles, one
//                    exchange of maxima per step.  While one tile's weights are formed, the tensor cores work for the other
//   warps 16-19      turn the e4m3 codes into fp16 (exact) and store them in the swizzled layout that the products read
//   warp 20          one thread issues every product
//   warp 21          brings the codes by TMA, 64 positions of keys or values per slot of a small ring, and the pages' scales
//                    (with the converting warps loading for themselves the latency of a step's loads showed: they have
//                    no registers for a second set)
// Measured: 2 sequences of 2048 new tokens at 8192 positions, 32 heads over 8 of 128, 526 us (875 TFLOP/s, 0.52 of the measured
// burst rate of dense products, 0.63 of the sustained one).  A step of 128 positions takes 4500 cycles against 2048 for its
// products: a row tile's scores wait 1400 for both tiles' products, its maxima take 700, their exchange 270, its weights 1850
// (2048 for both tiles by the exponentials' rate), and the next products wait for them.  Copying and converting (1900 and
// 3100 cycles a step, on their own warps) hide behind that.
// Numbers are those of the kernel for few rows: queries divided by a power of two per row, weights relative to each
// token's contribution (logit + exponent of its page's value scale), sums of weights divided by that scale again.
// The reference maximum follows the running maximum once that is 2^8 above it, so O is rescaled in TMEM a few times
// per row; weights stay between 2^-24 and 2^15.
#include <cmath>
#include <type_traits>

#include "kv8_attention.cuh"

namespace szo {
namespace kv8 {

namespace {

constexpr int kTile = 128;                     // rows of a row tile, positions of a step
constexpr int kSoft = 16, kConv = 4, kMmaWarp = kSoft + kConv, kLoadWarp = kMmaWarp + 1, kTcThreads = (kLoadWarp + 1) * 32;      // (22 warps: 80 registers)
constexpr int kRawTokens = 64, kRawSlots = 3;  // ring of codes as they come: half a step of keys or values per slot
constexpr float kTcOffset = 7.0f, kTcSlack = 8.0f;
constexpr float kTiny = 1e-37f;                // factors of scores are kept above it: a zero would make NaN of a masked -inf
constexpr uint32_t kTmemCols = 512;

__device__ __forceinline__ void tmem_alloc(uint32_t result_smem, uint32_t ncols) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(result_smem), "r"(ncols) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_dealloc(uint32_t taddr, uint32_t ncols) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols) : "memory");
}
// D += A B, A and B in shared memory
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
// D += A B, A in TMEM
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Arrives on the barrier when the products issued so far are done
__device__ __forceinline__ void mma_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t (&v)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]),
        "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]),
        "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]),
        "=r"(v[31])
      : "r"(addr)
      : "memory");
}
// Waits for this thread's TMEM loads; v is an operand so that its uses stay behind
__device__ __forceinline__ void tmem_load_wait(uint32_t (&v)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]),
                 "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]), "+r"(v[16]), "+r"(v[17]), "+r"(v[18]),
                 "+r"(v[19]), "+r"(v[20]), "+r"(v[21]), "+r"(v[22]), "+r"(v[23]), "+r"(v[24]), "+r"(v[25]), "+r"(v[26]), "+r"(v[27]),
                 "+r"(v[28])
               :
               : "memory");
  asm volatile("" : "+r"(v[29]), "+r"(v[30]), "+r"(v[31])::"memory");
}
__device__ __forceinline__ void tmem_store32(uint32_t addr, const uint32_t (&v)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};" ::"r"(v[0]),
      "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]),
      "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]),
      "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31]), "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tmem_store16(uint32_t addr, const uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(v[0]),
      "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]),
      "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tmem_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

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

__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// fp16 operand tiles in shared memory: 128 rows in blocks of 64 columns (one 128-byte row each), 128-byte swizzle.
__device__ __forceinline__ uint32_t tile_chunk(uint32_t base, int row, int chunk) {      // 16-byte chunk (8 columns) of a row
  return base + (chunk >> 3) * (kTile * 128) + row * 128 + (((chunk & 7) ^ (row & 7)) << 4);
}
__device__ __forceinline__ uint2 lds8(uint32_t a) {
  uint2 r;
  asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(r.x), "=r"(r.y) : "r"(a) : "memory");
  return r;
}
__device__ __forceinline__ void sts16(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
// Descriptor of such a tile as an operand whose rows are the contracted dimension (columns of the result contiguous):
// blocks of 64 columns kTile * 128 bytes apart, groups of 8 rows 1024 bytes apart
__device__ __forceinline__ uint64_t make_desc_rows_contracted(uint32_t smem_addr) {
  return static_cast<uint64_t>((smem_addr & 0x3FFFFu) >> 4) | (static_cast<uint64_t>((kTile * 128) >> 4) << 16) |
         (static_cast<uint64_t>(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// Instruction descriptors, kind::f16, fp16 x fp16 with fp32 sums; bit 16: B's rows are the contracted dimension
constexpr uint32_t make_idesc_f16(int M, int N, bool b_rows_contracted) {
  return (1u << 4) | (b_rows_contracted ? 1u << 16 : 0u) | (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(M >> 4) << 24);
}

__host__ __device__ __forceinline__ int box_tokens(const View& V) { return V.page_shift < 6 ? 1 << V.page_shift : kRawTokens; }

// Items (row tile, sequence, head) from `whole` on are cut into `nsplit` shares of their positions, a block each
struct TcSplit {
  unsigned whole;
  int nsplit;
};

template <typename T, int HD>
__global__ void __launch_bounds__(kTcThreads, 1)
kv8_attention_tc_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, View V, const T* __restrict__ q, int64_t q_stride, T* __restrict__ o, int64_t o_stride, int H, float scale, int row_tiles, TcSplit part, float* __restrict__ ws) {
  constexpr int kBytes = kTile * HD * 2;                          // of an operand tile
  constexpr int kLanes = HD / 16, kRowsPass = kConv * 32 / kLanes;
  extern __shared__ __align__(1024) unsigned char smem_tc[];
  struct alignas(16) Step {
    float ks, fe, el;                                             // 2^(keys' exponent), values' exponent, its inverse power; no page: 1, -inf, 0
    float pad;
  };
  __shared__ Step meta[4][kTile / kStep];
  __shared__ int nan_at[HD];
  __shared__ float peaks[2][2][2][kTile];                         // [step parity][row tile][half][row]; in the end sums of weights
  __shared__ __align__(8) uint64_t bars[20 + 2 * kRawSlots];
  __shared__ uint32_t tmem_ptr;
  __shared__ int abort_flag;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int64_t others = static_cast<int64_t>(V.batch) * V.hkv;
  const bool cut = blockIdx.x >= part.whole;
  const unsigned item = cut ? part.whole + (blockIdx.x - part.whole) / part.nsplit : blockIdx.x;
  const int split = cut ? (blockIdx.x - part.whole) % part.nsplit : 0, nsplit = cut ? part.nsplit : 1;
  const int rt = row_tiles - 1 - static_cast<int>(item / others);                // the longest rows first
  const int h = static_cast<int>(item % others) % V.hkv, b = static_cast<int>(item % others) / V.hkv, G = H / V.hkv;
  const Seq seq = load_seq(V, b);
  const unsigned r0 = static_cast<unsigned>(rt) * 2 * kTile;                     // (rows and heads of a call stay below 2^31)
  const int64_t left = static_cast<int64_t>(seq.n) * G - r0;
  if (left <= 0) return;
  const int n_rows = static_cast<int>(left < 2 * kTile ? left : 2 * kTile);
  const int first = seq.len - seq.n;                              // position of the sequence's row 0; negative: padding
  auto pos_of = [&](int r) { return first + static_cast<int>((r0 + r) / static_cast<unsigned>(G)); };
  int n_kv[2], lo[2];                                             // steps of each row tile; position of its first row
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int rows = n_rows - kTile * i < kTile ? n_rows - kTile * i : kTile;
    lo[i] = pos_of(kTile * i);
    const int hi = rows > 0 ? pos_of(kTile * i + rows - 1) : -1;
    n_kv[i] = hi < 0 ? 0 : hi / kTile + 1;
  }
  // this block's steps [j0, j0 + n), counted from j0 from here on
  const int n_all = n_kv[1] > n_kv[0] ? n_kv[1] : n_kv[0];
  const int j0 = static_cast<int>(static_cast<int64_t>(n_all) * split / nsplit), n = static_cast<int>(static_cast<int64_t>(n_all) * (split + 1) / nsplit) - j0;
  const int p0 = j0 * kTile;                                      // position of the first column of step 0
#pragma unroll
  for (int i = 0; i < 2; ++i) n_kv[i] = min(max(n_kv[i] - j0, 0), n);
  const int n_steps = (pos_of(n_rows - 1) < 0 ? -1 : pos_of(n_rows - 1) / kStep) + 1;      // of 16 positions

  const uint32_t base = (tc::smem_u32(smem_tc) + 1023u) & ~1023u;
  auto v_tile = [&](int s) { return base + s * kBytes; };
  auto k_tile = [&](int s) { return base + (2 + s) * kBytes; };
  auto q_tile = [&](int i) { return base + (4 + i) * kBytes; };
  auto raw_slot = [&](int s) { return base + 6 * kBytes + s * kRawTokens * HD; };
  auto bar = [&](int i) { return tc::smem_u32(&bars[i]); };
  const int kSFull = 0, kPFull = 2, kODone = 4, kKFull = 6, kKEmpty = 8, kVFull = 10, kVEmpty = 12, kQFull = 14, kDrain = 15, kMeta = 16, kRawFull = 20, kRawEmpty = 20 + kRawSlots;
  if (tid == 0) {
    abort_flag = 0;
    for (int i = 0; i < 2; ++i) {
      tc::mbar_init(bar(kSFull + i), 1);
      tc::mbar_init(bar(kPFull + i), kSoft / 2);
      tc::mbar_init(bar(kODone + i), 1);
      tc::mbar_init(bar(kKFull + i), kConv);
      tc::mbar_init(bar(kKEmpty + i), 1);
      tc::mbar_init(bar(kVFull + i), kConv);
      tc::mbar_init(bar(kVEmpty + i), 1);
    }
    tc::mbar_init(bar(kQFull), kSoft);
    tc::mbar_init(bar(kDrain), 1);
    for (int i = 0; i < 4; ++i) tc::mbar_init(bar(kMeta + i), 1);
    for (int i = 0; i < kRawSlots; ++i) {
      tc::mbar_init(bar(kRawFull + i), 1);
      tc::mbar_init(bar(kRawEmpty + i), kConv);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  for (int i = tid; i < HD; i += kTcThreads) nan_at[i] = 0x7fffffff;
  if (warp == kMmaWarp) tmem_alloc(tc::smem_u32(&tmem_ptr), kTmemCols);
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = tmem_ptr;
  auto wait = [&](int i, int phase, unsigned backoff) { return tc::mbar_wait(bar(i), phase & 1, &abort_flag, V.status, backoff); };
  auto wait_warp = [&](int i, int phase, unsigned backoff) { return __all_sync(0xffffffffu, wait(i, phase, backoff)) != 0; };

  if (warp < kSoft) {
    // ------------------------------------------------------------------ softmax: two threads per row, 64 columns each
    const int i = warp >> 3, half = (warp >> 2) & 1, rr = (warp & 3) * 32 + lane, r = i * kTile + rr;      // row tile, columns, row of it, of the block
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t s_addr = tmem + lanes + i * kTile + half * (kTile / 2), o_addr = tmem + lanes + 2 * kTile + i * kTile + half * (HD / 2);
    const int rpos = pos_of(r < n_rows ? r : n_rows - 1);         // (rows that are not there: anything, they are not stored)
    // The queries: a warp brings 16 rows, a row's dims over kQLanes lanes, all loads before the first use
    {
      constexpr int kQLanes = HD / 8, kQRows = 32 / kQLanes, kPasses = 16 / kQRows;
      const int row0 = (warp & 3) * 32 + half * 16 + lane / kQLanes, c = lane % kQLanes;
      Vec<T> x[kPasses];
#pragma unroll
      for (int k = 0; k < kPasses; ++k) {
        const int qr = i * kTile + row0 + k * kQRows;
        const unsigned at = r0 + qr;
        x[k] = {};
        if (qr < n_rows)
          x[k] = *reinterpret_cast<const Vec<T>*>(q + (seq.row0 + at / static_cast<unsigned>(G)) * q_stride +
                                                  (h * G + at % static_cast<unsigned>(G)) * static_cast<int64_t>(HD) + 8 * c);
      }
#pragma unroll
      for (int k = 0; k < kPasses; ++k) {
        int top = 0;                                              // the largest magnitude's bits: NaN above infinity above the rest
#pragma unroll
        for (int u = 0; u < 8; ++u) top = max(top, __float_as_int(widen<T>(x[k].x[u])) & 0x7fffffff);
#pragma unroll
        for (int s = 1; s < kQLanes; s *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, s));
        const int e = min(max((top >> 23) - 127, -126), 126);
        const float inv = scale < 0.f ? -exp2_int(-e) : exp2_int(-e);
        uint32_t p[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) p[u] = pack_f16(widen<T>(x[k].x[2 * u]) * inv, widen<T>(x[k].x[2 * u + 1]) * inv);
        const int row = row0 + k * kQRows;
        sts16(tile_chunk(q_tile(i), row, c), p[0], p[1], p[2], p[3]);
        if (c == 0) {
          peaks[1][i][0][row] = exp2_int(e) * (fabsf(scale) * 1.4426950408889634f);
          peaks[1][i][1][row] = top < 0x7f800000 ? 0.f : __int_as_float(0x7fffffff);      // a row that holds NaN or an infinity is NaN
        }
      }
      tc::fence_async_smem();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(bar(kQFull));
      asm volatile("bar.sync %0, %1;" ::"r"(1 + 4 * i + (warp & 3)), "r"(64) : "memory");
    }
    const float rs = peaks[1][i][0][rr], poison = rpos < 0 ? 0.f : peaks[1][i][1][rr];      // (padding rows are zeros whatever they hold)
    float m = -INFINITY, l = 0.f;
    const int limit0 = rpos - p0 - half * (kTile / 2);
    // (a wait that gave up changes nothing here: every warp of a row tile meets the others as often, whatever it read)
    for (int j = 0; j < n_kv[i]; ++j) {
      wait_warp(kMeta + (j & 3), j >> 2, 20);
      wait_warp(kSFull + i, j, 20);
      tc::tc_fence_after();
      const Step* st = &meta[j & 3][half * (kTile / kStep / 2)];
      uint32_t v[32];
      if (p0 + j * kTile + kTile - 1 > lo[i]) {                   // what a row does not see becomes -inf in S itself: one form of the rest
#pragma unroll 1
        for (int c = 0; c < 2; ++c) {
          tmem_load32(s_addr + 32 * c, v);
          tmem_load_wait(v);
          const int limit = limit0 - j * kTile - 32 * c;          // columns up to this one are seen
#pragma unroll
          for (int u = 0; u < 32; ++u)
            if (u > limit) v[u] = 0xff800000u;
          tmem_store32(s_addr + 32 * c, v);
        }
        tmem_store_wait();
      }
      // (loops and not copies, here and below: instruction fetch is what straight code would wait for)
      float mx = -INFINITY;
#pragma unroll 1
      for (int c = 0; c < 2; ++c) {
        tmem_load32(s_addr + 32 * c, v);
        tmem_load_wait(v);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const float2 kf = *reinterpret_cast<const float2*>(&st[2 * c + s]);
          float t[4];
#pragma unroll
          for (int u = 0; u < 4; ++u) t[u] = max3(__uint_as_float(v[16 * s + 3 * u]), __uint_as_float(v[16 * s + 3 * u + 1]), __uint_as_float(v[16 * s + 3 * u + 2]));
          t[0] = max3(t[0], __uint_as_float(v[16 * s + 12]), __uint_as_float(v[16 * s + 13]));
          t[1] = max3(t[1], __uint_as_float(v[16 * s + 14]), __uint_as_float(v[16 * s + 15]));
          t[0] = fmaxf(max3(t[0], t[1], t[2]), t[3]);
          mx = fmaxf(mx, fmaf(t[0], fmaxf(rs * kf.x, kTiny), kf.y));
        }
      }
      // the row's other half
      peaks[j & 1][i][half][rr] = mx;
      asm volatile("bar.sync %0, %1;" ::"r"(1 + 4 * i + (warp & 3)), "r"(64) : "memory");
      mx = fmaxf(mx, peaks[j & 1][i][half ^ 1][rr]);
      const bool need = mx > m + kTcSlack || (m == -INFINITY && mx > -INFINITY);
      if (__any_sync(0xffffffffu, need)) {
        const float m_new = need ? mx : m, corr = need ? ex2(m - m_new) : 1.f;       // (mx > m there; ex2(-inf) = 0)
        if (j > 0) {
          wait_warp(kODone + i, j - 1, 0);
          tc::tc_fence_after();
#pragma unroll 1
          for (int c = 0; c < HD / 64; ++c) {
            tmem_load32(o_addr + 32 * c, v);
            tmem_load_wait(v);
#pragma unroll
            for (int u = 0; u < 32; ++u) v[u] = __float_as_uint(__uint_as_float(v[u]) * corr);
            tmem_store32(o_addr + 32 * c, v);
          }
          l *= corr;
        }
        m = m_new;
      }
      const float ref = (m == -INFINITY ? 0.f : m) - kTcOffset + poison;
#pragma unroll 1
      for (int c = 0; c < 2; ++c) {
        tmem_load32(s_addr + 32 * c, v);
        tmem_load_wait(v);
        uint32_t p[16];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const float4 x = *reinterpret_cast<const float4*>(&st[2 * c + s]);
          const float f = fmaxf(rs * x.x, kTiny), d = x.y - ref;
          const uint64_t f2 = pair(f, f), d2 = pair(d, d);
          uint64_t sum = 0;
#pragma unroll
          for (int u = 0; u < 16; u += 2) {
            float2 y = unpair(fma2(pair(__uint_as_float(v[16 * s + u]), __uint_as_float(v[16 * s + u + 1])), f2, d2));
            y = make_float2(ex2(y.x), ex2(y.y));
            sum = add2(sum, pair(y.x, y.y));
            p[8 * s + u / 2] = pack_f16(y.x, y.y);
          }
          const float2 t = unpair(sum);
          l = fmaf(x.z, t.x + t.y, l);
        }
        tmem_store16(s_addr + 16 * c, p);                         // over columns that this thread has read
      }
      tmem_store_wait();
      tc::tc_fence_before();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(bar(kPFull + i));
    }
    if (n_kv[i] > 0) wait_warp(kODone + i, n_kv[i] - 1, 20);
    __syncthreads();                                              // (nan_at is complete; see the other warps' ends)
    peaks[0][i][half][rr] = l;
    asm volatile("bar.sync %0, %1;" ::"r"(1 + 4 * i + (warp & 3)), "r"(64) : "memory");
    l = peaks[0][i][0][rr] + peaks[0][i][1][rr];
    tc::tc_fence_after();
    const int d0 = half * (HD / 2);                               // this thread's share of the row's dims
    float* wp = ws + static_cast<int64_t>(blockIdx.x - part.whole) * (2 * kTile * (HD + 2));       // (a share's: sums, maxima, sums of weights)
    const float inv = cut ? 1.f : l == 0.f ? 0.f : 1.0f / l;
    const unsigned at = r0 + r;
    const int64_t mine = cut ? static_cast<int64_t>(r) * HD + d0
                             : (seq.row0 + at / static_cast<unsigned>(G)) * o_stride + (h * G + at % static_cast<unsigned>(G)) * static_cast<int64_t>(HD) + d0;
    // Rows go out through shared memory (all of its tiles are done with), 32 rows of at most 128 bytes per warp: whole
    // lines per store, where a thread that stored its own row would touch 32 lines with each
    const uint32_t stage = base + warp * 4096;
    auto put = [&](int chunk, uint32_t x, uint32_t y, uint32_t z, uint32_t w) { sts16(stage + lane * 128 + ((chunk ^ (lane & 7)) << 4), x, y, z, w); };
    auto flush = [&](auto chunks, auto* to) {                     // `chunks` 16-byte pieces of every row to to[its offset]
      constexpr int kC = decltype(chunks)::value;
      __syncwarp();
#pragma unroll
      for (int k = 0; k < kC; ++k) {
        const int row = k * (32 / kC) + lane / kC, chunk = lane % kC;
        const int64_t off = __shfl_sync(0xffffffffu, mine, row);
        uint32_t x[4];
        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
                     : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3])
                     : "r"(stage + row * 128 + ((chunk ^ (row & 7)) << 4))
                     : "memory");
        if (r - lane + row < n_rows) *reinterpret_cast<uint4*>(reinterpret_cast<unsigned char*>(to + off) + 16 * chunk) = make_uint4(x[0], x[1], x[2], x[3]);
      }
      __syncwarp();
    };
#pragma unroll 1
    for (int c = 0; c < HD / 64; ++c) {
      uint32_t v[32];
      if (n_kv[i] > 0) {
        tmem_load32(o_addr + 32 * c, v);
        tmem_load_wait(v);
      }
#pragma unroll
      for (int u = 0; u < 32; ++u) {
        v[u] = l == 0.f ? 0u : __float_as_uint(__uint_as_float(v[u]) * inv);      // nothing attended to: zeros
        if (rpos >= nan_at[d0 + 32 * c + u]) v[u] = 0x7fffffffu;
      }
      if (cut) {
#pragma unroll
        for (int u = 0; u < 8; ++u) put(u, v[4 * u], v[4 * u + 1], v[4 * u + 2], v[4 * u + 3]);
        flush(std::integral_constant<int, 8>{}, wp + 32 * c);
      } else {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          Vec<T> x;
#pragma unroll
          for (int k = 0; k < 8; ++k) x.x[k] = narrow<T>(__uint_as_float(v[8 * u + k]));
          const uint4 y = *reinterpret_cast<const uint4*>(&x);
          put(4 * c + u, y.x, y.y, y.z, y.w);
        }
      }
    }
    if (!cut) flush(std::integral_constant<int, HD / 16>{}, o);
    if (cut && r < n_rows && half == 0) {
      wp[2 * kTile * HD + r] = m;
      wp[2 * kTile * (HD + 1) + r] = l;
    }
    tc::tc_fence_before();
  } else if (warp < kMmaWarp) {
    // ------------------------------------------------------------------ codes to fp16 operand tiles
    const int w = warp - kSoft, piece = lane % kLanes, row_a = w * (32 / kLanes) + lane / kLanes;
    // (kRowsPass is a multiple of 8: every pass is the same place of the swizzle, kRowsPass rows further)
    static_assert(kRowsPass % 8 == 0 && kRawTokens % kRowsPass == 0, "");
    // (the second block's lanes take their upper 8 codes first: no bank is stored to twice)
    const bool other = (piece & 4) != 0;
    const int half0 = other ? 8 : 0;
    const uint32_t place0 = tile_chunk(0, row_a, 2 * piece + (other ? 1 : 0)), place1 = tile_chunk(0, row_a, 2 * piece + (other ? 0 : 1));
    int raw = 0;
    uint32_t raw_phase = 0;
    // a tile of step j, a slot of the ring after the other
    auto convert = [&](uint32_t tile, int j, bool values) {
      const bool partial = values && p0 + j * kTile + kTile - 1 > lo[0];
#pragma unroll 1
      for (int hf = 0; hf < kTile / kRawTokens; ++hf) {
        if (!wait_warp(kRawFull + raw, raw_phase, 20)) return false;
        const uint32_t src = raw_slot(raw) + row_a * HD + 16 * piece, dst = tile + hf * kRawTokens * 128;
#pragma unroll
        for (int p = 0; p < kRawTokens / kRowsPass; ++p) {
          uint2 x = lds8(src + half0 + p * kRowsPass * HD), y = lds8(src + (8 - half0) + p * kRowsPass * HD);
          if (partial) {
            // 0 * NaN: where rows do not see the whole step a NaN value is taken out, and the rows that do see it are set to NaN
            // at the end
            auto clear = [&](uint32_t& z, int byte0) {
              uint32_t bad = ((z & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
              z &= ~((bad >> 7) * 0xffu);
              while (bad) {
                const int byte = (__ffs(bad) - 1) >> 3;
                bad &= bad - 1;
                atomicMin(nan_at + 16 * piece + byte0 + byte, p0 + j * kTile + hf * kRawTokens + p * kRowsPass + row_a);
              }
            };
            clear(x.x, half0);
            clear(x.y, half0 + 4);
            clear(y.x, 8 - half0);
            clear(y.y, 12 - half0);
          }
          sts16(dst + place0 + p * kRowsPass * 128, decode2(x.x), decode2(x.x >> 16), decode2(x.y), decode2(x.y >> 16));
          sts16(dst + place1 + p * kRowsPass * 128, decode2(y.x), decode2(y.x >> 16), decode2(y.y), decode2(y.y >> 16));
        }
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(bar(kRawEmpty + raw));
        if (++raw == kRawSlots) {
          raw = 0;
          raw_phase ^= 1;
        }
      }
      tc::fence_async_smem();
      __syncwarp();
      return true;
    };
    for (int j = 0; j < n; ++j) {
      const int s = j & 1;
      if (j >= 2 && !wait_warp(kKEmpty + s, (j >> 1) - 1, 20)) break;
      if (!convert(k_tile(s), j, false)) break;
      if (lane == 0) tc::mbar_arrive(bar(kKFull + s));
      if (j >= 2 && !wait_warp(kVEmpty + s, (j >> 1) - 1, 20)) break;
      if (!convert(v_tile(s), j, true)) break;
      if (lane == 0) tc::mbar_arrive(bar(kVFull + s));
    }
    __syncthreads();
  } else if (warp == kLoadWarp) {
    // ------------------------------------------------------------------ codes and scales from global memory
    // Lane s < 8 keeps the page of the s-th 16 positions of a step: the table's entry two steps ahead, its row in the tensor
    // maps (-1: no page) and its scales one step ahead
    // A box of the maps is a page's tokens or 64 of them (32 sequences of 12 tokens at 4096 positions, pages of
    // 32: 158 us, in boxes of 16 163)
    const int box = box_tokens(V), boxes = kRawTokens / box;
    const int32_t* table = V.table + static_cast<int64_t>(b) * V.max_pages;
    auto needed = [&](int j) { return lane < kTile / kStep && (j0 + j) * (kTile / kStep) + lane < n_steps; };
    auto load_entry = [&](int j) { return needed(j) ? __ldg(table + (((j0 + j) * (kTile / kStep) + lane) >> (V.page_shift - 4))) : -1; };
    int entry = load_entry(0), place = -1, raw = 0;
    uint32_t raw_phase = 1;
    float2 sc = make_float2(0.f, 0.f);
    auto take_entry = [&](int j) {
      const bool there = static_cast<uint32_t>(entry) < static_cast<uint64_t>(V.n_pages);
      if (!there && needed(j)) report_page(V);                    // (any value may stand in the table)
      place = there ? ((entry * V.hkv + h) << V.page_shift) + ((p0 + j * kTile + lane * kStep) & ((1 << V.page_shift) - 1)) : -1;
      if (there) sc = __ldg(V.scales + static_cast<int64_t>(entry) * V.hkv + h);
    };
    take_entry(0);
    entry = load_entry(1);
    for (int j = 0; j < n; ++j) {
      bool ok = true;
#pragma unroll 1
      for (int part4 = 0; part4 < 2 * (kTile / kRawTokens) && ok; ++part4) {      // keys, keys, values, values
        if (!(ok = wait_warp(kRawEmpty + raw, raw_phase, 20))) break;
        if (part4 == 0) {                                         // (the readers of step j - 4's scales are done: see the ring's bound)
          if (lane < kTile / kStep) {
            const int ev = scale_exponent(sc.y);
            meta[j & 3][lane] = place >= 0 ? Step{exp2_int(scale_exponent(sc.x)), static_cast<float>(ev), exp2_int(-ev), 0.f} : Step{1.f, -INFINITY, 0.f, 0.f};
          }
          __syncwarp();
          if (lane == 0) tc::mbar_arrive(bar(kMeta + (j & 3)));
        }
        const bool values = part4 >= kTile / kRawTokens;
        const int row = __shfl_sync(0xffffffffu, place, part4 % (kTile / kRawTokens) * (kRawTokens / kStep) + (lane % boxes) * (box / kStep));
        const unsigned live = __ballot_sync(0xffffffffu, lane < boxes && row >= 0);
        if (live != (1u << boxes) - 1) {                          // positions without a page (or in a box behind the last) are zeros
          for (int i = lane; i < kRawTokens * HD / 16; i += 32) sts16(raw_slot(raw) + 16 * i, 0u, 0u, 0u, 0u);
          tc::fence_async_smem();
          __syncwarp();
        }
        if (lane == 0) tc::mbar_expect_tx(bar(kRawFull + raw), __popc(live) * box * HD);
        __syncwarp();
        if (lane < boxes && row >= 0) tc::tma_load_2d(raw_slot(raw) + lane * box * HD, values ? &map_v : &map_k, 0, row, bar(kRawFull + raw));
        if (++raw == kRawSlots) {
          raw = 0;
          raw_phase ^= 1;
        }
      }
      if (!ok) break;
      take_entry(j + 1);
      entry = load_entry(j + 2);
    }
    __syncthreads();
  } else {
    // ------------------------------------------------------------------ one thread issues the products
    // (elected and not lane 0: the compiler then knows that one thread is left, and issues in half the instructions)
    uint32_t elected;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(elected));
    if (elected && n > 0) {
      constexpr uint32_t kIdS = make_idesc_f16(kTile, kTile, false), kIdO = make_idesc_f16(kTile, HD, true);
      auto scores = [&](int i, int s) {
        const uint64_t a = tc::make_desc_sw128(q_tile(i)), bd = tc::make_desc_sw128(k_tile(s));
#pragma unroll
        for (int k = 0; k < HD / 16; ++k) {
          const int off = ((k >> 2) * (kTile * 128) + (k & 3) * 32) >> 4;
          mma_ss(tmem + i * kTile, a + off, bd + off, kIdS, k > 0);
        }
        mma_commit(bar(kSFull + i));
      };
      auto values = [&](int i, int s, int j) {
        const uint64_t bd = make_desc_rows_contracted(v_tile(s));
#pragma unroll
        for (int k = 0; k < kTile / 16; ++k)
          mma_ts(tmem + 2 * kTile + i * kTile, tmem + i * kTile + (k >> 2) * (kTile / 2) + 8 * (k & 3), bd + (k * 2048 >> 4), kIdO, j > 0 || k > 0);
        mma_commit(bar(kODone + i));
      };
      bool ok = wait(kQFull, 0, 0) && wait(kKFull, 0, 0);
      if (ok) {
        tc::tc_fence_after();
        if (n_kv[0] > 0) scores(0, 0);
        if (n_kv[1] > 0) scores(1, 0);
        mma_commit(bar(kKEmpty));
      }
      for (int j = 0; j < n && ok; ++j) {
        const int s = j & 1, s1 = s ^ 1;
        if (j + 1 < n && !(ok = wait(kKFull + s1, (j + 1) >> 1, 0))) break;
        if (!(ok = wait(kVFull + s, j >> 1, 0))) break;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if (j < n_kv[i]) {
            if (!(ok = wait(kPFull + i, j, 0))) break;
            tc::tc_fence_after();
            values(i, s, j);
          }
          if (i == 1) mma_commit(bar(kVEmpty + s));
          if (j + 1 < n_kv[i]) scores(i, s1);
          if (i == 1 && j + 1 < n) mma_commit(bar(kKEmpty + s1));
        }
      }
      mma_commit(bar(kDrain));                                    // nothing is in flight when the TMEM goes
      wait(kDrain, 0, 20);
    }
    __syncwarp();
    __syncthreads();
  }
  __syncthreads();
  if (warp == kMmaWarp) {
    tc::tc_fence_after();
    tmem_dealloc(tmem, kTmemCols);
  }
}

}  // namespace

// The blocks of the last, partial round of SMs (all, where there are fewer than SMs) are cut along the positions as far as
// SMs are idle: into shares of 2 steps of 128 positions at least (of what the page table could hold) where there is no full
// round (1 sequence of 1024 positions, 256 rows per head, 8 heads: 23 us, uncut 32; 65536 positions in 16 shares 106 us, in 8
// 177, uncut 1145), of 8 steps behind full ones (8 sequences of 1024, 512 blocks: cut 127 us, uncut 117).
struct TcCut {
  int64_t tiles, items, whole;
  int nsplit;
};
static TcCut tc_plan(const View& V, int H) {
  TcCut p;
  p.tiles = ceil_div(static_cast<int64_t>(V.max_new) * (H / V.hkv), 2 * kTile);
  p.items = p.tiles * V.batch * V.hkv;
  const int64_t tail = p.items % 148, steps = (static_cast<int64_t>(V.max_pages) << V.page_shift) / kTile;
  p.nsplit = 1;
  while (p.nsplit < 16 && tail > 0 && tail * (p.nsplit + 1) <= 148 && steps >= (p.items < 148 ? 2 : 8) * (p.nsplit + 1)) ++p.nsplit;
  p.whole = p.nsplit > 1 ? p.items - tail : p.items;
  return p;
}

size_t workspace_bytes_tc(const View& V, int H, int hd) {
  const TcCut p = tc_plan(V, H);
  return static_cast<size_t>(p.items - p.whole) * p.nsplit * 2 * kTile * (hd + 2) * sizeof(float);
}

template <typename T, int HD>
szo_status launch_attention_tc(const View& V, const Rows& A, float* ws, cudaStream_t st) {
  const TcCut p = tc_plan(V, A.H);
  SZO_REQUIRE(p.items <= 0x7fffffff, SZO_ERR_SHAPE, "too many rows, heads and sequences for one launch");
  const int smem = 6 * kTile * HD * 2 + kRawSlots * kRawTokens * HD + 1024;
  CUtensorMap map_k, map_v;
  const int64_t rows = (V.n_pages * V.hkv) << V.page_shift;
  SZO_TRY(encode_map_2d(&map_k, CU_TENSOR_MAP_DATA_TYPE_UINT8, V.k, rows, HD, 1, box_tokens(V), HD, CU_TENSOR_MAP_SWIZZLE_NONE));
  SZO_TRY(encode_map_2d(&map_v, CU_TENSOR_MAP_DATA_TYPE_UINT8, V.v, rows, HD, 1, box_tokens(V), HD, CU_TENSOR_MAP_SWIZZLE_NONE));
  auto kern = kv8_attention_tc_kernel<T, HD>;
  SZO_CHECK_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  const unsigned blocks = static_cast<unsigned>(p.whole + (p.items - p.whole) * p.nsplit);
  kern<<<blocks, kTcThreads, smem, st>>>(map_k, map_v, V, static_cast<const T*>(A.q), A.q_stride, static_cast<T*>(A.o), A.o_stride, A.H, A.scale,
                                         static_cast<int>(p.tiles), TcSplit{static_cast<unsigned>(p.whole), p.nsplit}, ws);
  count_launch();
  SZO_CHECK_LAUNCH("kv8_attention_tc_kernel");
  if (p.whole == p.items) return SZO_OK;
  return launch_join<T, HD>(V, A, ws, 2 * kTile, static_cast<int>(p.tiles), p.nsplit, true, p.whole, p.items - p.whole, st);
}
template szo_status launch_attention_tc<__nv_bfloat16, 64>(const View&, const Rows&, float*, cudaStream_t);
template szo_status launch_attention_tc<__nv_bfloat16, 128>(const View&, const Rows&, float*, cudaStream_t);
template szo_status launch_attention_tc<__half, 64>(const View&, const Rows&, float*, cudaStream_t);
template szo_status launch_attention_tc<__half, 128>(const View&, const Rows&, float*, cudaStream_t);

}  // namespace kv8
}  // namespace szo
