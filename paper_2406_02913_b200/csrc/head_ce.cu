// Next-token cross entropy straight from hidden states, and its gradient: the logits x = scale * h W^T of a tile are
// formed, used and dropped.
//
// Forward: every (row, tile of the vocabulary) leaves (m, s): m the tile's largest logit and s = sum 2^(x - m) over it in base 2,
// WITHOUT the target's own term, which is kept apart.  Joined over the tiles with S and M,
//   lse = M + log2(S + 2^(x_t - M)),   loss = log(1 + S 2^(M - x_t)):
// loss does not come from the difference of two numbers of the size of lse, so a confident row's keeps its relative precision.
// Backward: G = scale ((a + b) p - a 1[t]) (a = d_loss, b = d_lse), p = 2^(x - lse), for a piece of the vocabulary at a time, in the
// 16-bit type of the products that follow; p - 1 of the target is formed before the rounding.
#include <cmath>

#include "head_ce.cuh"
#include "tc_common.cuh"

namespace szo {
namespace head {

namespace {

constexpr int kNoExponent = static_cast<int>(0x80808080u);       // (below every exponent)
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

template <typename T> __device__ __forceinline__ float widen(T x);
template <> __device__ __forceinline__ float widen<__half>(__half x) { return __half2float(x); }
template <> __device__ __forceinline__ float widen<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T narrow(float x);
template <> __device__ __forceinline__ __half narrow<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// Joins a row's parts: kRows rows per block, 256 / kRows threads over the parts of each, joined in their order.  (Few rows: a
// block each, or a thread's chain of loads is what it waits for: 8 rows of 1000 parts 16 us with 32 rows per block.)
template <int kRows>
__global__ void __launch_bounds__(256) head_join_kernel(const float2* __restrict__ part, const float* __restrict__ xt, const int32_t* __restrict__ targets,
                                                        int64_t rows, int64_t vocab, int parts, float* __restrict__ loss, float* __restrict__ lse,
                                                        int32_t* status) {
  constexpr int kLanes = 256 / kRows;                             // threads of a row
  __shared__ float ms[8][kRows], ss[8][kRows];
  chain_release();
  chain_wait();
  const int lane = threadIdx.x % kRows, w = threadIdx.x / kRows, warp = threadIdx.x / 32;
  const int64_t r = static_cast<int64_t>(blockIdx.x) * kRows + lane;
  const bool there = r < rows;
  const float2* p = part + (there ? r : rows - 1);
  float m = -INFINITY, s = 0.f;
#pragma unroll 8
  for (int i = w; i < parts; i += kLanes) m = fmaxf(m, p[i * rows].x);
#pragma unroll
  for (int o = kRows; o < 32; o *= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (threadIdx.x % 32 < kRows) ms[warp][lane] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, ms[i][lane]);
  const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll 8
  for (int i = w; i < parts; i += kLanes) {
    const float2 x = p[i * rows];
    s += x.y * exp2f(x.x - ref);
  }
#pragma unroll
  for (int o = kRows; o < 32; o *= 2) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (threadIdx.x % 32 < kRows) ss[warp][lane] = s;
  __syncthreads();
  if (threadIdx.x >= kRows || !there) return;
  s = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) s += ss[i][lane];
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
    // (the target as far below everything as all else is: lse - x is the difference of two infinities)
    if (isnan(total) || top == -INFINITY) out = __int_as_float(0x7fffffff);
  }
  if (isnan(total) || total == INFINITY) {
    total = __int_as_float(0x7fffffff);
    if (t >= 0) out = total;                                      // (a row without a target may hold anything: no loss)
  }
  loss[r] = out;
  if (lse != nullptr) lse[r] = total;
}

// What the gradient needs of a row: x = lse in base 2, y = weight of p, z = weight of the target (both times scale and, for fp16, a
// power of two that brings the larger to [2^13, 2^14)), w = that power's inverse.  Rows that weigh nothing have y = z = 0.
struct RowArgs {
  const int32_t* targets;
  const float *lse, *d_loss, *d_lse;
  int64_t rows, vocab;
  float scale;
};
template <typename T> constexpr bool kIsHalf = std::is_same<T, __half>::value;
template <typename T> __device__ __forceinline__ float4 row_info(const RowArgs& A, int64_t r, int* exponent) {
  const int32_t t = A.targets[r];
  const float d = A.d_loss[r], b = A.d_lse != nullptr ? A.d_lse[r] : 0.f, l = A.lse[r], a = t >= 0 && t < A.vocab ? d : 0.f;
  float y = A.scale * (a + b), z = A.scale * a, inv = 1.f;
  *exponent = kNoExponent;
  if (l == -INFINITY) y = z = 0.f;
  if (kIsHalf<T> && (y != 0.f || z != 0.f)) {
    const float top = fmaxf(fmaxf(fabsf(y), fabsf(z)), fabsf(A.scale * b));
    const int e = min(max(((__float_as_int(top) >> 23) & 255) - 127, -100), 100);      // (rows beyond: as near as it goes)
    const float f = __int_as_float((13 - e + 127) << 23);
    y *= f;
    z *= f;
    inv = __int_as_float((e - 13 + 127) << 23);
    *exponent = e;
  }
  return make_float4(l * kLog2e, y, z, inv);
}
// The largest exponent of all rows, in every thread of the block
template <typename T> __device__ __forceinline__ int largest_exponent(const RowArgs& A) {
  __shared__ int tops[32];
  int most = kNoExponent;
#pragma unroll 4
  for (int64_t r = threadIdx.x; r < A.rows; r += blockDim.x) {
    int e;
    row_info<T>(A, r, &e);
    most = max(most, e);
  }
  most = __reduce_max_sync(0xffffffffu, most);
  if (threadIdx.x % 32 == 0) tops[threadIdx.x / 32] = most;
  __syncthreads();
  most = tops[0];
  for (int i = 1; i < static_cast<int>(blockDim.x) / 32; ++i) most = max(most, tops[i]);
  return most;
}
// Up to this many rows every block of the next kernel looks for the largest itself; more are looked at once, before it
constexpr int64_t kScanRows = 2048;
template <typename T> __global__ void __launch_bounds__(1024) head_exponent_kernel(RowArgs A, int32_t* __restrict__ exponent) {
  chain_release();
  chain_wait();
  const int most = largest_exponent<T>(A);
  if (threadIdx.x == 0) *exponent = most;
}
// Rows' infos, zeroed counters and, for dW (`copy`), h with rows that weigh nothing as zeros and fp16 rows brought to the largest weight
// (exactly but for what falls below fp16's range): eight elements per thread
template <typename T>
__global__ void __launch_bounds__(256) head_prepare_kernel(RowArgs A, const T* __restrict__ h, int64_t h_stride, int64_t d, float4* __restrict__ info,
                                                           int32_t* __restrict__ exponent, T* __restrict__ copy, int32_t* __restrict__ counters,
                                                           int64_t n_counters) {
  chain_release();
  chain_wait();
  if (blockIdx.x == 0)
    for (int64_t i = threadIdx.x; i < n_counters; i += blockDim.x) counters[i] = 0;
  int most = kNoExponent;
  if (kIsHalf<T> && copy != nullptr) {
    if (A.rows <= kScanRows) {
      most = largest_exponent<T>(A);
      if (blockIdx.x == 0 && threadIdx.x == 0) *exponent = most;
    } else {
      most = *exponent;
    }
  }
  const int64_t per = copy != nullptr ? d / 8 : 1, i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
  if (i >= A.rows * per) return;
  const int64_t r = i / per, c = i % per * 8;
  int e;
  const float4 f = row_info<T>(A, r, &e);
  if (c == 0) info[r] = f;
  if (copy == nullptr) return;
  uint4 x = make_uint4(0u, 0u, 0u, 0u);
  if (f.y != 0.f || f.z != 0.f) {
    x = *reinterpret_cast<const uint4*>(h + r * h_stride + c);
    if constexpr (kIsHalf<T>) {
      const float to = f.w * __int_as_float((13 - most + 127) << 23);
      T* el = reinterpret_cast<T*>(&x);
#pragma unroll
      for (int k = 0; k < 8; ++k) el[k] = narrow<T>(widen<T>(el[k]) * to);
    }
  }
  *reinterpret_cast<uint4*>(copy + r * d + c) = x;
}

// dh: the sums of a row (of `parts` parts, in their order) times its power of two, rounded
template <typename T>
__global__ void head_round_kernel(const float* __restrict__ acc, int parts, int64_t rows, int64_t d, const float4* __restrict__ info,
                                  T* __restrict__ out, int64_t stride) {
  chain_release();
  chain_wait();
  const int64_t per = d / 8, i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
  if (i >= rows * per) return;
  const int64_t r = i / per, c = i % per * 8;
  const float4 of = info[r];
  const float f = of.w;
  float x[8] = {};
  if (of.y == 0.f && of.z == 0.f) parts = 0;                      // a row that weighs nothing: zeros, whatever W holds
  for (int p = 0; p < parts; ++p) {
    const float4* from = reinterpret_cast<const float4*>(acc + (p * rows + r) * d + c);
    const float4 lo = from[0], hi = from[1];
    x[0] += lo.x, x[1] += lo.y, x[2] += lo.z, x[3] += lo.w, x[4] += hi.x, x[5] += hi.y, x[6] += hi.z, x[7] += hi.w;
  }
  alignas(16) T y[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) y[k] = narrow<T>(x[k] * f);
  *reinterpret_cast<uint4*>(out + r * stride + c) = *reinterpret_cast<const uint4*>(y);
}

// ------------------------------------------------------------------------------ host side
struct Shape {
  int64_t rows, vocab, d;
};
struct Plan {
  size_t part, xt;                                                // of a workspace, in bytes from its start
  size_t info, exponent, counters, copy, G, acc;
  size_t total;
  int parts;                                                      // forward: of the vocabulary
  int64_t piece;                                                  // vocabulary entries of a piece of G
  int pieces, buffers;
  int dh_parts, sums;                                             // shares of dh's sum over a piece; sums kept apart in all
};
struct Taker {
  size_t at = 0;
  size_t operator()(size_t bytes) {
    const size_t from = at;
    at += round_up(bytes, 256);
    return from;
  }
};
int tiles_of(int64_t n) { return static_cast<int>(ceil_div(n, kTile)); }
constexpr int kPairs = 74;                                        // (of a B200; the rules below only lose balance on another number)
// Up to this many rows of hidden states are the columns of a product, and not its rows: at 128 both ways take as long
constexpr int64_t kFewRows = 128;
bool few(int64_t rows) { return rows <= kFewRows; }
// Height of tiles over n vocabulary entries that gives every pair of SMs the same share
int step_of(int64_t n) {
  const int64_t rounds = ceil_div(tiles_of(n), kPairs);
  return static_cast<int>(round_up(static_cast<size_t>(ceil_div(n, rounds * kPairs)), 16));
}
Plan forward_plan(const Shape& s) {
  Plan p = {};
  Taker take;
  const int step = step_of(s.vocab);
  p.parts = few(s.rows) ? static_cast<int>(ceil_div(s.vocab, step) * 2 * ceil_div(step / 2, 32)) : 2 * tiles_of(s.vocab);
  p.part = take(static_cast<size_t>(p.parts) * s.rows * sizeof(float2));
  p.xt = take(static_cast<size_t>(s.rows) * sizeof(float));
  p.total = take.at;
  return p;
}
// Gradient.  G of a piece is about 64 MB (half of L2), and a piece 4096 to 65536 entries: so up to 8192 rows three pieces' G stay below 200 MB, and
// more rows take 24 KB each (32768 x 32000 x 4096, both gradients: least pieces of 2048 entries 24.0 ms, 4096 22.7, 8192 23.9: dh's sums are
// written and read once per piece).  Many rows: one launch for all pieces, dh and dW
// following G a piece behind (of 256 units of logits at least, more than three for every pair of SMs), so that hardly a unit waits for one that
// runs beside it, and no SM for the end of a piece (4096 rows of 32000 x 4096 in a launch per piece 1614 us, in one 1476); the sums of dh are kept in one place, piece after piece.  Few rows: a launch per
// piece, since units that wait for others cost more than the end of a launch there (16 rows of 32000 x 4096 84 us, in one launch
// 107, with dh so close behind G that it finds W in L2); the sums of the pieces are kept apart.
constexpr int64_t kLeastPiece = 4096;
Plan backward_plan(const Shape& s, bool dh, bool dw) {
  Plan p = {};
  Taker take;
  const bool is_few = few(s.rows);
  int64_t piece = (int64_t(64) << 20) / (2 * s.rows);
  piece = piece < kLeastPiece ? kLeastPiece : piece > 65536 ? 65536 : piece;
  if (piece > s.vocab) piece = s.vocab;
  p.piece = static_cast<int64_t>(round_up(static_cast<size_t>(piece), kTile));
  p.pieces = static_cast<int>(ceil_div(s.vocab, p.piece));
  p.buffers = p.pieces < 3 ? p.pieces : 3;                        // (written, read, and the one whose last readers may still run)
  p.info = take(static_cast<size_t>(s.rows) * sizeof(float4));
  p.exponent = take(sizeof(int32_t));
  p.counters = take(static_cast<size_t>(counters_of(p.pieces)) * sizeof(int32_t));
  if (dw) p.copy = take(static_cast<size_t>(s.rows) * s.d * 2);
  p.G = take(static_cast<size_t>(s.rows) * p.piece * p.buffers * 2);
  // few tiles of dh: its sums over a piece are cut so that the rounds of tiles over the pairs of SMs are as full as they get, in shares of
  // 8 blocks of 64 at least
  p.dh_parts = 1;
  const int64_t tiles = static_cast<int64_t>(is_few ? p.pieces : tiles_of(s.rows)) * tiles_of(s.d), nkb = p.piece / kBlockK;
  double best = 1e30;
  for (int n = 1; n <= 16 && nkb >= 8 * n && (n == 1 || tiles * n <= 2 * kPairs); ++n) {
    const double cost = static_cast<double>(ceil_div(tiles * n, kPairs)) * (static_cast<double>(nkb) / n + 8);      // (a unit's fixed part: about 8 blocks)
    if (cost < best * 0.98) {
      best = cost;
      p.dh_parts = n;
    }
  }
  const int64_t last = ceil_div(s.vocab - (p.pieces - 1) * p.piece, kBlockK);
  p.sums = is_few ? (p.pieces - 1) * p.dh_parts + static_cast<int>(last < p.dh_parts ? last : p.dh_parts)
                  : static_cast<int>(p.pieces > 1 || last >= p.dh_parts ? p.dh_parts : last);
  if (dh) p.acc = take(static_cast<size_t>(p.sums) * s.rows * s.d * sizeof(float));
  p.total = take.at;
  return p;
}
// dh alone of more rows, where G is more than the pieces that are kept: up to 8192 of them at a time, in equal shares, which bounds the workspace
// (65536 x 32000 x 4096: 320 MB and 29.0 ms, at once 2.5 GB and 31.4)
int64_t rows_at_once(const Shape& s, bool dw) {
  constexpr int64_t kMost = 8192;
  if (dw || s.rows <= kMost || s.vocab <= 3 * kLeastPiece) return s.rows;
  return static_cast<int64_t>(round_up(static_cast<size_t>(ceil_div(s.rows, ceil_div(s.rows, kMost))), kTile));
}
bool fits(int64_t rows, int64_t vocab, int64_t d) {
  constexpr int64_t kMost = 0x7fffff00, kTiles = 1 << 25;        // (tiles of a product, and blocks of a launch, are counted in 32 bits)
  if (rows < 0 || vocab <= 0 || d <= 0 || d % 8 != 0 || rows > kMost || vocab > kMost || d > kMost) return false;
  const int64_t m = ceil_div(rows, kTile), n = ceil_div(vocab, kTile), k = ceil_div(d, kTile);
  return m * n <= kTiles && m * k <= kTiles && n * k <= kTiles;
}
szo_status check(const void* h, int64_t h_stride, const void* W, int64_t w_stride, szo_dtype dtype, int64_t rows, int64_t vocab, int64_t d,
                 float scale, const int32_t* targets) {
  SZO_REQUIRE(dtype == SZO_BF16 || dtype == SZO_F16, SZO_ERR_UNSUPPORTED, "dtype must be bf16 or f16");
  SZO_REQUIRE(fits(rows, vocab, d), SZO_ERR_SHAPE, "rows >= 0, vocab > 0 and d a positive multiple of 8, below 2^31 - 256, and each two of them below 2^25 tiles of 256 x 256");
  SZO_REQUIRE(std::isfinite(scale) && scale >= 1e-30f && scale <= 1e30f, SZO_ERR_INVALID_ARG, "scale must be in [1e-30, 1e30]");
  SZO_REQUIRE(W != nullptr && (rows == 0 || (h != nullptr && targets != nullptr)), SZO_ERR_INVALID_ARG, "NULL h, W or targets");
  SZO_REQUIRE(h_stride >= d && w_stride >= d, SZO_ERR_SHAPE, "row strides must be at least d");
  SZO_REQUIRE(aligned16(h) && aligned16(W) && aligned16(targets) && h_stride % 8 == 0 && w_stride % 8 == 0, SZO_ERR_ALIGNMENT,
              "buffers and rows must be 16-byte aligned");
  return SZO_OK;
}
unsigned blocks_of(int64_t n, int per) { return static_cast<unsigned>(ceil_div(n, per)); }

template <typename T> constexpr CUtensorMapDataType kMapType =
    std::is_same<T, __nv_bfloat16>::value ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
// A 16-bit matrix in boxes of 64 elements of `rows_box` rows
template <typename T>
szo_status matrix_map(CUtensorMap* map, const T* base, int64_t rows, int64_t cols, int64_t stride, int rows_box) {
  const uint64_t dims[2] = {static_cast<uint64_t>(cols), static_cast<uint64_t>(rows)}, strides[1] = {static_cast<uint64_t>(stride) * 2};
  const uint32_t box[2] = {64, static_cast<uint32_t>(rows_box)};
  return encode_map(map, kMapType<T>, base, 2, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}
// Operands.  `rows_box`: rows that a CTA brings per stage where they are not contracted (64 of them, twice 64 elements, where they are)
template <typename T>
szo_status operand_a(Job* j, const T* base, int64_t rows, int64_t cols, int64_t stride, bool mn, Offset from, int rows_box) {
  j->a_mn = mn;
  j->a_from = from;
  j->a_bytes = (mn ? 128 : rows_box) * kBlockK * 2;
  return matrix_map(&j->a, base, rows, cols, stride, mn ? 64 : rows_box);
}
template <typename T>
szo_status operand_b(Job* j, const T* base, int64_t rows, int64_t cols, int64_t stride, bool mn, Offset from, int rows_box) {
  j->b_mn = mn;
  j->b_from = from;
  j->b_bytes = (mn ? 128 : rows_box) * kBlockK * 2;
  return matrix_map(&j->b, base, rows, cols, stride, mn ? 64 : rows_box);
}
// The product's extent: m, n or k (vocab_dim 0, 1, 2) is the piece of the vocabulary, `piece` entries, `last` in the last one
void sizes(Job* j, Kind kind, int vocab_dim, int64_t m, int64_t n, int64_t k, int64_t piece, int64_t last, int parts = 1, int m_step = kTile,
           int n_step = kTile) {
  j->kind = kind;
  j->vocab_dim = vocab_dim;
  j->keep_from = -1;
  j->m_limit = static_cast<int>(m);
  j->m_step = m_step;
  j->n_step = n_step;
  auto extent = [&](int64_t v) {
    Extent e;
    e.m_tiles = static_cast<int>(ceil_div(vocab_dim == 0 ? v : m, m_step));
    e.n_tiles = static_cast<int>(ceil_div(vocab_dim == 1 ? v : n, n_step));
    e.nkb = static_cast<int>(ceil_div(vocab_dim == 2 ? v : k, kBlockK));
    e.parts = parts < e.nkb ? parts : e.nkb;
    e.units = e.m_tiles * e.n_tiles * e.parts;
    return e;
  };
  j->full = extent(piece);
  j->last = extent(last);
}
// Tiles of m in equal bands whose part of A (16-bit) is at most 48 MB: it stays in L2 while B goes by (loss in bands / in one: 8192 rows of
// 32000 x 4096 1.30 / 1.39 ms, 16384 2.8 to 3.0 / 3.7 to 3.8, 8192 of 50272 x 8192 5.1 / 5.9)
int band_of(int64_t m, int64_t k) {
  const int64_t tiles = tiles_of(m), most = (int64_t(48) << 20) / (kTile * k * 2);
  if (tiles <= most || most < 1) return 0;
  return static_cast<int>(ceil_div(tiles, ceil_div(tiles, most)));
}

template <typename T> struct Inputs {
  const T* h;
  int64_t hs;
  const T* W;
  int64_t ws;
  float scale;
  const int32_t* targets;
};

// The logits' product over a piece of the vocabulary; few rows: in tiles of `step` vocabulary entries
template <typename T> szo_status logits_job(Job* j, const Shape& s, const Inputs<T>& in, int64_t piece, int64_t last, int step, Kind kind, Kind kind_few) {
  if (few(s.rows)) {
    const int cols = static_cast<int>(round_up(s.rows, 32));
    SZO_TRY(operand_a(j, in.W, s.vocab, s.d, in.ws, false, kVocab, step / 2));
    SZO_TRY(operand_b(j, in.h, s.rows, s.d, in.hs, false, kNone, cols / 2));
    sizes(j, kind_few, 0, 0, s.rows, s.d, piece, last, 1, step, cols);
    return SZO_OK;
  }
  SZO_TRY(operand_a(j, in.h, s.rows, s.d, in.hs, false, kNone, 128));
  SZO_TRY(operand_b(j, in.W, s.vocab, s.d, in.ws, false, kVocab, 128));
  sizes(j, kind, 1, s.rows, 0, s.d, piece, last);
  j->m_band = band_of(s.rows, s.d);
  return SZO_OK;
}
Jobs no_jobs() {
  Jobs P = {};
  for (Job& j : P.job) j.kind = -1;
  P.pieces = P.buffers = 1;
  return P;
}

template <typename T>
szo_status forward(const Shape& s, const Inputs<T>& in, float* loss, float* lse, unsigned char* ws, int32_t* status, cudaStream_t st) {
  const Plan p = forward_plan(s);
  Jobs P = no_jobs();
  SZO_TRY(logits_job(&P.job[0], s, in, s.vocab, s.vocab, step_of(s.vocab), kStats, kStatsT));
  P.vocab = P.piece = static_cast<int>(s.vocab);
  P.units = P.job[0].last.units;
  P.targets = in.targets;
  P.part = reinterpret_cast<float2*>(ws + p.part);
  P.xt = reinterpret_cast<float*>(ws + p.xt);
  P.rows = s.rows;
  P.c = in.scale * kLog2e;
  P.status = status;
  SZO_TRY(launch_jobs<T>(P, few(s.rows), true, st));
  auto join = [&](auto kern, int rows) {
    return launch_maybe_chained(kern, dim3(blocks_of(s.rows, rows)), dim3(256), 0, st, true, P.part, P.xt, in.targets, s.rows, s.vocab, p.parts, loss, lse,
                                status);
  };
  SZO_CHECK_CUDA(s.rows <= 512 ? join(head_join_kernel<1>, 1) : join(head_join_kernel<8>, 8));
  count_launch();
  return SZO_OK;
}

template <typename T>
szo_status backward(const Shape& s, const Inputs<T>& in, const float* lse, const float* d_loss, const float* d_lse, T* dh, int64_t dhs, T* dw, int64_t dws,
                    unsigned char* ws, int32_t* status, cudaStream_t st) {
  const Plan p = backward_plan(s, dh != nullptr, dw != nullptr);
  float4* info = reinterpret_cast<float4*>(ws + p.info);
  int32_t *exponent = reinterpret_cast<int32_t*>(ws + p.exponent), *counters = reinterpret_cast<int32_t*>(ws + p.counters);
  T *copy = dw != nullptr ? reinterpret_cast<T*>(ws + p.copy) : nullptr, *G = reinterpret_cast<T*>(ws + p.G);
  float* acc = reinterpret_cast<float*>(ws + p.acc);
  const RowArgs rows{in.targets, lse, d_loss, d_lse, s.rows, s.vocab, in.scale};
  const bool scan = kIsHalf<T> && dw != nullptr && s.rows > kScanRows;
  if (scan) {
    SZO_CHECK_CUDA(launch_maybe_chained(head_exponent_kernel<T>, dim3(1), dim3(1024), 0, st, true, rows, exponent));
    count_launch();
  }
  const unsigned vec_blocks = blocks_of(s.rows * (s.d / 8), 256);
  SZO_CHECK_CUDA(launch_maybe_chained(head_prepare_kernel<T>, dim3(dw != nullptr ? vec_blocks : blocks_of(s.rows, 256)), dim3(256), 0, st, true, rows, in.h,
                                      in.hs, s.d, info, exponent, copy, counters, counters_of(p.pieces)));
  count_launch();

  Jobs P = no_jobs();
  P.vocab = static_cast<int>(s.vocab);
  P.piece = static_cast<int>(p.piece);
  P.pieces = p.pieces;
  P.buffers = p.buffers;
  P.targets = in.targets;
  P.info = info;
  P.exponent = exponent;
  P.rows = s.rows;
  P.c = in.scale * kLog2e;
  P.G = G;
  P.g_stride = p.piece * p.buffers;
  P.sums = acc;
  P.d = static_cast<int>(s.d);
  P.status = status;
  const int64_t last = s.vocab - (p.pieces - 1) * p.piece;
  // (G is contracted in blocks of 64: it ends on one)
  SZO_TRY(logits_job(&P.job[0], s, in, p.piece, static_cast<int64_t>(round_up(static_cast<size_t>(last), kBlockK)), step_of(p.piece), kGrad, kGradT));
  if (!few(s.rows)) SZO_TRY(matrix_map(&P.job[0].out, G, s.rows, P.g_stride, P.g_stride, 32));
  if (dh != nullptr) {
    Job& j = P.job[1];
    if (few(s.rows)) {
      const int cols = static_cast<int>(round_up(s.rows, 32));
      SZO_TRY(operand_a(&j, in.W, s.vocab, s.d, in.ws, true, kVocab, 0));
      SZO_TRY(operand_b(&j, G, s.rows, P.g_stride, P.g_stride, false, kBuffer, cols / 2));
      sizes(&j, kSumT, 2, s.d, s.rows, 0, p.piece, last, p.dh_parts, kTile, cols);
    } else {
      SZO_TRY(operand_a(&j, G, s.rows, P.g_stride, P.g_stride, false, kBuffer, 128));
      SZO_TRY(operand_b(&j, in.W, s.vocab, s.d, in.ws, true, kVocab, 0));
      const uint64_t dims[3] = {static_cast<uint64_t>(s.d), static_cast<uint64_t>(s.rows), static_cast<uint64_t>(p.sums)};
      const uint64_t strides[2] = {static_cast<uint64_t>(s.d) * 4, static_cast<uint64_t>(s.rows) * s.d * 4};
      const uint32_t box[3] = {32, 32, 1};
      SZO_TRY(encode_map(&j.out, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, acc, 3, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B));
      sizes(&j, kSum, 2, s.rows, s.d, 0, p.piece, last, p.dh_parts);
    }
  }
  if (dw != nullptr) {
    Job& j = P.job[2];
    SZO_TRY(operand_a(&j, G, s.rows, P.g_stride, P.g_stride, true, kBuffer, 0));
    SZO_TRY(operand_b(&j, copy, s.rows, s.d, s.d, true, kNone, 0));
    SZO_TRY(matrix_map(&j.out, dw, s.vocab, s.d, dws, 32));
    sizes(&j, kOut, 0, 0, s.d, s.rows, p.piece, last);
  }
  auto units = [&](int job, int i) -> int64_t {
    const Job& j = P.job[job];
    return j.kind < 0 || i < 0 || i >= p.pieces ? 0 : i == p.pieces - 1 ? j.last.units : j.full.units;
  };
  // Few rows read W twice: where it is larger than that, its last 64 MB are kept in L2 (126 MB) for dh, the rest goes by (16 rows of 32000 x
  // 4096: 89 us without, 84 with 40 to 80 MB, 86 with 100)
  constexpr int64_t kKept = int64_t(64) << 20;
  if (few(s.rows) && dh != nullptr && s.vocab * s.d * 2 > kKept) {
    P.job[0].keep_from = static_cast<int>(s.vocab - kKept / (s.d * 2));
    P.job[1].keep_from = 0;
  }
  const int steps = p.pieces + 1;
  int64_t all = 0;                                                // (below 2^31: see fits)
  for (int i = 0; i < steps; ++i) {
    const int64_t n = units(0, i) + units(1, i - 1) + units(2, i - 1);
    if (few(s.rows)) {
      P.step = i;
      P.units = static_cast<int>(n);
      P.idle = 0;
      for (int k = 0; k < 3; ++k) P.idle |= units(k, k == 0 ? i : i - 1) == 0 ? 1 << k : 0;
      SZO_TRY(launch_jobs<T>(P, true, true, st));
    }
    all += n;
  }
  if (!few(s.rows)) {
    P.counters = counters;
    P.units = static_cast<int>(all);
    SZO_TRY(launch_jobs<T>(P, false, true, st));
  }
  if (dh != nullptr) {
    SZO_CHECK_CUDA(launch_maybe_chained(head_round_kernel<T>, dim3(vec_blocks), dim3(256), 0, st, true, acc, p.sums, s.rows, s.d, info, dh, dhs));
    count_launch();
  }
  return SZO_OK;
}

}  // namespace
}  // namespace head
}  // namespace szo

using namespace szo;

extern "C" {

size_t szo_head_ce_workspace_bytes(int64_t rows, int64_t vocab, int64_t d) {
  return head::fits(rows, vocab, d) && rows > 0 ? head::forward_plan({rows, vocab, d}).total : 0;
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
  auto run = [&](auto zero) {
    using T = decltype(zero);
    return head::forward<T>(s, {static_cast<const T*>(h), h_stride, static_cast<const T*>(W), w_stride, scale, targets}, loss, lse, ws, status, st);
  };
  return dtype == SZO_BF16 ? run(__nv_bfloat16{}) : run(__half{});
}

size_t szo_head_ce_bwd_workspace_bytes(int64_t rows, int64_t vocab, int64_t d, int32_t want_dh, int32_t want_dw) {
  if (!head::fits(rows, vocab, d) || rows == 0 || (!want_dh && !want_dw)) return 0;
  const int64_t most = head::rows_at_once({rows, vocab, d}, want_dw != 0), last = rows - (ceil_div(rows, most) - 1) * most;
  const size_t a = head::backward_plan({most, vocab, d}, want_dh != 0, want_dw != 0).total;
  const size_t b = head::backward_plan({last, vocab, d}, want_dh != 0, want_dw != 0).total;      // (fewer rows may sum dh in more shares)
  return a > b ? a : b;
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
  auto* ws = static_cast<unsigned char*>(workspace);
  int32_t* status = device_status_word();
  SZO_REQUIRE(status != nullptr, SZO_ERR_CUDA, "no device status word (no CUDA device?)");
  const int64_t most = head::rows_at_once({rows, vocab, d}, dW != nullptr);
  auto run = [&](auto zero) -> szo_status {
    using T = decltype(zero);
    for (int64_t r = 0; r < rows; r += most) {                    // (r is a multiple of 256: everything stays aligned)
      const head::Shape s{rows - r < most ? rows - r : most, vocab, d};
      SZO_TRY(head::backward<T>(s, {static_cast<const T*>(h) + r * h_stride, h_stride, static_cast<const T*>(W), w_stride, scale, targets + r}, lse + r,
                                d_loss + r, d_lse != nullptr ? d_lse + r : nullptr, dh != nullptr ? static_cast<T*>(dh) + r * dh_stride : nullptr, dh_stride,
                                static_cast<T*>(dW), dw_stride, ws, status, st));
    }
    return SZO_OK;
  };
  return dtype == SZO_BF16 ? run(__nv_bfloat16{}) : run(__half{});
}

}  // extern "C"
