// Writing new keys and values into the 8-bit paged cache and reading cached positions back.
//
// Both are streams: per element one 2- or 4-byte access of a row buffer and one byte of the cache, so HBM
// bandwidth bounds them once there are enough pages, and the latency of one dependent chain
// (lengths -> page id -> rows -> amax -> codes) when there are few.  One block owns one (page, head): the
// amax that sets its scale then needs no second pass and no atomics, and the rows stay in registers
// between the two uses.  Inside a block a warp owns 16 slots of the keys or of the values, and all its loads are under way
// before the first is used.  Measured (8 heads of 128; inputs of several calls in turn, together larger than L2): 8 x 2048 new
// positions written in 20.8 us from bf16 (4.3 TB/s, 0.67 of the measured copy bandwidth; 18.5 us where the same 90 MB come again and
// partly stay in L2), 35.7 us from fp32 (4.2 TB/s): what is left is the chain above, with 2 blocks per SM (fp32: 1); contexts of 4 x
// 8192 read in 34.2 us to bf16 (5.8 TB/s, 0.90), 56.9 us to fp32 (5.8 TB/s); 32 single tokens written in 3.6 us, which is launch and chain.
#include "kv8.cuh"

namespace szo {
namespace kv8 {

szo_status make_view(const szo_kv8_cache* c, const szo_kv8_batch* b, View* out) {
  SZO_REQUIRE(c && b, SZO_ERR_INVALID_ARG, "NULL cache or batch");
  SZO_REQUIRE(c->k_codes && c->v_codes && c->scales, SZO_ERR_INVALID_ARG, "NULL cache buffer");
  SZO_REQUIRE(b->page_table && b->kv_len, SZO_ERR_INVALID_ARG, "NULL page_table or kv_len");
  SZO_REQUIRE(c->page_tokens == 16 || c->page_tokens == 32 || c->page_tokens == 64 || c->page_tokens == 128,
              SZO_ERR_UNSUPPORTED, "page_tokens must be 16, 32, 64 or 128 (got %d)", c->page_tokens);
  SZO_REQUIRE(c->head_dim == 64 || c->head_dim == 128, SZO_ERR_UNSUPPORTED, "head_dim must be 64 or 128 (got %d)", c->head_dim);
  SZO_REQUIRE(c->n_kv_heads > 0 && c->n_pages > 0 && c->n_pages < (int64_t(1) << 31), SZO_ERR_SHAPE, "bad cache shape");
  SZO_REQUIRE(b->batch >= 0 && b->rows >= 0 && b->max_new >= 0 && b->max_pages > 0, SZO_ERR_SHAPE, "bad batch shape");
  SZO_REQUIRE(static_cast<int64_t>(b->max_pages) * c->page_tokens <= (int64_t(1) << 30), SZO_ERR_SHAPE,
              "max_pages * page_tokens must not pass 2^30 positions");
  SZO_REQUIRE(b->max_new <= (1 << 30), SZO_ERR_SHAPE, "max_new must not pass 2^30");
  SZO_REQUIRE(b->start != nullptr || static_cast<int64_t>(b->batch) * b->max_new <= b->rows, SZO_ERR_SHAPE,
              "without start, rows must hold batch * max_new rows");
  SZO_REQUIRE(aligned16(c->k_codes) && aligned16(c->v_codes) && aligned16(c->scales) && aligned16(b->page_table) &&
                  aligned16(b->kv_len) && aligned16(b->start),
              SZO_ERR_ALIGNMENT, "buffers must be 16-byte aligned");
  int shift = 4;
  while ((1 << shift) < c->page_tokens) ++shift;
  *out = View{c->k_codes, c->v_codes, reinterpret_cast<float2*>(c->scales), c->n_pages, c->n_kv_heads, shift, b->batch,
              b->max_pages, b->max_new, b->rows, b->page_table, b->kv_len, b->start, nullptr};
  return SZO_OK;
}

szo_status set_status_word(View* V) {
  V->status = device_status_word();
  SZO_REQUIRE(V->status != nullptr, SZO_ERR_CUDA, "no device status word (no CUDA device?)");
  return SZO_OK;
}

szo_status grid_items(int64_t per_head, const View& V, unsigned* blocks) {
  const int64_t heads = static_cast<int64_t>(V.batch) * V.hkv;
  SZO_REQUIRE(per_head <= 0x7fffffff / heads, SZO_ERR_SHAPE, "too many pages, heads and sequences for one launch");
  *blocks = static_cast<unsigned>(per_head * heads);
  return SZO_OK;
}

namespace {

// Rows of a warp's 16 slots, kN elements per lane and load: kLR lanes share a row.
template <typename T, int HD> struct Slots {
  static constexpr int kN = Vec<T>::kN, kLR = HD / kN, kRows = 32 / kLR, kLoads = 16 / kRows;
};

// Bits of |x| of both 16-bit halves
__device__ __forceinline__ uint32_t magnitudes(uint32_t w) { return w & 0x7fff7fffu; }
// Largest magnitude of a vector: of the finite elements within the format's range, and whether there are others.  For 16-bit
// types the order of magnitudes is that of their bits, two at a time.
__device__ __forceinline__ float largest(const Vec<float>& v, bool& others) {
  float a = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float m = fabsf(v.x[i]);
    others = others || !(m <= kLargest);
    a = fmaxf(a, m <= kLargest ? m : 0.f);
  }
  return a;
}
template <typename T> __device__ __forceinline__ float largest(const Vec<T>& v, bool& others) {
  const uint32_t* w = reinterpret_cast<const uint32_t*>(v.x);
  const uint32_t m = __vmaxu2(__vmaxu2(magnitudes(w[0]), magnitudes(w[1])), __vmaxu2(magnitudes(w[2]), magnitudes(w[3])));
  const uint16_t top = static_cast<uint16_t>(max(m & 0xffffu, m >> 16));
  const float a = widen<T>(*reinterpret_cast<const T*>(&top));
  if (a <= kLargest) return a;
  others = true;
  float b = 0.f;
#pragma unroll
  for (int i = 0; i < Vec<T>::kN; ++i) {
    const float x = fabsf(widen<T>(v.x[i]));
    b = fmaxf(b, x <= kLargest ? x : 0.f);
  }
  return b;
}
// Elements 2 i, 2 i + 1 in fp32
__device__ __forceinline__ float2 widen2(const Vec<float>& v, int i) { return make_float2(v.x[2 * i], v.x[2 * i + 1]); }
__device__ __forceinline__ float2 widen2(const Vec<__half>& v, int i) { return __half22float2(reinterpret_cast<const __half2*>(v.x)[i]); }
__device__ __forceinline__ float2 widen2(const Vec<__nv_bfloat16>& v, int i) {
  const uint32_t w = reinterpret_cast<const uint32_t*>(v.x)[i];
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}

// Block = (touched page, head, sequence); warps 2 i and 2 i + 1 take slots [16 i, 16 i + 16) of keys and values.
template <typename T, int HD>
__global__ void __launch_bounds__(512, sizeof(T) == 2 ? 2 : 1)
kv8_write_kernel(View V, const T* __restrict__ k, const T* __restrict__ v, int64_t k_stride, int64_t v_stride, int per_seq) {
  using S = Slots<T, HD>;
  __shared__ float amax[2][8];
  chain_release();
  chain_wait();
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, which = w & 1, sub = w >> 1;
  const unsigned item = blockIdx.x;
  const int h = item % V.hkv, j = (item / V.hkv) % per_seq, b = item / V.hkv / per_seq;
  const Seq seq = load_seq(V, b);
  const int pos0 = max(seq.len - seq.n, 0);                       // first position stored
  const int pj = (pos0 >> V.page_shift) + j, base = pj << V.page_shift;
  if (seq.n == 0 || pj >= V.max_pages || base >= seq.len) return;
  const int page = load_page(V, b, pj);
  if (page < 0) return;
  const T* rows = (which ? v : k) + (seq.row0 - (seq.len - seq.n)) * (which ? v_stride : k_stride) + h * HD;   // + pos * stride
  const int64_t stride = which ? v_stride : k_stride;
  uint8_t* codes = (which ? V.v : V.k) + page_offset(V, page, h, HD);
  float* scale = reinterpret_cast<float*>(V.scales + static_cast<int64_t>(page) * V.hkv + h) + which;
  const bool fresh = base >= pos0;
  const int e_old = fresh ? kEMin : scale_exponent(*scale);

  const int r0 = sub * 16 + lane / S::kLR, c0 = lane % S::kLR * S::kN;
  Vec<T> x[S::kLoads];
#pragma unroll
  for (int i = 0; i < S::kLoads; ++i) {
    const int pos = base + r0 + i * S::kRows;
    x[i] = Vec<T>{};
    if (pos >= pos0 && pos < seq.len) x[i] = *reinterpret_cast<const Vec<T>*>(rows + pos * stride + c0);
  }
  float a = 0.f;
  bool others = false;                                            // elements that are not finite, or too large: they do not set the scale
#pragma unroll
  for (int i = 0; i < S::kLoads; ++i) a = fmaxf(a, largest(x[i], others));
#pragma unroll
  for (int o = 16; o; o >>= 1) a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, o));
  if (lane == 0) amax[which][sub] = a;
  __syncthreads();
  for (int i = 0; i < static_cast<int>(blockDim.x >> 6); ++i) a = fmaxf(a, amax[which][i]);
  const int e = max(needed_exponent(a), e_old);
  if (sub == 0 && lane == 0) *scale = exp2_int(e);                // (every warp has read the old one)
  const float inv = exp2_int(-e);
  const bool rescale = !fresh && e != e_old;
  const float shift = exp2_int(max(e_old - e, -126));
#pragma unroll
  for (int i = 0; i < S::kLoads; ++i) {
    const int slot = r0 + i * S::kRows, pos = base + slot;
    uint8_t* dst = codes + slot * HD + c0;
    uint32_t out[S::kN / 4];
    if (pos >= pos0 && pos < seq.len) {
#pragma unroll
      for (int u = 0; u < S::kN; u += 4) {
        float2 lo = widen2(x[i], u / 2), hi = widen2(x[i], u / 2 + 1);
        if (others) {
          const float nan = __int_as_float(0x7fffffff);
          lo = make_float2(fabsf(lo.x) <= kLargest ? lo.x : nan, fabsf(lo.y) <= kLargest ? lo.y : nan);
          hi = make_float2(fabsf(hi.x) <= kLargest ? hi.x : nan, fabsf(hi.y) <= kLargest ? hi.y : nan);
        }
        out[u / 4] = encode2(lo.x * inv, lo.y * inv) | encode2(hi.x * inv, hi.y * inv) << 16;
      }
    } else if (rescale && pos < pos0) {
#pragma unroll
      for (int u = 0; u < S::kN; u += 4) {
        const uint32_t old = *reinterpret_cast<const uint32_t*>(dst + u);
        const float2 lo = decode2f(old), hi = decode2f(old >> 16);
        out[u / 4] = encode2(lo.x * shift, lo.y * shift) | encode2(hi.x * shift, hi.y * shift) << 16;
      }
    } else {
      continue;
    }
    if constexpr (S::kN == 8) *reinterpret_cast<uint2*>(dst) = make_uint2(out[0], out[1]);
    else *reinterpret_cast<uint32_t*>(dst) = out[0];
  }
}

// Same blocks: the positions of one page that the batch's rows stand for, one 16-byte store per lane and load.
template <typename T, int HD>
__global__ void __launch_bounds__(512)
kv8_read_kernel(View V, T* __restrict__ k, T* __restrict__ v, int64_t k_stride, int64_t v_stride, int per_seq) {
  using S = Slots<T, HD>;
  chain_release();
  chain_wait();
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, which = w & 1, sub = w >> 1;
  const unsigned item = blockIdx.x;
  const int h = item % V.hkv, j = (item / V.hkv) % per_seq, b = item / V.hkv / per_seq;
  const Seq seq = load_seq(V, b);
  T* rows = (which ? v : k) + h * HD;
  const int64_t stride = which ? v_stride : k_stride;
  const int pos0 = seq.len - seq.n;
  const int r0 = sub * 16 + lane / S::kLR, c0 = lane % S::kLR * S::kN;
  if (j == 0 && pos0 < 0) {                                       // padding rows: zeros
    const Vec<T> zero = {};
    for (int i = sub * S::kRows + lane / S::kLR; i < -pos0; i += S::kRows * static_cast<int>(blockDim.x >> 6))
      *reinterpret_cast<Vec<T>*>(rows + (seq.row0 + i) * stride + c0) = zero;
  }
  const int first = max(pos0, 0);
  const int pj = (first >> V.page_shift) + j, base = pj << V.page_shift;
  if (seq.n == 0 || pj >= V.max_pages || base >= seq.len) return;
  const int page = load_page(V, b, pj);
  const uint8_t* codes = (which ? V.v : V.k) + page_offset(V, page < 0 ? 0 : page, h, HD);
  const float2 sc = V.scales[static_cast<int64_t>(page < 0 ? 0 : page) * V.hkv + h];
  const float scale = exp2_int(scale_exponent(which ? sc.y : sc.x));
  uint32_t word[S::kLoads][S::kN / 4];
#pragma unroll
  for (int i = 0; i < S::kLoads; ++i) {                           // (all loads first; a page is whole, so slots behind the last position may be read)
    const uint8_t* p = codes + (r0 + i * S::kRows) * HD + c0;
    if constexpr (S::kN == 8) {
      const uint2 t = *reinterpret_cast<const uint2*>(p);
      word[i][0] = t.x;
      word[i][1] = t.y;
    } else {
      word[i][0] = *reinterpret_cast<const uint32_t*>(p);
    }
  }
#pragma unroll
  for (int i = 0; i < S::kLoads; ++i) {
    const int pos = base + r0 + i * S::kRows;
    if (pos < first || pos >= seq.len) continue;
    Vec<T> out;
#pragma unroll
    for (int u = 0; u < S::kN; u += 4) {
      const float2 lo = decode2f(word[i][u / 4]), hi = decode2f(word[i][u / 4] >> 16);
      out.x[u] = narrow<T>(lo.x * scale);
      out.x[u + 1] = narrow<T>(lo.y * scale);
      out.x[u + 2] = narrow<T>(hi.x * scale);
      out.x[u + 3] = narrow<T>(hi.y * scale);
    }
    if (page < 0) out = Vec<T>{};                                 // no such page: zeros, and the status word says so
    *reinterpret_cast<Vec<T>*>(rows + (seq.row0 + (pos - pos0)) * stride + c0) = out;
  }
}

szo_status check_rows(const szo_kv8_cache* c, const void* k, const void* v, szo_dtype dt, int64_t ks, int64_t vs) {
  SZO_REQUIRE(k && v, SZO_ERR_INVALID_ARG, "NULL row buffer");
  SZO_REQUIRE(dt == SZO_F32 || dt == SZO_BF16 || dt == SZO_F16, SZO_ERR_UNSUPPORTED, "dtype must be f32, bf16 or f16");
  const int64_t width = static_cast<int64_t>(c->n_kv_heads) * c->head_dim, vec = dt == SZO_F32 ? 4 : 8;
  SZO_REQUIRE(ks >= width && vs >= width, SZO_ERR_SHAPE, "row strides must be at least n_kv_heads * head_dim");
  SZO_REQUIRE(aligned16(k) && aligned16(v) && ks % vec == 0 && vs % vec == 0, SZO_ERR_ALIGNMENT,
              "row buffers and rows must be 16-byte aligned");
  return SZO_OK;
}

// pages that a sequence's max_new newest positions can touch
int64_t pages_touched(const View& V) {
  const int64_t p = int64_t(1) << V.page_shift, n = (V.max_new + p - 2) / p + 1;
  return n < V.max_pages ? n : V.max_pages;
}

}  // namespace
}  // namespace kv8
}  // namespace szo

using namespace szo;

extern "C" {

szo_status szo_kv8_write(const szo_kv8_cache* cache, const szo_kv8_batch* batch, const void* k, const void* v, szo_dtype dtype,
                         int64_t k_stride, int64_t v_stride, void* stream) {
  kv8::View V;
  SZO_TRY(kv8::make_view(cache, batch, &V));
  SZO_TRY(kv8::check_rows(cache, k, v, dtype, k_stride, v_stride));
  if (V.batch == 0 || V.max_new == 0 || V.rows == 0) return SZO_OK;
  const int64_t per_seq = kv8::pages_touched(V);
  unsigned blocks;
  SZO_TRY(kv8::grid_items(per_seq, V, &blocks));
  const unsigned threads = static_cast<unsigned>(cache->page_tokens) * 4;
  SZO_TRY(kv8::set_status_word(&V));
  cudaStream_t st = static_cast<cudaStream_t>(stream);
#define SZO_KV8_WRITE(T, HD) \
  kv8::kv8_write_kernel<T, HD><<<blocks, threads, 0, st>>>(V, static_cast<const T*>(k), static_cast<const T*>(v), k_stride, v_stride, static_cast<int>(per_seq))
  const bool wide = cache->head_dim == 128;
  if (dtype == SZO_F32) { if (wide) SZO_KV8_WRITE(float, 128); else SZO_KV8_WRITE(float, 64); }
  else if (dtype == SZO_BF16) { if (wide) SZO_KV8_WRITE(__nv_bfloat16, 128); else SZO_KV8_WRITE(__nv_bfloat16, 64); }
  else { if (wide) SZO_KV8_WRITE(__half, 128); else SZO_KV8_WRITE(__half, 64); }
#undef SZO_KV8_WRITE
  count_launch();
  SZO_CHECK_LAUNCH("kv8_write_kernel");
  return SZO_OK;
}

szo_status szo_kv8_read(const szo_kv8_cache* cache, const szo_kv8_batch* batch, void* k, void* v, szo_dtype dtype,
                        int64_t k_stride, int64_t v_stride, void* stream) {
  kv8::View V;
  SZO_TRY(kv8::make_view(cache, batch, &V));
  SZO_TRY(kv8::check_rows(cache, k, v, dtype, k_stride, v_stride));
  if (V.batch == 0 || V.max_new == 0 || V.rows == 0) return SZO_OK;
  const int64_t per_seq = kv8::pages_touched(V);
  unsigned blocks;
  SZO_TRY(kv8::grid_items(per_seq, V, &blocks));
  const unsigned threads = static_cast<unsigned>(cache->page_tokens) * 4;
  SZO_TRY(kv8::set_status_word(&V));
  cudaStream_t st = static_cast<cudaStream_t>(stream);
#define SZO_KV8_READ(T, HD) \
  kv8::kv8_read_kernel<T, HD><<<blocks, threads, 0, st>>>(V, static_cast<T*>(k), static_cast<T*>(v), k_stride, v_stride, static_cast<int>(per_seq))
  const bool wide = cache->head_dim == 128;
  if (dtype == SZO_F32) { if (wide) SZO_KV8_READ(float, 128); else SZO_KV8_READ(float, 64); }
  else if (dtype == SZO_BF16) { if (wide) SZO_KV8_READ(__nv_bfloat16, 128); else SZO_KV8_READ(__nv_bfloat16, 64); }
  else { if (wide) SZO_KV8_READ(__half, 128); else SZO_KV8_READ(__half, 64); }
#undef SZO_KV8_READ
  count_launch();
  SZO_CHECK_LAUNCH("kv8_read_kernel");
  return SZO_OK;
}

}  // extern "C"
