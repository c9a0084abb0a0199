// The 8-bit paged key/value cache: kernel-side view, the checks of its arguments and the number format.
//
// Format.  A cached element is an e4m3 code times 2^e, one e per (page, key/value head), keys and values
// apart.  With a = the largest magnitude to be stored, e is the smallest integer with a <= 448 * 2^e (448 is
// the largest e4m3 number), kept in [kEMin, kEMax].  Powers of two because e4m3 carries its own exponent: a
// real-valued scale would gain precision only for the elements that fall into e4m3's subnormals (below
// 2^-15 of the largest), while with a power of two (1) no product or quotient by the scale rounds, (2) a
// page whose scale has to grow when a louder token is appended can be rescaled by shifting exponents,
// exact but for those subnormals, and (3) a dequantised element has four significant bits, exact in bf16.
#pragma once
#include <cuda_fp8.h>

#include "common.cuh"

namespace szo {
namespace kv8 {

constexpr int kEMin = -63, kEMax = 63;
constexpr uint8_t kNaNCode = 0x7f;

// Kernel parameters common to every operator on the cache.
struct View {
  uint8_t *k, *v;              // [n_pages][hkv][page_tokens][hd]
  float2* scales;              // [n_pages][hkv]: (keys, values)
  int64_t n_pages;
  int hkv, page_shift;         // page_tokens = 1 << page_shift
  int batch, max_pages, max_new;
  int64_t rows;
  const int32_t *table, *kv_len, *start;
  int32_t* status;
};

szo_status make_view(const szo_kv8_cache* cache, const szo_kv8_batch* batch, View* out);
szo_status set_status_word(View* V);
// grid of one block per (item, key/value head, sequence), refused where it passes the launch limit
szo_status grid_items(int64_t per_head, const View& V, unsigned* blocks);

#ifdef __CUDACC__
// Sequence b of a batch: n rows from row0 on, the last of them at position len - 1.  A sequence whose
// description does not fit its buffers is reported in the status word and skipped (n = 0, len = 0).
struct Seq {
  int n, len;
  int64_t row0;
};
__device__ __forceinline__ Seq load_seq(const View& V, int b) {
  Seq s{V.max_new, V.kv_len[b], static_cast<int64_t>(b) * V.max_new};
  bool ok = s.len >= 0 && s.len <= static_cast<int64_t>(V.max_pages) << V.page_shift;
  if (V.start != nullptr) {
    const int s0 = V.start[b], s1 = V.start[b + 1];
    s.row0 = s0;
    s.n = s1 - s0;
    ok = ok && s0 >= 0 && s1 >= s0 && s1 <= V.rows && s.n <= V.max_new;
  }
  if (!ok) {
    atomicExch(V.status, static_cast<int32_t>(SZO_ERR_SHAPE));
    s.n = s.len = 0;
  }
  return s;
}
__device__ __forceinline__ void report_page(const View& V) { atomicExch(V.status, static_cast<int32_t>(SZO_ERR_INVALID_ARG)); }
// Page id of the j-th page of sequence b, or -1 (reported) where the table holds none
__device__ __forceinline__ int load_page(const View& V, int b, int j) {
  const int p = V.table[static_cast<int64_t>(b) * V.max_pages + j];
  if (static_cast<uint32_t>(p) >= static_cast<uint64_t>(V.n_pages)) {
    report_page(V);
    return -1;
  }
  return p;
}
// First byte of (page, head) in k or v
__device__ __forceinline__ int64_t page_offset(const View& V, int page, int h, int hd) {
  return ((static_cast<int64_t>(page) * V.hkv + h) << V.page_shift) * hd;
}

__device__ __forceinline__ float exp2_int(int e) { return __int_as_float((e + 127) << 23); }   // e in [-126, 127]
// Exponent of a stored scale.  Scales are written by szo_kv8_write only; zeroed memory reads as kEMin.
__device__ __forceinline__ int scale_exponent(float s) {
  const int e = ((__float_as_int(s) >> 23) & 255) - 127;
  return min(max(e, kEMin), kEMax);
}
// The smallest e in [kEMin, kEMax] with a <= 448 * 2^e, a finite and >= 0 (448 = 1.75 * 2^8)
__device__ __forceinline__ int needed_exponent(float a) {
  const int bits = __float_as_int(a);
  const int e = (bits >> 23) - 127 - 8 + ((bits & 0x7fffff) > 0x600000 ? 1 : 0);
  return min(max(e, kEMin), kEMax);
}
constexpr float kLargest = 448.0f * 9223372036854775808.0f;      // 448 * 2^63: beyond it an element is stored as NaN

// Two floats to e4m3 (round to nearest even, NaN to 0x7f), `lo` in the low byte.  |x| <= 448 or NaN.
__device__ __forceinline__ uint32_t encode2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
// Two e4m3 codes (low 16 bits of w) to packed f16, exactly
__device__ __forceinline__ uint32_t decode2(uint32_t w) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(static_cast<uint16_t>(w)));
  return r;
}
__device__ __forceinline__ float2 decode2f(uint32_t w) {
  const uint32_t h = decode2(w);
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

template <typename T> __device__ __forceinline__ float widen(T x);
template <> __device__ __forceinline__ float widen<float>(float x) { return x; }
template <> __device__ __forceinline__ float widen<__half>(__half x) { return __half2float(x); }
template <> __device__ __forceinline__ float widen<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T narrow(float x);
template <> __device__ __forceinline__ float narrow<float>(float x) { return x; }
template <> __device__ __forceinline__ __half narrow<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// 16 bytes of T
template <typename T> struct alignas(16) Vec {
  static constexpr int kN = 16 / static_cast<int>(sizeof(T));
  T x[kN];
};
#endif

}  // namespace kv8
}  // namespace szo
