// What the two attention kernels over the 8-bit cache share (kv8_attention.cu: few query rows per key/value head;
// kv8_attention_tc.cu: many).
#pragma once
#include "kv8.cuh"
#include "tc_common.cuh"

namespace szo {
namespace kv8 {

constexpr int kStep = 16;                      // positions that certainly share a page

// The row buffers and heads of a call
struct Rows {
  const void* q;
  void* o;
  int64_t q_stride, o_stride;
  int H;
  float scale;
};

// Many query rows per key/value head (kv8_attention_tc.cu); 16-bit types only
template <typename T, int HD> szo_status launch_attention_tc(const View& V, const Rows& A, float* ws, cudaStream_t st);
size_t workspace_bytes_tc(const View& V, int H, int hd);
// Joins the partial results of n_items items from item0 on, cut into nsplit shares each (kv8_attention.cu).  ws: per item and
// share R * HD sums, R maxima (base 2), R sums of weights.  long_first: items are counted as kv8_attention_tc.cu does.
template <typename T, int HD>
szo_status launch_join(const View& V, const Rows& A, const float* ws, int R, int row_tiles, int nsplit, bool long_first, int64_t item0,
                       int64_t n_items, cudaStream_t st);

#ifdef __CUDACC__
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
#endif

}  // namespace kv8
}  // namespace szo
