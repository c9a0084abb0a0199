// What the two attention kernels over the 8-bit cache share (kv8_attention.cu: few query rows per key/value head;
// kv8_attention_tc.cu: many).
#pragma once
#include "kv8.cuh"
#include "tc_common.cuh"

namespace szo {
namespace kv8 {

constexpr int kPrefixRows = 32;                // rows of a group, 16-bit types, that one block takes
constexpr int kStep = 16;                      // positions that certainly share a page

// The row buffers and heads of a call
struct Rows {
  const void* q;
  void* o;
  int64_t q_stride, o_stride;
  int H;
  float scale;
};

// One pass of attention over groups that share their first positions (kv8_prefix.cu): a row's result is left unfinished, for
// every (share of the positions, row, head) HD sums in `sums` and (reference, sum of weights) in `stats`, the weights of position j being
// 2^(t_j - reference); row-heads are counted row * H + head in each share.
struct Part {
  const int4* groups;          // per group: first row, rows, shared positions (0: none), sequence whose table holds them
  const int32_t* pos;          // position of every row
  const int32_t* shared;       // per sequence: positions that its group shares
  float* sums;
  float2* stats;
  int64_t row_heads;           // of a share
  int prefix;                  // 1: the rows of a group over the shared positions; 0: a sequence's rows over the rest
  int items;                   // groups or sequences
  int max_rows;                // the most rows of one
};
// (chained launches, see kv8_prefix.cu)
template <typename T, int HD> szo_status launch_part(const View& V, const Rows& A, const Part& part, int nsplit, cudaStream_t st);
template <typename T, int HD> szo_status launch_part_tc(const View& V, const Rows& A, const Part& part, int nsplit, cudaStream_t st);

// The checks of a call's row buffers, and of what its kernels count in 32 bits (kv8_attention.cu)
szo_status check_rows(const szo_kv8_cache* cache, const void* q, int64_t q_stride, const void* o, int64_t o_stride, szo_dtype dtype,
                      int32_t n_heads, float scale, const void* workspace);
szo_status check_sizes(const szo_kv8_cache* cache, const View& V, int32_t n_heads);

// Many query rows per key/value head (kv8_attention_tc.cu); 16-bit types only
template <typename T, int HD> szo_status launch_attention_tc(const View& V, const Rows& A, float* ws, cudaStream_t st);
size_t workspace_bytes_tc(const View& V, int H, int hd);
// Joins the partial results of n_items items from item0 on, cut into nsplit shares each (kv8_attention.cu).  ws: per item and
// share R * HD sums, R maxima (base 2), R sums of weights.  long_first: items are counted as kv8_attention_tc.cu does.
template <typename T, int HD>
szo_status launch_join(const View& V, const Rows& A, const float* ws, int R, int row_tiles, int nsplit, bool long_first, int64_t item0,
                       int64_t n_items, cudaStream_t st);

#ifdef __CUDACC__
// What a block works on: rows seq.row0 .. of a sequence or of a group, whose last stands at position seq.len - 1 counted from
// `skip` on, in the table of sequence `owner`.  (A group's rows stand anywhere at or behind its shared positions [0, len), or inside them.)
struct Work {
  Seq seq;
  int skip, owner;
};
__device__ __forceinline__ Work load_work(const View& V, const Part& part, int b) {
  if (part.prefix) {
    const int4 g = __ldcg(part.groups + b);
    return Work{Seq{g.z > 0 ? g.y : 0, g.z, g.x}, 0, g.w};
  }
  Work w{load_seq(V, b), __ldcg(part.shared + b), b};
  w.seq.len -= w.skip;
  return w;
}
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
