// What the two files of the cross entropy from hidden states share: the products of its forward and backward passes as jobs of
// one kernel (head_ce_tc.cu), planned by head_ce.cu.
#pragma once
#include <cuda.h>

#include <type_traits>

#include "common.cuh"

namespace szo {
namespace head {

constexpr int kTile = 256;                     // rows and columns of a tile
constexpr int kBlockK = 64;                    // contracted elements of a stage

// A product D[m][n] = sum_k A(m, k) B(n, k) in tiles of 256 x 256, and what becomes of a tile
enum Kind : int {
  kStats,      // (m, s) of every row and 128 columns, the target's logit
  kGrad,       // G in the 16-bit type
  kSum,        // fp32 sums, stored or (add) added to what is there
  kOut         // times a power of two, rounded to the 16-bit type
};
struct Job {
  CUtensorMap a, b, out;                       // operands by boxes of 64 elements; out: boxes of 32 rows
  int kind;
  int a_mn, b_mn;                              // the operand's rows are the contracted dimension
  int a_bytes;                                 // of A per stage and CTA (fewer where there are fewer than 128 rows)
  int b_k0, b_n0;                              // where B's piece starts, in its contracted / other dimension
  int m_tiles, n_tiles, m_band;                // tiles of m are taken in bands of m_band (0: all)
  int nkb, parts, units;                       // blocks of 64 contracted elements, cut into `parts`; units = tiles * parts
  int out_row0;                                // the tile's first row in `out`
  int m_limit;                                 // rows of D that there are
  int add;
};
struct Jobs {
  Job job[3];
  int n_jobs, units;
  // kStats, kGrad
  const int32_t* targets;
  const float4* info;
  const int32_t* exponent;                     // of the largest weight (fp16)
  float2* part;                                // [2 * n_tiles][rows]
  float* xt;
  int64_t rows;
  int n_end;                                   // columns that there are (of this piece)
  int target0;                                 // the vocabulary index of column 0
  float c;                                     // scale * log2 e
  int32_t* status;
};
template <typename T> szo_status launch_jobs(const Jobs& P, cudaStream_t st);

#ifdef __CUDACC__
// For dW of fp16 the rows of G stand at 2^13 times their weight's power of two and those of h at that power over the largest
// one's: what is left of the product is 2^(exponent - 13).  (No row weighs anything: the sums are zeros.)
template <typename T> __device__ __forceinline__ float weight_of(const int32_t* exponent) {
  if constexpr (std::is_same<T, __nv_bfloat16>::value) return 1.f;
  const int e = *exponent;
  return e < -126 ? 1.f : __int_as_float((e - 13 + 127) << 23);
}
#endif

}  // namespace head
}  // namespace szo
