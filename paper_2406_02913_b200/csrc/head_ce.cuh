// What the two files of the cross entropy from hidden states share: the products of its forward and backward passes as jobs of
// one kernel (head_ce_tc.cu), planned by head_ce.cu.
#pragma once
#include <cuda.h>

#include <type_traits>

#include "common.cuh"

namespace szo {
namespace head {

constexpr int kTile = 256;                     // rows and columns of a tile, at most
constexpr int kBlockK = 64;                    // contracted elements of a stage

// A product D[m][n] = sum_k A(m, k) B(n, k) in tiles of up to 256 x 256, and what becomes of a tile
enum Kind : int {
  kStats,      // (m, s) of every row and 128 columns, the target's logit
  kGrad,       // G in the 16-bit type
  kSum,        // fp32 sums, stored or (add) added to what is there
  kOut,        // times a power of two, rounded to the 16-bit type
  // few rows of hidden states: they are the columns of D
  kStatsT,     // (m, s) of every column and 32 rows, the target's logit
  kGradT,
  kSumT
};
struct Job {
  CUtensorMap a, b, out;                       // operands by boxes of 64 elements; out: boxes of 32 rows
  int kind;
  int a_mn, b_mn;                              // the operand's rows are the contracted dimension
  int a_bytes, b_bytes;                        // of the operands per stage and CTA
  int a_m0, a_k0, b_n0, b_k0;                  // where the operands' pieces start
  int m_step, n_step;                          // a tile's rows and columns; each CTA brings half of either
  int m_tiles, n_tiles, m_band;                // tiles of m are taken in bands of m_band (0: all)
  int nkb, parts, units;                       // blocks of 64 contracted elements, cut into `parts`; units = tiles * parts
  int out_row0;                                // the tile's first row in `out`
  int m_limit;                                 // rows of D that there are
  int add;
};
struct Jobs {
  Job job[3];
  int n_jobs, units;
  int b_at, stage_bytes, stages;               // the ring: B's place in a stage (set by launch_jobs)
  // kStats, kGrad
  const int32_t* targets;
  const float4* info;
  const int32_t* exponent;                     // of the largest weight (fp16)
  float2* part;                                // [parts of the vocabulary][rows]
  float* xt;
  int64_t rows;
  int n_end;                                   // vocabulary entries that there are (of this piece)
  int target0;                                 // index of the first
  float c;                                     // scale * log2 e
  // kGradT, kSumT
  void* G;
  int64_t g_stride;
  float* sums;                                 // [parts][rows][d]
  int d;
  int32_t* status;
};
template <typename T> szo_status launch_jobs(Jobs& P, bool chained, cudaStream_t st);

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
