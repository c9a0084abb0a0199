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
enum Offset : int { kNone, kVocab, kBuffer };  // of an operand's vocabulary dimension: the piece's first entry, or its buffer of G
struct Extent {                                // of a product over a piece: tiles, blocks of 64 contracted elements, and the shares that these are cut into
  int m_tiles, n_tiles, nkb, parts, units;     // units = m_tiles * n_tiles * parts
};
struct Job {
  CUtensorMap a, b, out;                       // operands by boxes of 64 elements; out: boxes of 32 rows
  int kind;                                    // -1: no such job
  int vocab_dim;                               // which dimension is the piece of the vocabulary: 0 m, 1 n, 2 k
  int a_mn, b_mn;                              // the operand's rows are the contracted dimension
  int a_from, b_from;                          // Offset
  int a_bytes, b_bytes;                        // of the operands per stage and CTA
  int keep_from;                               // few rows: entry of W from which on L2 is to keep what is read (-1: no matter)
  int m_step, n_step;                          // a tile's rows and columns; each CTA brings half of either
  int m_limit;                                 // rows of D that there are (where they are not the vocabulary)
  int m_band;                                  // tiles of m are taken in bands of m_band (0: all)
  Extent full, last;                           // over a piece, over the last one
};
// The units of work, in their order: for s = 0, 1, ..  job 0 of piece s, then jobs 1 and 2 of piece s - 1.  Jobs 1 and 2 read what job 0
// has written of their piece, in a ring of buffers.  A launch takes all steps s, its units handed out as they are asked for and waiting for
// what they read (`counters`), or one step, its units dealt out in turn.
struct Jobs {
  Job job[3];
  int vocab, piece, pieces, buffers;
  int step, units;                             // the first step of the launch, and its units
  int idle;                                    // bit j: the launch has no units of job j (the ring need not hold its operands)
  int b_at, stage_bytes, stages;               // the ring of operands: B's place in a stage (set by launch_jobs)
  int32_t* counters;                           // NULL, or zeroed: the next unit, and per piece the epilogues' arrivals for job 0 and for
                                               // jobs 1 and 2
  const int32_t* targets;
  const float4* info;
  const int32_t* exponent;                     // of the largest weight (fp16)
  float2* part;                                // [parts of the vocabulary][rows]
  float* xt;
  int64_t rows;
  float c;                                     // scale * log2 e
  // kGradT, kSumT
  void* G;
  int64_t g_stride;
  float* sums;                                 // [parts][rows][d]
  int d;
  int32_t* status;
};
inline int64_t counters_of(int64_t pieces) { return 1 + 2 * pieces; }
// few: the jobs are those of few rows of hidden states (kStatsT, kGradT, kSumT)
template <typename T> szo_status launch_jobs(Jobs& P, bool few, bool chained, cudaStream_t st);

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
