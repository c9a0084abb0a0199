// Groups of sequences that share their first positions: kernel-side view (kv8_prefix.cu).
#pragma once
#include "kv8_attention.cuh"

namespace szo {
namespace kv8 {

struct Prefix {
  const int32_t *len, *seqs;
  int n_groups, max_seqs;
};

#ifdef __CUDACC__
// What a group shares: sequences [first, last), len positions (whole pages) read through the table of `first`
struct Shared {
  int first, last, len;
};
__device__ __forceinline__ Shared load_shared(const View& V, const Prefix& P, int g, bool report) {
  Shared s{0, 0, 0};
  if (g < 0) return s;
  s.last = V.batch;
  if (P.seqs != nullptr) {
    s.first = P.seqs[g];
    s.last = P.seqs[g + 1];
  }
  const int n = P.len[g];
  if (s.first < 0 || s.last < s.first || s.last > V.batch || s.last - s.first > P.max_seqs || n < 0 ||
      n > static_cast<int64_t>(V.max_pages) << V.page_shift) {
    if (report) atomicExch(V.status, static_cast<int32_t>(SZO_ERR_SHAPE));
    return Shared{0, 0, 0};
  }
  s.len = s.first == s.last ? 0 : n >> V.page_shift << V.page_shift;
  return s;
}
// The group of sequence b, or -1: the last one that starts at or before b, if it holds b
__device__ __forceinline__ int group_of(const Prefix& P, int b) {
  if (P.n_groups == 0 || P.seqs == nullptr) return P.n_groups - 1;
  int lo = 0, hi = P.n_groups;                                    // seqs[lo] <= b < seqs[hi], as far as they ascend
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (P.seqs[mid] <= b) lo = mid;
    else hi = mid;
  }
  return P.seqs[lo] <= b && b < P.seqs[lo + 1] ? lo : -1;
}
#endif

}  // namespace kv8
}  // namespace szo
