// Groups of sequences that share their first positions: kernel-side view (kv8_prefix.cu).
#pragma once
#include "kv8_attention.cuh"

namespace szo {
namespace kv8 {

struct Prefix {
  const int32_t *len, *seqs;
  int n_groups, max_seqs;
};

}  // namespace kv8
}  // namespace szo
