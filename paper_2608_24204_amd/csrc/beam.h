// Beam search: the selection over beams and vocabulary, and the reordering of paged caches.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kv8.h"

namespace wici {

struct BeamSelect {
  const void* logits;  // [n * beams] rows, row_stride elements apart
  int bf16;
  int64_t row_stride;
  int n, beams, vocab, k;
  const float* scores;  // [n][beams]
  float* out_scores;    // [n][k]
  int32_t* out_parent;
  int32_t* out_token;
  char* work;           // beam_space bytes
};
hipError_t launch_beam_select(const BeamSelect& a, hipStream_t st);

constexpr int kPoolsALaunch = 64;
// c: the caches' geometry and table (its pool is not used); page_bytes of each page of each pool.
hipError_t launch_beam_reorder(const Kv8& c, size_t page_bytes, void* const* pools, int n_pools,
                               int n, int beams, const int32_t* parent, const int32_t* length,
                               int32_t* table, int32_t* spare, hipStream_t st);

}  // namespace wici
