// What hs_sample's entry point hands to its kernel.
#pragma once

#include "hs_internal.cuh"

namespace hs {

struct SampleParams {
  const uint16_t* logits;
  int64_t stride;
  int32_t n_rows;
  int32_t vocab;
  const int32_t* row_of;
  int32_t n;
  const int32_t* n_dev;
  const float* temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  const float* u;
  int32_t* tokens;
  float* logprob;
  int32_t* kept;
  bool whole;  // all of a row is its head
  bool either; // whether head_kernel sees a row at all depends on the number of draws
  bool all;    // order_kernel takes all draws, not those that are left
  unsigned* err;
};

hs_status launch_sample(SampleParams p, bool fp16, cudaStream_t stream);

}  // namespace hs
