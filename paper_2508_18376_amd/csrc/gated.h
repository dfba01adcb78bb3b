// The gated half of a block of experts: arguments of the launches.
#pragma once
#include "grouped.h"

namespace dsmoe {

struct GatedArgs {
  const void *x, *w1, *w3;
  const int32_t* offsets;
  void* h;       // forward
  float* saved;  // [2][R][N], written by the forward pass (or nullptr), read by the backward pass
  const void* dh;  // backward
  void *dx, *dw1, *dw3;
  int64_t x_row, w_row, w_group, h_row;  // in values; h_row: of h, or of dh
  int32_t R, G, K, N, type, act;
  char* workspace;
};

size_t gated_workspace_bytes(const GatedArgs& a);
size_t gated_backward_workspace_bytes(const GatedArgs& a);
hipError_t launch_gated(const GatedArgs& a, hipStream_t s);
hipError_t launch_gated_backward(const GatedArgs& a, hipStream_t s);

// the products (gated_pair.hip: kGatedPair; gated_sum.hip: kSumOfTwo)
size_t gated_pair_bytes(const GroupedArgs& g, int type);
hipError_t launch_gated_pair(const GroupedArgs& g, int type, hipStream_t s);
size_t sum_of_two_bytes(const GroupedArgs& g, int type);
hipError_t launch_sum_of_two(const GroupedArgs& g, int type, hipStream_t s);

}  // namespace dsmoe
