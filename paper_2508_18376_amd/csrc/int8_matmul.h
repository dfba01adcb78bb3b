// Products in 8-bit integers: arguments of the launches.
#pragma once
#include "grouped.h"

namespace dsmoe {

struct Int8Args {
  const void* x;
  int64_t x_row;  // in values
  const int8_t* w;
  int64_t w_row, w_group;
  const float* w_scale;
  int64_t ws_group;
  const int32_t* offsets;
  void* y;
  int64_t y_row;  // in values
  int32_t R, G, N, K, type;
  char* workspace;
};

size_t int8_workspace_bytes(int R, int G, int K, int N);
hipError_t launch_int8_matmul(const Int8Args& a, hipStream_t s);

}  // namespace dsmoe
