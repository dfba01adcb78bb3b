// The norms around a block: arguments of the launches.
#pragma once
#include "common.h"

namespace dsmoe {

struct BlockNormArgs {
  const void *x, *branch, *gate, *branch_weight, *weight;
  int64_t x_row, branch_row, gate_row;  // in values
  int32_t T, D, gate_kind, type;
  float scale, offset, eps;
  float* stats;  // [2][T]: 1 / rms of the branch's rows and of y's
  // forward
  void *y, *h;
  // backward
  const void *dy, *dh;
  int64_t dy_row, dh_row;
  void *dx, *dbranch, *dgate, *dbranch_weight, *dweight;
  float* partial;  // column sums of a workgroup's rows
};

size_t block_norm_backward_bytes(int T, int D, int gate_kind);
hipError_t launch_block_norm(const BlockNormArgs& a, hipStream_t s);
hipError_t launch_block_norm_backward(const BlockNormArgs& a, hipStream_t s);

}  // namespace dsmoe
