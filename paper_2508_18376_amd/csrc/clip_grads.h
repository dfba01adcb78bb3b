// The norm over all gradients, and clipping by it: arguments of the launches.
#pragma once
#include "common.h"

namespace dsmoe {

constexpr int kMostNormSums = 2048;  // workgroups of a launch, and sums that they leave

size_t clip_grads_bytes();
// max_norm is not looked at where no gradient is written (clip false)
hipError_t launch_clip_grads(const dsmoe_grad* grads, int count, bool clip, float max_norm, float eps, float* norm, double* sums, hipStream_t s);

}  // namespace dsmoe
