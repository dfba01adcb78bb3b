// Products with weights in 4 bits: arguments of the launches, and what the kernels share.
#pragma once
#include "grouped.h"

namespace dsmoe {

// y[r][c] = sum over the blocks j of a row of s[c][j] * sum over k in block j of x[r][k] (q[c][k] - z[c][j]), for the rows of each group.
struct Int4Args {
  const char* x;
  const uint8_t* w;     // [G][N][(K + 1) / 2], the weight of an even k in the low half of a byte
  const char* scale;    // [G][N][blocks]
  const uint8_t* zero;  // like scale, or nullptr: 8 everywhere
  const int32_t* off;
  char* y;
  int64_t x_row, y_row;                           // in bytes
  int64_t w_row, w_group;                         // in bytes
  int64_t s_row, s_group, z_row, z_group;         // in values (s: of scale_type)
  int32_t R, G, N, K, type, scale_type, shift;    // a block has 2^shift values
  int32_t blocks;
  int32_t parts;  // of the contraction (int4_short.hip), whose sums go to the workspace
  char* partial;  // workspace, or nullptr: none is split
};

hipError_t launch_int4_plain(const Int4Args& a, hipStream_t s);
bool int4_stream_fits(const Int4Args& a);
hipError_t launch_int4_stream(const Int4Args& a, hipStream_t s);
bool int4_short_fits(const Int4Args& a);
size_t int4_short_bytes(const Int4Args& a);  // what a's pointers and strides are does not matter
hipError_t launch_int4_short(Int4Args a, hipStream_t s);
bool int4_tiles_fit(const Int4Args& a);
size_t int4_tiles_bytes(const Int4Args& a);  // what a's pointers and strides are does not matter
hipError_t launch_int4_tiles(const Int4Args& a, hipStream_t s);
size_t int4_workspace_bytes(const Int4Args& a);
hipError_t launch_int4_matmul(const Int4Args& a, hipStream_t s);

__device__ __forceinline__ float int4_scale(const Int4Args& a, int64_t i) { return elem_to_f32(a.scale + i * elem_bytes(a.scale_type), a.scale_type); }

// Half precision has room for 2^-14 .. 2^15 at full precision, and a weight can be of any size.  Where weights go to half precision with their scales, the
// scales of an output channel are taken times the power of two that brings the largest of them to [1, 2) (so weights are below 512), and its sums times
// the inverse.  largest: bits of the largest |scale|; 0, infinite and NaN scales stay as they are.
__device__ __forceinline__ int int4_exponent(uint32_t largest) {
  const float v = __uint_as_float(largest);
  int e = 0;
  if (largest > 0 && largest < 0x7f800000u) (void)frexpf(v, &e);
  return e - (largest > 0 && largest < 0x7f800000u ? 1 : 0);
}

}  // namespace dsmoe
