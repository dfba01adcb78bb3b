// Reading, writing and summing up rows of values that may start on any value, 8 values a thread at a time.
#pragma once
#include "common.h"

namespace dsmoe {

constexpr int kRowThreads = 256;

template <int TY>
struct RowElem {
  static constexpr int bytes = TY == DSMOE_F32 ? 4 : 2;
};

template <int TY>
__device__ __forceinline__ float widen(uint16_t v) {
  return TY == DSMOE_BF16 ? bf16_to_f32(v) : (float)__builtin_bit_cast(_Float16, v);
}

// 8 values from i on of the n >= i that p holds, zeros behind them.  Rows may start on any value: a whole chunk is loaded in 16-byte
// pieces wherever it lies.
template <int TY>
__device__ __forceinline__ void load8(const void* p, int64_t i, int left, float (&v)[8]) {
  const char* q = (const char*)p + i * RowElem<TY>::bytes;
  if (left >= 8) {
    if (TY == DSMOE_F32) {
      __builtin_memcpy(v, q, 32);
    } else {
      uint16_t h[8];
      __builtin_memcpy(h, q, 16);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = widen<TY>(h[e]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] = 0.f;
      if (e < left) v[e] = TY == DSMOE_F32 ? ((const float*)q)[e] : widen<TY>(((const uint16_t*)q)[e]);
    }
  }
}

template <int TY>
__device__ __forceinline__ uint16_t narrow(float v) {
  return TY == DSMOE_BF16 ? __builtin_bit_cast(uint16_t, (__bf16)v) : __builtin_bit_cast(uint16_t, (_Float16)v);
}

template <int TY>
__device__ __forceinline__ void store8(void* p, int64_t i, int left, const float (&v)[8]) {
  char* q = (char*)p + i * RowElem<TY>::bytes;
  if (TY == DSMOE_F32) {
    if (left >= 8) {
      __builtin_memcpy(q, v, 32);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < left) ((float*)q)[e] = v[e];
    }
    return;
  }
  uint16_t h[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) h[e] = narrow<TY>(v[e]);
  if (left >= 8) {
    __builtin_memcpy(q, h, 16);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < left) ((uint16_t*)q)[e] = h[e];
  }
}

template <int TY>
__device__ __forceinline__ float load1(const void* p, int64_t i) {
  return TY == DSMOE_F32 ? ((const float*)p)[i] : widen<TY>(((const uint16_t*)p)[i]);
}
template <int TY>
__device__ __forceinline__ void store1(void* p, int64_t i, float v) {
  if (TY == DSMOE_F32)
    ((float*)p)[i] = v;
  else
    ((uint16_t*)p)[i] = narrow<TY>(v);
}

// Sums over the TPR threads of a row, the same bits in each of them.  lds: N * 4 floats, not in use by a sum before the last one.
template <int TPR, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float* lds) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[i] = row_sum(v[i]);
    v[i] += __shfl_xor(v[i], 16);
    v[i] += __shfl_xor(v[i], 32);
  }
  if (TPR > 64) {
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) lds[i * 4 + (threadIdx.x >> 6)] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = (lds[i * 4] + lds[i * 4 + 1]) + (lds[i * 4 + 2] + lds[i * 4 + 3]);
  }
}

}  // namespace dsmoe
