// norm = sqrt(sum of all squares of all gradients), and out = grad * min(1, max_norm / (norm + eps)).
//
// Two passes of launches, both bound by memory: the first reads the gradients and leaves a sum for each workgroup, the second has each workgroup add those
// up (in the same order, so all get the same bits), and reads and writes the gradients.  Squares and sums are in 64 bits: the largest fp32 or bf16
// value's square is finite there, the smallest one's not zero, and 2^32 terms cost no precision; the vector units do them as fast as fp32 ones.
//
// 2.8 GB of gradients in bf16: 1486 us, 5.7 TB/s.  2 MB in fp32: 4 + 5 us, the launches; the host's call takes 20.
//
// The gradients are dealt out in chunks of 16-byte vectors.  What the workgroups have to know of a tensor travels with the launch, up to kMost tensors in each;
// further launches of the first pass add to the sums that the earlier ones left.
#include "clip_grads.h"

#include "rows.h"

namespace dsmoe {

namespace {

constexpr int kThreads = 256, kMost = 48;
constexpr int64_t kLastLevelBytes = 256ll << 20;

struct Entry {
  const char* in;
  char* out;
  int64_t vectors, first_chunk;    // all of its vectors; chunks of the tensors before it
  int64_t width;                   // values of a row
  int64_t in_row, out_row;         // in bytes
  int32_t per_row, type;           // vectors of a row (of several)
};
struct Entries {
  Entry e[kMost];
  int64_t chunks;
  int32_t count, per_chunk;  // vectors of a chunk
};
static_assert(sizeof(Entries) + 64 <= 4096, "a launch takes 4 KiB of arguments");

typedef uint32_t words_t __attribute__((ext_vector_type(4), aligned(2)));

template <int TY>
struct Vec {
  static constexpr int N = 16 / RowElem<TY>::bytes;
  float v[N];
  // n values exist
  template <bool ONCE>
  __device__ __forceinline__ void load(const char* p, int n) {
    if (n >= N) {
      const words_t x = ONCE ? __builtin_nontemporal_load((const words_t*)p) : *(const words_t*)p;
      uint32_t w[4];
      __builtin_memcpy(w, &x, 16);
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = TY == DSMOE_F32 ? __uint_as_float(w[i * 4 / N]) : widen<TY>((uint16_t)(w[i >> 1] >> (16 * (i & 1))));
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = i < n ? load1<TY>(p, i) : 0.f;
    }
  }
  template <bool ONCE>
  __device__ __forceinline__ void store(char* p, int n) const {
    if (n >= N) {
      uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (TY == DSMOE_F32)
          w[i * 4 / N] = __float_as_uint(v[i]);
        else
          w[i >> 1] |= (uint32_t)narrow<TY>(v[i]) << (16 * (i & 1));
      }
      words_t x;
      __builtin_memcpy(&x, w, 16);
      if (ONCE)
        __builtin_nontemporal_store(x, (words_t*)p);
      else
        *(words_t*)p = x;
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (i < n) store1<TY>(p, i, v[i]);
    }
  }
};

// body(in, out, values that exist) for the thread's vectors of chunk `chunk` of e
template <int TY, class Body>
__device__ __forceinline__ void chunk_vectors(const Entry& e, int64_t chunk, int per_chunk, Body&& body) {
  constexpr int N = Vec<TY>::N, B = RowElem<TY>::bytes;
  const int64_t base = (chunk - e.first_chunk) * per_chunk;
  const int n = (int)min((int64_t)per_chunk, e.vectors - base);
  if (e.per_row == 0) {  // one row
    const int64_t left = e.width - base * N;
    if (n == per_chunk && left >= (int64_t)per_chunk * N) {
#pragma unroll 8
      for (int i = threadIdx.x; i < per_chunk; i += kThreads) body(e.in + (base + i) * 16, e.out + (base + i) * 16, N);
    } else {
      for (int i = threadIdx.x; i < n; i += kThreads) body(e.in + (base + i) * 16, e.out + (base + i) * 16, (int)min((int64_t)N, left - (int64_t)i * N));
    }
    return;
  }
  const int64_t row0 = base / e.per_row;
  const int at0 = (int)(base - row0 * e.per_row);
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const uint32_t at = (uint32_t)at0 + (uint32_t)i, down = at / (uint32_t)e.per_row;
    const int64_t row = row0 + down, c = (int64_t)(at - down * (uint32_t)e.per_row) * N;
    body(e.in + row * e.in_row + c * B, e.out + row * e.out_row + c * B, (int)min((int64_t)N, e.width - c));
  }
}
__device__ __forceinline__ const Entry& entry_of(const Entries& t, int64_t chunk) {
  int i = 0;
  for (int left = t.count; left > 1;) {  // the last tensor that begins at or before the chunk is among t.e[i] .. t.e[i + left - 1]
    const int half = left >> 1;
    if (t.e[i + half].first_chunk <= chunk) {
      i += half;
      left -= half;
    } else {
      left = half;
    }
  }
  return t.e[i];
}

__device__ __forceinline__ double block_sum(double v) {
  __shared__ double lds[kThreads / 64];
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

__global__ __launch_bounds__(kThreads) void norm_sums_kernel(Entries t, double* sums, int first) {
  double sum = 0;
  for (int64_t c = blockIdx.x; c < t.chunks; c += gridDim.x) {
    const Entry& e = entry_of(t, c);
    auto add = [&](auto ty) {
      constexpr int TY = decltype(ty)::value;
      chunk_vectors<TY>(e, c, t.per_chunk, [&](const char* in, char*, int n) {
        Vec<TY> v;
        v.template load<false>(in, n);
#pragma unroll
        for (int i = 0; i < Vec<TY>::N; ++i) sum = fma((double)v.v[i], (double)v.v[i], sum);
      });
    };
    if (e.type == DSMOE_F32)
      add(std::integral_constant<int, DSMOE_F32>());
    else if (e.type == DSMOE_BF16)
      add(std::integral_constant<int, DSMOE_BF16>());
    else
      add(std::integral_constant<int, DSMOE_F16>());
  }
  sum = block_sum(sum);
  if (threadIdx.x == 0) sums[blockIdx.x] = first ? sum : sums[blockIdx.x] + sum;
}

// the norm, from n sums: the same bits in every workgroup
__device__ __forceinline__ float norm_of(const double* sums, int n) {
  double v = 0;
  for (int i = threadIdx.x; i < n; i += kThreads) v += sums[i];
  return (float)sqrt(block_sum(v));
}

__global__ __launch_bounds__(kThreads) void norm_kernel(const double* sums, int n, float* norm) {
  const float v = norm_of(sums, n);
  if (threadIdx.x == 0) *norm = v;
}

// Chunks are taken from the last one on: what the first pass read last is in the last-level cache still.  ONCE: gradients that do not fit that cache are
// loaded and stored past it (1.4 G values in bf16: both passes 1580 -> 1486 us; 5.9 TB/s in the first, 5.6 in the second).
template <bool ONCE>
__global__ __launch_bounds__(kThreads) void clip_kernel(Entries t, const double* sums, int n, float max_norm, float eps, float* norm) {
  const float length = norm_of(sums, n), ratio = max_norm / (length + eps), factor = ratio >= 1.f ? 1.f : ratio;
  if (blockIdx.x == 0 && threadIdx.x == 0) *norm = length;
  for (int64_t c = t.chunks - 1 - blockIdx.x; c >= 0; c -= gridDim.x) {
    const Entry& e = entry_of(t, c);
    if (factor == 1.f && e.in == e.out) continue;
    auto scale = [&](auto ty) {
      constexpr int TY = decltype(ty)::value;
      chunk_vectors<TY>(e, c, t.per_chunk, [&](const char* in, char* out, int k) {
        Vec<TY> v;
        v.template load<ONCE>(in, k);
#pragma unroll
        for (int i = 0; i < Vec<TY>::N; ++i) v.v[i] *= factor;
        v.template store<ONCE>(out, k);
      });
    };
    if (e.type == DSMOE_F32)
      scale(std::integral_constant<int, DSMOE_F32>());
    else if (e.type == DSMOE_BF16)
      scale(std::integral_constant<int, DSMOE_BF16>());
    else
      scale(std::integral_constant<int, DSMOE_F16>());
  }
}

inline int64_t vectors_of(const dsmoe_grad& g) {
  const int64_t n = g.dtype == DSMOE_F32 ? 4 : 8;
  return (g.width + n - 1) / n * g.rows;
}

}  // namespace

size_t clip_grads_bytes() { return kMostNormSums * sizeof(double); }

hipError_t launch_clip_grads(const dsmoe_grad* grads, int count, bool clip, float max_norm, float eps, float* norm, double* sums, hipStream_t s) {
  int64_t all = 0;
  for (int i = 0; i < count; ++i) all += vectors_of(grads[i]);
  const int per_chunk = all >= (int64_t)kMostNormSums * 2048 ? 2048 : 512;
  // tensors [from, to) of a launch; each launch of a pass has the same workgroups
  auto fill = [&](Entries& t, int from, int& to) {
    t.chunks = t.count = 0;
    t.per_chunk = per_chunk;
    for (to = from; to < count && t.count < kMost; ++to) {
      const dsmoe_grad& g = grads[to];
      Entry& e = t.e[t.count];
      e.vectors = vectors_of(g);
      if (e.vectors == 0) continue;
      e.in = (const char*)g.grad;
      e.out = (char*)g.out;
      e.first_chunk = t.chunks;
      e.width = g.width;
      e.in_row = g.grad_stride * (g.dtype == DSMOE_F32 ? 4 : 2);
      e.out_row = g.out_stride * (g.dtype == DSMOE_F32 ? 4 : 2);
      e.per_row = g.rows > 1 ? (int32_t)(e.vectors / g.rows) : 0;
      e.type = g.dtype;
      t.chunks += (e.vectors + per_chunk - 1) / per_chunk;
      ++t.count;
    }
  };
  Entries t;
  int64_t most = 1;
  for (int from = 0, to; from < count; from = to) {
    fill(t, from, to);
    most = t.chunks > most ? t.chunks : most;
  }
  const int blocks = (int)(most < kMostNormSums ? most : kMostNormSums);
  hipError_t e = hipSuccess;
  for (int from = 0, to; from < count && e == hipSuccess; from = to) {
    fill(t, from, to);
    norm_sums_kernel<<<dim3(blocks), dim3(kThreads), 0, s>>>(t, sums, from == 0);
    e = hipGetLastError();
  }
  if (e != hipSuccess) return e;
  if (!clip) {
    norm_kernel<<<dim3(1), dim3(kThreads), 0, s>>>(sums, blocks, norm);
    return hipGetLastError();
  }
  for (int from = 0, to; from < count && e == hipSuccess; from = to) {
    fill(t, from, to);
    if (all * 16 > kLastLevelBytes)
      clip_kernel<true><<<dim3(blocks), dim3(kThreads), 0, s>>>(t, sums, blocks, max_norm, eps, norm);
    else
      clip_kernel<false><<<dim3(blocks), dim3(kThreads), 0, s>>>(t, sums, blocks, max_norm, eps, norm);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace dsmoe
