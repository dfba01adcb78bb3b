// Products in 8-bit integers: y = x W^T with W held as 8-bit integers and a factor for each output channel, and the rows of x brought to 8 bits
// within the call, each with a factor of its own:
//   s[r] = max |x[r]| / 127  (times the fp32 value of 1 / 127: what a tensor's division by 127 is in torch on the GPU, so that a program
//                              that quantizes rows itself finds the same bits; within one unit of the last place of the quotient)
//   q[r] = round(x[r] / s[r])      y[r][n] = s[r] * w_scale[n] * sum over k of q[r][k] w[n][k]
// The sum is exact in int32 (k is at most 2^17: 127 * 127 * 2^17 < 2^31); s and the products around it are fp32.
#include "int8_matmul.h"

#include "rows.h"

namespace dsmoe {

namespace {

// TPR threads a row (a wavefront or a workgroup).  NCH chunks of 8 values a thread stay in registers between the maximum and the rounding; NCH == 0: the row is read
// twice.  The maximum is that of the bits without the sign, so a NaN or an infinity comes out on top: the row's factor is then not finite
// and its values are set to zero, which makes its outputs NaN.  A row whose factor is zero has q = 0.
template <int TY, int TPR, int NCH>
__global__ __launch_bounds__(kRowThreads) void quantize_rows_kernel(const void* x, int64_t x_row, int R, int K, int8_t* q, int64_t q_row, float* scale) {
  __shared__ uint32_t lds[4];
  constexpr int N = NCH ? NCH : 1;
  const int64_t r = (int64_t)blockIdx.x * (kRowThreads / TPR) + threadIdx.x / TPR;
  if (r >= R) return;  // (whole wavefronts)
  const int i0 = threadIdx.x % TPR * 8, n = NCH ? NCH : (int)((q_row + TPR * 8 - 1) / (TPR * 8));
  float v[N][8];
  uint32_t top = 0;
#pragma unroll N
  for (int j = 0; j < n; ++j) {
    const int c = i0 + j * TPR * 8, k = NCH ? j : 0;
    load8<TY>(x, r * x_row + c, K - c, v[k]);
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(v[k][e]) & 0x7fffffffu);
  }
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m));
  if (TPR > 64) {
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = top;
    __syncthreads();
    top = max(max(lds[0], lds[1]), max(lds[2], lds[3]));
  }
  const float s = __uint_as_float(top) * (1.f / 127.f);
  const bool zero = s == 0.f || top >= 0x7f800000u;
  // (a factor below 2^-125 has no finite reciprocal, or one that has lost bits: its quotients are all computed)
  const float inv = s < 0x1p-120f ? 0.f : 1.f / s;
#pragma unroll N
  for (int j = 0; j < n; ++j) {
    const int c = i0 + j * TPR * 8, k = NCH ? j : 0;
    if (c >= q_row) continue;
    if (!NCH) load8<TY>(x, r * x_row + c, K - c, v[k]);
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float t = v[k][e] * inv;
      // within 2^-13 of a half the product with the reciprocal (off by less than 127 * 2^-22) may lie on the other side: there the quotient decides
      if (inv == 0.f || fabsf(fabsf(t - rintf(t)) - 0.5f) < 1.f / 8192) t = v[k][e] / s;
      const int i = zero ? 0 : (int)fminf(fmaxf(rintf(t), -127.f), 127.f);
      w[e >> 2] |= (uint32_t)(i & 0xff) << (8 * (e & 3));
    }
    *(uint2*)(q + r * q_row + c) = make_uint2(w[0], w[1]);  // (rows of q are whole chunks, zeros behind K)
  }
  if (i0 == 0) scale[r] = s;
}

template <int TY, int TPR, int NCH>
void launch_quantize(const Int8Args& a, int8_t* q, int64_t q_row, float* scale, hipStream_t s) {
  const int rows = kRowThreads / TPR;
  quantize_rows_kernel<TY, TPR, NCH><<<dim3((unsigned)((a.R + rows - 1) / rows)), dim3(kRowThreads), 0, s>>>(a.x, a.x_row, a.R, a.K, q, q_row, scale);
}

// Many short rows: a wavefront each, since half of a workgroup would have nothing (whole product, 1024 columns: 6007 rows of 1024 29 -> 27 us, 2101 of
// 512 16.3 -> 14.3; rows of 2048 values 22 -> 24, so those keep a workgroup).
template <int TY>
hipError_t quantize(const Int8Args& a, int8_t* q, int64_t q_row, float* scale, hipStream_t s) {
  if (a.R >= 512 && a.K <= 512)
    launch_quantize<TY, 64, 1>(a, q, q_row, scale, s);
  else if (a.R >= 512 && a.K <= 1024)
    launch_quantize<TY, 64, 2>(a, q, q_row, scale, s);
  else if (a.K <= 2048)
    launch_quantize<TY, kRowThreads, 1>(a, q, q_row, scale, s);
  else if (a.K <= 4096)
    launch_quantize<TY, kRowThreads, 2>(a, q, q_row, scale, s);
  else if (a.K <= 16384)
    launch_quantize<TY, kRowThreads, 8>(a, q, q_row, scale, s);
  else
    launch_quantize<TY, kRowThreads, 0>(a, q, q_row, scale, s);
  return hipGetLastError();
}

// (a stage of the products takes 128 values: zeros to there)
inline int64_t quantized_row(int K) { return ((int64_t)K + 127) / 128 * 128; }
inline int64_t scale_offset(int64_t R, int K) { return (R * quantized_row(K) + 255) / 256 * 256; }

}  // namespace

inline int64_t partial_offset(int64_t R, int K) { return (scale_offset(R, K) + R * 4 + 255) / 256 * 256; }

size_t int8_workspace_bytes(int R, int G, int K, int N) {
  static const int32_t some = 0;
  GroupedArgs g = {};
  g.off = &some;
  g.R = R;
  g.G = G;
  g.K = K;
  g.N = N;
  return (size_t)partial_offset(R, K) + grouped_workspace_bytes(g, kElemI8, true);
}

hipError_t launch_int8_matmul(const Int8Args& a, hipStream_t s) {
  if (a.R == 0) return hipSuccess;
  int8_t* q = (int8_t*)a.workspace;
  float* scale = (float*)(a.workspace + scale_offset(a.R, a.K));
  const int64_t q_row = quantized_row(a.K);
  hipError_t e = a.type == DSMOE_F32    ? quantize<DSMOE_F32>(a, q, q_row, scale, s)
                 : a.type == DSMOE_BF16 ? quantize<DSMOE_BF16>(a, q, q_row, scale, s)
                                        : quantize<DSMOE_F16>(a, q, q_row, scale, s);
  if (e != hipSuccess) return e;
  GroupedArgs g = {};
  g.a = (const char*)q;
  g.b = (const char*)a.w;
  g.c = (char*)a.y;
  g.off = a.offsets;
  g.a_row = q_row;
  g.b_row = a.w_row;
  g.b_group = a.w_group;
  g.c_row = a.y_row * elem_bytes(a.type);
  g.R = a.R;
  g.G = a.G;
  g.N = a.N;
  g.K = a.K;
  g.a_scale = scale;
  g.b_scale = a.w_scale;
  g.bs_group = a.ws_group;
  g.out_type = a.type;
  g.partial = a.workspace + partial_offset(a.R, a.K);
  return launch_grouped(g, kElemI8, true, s);
}

}  // namespace dsmoe
