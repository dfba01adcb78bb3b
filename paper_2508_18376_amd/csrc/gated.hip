// The gated half of a block of experts, over groups of rows:
//   forward    a = x W1, b = x W3, h = f(a) * b                                    one launch of pairs of products (gated_pair.hip)
//   backward   da = dh * b * f'(a), db = dh * f(a)                                 the kernel below, from a and b as the forward pass summed them, in fp32
//              dx = da W1^T + db W3^T                                              one launch of sums of two products (gated_sum.hip)
//              dW1 = x^T da, dW3 = x^T db                                          the products of moe_grouped_matmul_dw
// The matrix instructions take operands of 16 bits, so da and db are rounded to x's type, once; a and b are not: kept in 16 bits they would put as much
// error again into each of da and db as that rounding does.
#include "gated.h"

#include "rows.h"

namespace dsmoe {

namespace {

// 8 values a thread, TPR threads a row.  Bound by memory: dh, a, b in, da, db out (65536 rows of 1024 in bf16: 940 MB in 167 us, 5.6 TB/s).
template <int TY, int TPR>
__global__ __launch_bounds__(kRowThreads) void gated_slopes_kernel(const void* dh, int64_t dh_row, const float* saved, int R, int N, int act, void* da, void* db,
                                                                    int64_t out_row) {
  const int64_t r = (int64_t)blockIdx.x * (kRowThreads / TPR) + threadIdx.x / TPR;
  if (r >= R) return;
  const float *a = saved + r * N, *b = a + (int64_t)R * N;
  for (int c = threadIdx.x % TPR * 8; c < N; c += TPR * 8) {
    float d[8], u[8], v[8], du[8], dv[8];
    load8<TY>(dh, r * dh_row + c, N - c, d);
    load8<DSMOE_F32>(a, c, N - c, u);
    load8<DSMOE_F32>(b, c, N - c, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float f, slope;
      activation_slope(act, u[e], f, slope);
      du[e] = d[e] * v[e] * slope;
      dv[e] = d[e] * f;
    }
    store8<TY>(da, r * out_row + c, N - c, du);
    store8<TY>(db, r * out_row + c, N - c, dv);
  }
}

template <int TY>
hipError_t slopes(const GatedArgs& a, void* da, void* db, int64_t row, hipStream_t s) {
  const int chunks = (a.N + 7) / 8;
  auto go = [&](auto kernel, int tpr) {
    const int rows = kRowThreads / tpr;
    kernel<<<dim3((unsigned)((a.R + rows - 1) / rows)), dim3(kRowThreads), 0, s>>>(a.dh, a.h_row, a.saved, a.R, a.N, a.act, da, db, row);
    return hipGetLastError();
  };
  if (chunks <= 16) return go(gated_slopes_kernel<TY, 16>, 16);
  if (chunks <= 64) return go(gated_slopes_kernel<TY, 64>, 64);
  return go(gated_slopes_kernel<TY, 256>, 256);
}

inline int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
// rows of da and db start on 16 bytes whatever N is
inline int64_t slope_row(const GatedArgs& a) { return up(a.N, 16 / elem_bytes(a.type)); }
inline int64_t slope_bytes(const GatedArgs& a) { return up(a.R * slope_row(a) * elem_bytes(a.type), 256); }

GroupedArgs base(const GatedArgs& a) {
  static const int32_t some = 0;
  GroupedArgs g = {};
  g.off = a.offsets ? a.offsets : a.G > 1 ? &some : nullptr;  // (sizes of workspaces are asked for without a table)
  g.R = a.R;
  g.G = a.G;
  return g;
}
GroupedArgs forward_args(const GatedArgs& a) {
  const int64_t e = elem_bytes(a.type);
  GroupedArgs g = base(a);
  g.a = (const char*)a.x;
  g.b = (const char*)a.w1;
  g.b2 = (const char*)a.w3;
  g.c = (char*)a.h;
  g.a_row = a.x_row * e;
  g.b_row = a.w_row * e;
  g.b_group = a.w_group * e;
  g.c_row = a.h_row * e;
  g.N = a.N;
  g.K = a.K;
  g.sums = a.saved;
  g.act = a.act;
  g.partial = a.workspace;
  return g;
}
GroupedArgs dx_args(const GatedArgs& a) {
  const int64_t e = elem_bytes(a.type);
  GroupedArgs g = base(a);
  g.a = a.workspace;
  g.a2 = a.workspace + slope_bytes(a);
  g.b = (const char*)a.w1;
  g.b2 = (const char*)a.w3;
  g.c = (char*)a.dx;
  g.a_row = slope_row(a) * e;
  g.b_row = a.w_row * e;
  g.b_group = a.w_group * e;
  g.c_row = a.K * e;
  g.N = a.K;
  g.K = a.N;
  g.partial = a.workspace + 2 * slope_bytes(a);
  return g;
}
GroupedArgs dw_args(const GatedArgs& a) {
  const int64_t e = elem_bytes(a.type);
  GroupedArgs g = base(a);
  g.a = (const char*)a.x;
  g.b = a.workspace;
  g.b2 = a.workspace + slope_bytes(a);
  g.c = (char*)a.dw1;
  g.c2 = (char*)a.dw3;
  g.a_row = a.x_row * e;
  g.b_row = slope_row(a) * e;
  g.c_row = a.N * e;
  g.c_group = (int64_t)a.K * a.N * e;
  g.M = a.K;
  g.N = a.N;
  g.partial = a.workspace + 2 * slope_bytes(a);
  return g;
}

}  // namespace

size_t gated_workspace_bytes(const GatedArgs& a) { return gated_pair_bytes(forward_args(a), a.type); }
size_t gated_backward_workspace_bytes(const GatedArgs& a) {
  const size_t dx = sum_of_two_bytes(dx_args(a), a.type), dw = grouped_dw_workspace_bytes(dw_args(a), a.type);
  return (size_t)(2 * slope_bytes(a)) + (dx > dw ? dx : dw);
}

hipError_t launch_gated(const GatedArgs& a, hipStream_t s) { return launch_gated_pair(forward_args(a), a.type, s); }

hipError_t launch_gated_backward(const GatedArgs& a, hipStream_t s) {
  hipError_t e = hipSuccess;
  if (a.R > 0) {
    char *da = a.workspace, *db = da + slope_bytes(a);
    e = a.type == DSMOE_F32    ? slopes<DSMOE_F32>(a, da, db, slope_row(a), s)
        : a.type == DSMOE_BF16 ? slopes<DSMOE_BF16>(a, da, db, slope_row(a), s)
                               : slopes<DSMOE_F16>(a, da, db, slope_row(a), s);
    if (e == hipSuccess) e = launch_sum_of_two(dx_args(a), a.type, s);
  }
  return e == hipSuccess ? launch_grouped_dw(dw_args(a), a.type, s) : e;
}

}  // namespace dsmoe
