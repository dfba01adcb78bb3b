// Norms around a block, with its gate and residual scale:
//   b'  = branch * rsqrt(mean(branch^2) + eps)          y = x + scale * gate * b' * (branch_weight + offset)
//   y'  = y * rsqrt(mean(y^2) + eps)                    h = y' * (weight + offset)
// and the gradients, with g = scale * gate and u = dh * (weight + offset):
//   dx  = dy + (u - y' mean(u y')) / rms(y)             v = g * dx * (branch_weight + offset)
//   dbranch = (v - b' mean(v b')) / rms(branch)         dbranch_weight = sum over tokens of g dx b', dweight of dh y'
//   dgate = scale * dx * b' * (branch_weight + offset), summed over what the gate is broadcast over
// All of it is a few operations a value: memory bounds it.  A row is read once and stays in registers (up to 8192 values) between the two
// sums that it needs, one after the other; y is not rounded before its norm.  All arithmetic is fp32.
#include "block_norm.h"
#include "rows.h"

namespace dsmoe {

namespace {

enum GateKind { kGateNone = 0, kGateToken = 1, kGateChannel = 2, kGateFull = 3 };

constexpr int kThreads = kRowThreads;

// What the values of one chunk take: everything that both directions compute from x, branch, gate and branch_weight.
template <int TY>
__device__ __forceinline__ void gate8(const BlockNormArgs& a, int64_t t, int c, int left, float (&g)[8]) {
  if (a.gate_kind == kGateChannel) {
    load8<TY>(a.gate, c, left, g);
  } else if (a.gate_kind == kGateFull) {
    load8<TY>(a.gate, t * a.gate_row + c, left, g);
  } else {
    const float v = a.gate_kind == kGateToken ? load1<TY>(a.gate, t * a.gate_row) : 1.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) g[e] = v;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) g[e] *= a.scale;
}

// NCH chunks of 8 values a thread, TPR threads a row; NCH == 0: rows longer than 8192, read again in each step.
template <int TY, int TPR, int NCH>
__global__ __launch_bounds__(kThreads) void block_norm_kernel(BlockNormArgs a) {
  __shared__ float lds[8];
  const int64_t t = (int64_t)blockIdx.x * (kThreads / TPR) + threadIdx.x / TPR;
  const int i0 = (threadIdx.x % TPR) * 8, D = a.D;
  if (t >= a.T) return;  // (whole wavefronts: rows share a workgroup only where each has a wavefront)
  constexpr int N = NCH ? NCH : 1;
  const int n = NCH ? NCH : (D + TPR * 8 - 1) / (TPR * 8);
  const float inv_d = 1.f / D;

  float b[N][8], y[N][8], sum[1] = {0.f};
  auto load_branch = [&](int k, int c) { load8<TY>(a.branch, t * a.branch_row + c, D - c, b[k]); };
#pragma unroll N
  for (int j = 0; j < n; ++j) {
    const int k = NCH ? j : 0, c = i0 + j * TPR * 8;
    load_branch(k, c);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[0] += b[k][e] * b[k][e];
  }
  auto residual = [&](int k, int c, float inv_b) {  // y of chunk k
    float x[8], g[8], w[8];
    if (!NCH) load_branch(k, c);
    load8<TY>(a.x, t * a.x_row + c, D - c, x);
    gate8<TY>(a, t, c, D - c, g);
    load8<TY>(a.branch_weight, c, D - c, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) y[k][e] = c + e < D ? x[e] + g[e] * (b[k][e] * inv_b * (w[e] + a.offset)) : 0.f;
  };
  row_sums<TPR>(sum, lds);
  const float inv_b = 1.f / sqrtf(sum[0] * inv_d + a.eps);
  sum[0] = 0.f;
#pragma unroll N
  for (int j = 0; j < n; ++j) {
    const int k = NCH ? j : 0, c = i0 + j * TPR * 8;
    residual(k, c, inv_b);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[0] += y[k][e] * y[k][e];
    store8<TY>(a.y, t * D + c, D - c, y[k]);
  }
  row_sums<TPR>(sum, lds + 4);
  const float inv_y = 1.f / sqrtf(sum[0] * inv_d + a.eps);
#pragma unroll N
  for (int j = 0; j < n; ++j) {
    const int k = NCH ? j : 0, c = i0 + j * TPR * 8;
    if (!NCH) residual(k, c, inv_b);
    float w[8];
    load8<TY>(a.weight, c, D - c, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = y[k][e] * inv_y * (w[e] + a.offset);
    store8<TY>(a.h, t * D + c, D - c, w);
  }
  if (a.stats != nullptr && i0 == 0) {
    a.stats[t] = inv_b;
    a.stats[a.T + t] = inv_y;
  }
}

// Column sums: S = 2 (dbranch_weight, dweight), 3 with a gate per channel.  Each set of TPR threads keeps those of its rows in registers and
// leaves them as a row of the partial table; NCH == 0 keeps them in that table, each thread its own columns.
template <int TY, int TPR, int NCH, int S>
__global__ __launch_bounds__(kThreads) void block_norm_backward_kernel(BlockNormArgs a) {
  __shared__ float lds[12];
  constexpr int RW = kThreads / TPR, N = NCH ? NCH : 1;
  const int i0 = (threadIdx.x % TPR) * 8, D = a.D;
  const int n = NCH ? NCH : (D + TPR * 8 - 1) / (TPR * 8);
  const int set = blockIdx.x * RW + threadIdx.x / TPR, sets = gridDim.x * RW;
  const float inv_d = 1.f / D;
  float* part = a.partial + (int64_t)set * S * D;
  float cs[S][N][8];
#pragma unroll
  for (int s = 0; s < S; ++s)
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) cs[s][k][e] = 0.f;
  if (!NCH)
    for (int s = 0; s < S; ++s)
      for (int c = i0; c < D; c += TPR * 8)
        for (int e = 0; e < 8 && c + e < D; ++e) part[s * D + c + e] = 0.f;

  for (int64_t t = set; t < a.T; t += sets) {  // (a workgroup of one row at a time, or wavefronts on their own)
    const float inv_b = a.stats[t], inv_y = a.stats[a.T + t];
    float bh[N][8], yh[N][8], dx[N][8], w[N][8], g[N][8], dh[N][8];  // b', y', dx, then v, branch_weight + offset
    float sum[1] = {0.f};
    auto forward = [&](int k, int c) {
      float x[8], wy[8];
      load8<TY>(a.branch, t * a.branch_row + c, D - c, bh[k]);
      load8<TY>(a.x, t * a.x_row + c, D - c, x);
      load8<TY>(a.dh, t * a.dh_row + c, D - c, dh[k]);
      load8<TY>(a.dy, t * a.dy_row + c, D - c, dx[k]);
      gate8<TY>(a, t, c, D - c, g[k]);
      load8<TY>(a.branch_weight, c, D - c, w[k]);
      load8<TY>(a.weight, c, D - c, wy);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool in = c + e < D;
        bh[k][e] = in ? bh[k][e] * inv_b : 0.f;
        w[k][e] += a.offset;
        yh[k][e] = in ? (x[e] + g[k][e] * (bh[k][e] * w[k][e])) * inv_y : 0.f;
        const float u = in ? dh[k][e] * (wy[e] + a.offset) : 0.f;
        dh[k][e] *= yh[k][e];  // from here on what dweight sums up
        sum[0] += u * yh[k][e];
        dx[k][e] += inv_y * u;  // the rest follows with the sum
      }
    };
#pragma unroll N
    for (int j = 0; j < n; ++j) forward(NCH ? j : 0, i0 + j * TPR * 8);
    row_sums<TPR>(sum, lds);
    const float m = sum[0] * inv_d * inv_y;
    float two[2] = {0.f, 0.f};  // of v b', and of a gate per token
    auto through = [&](int k) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        dx[k][e] -= yh[k][e] * m;
        const float db = dx[k][e] * bh[k][e], dg = db * w[k][e];
        two[0] += g[k][e] * dg;
        two[1] += dg;
      }
    };
    if (!NCH) sum[0] = 0.f;
#pragma unroll N
    for (int j = 0; j < n; ++j) {
      const int k = NCH ? j : 0, c = i0 + j * TPR * 8;
      if (!NCH) forward(k, c);
      through(k);
    }
    row_sums<TPR>(two, lds + 4);
    const float mv = two[0] * inv_d;
#pragma unroll N
    for (int j = 0; j < n; ++j) {
      const int k = NCH ? j : 0, c = i0 + j * TPR * 8;
      if (!NCH) {
        forward(k, c);
        float keep[2] = {two[0], two[1]};
        through(k);
        two[0] = keep[0];
        two[1] = keep[1];
      }
      float db[8], dg[8], first[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        first[e] = dx[k][e] * bh[k][e];
        dg[e] = a.scale * (first[e] * w[k][e]);
        db[e] = inv_b * (g[k][e] * dx[k][e] * w[k][e] - bh[k][e] * mv);
        first[e] *= g[k][e];
      }
      store8<TY>(a.dx, t * D + c, D - c, dx[k]);
      store8<TY>(a.dbranch, t * D + c, D - c, db);
      if (a.gate_kind == kGateFull) store8<TY>(a.dgate, t * D + c, D - c, dg);
      if (NCH) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          cs[0][k][e] += first[e];
          cs[1][k][e] += dh[k][e];
          if (S > 2) cs[S - 1][k][e] += dg[e];
        }
      } else {
        for (int e = 0; e < 8 && c + e < D; ++e) {
          part[c + e] += first[e];
          part[D + c + e] += dh[k][e];
          if (S > 2) part[2 * (int64_t)D + c + e] += dg[e];
        }
      }
    }
    if (a.gate_kind == kGateToken && i0 == 0) store1<TY>(a.dgate, t, a.scale * two[1]);
  }
  if (NCH) {
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int k = 0; k < N; ++k) store8<DSMOE_F32>(part, (int64_t)s * D + i0 + k * TPR * 8, D - i0 - k * TPR * 8, cs[s][k]);
  }
}

// Sums of the partial table's rows, 64 columns a workgroup: 16 threads a column, each every 16th row.
template <int TY>
__global__ __launch_bounds__(1024) void block_norm_columns_kernel(BlockNormArgs a, int sets, int S) {
  __shared__ float lds[16][64];
  const int lane = threadIdx.x & 63, r = threadIdx.x >> 6, s = blockIdx.y;
  const int64_t c = (int64_t)blockIdx.x * 64 + lane;
  float v = 0.f;
  if (c < a.D) {
    const float* p = a.partial + (int64_t)s * a.D + c;
#pragma unroll 8
    for (int i = r; i < sets; i += 16) v += p[(int64_t)i * S * a.D];
  }
  lds[r][lane] = v;
  __syncthreads();
  if (r == 0 && c < a.D) {
    v = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) v += lds[i][lane];
    store1<TY>(s == 0 ? a.dbranch_weight : s == 1 ? a.dweight : a.dgate, c, v);
  }
}

// Threads of a row, and rows of the partial table
inline int threads_of(int D) { return D <= 512 ? 64 : kThreads; }
inline int partial_sets(int T, int D) {
  const int most = D > 8192 ? 256 : D <= 512 ? 2048 : 512, rw = kThreads / threads_of(D);
  const int sets = T < most ? T : most;
  return (sets + rw - 1) / rw * rw;
}

template <int TY>
hipError_t forward(const BlockNormArgs& a, hipStream_t s) {
  const int D = a.D, rw = kThreads / threads_of(D);
  const dim3 grid((unsigned)((a.T + rw - 1) / rw)), block(kThreads);
  if (D <= 512)
    block_norm_kernel<TY, 64, 1><<<grid, block, 0, s>>>(a);
  else if (D <= 2048)
    block_norm_kernel<TY, kThreads, 1><<<grid, block, 0, s>>>(a);
  else if (D <= 4096)
    block_norm_kernel<TY, kThreads, 2><<<grid, block, 0, s>>>(a);
  else if (D <= 8192)
    block_norm_kernel<TY, kThreads, 4><<<grid, block, 0, s>>>(a);
  else
    block_norm_kernel<TY, kThreads, 0><<<grid, block, 0, s>>>(a);
  return hipGetLastError();
}

template <int TY, int S>
hipError_t backward(const BlockNormArgs& a, hipStream_t s) {
  const int D = a.D, sets = partial_sets(a.T, D), rw = kThreads / threads_of(D);
  if (a.T > 0) {
    const dim3 grid((unsigned)(sets / rw)), block(kThreads);
    if (D <= 512)
      block_norm_backward_kernel<TY, 64, 1, S><<<grid, block, 0, s>>>(a);
    else if (D <= 2048)
      block_norm_backward_kernel<TY, kThreads, 1, S><<<grid, block, 0, s>>>(a);
    else if (D <= 4096)
      block_norm_backward_kernel<TY, kThreads, 2, S><<<grid, block, 0, s>>>(a);
    else if (D <= 8192)
      block_norm_backward_kernel<TY, kThreads, 4, S><<<grid, block, 0, s>>>(a);
    else
      block_norm_backward_kernel<TY, kThreads, 0, S><<<grid, block, 0, s>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  block_norm_columns_kernel<TY><<<dim3((unsigned)((D + 63) / 64), S), dim3(1024), 0, s>>>(a, a.T > 0 ? sets : 0, S);
  return hipGetLastError();
}

}  // namespace

size_t block_norm_backward_bytes(int T, int D, int gate_kind) {
  return (size_t)partial_sets(T, D) * (gate_kind == kGateChannel ? 3 : 2) * (size_t)D * sizeof(float);
}

hipError_t launch_block_norm(const BlockNormArgs& a, hipStream_t s) {
  if (a.T == 0) return hipSuccess;
  return a.type == DSMOE_F32 ? forward<DSMOE_F32>(a, s) : a.type == DSMOE_BF16 ? forward<DSMOE_BF16>(a, s) : forward<DSMOE_F16>(a, s);
}

hipError_t launch_block_norm_backward(const BlockNormArgs& a, hipStream_t s) {
  const bool three = a.gate_kind == kGateChannel;
  switch (a.type) {
    case DSMOE_F32: return three ? backward<DSMOE_F32, 3>(a, s) : backward<DSMOE_F32, 2>(a, s);
    case DSMOE_BF16: return three ? backward<DSMOE_BF16, 3>(a, s) : backward<DSMOE_BF16, 2>(a, s);
    default: return three ? backward<DSMOE_F16, 3>(a, s) : backward<DSMOE_F16, 2>(a, s);
  }
}

}  // namespace dsmoe
