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

// The backward pass, TPR threads a row of up to 8 TPR values (8 a thread), S = 2 column sums (dbranch_weight, dweight), 3 with a gate per
// channel.  Rows are dealt out to the sets of TPR threads; each set keeps its rows' column sums in registers and leaves them as a row of the partial table.
// The two sums that a row needs depend on each other, but the second is linear in the first: with q = b' (branch_weight + offset), times the gate where that
// varies inside the row, and d = dy + u / rms(y),
//   sum of q dx = sum of q d - (sum of u y' / (d rms(y))) * sum of q y'
// so one exchange between the wavefronts gives all three.  Where dh lies along y the difference cancels more than q dx does: the error of a gate's gradient is
// then 1.1 - 1.2 times that of the sum as it stands (both in fp32 on the CPU, rms over 400 rows of 512 and of 4096; 1.0 otherwise).
// The next row's values are on their way while this one is worked on: without that and with two exchanges 8192 rows of 4096 took 145 us; now 84.
// A last chunk that is not whole is the row's last 8 values: what it has in common with the chunk before it comes out the same in both, and only
// counts once in the sums.
template <int TY>
struct RawRow {  // 8 values as they lie in memory
  static constexpr int W = TY == DSMOE_F32 ? 8 : 4;
  uint32_t w[W];
  template <bool SHORT>  // rows of fewer than 8 values, too
  __device__ __forceinline__ void load(const void* p, int64_t i, int n) {
    const char* q = (const char*)p + i * RowElem<TY>::bytes;
    if (n >= 8) {
      __builtin_memcpy(w, q, 4 * W);
    } else {
#pragma unroll
      for (int j = 0; j < W; ++j) w[j] = 0;
#pragma unroll
      for (int e = 0; e < (SHORT ? 8 : 0); ++e)
        if (e < n) {
          if (TY == DSMOE_F32)
            w[e % W] = ((const uint32_t*)q)[e];
          else
            w[e / 2 % W] |= (uint32_t)((const uint16_t*)q)[e] << (16 * (e & 1));
        }
    }
  }
  __device__ __forceinline__ float operator[](int e) const {
    if (TY == DSMOE_F32) return __uint_as_float(w[e % W]);
    if (TY == DSMOE_BF16) return __uint_as_float(e & 1 ? w[e / 2 % W] & 0xffff0000u : w[e / 2 % W] << 16);
    return (float)__builtin_bit_cast(_Float16, (uint16_t)(w[e / 2 % W] >> (16 * (e & 1))));
  }
};

// what fits into 128 registers with the next row's values in them: four wavefronts to a SIMD, two workgroups of 512 threads to a compute unit
constexpr bool lean(int type, int gate) { return type != DSMOE_F32 && gate <= kGateToken; }

template <int TY, int TPR, int GATE>
__global__ __launch_bounds__(TPR < kThreads ? kThreads : TPR, lean(TY, GATE) && TPR >= 256 ? 4 : 1) void block_norm_backward_kernel(BlockNormArgs a) {
  constexpr int THREADS = TPR < kThreads ? kThreads : TPR, RW = THREADS / TPR, S = GATE == kGateChannel ? 3 : 2, NW = TPR / 64;
  __shared__ float lds[2][3][NW];
  const int tid = threadIdx.x % TPR, D = a.D;
  const int n = tid * 8 >= D ? 0 : D < 8 ? D : 8;         // values of this thread
  const int c = tid * 8 + 8 > D && D >= 8 ? D - 8 : tid * 8;  // ... from this column on
  const int lead = n > 0 ? tid * 8 - c : 0;                  // ... of which the first ones are another thread's too
  const int set = blockIdx.x * RW + threadIdx.x / TPR, sets = gridDim.x * RW;
  const float inv_d = 1.f / D;
  float wb[8], wy[8], gc[8], cs[S][8];
  {
    RawRow<TY> rb, ry, rg;
    rb.template load<TPR == 64>(a.branch_weight, c, n);
    ry.template load<TPR == 64>(a.weight, c, n);
    if (GATE == kGateChannel) rg.template load<TPR == 64>(a.gate, c, n);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      wb[e] = rb[e] + a.offset;
      wy[e] = ry[e] + a.offset;
      gc[e] = GATE == kGateChannel ? rg[e] * a.scale : 0.f;
    }
  }
#pragma unroll
  for (int s = 0; s < S; ++s)
#pragma unroll
    for (int e = 0; e < 8; ++e) cs[s][e] = 0.f;
  constexpr bool AHEAD = TPR < 1024 || lean(TY, GATE);
  RawRow<TY> b, x, dh, dy, gf;
  float inv_b, inv_y, gt;
  auto load = [&](int64_t t) __attribute__((always_inline)) {
    b.template load<TPR == 64>(a.branch, t * a.branch_row + c, n);
    x.template load<TPR == 64>(a.x, t * a.x_row + c, n);
    dh.template load<TPR == 64>(a.dh, t * a.dh_row + c, n);
    dy.template load<TPR == 64>(a.dy, t * a.dy_row + c, n);
    if (GATE == kGateFull) gf.template load<TPR == 64>(a.gate, t * a.gate_row + c, n);
    inv_b = a.stats[t];
    inv_y = a.stats[a.T + t];
    gt = GATE == kGateToken ? load1<TY>(a.gate, t * a.gate_row) * a.scale : a.scale;
  };
  if (AHEAD && set < a.T) load(set);
  int turn = 0;
  for (int64_t t = set; t < a.T; t += sets, turn ^= 1) {  // (a workgroup of one row at a time, or wavefronts on their own)
    if (!AHEAD) load(t);
    const float ib = inv_b, iy = inv_y, g0 = gt;  // g0: the gate's factor that the whole row has
    float bh[8], yh[8], dx[8], g[8], dhy[8], sum[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (GATE == kGateChannel) g[e] = gc[e];
      if (GATE == kGateFull) g[e] = gf[e] * a.scale;
      if (GATE <= kGateToken) g[e] = 1.f;
      bh[e] = b[e] * ib;
      float q = bh[e] * wb[e];
      if (GATE > kGateToken) q *= g[e];
      yh[e] = (GATE > kGateToken ? x[e] + q : x[e] + g0 * q) * iy;
      const float u = dh[e] * wy[e];
      dhy[e] = dh[e] * yh[e];
      dx[e] = dy[e] + iy * u;
      const float us = e < lead ? 0.f : u, qs = e < lead ? 0.f : q;
      sum[0] += us * yh[e];
      sum[1] += qs * dx[e];
      sum[2] += qs * yh[e];
    }
    if (AHEAD && t + sets < a.T) load(t + sets);
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      sum[i] = row_sum(sum[i]);
      sum[i] += __shfl_xor(sum[i], 16);
      sum[i] += __shfl_xor(sum[i], 32);
      if (NW > 1 && (threadIdx.x & 63) == 0) lds[turn][i][threadIdx.x >> 6 & (NW - 1)] = sum[i];
    }
    if (NW > 1) {
      __syncthreads();  // (the other turn's sums have been read before this barrier)
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        sum[i] = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) sum[i] += lds[turn][i][w];
      }
    }
    const float m = sum[0] * inv_d * iy, dot = sum[1] - m * sum[2];  // dot: sum of q dx
    const float f = GATE <= kGateToken ? g0 : 1.f, mv = f * dot * inv_d * ib, fb = f * ib;
    float db[8], dg[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      dx[e] -= yh[e] * m;
      const float first = dx[e] * bh[e], w = GATE <= kGateToken ? wb[e] : wb[e] * g[e];
      db[e] = fb * (dx[e] * w) - bh[e] * mv;
      cs[0][e] += (GATE <= kGateToken ? f : g[e]) * first;
      cs[1][e] += dhy[e];
      if (GATE > kGateToken) dg[e] = a.scale * (first * wb[e]);
      if (S > 2) cs[S - 1][e] += dg[e];
    }
    if (n > 0) {
      store8<TY>(a.dx, t * D + c, TPR == 64 ? n : 8, dx);
      store8<TY>(a.dbranch, t * D + c, TPR == 64 ? n : 8, db);
      if (GATE == kGateFull) store8<TY>(a.dgate, t * D + c, TPR == 64 ? n : 8, dg);
    }
    if (GATE == kGateToken && tid == 0) store1<TY>(a.dgate, t, a.scale * dot);
  }
  if (n > 0) {
#pragma unroll
    for (int s = 0; s < S; ++s) store8<DSMOE_F32>(a.partial, ((int64_t)set * S + s) * D + c, TPR == 64 ? n : 8, cs[s]);
  }
}

// Rows longer than 8192: read again in each step, the column sums kept in the partial table, each thread its own columns.
template <int TY, int S>
__global__ __launch_bounds__(kThreads) void block_norm_backward_long_kernel(BlockNormArgs a) {
  __shared__ float lds[12];
  const int i0 = threadIdx.x * 8, D = a.D;
  const float inv_d = 1.f / D;
  float* part = a.partial + (int64_t)blockIdx.x * S * D;
  for (int s = 0; s < S; ++s)
    for (int c = i0; c < D; c += kThreads * 8)
      for (int e = 0; e < 8 && c + e < D; ++e) part[(int64_t)s * D + c + e] = 0.f;
  for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
    const float inv_b = a.stats[t], inv_y = a.stats[a.T + t];
    float bh[8], yh[8], dx[8], w[8], g[8], dh[8];  // dx without the part that hangs on the row's sum; dh times y'
    float sum[1] = {0.f};
    auto forward = [&](int c) __attribute__((always_inline)) {
      float x[8], wy[8];
      load8<TY>(a.branch, t * a.branch_row + c, D - c, bh);
      load8<TY>(a.x, t * a.x_row + c, D - c, x);
      load8<TY>(a.dh, t * a.dh_row + c, D - c, dh);
      load8<TY>(a.dy, t * a.dy_row + c, D - c, dx);
      gate8<TY>(a, t, c, D - c, g);
      load8<TY>(a.branch_weight, c, D - c, w);
      load8<TY>(a.weight, c, D - c, wy);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool in = c + e < D;
        bh[e] = in ? bh[e] * inv_b : 0.f;
        w[e] += a.offset;
        yh[e] = in ? (x[e] + g[e] * (bh[e] * w[e])) * inv_y : 0.f;
        const float u = in ? dh[e] * (wy[e] + a.offset) : 0.f;
        dh[e] *= yh[e];
        sum[0] += u * yh[e];
        dx[e] += inv_y * u;
      }
    };
    for (int c = i0; c < D; c += kThreads * 8) forward(c);
    row_sums<kThreads>(sum, lds);
    const float m = sum[0] * inv_d * inv_y;
    float two[2] = {0.f, 0.f};  // of v b', and of a gate per token
    for (int c = i0; c < D; c += kThreads * 8) {
      forward(c);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float dg = (dx[e] - yh[e] * m) * bh[e] * w[e];
        two[0] += g[e] * dg;
        two[1] += dg;
      }
    }
    row_sums<kThreads>(two, lds + 4);
    const float mv = two[0] * inv_d;
    for (int c = i0; c < D; c += kThreads * 8) {
      forward(c);
      float db[8], dg[8], first[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        dx[e] -= yh[e] * m;
        first[e] = dx[e] * bh[e];
        dg[e] = a.scale * (first[e] * w[e]);
        db[e] = inv_b * (g[e] * dx[e] * w[e] - bh[e] * mv);
        first[e] *= g[e];
      }
      store8<TY>(a.dx, t * D + c, D - c, dx);
      store8<TY>(a.dbranch, t * D + c, D - c, db);
      if (a.gate_kind == kGateFull) store8<TY>(a.dgate, t * D + c, D - c, dg);
      for (int e = 0; e < 8 && c + e < D; ++e) {
        part[c + e] += first[e];
        part[(int64_t)D + c + e] += dh[e];
        if (S > 2) part[2 * (int64_t)D + c + e] += dg[e];
      }
    }
    if (a.gate_kind == kGateToken && i0 == 0) store1<TY>(a.dgate, t, a.scale * two[1]);
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

// Rows of the partial table: as many sets of threads as the card holds of the kernel, but at least four rows each, so that the table does not become
// the larger part of what is written (1001 rows of 2047, both launches: 1001 sets 21.5 us, 256 sets 19.3).
inline int backward_threads(int D) { return D <= 512 ? 64 : D <= 2048 ? 256 : D <= 4096 ? 512 : 1024; }
inline int partial_sets(int T, int D) {
  if (D > 8192) return T < 256 ? T : 256;
  const int tpr = backward_threads(D), rw = tpr < kThreads ? kThreads / tpr : 1;
  const int most = tpr == 64 ? 4096 : tpr == 256 ? 1024 : tpr == 512 ? 512 : 256, least = 256;
  int sets = T / 4 < least ? (T < least ? T : least) : T / 4;
  if (sets > most) sets = most;
  return (sets + rw - 1) / rw * rw;
}

template <int TY>
hipError_t forward(const BlockNormArgs& a, hipStream_t s) {
  const int D = a.D, rw = D <= 512 ? kThreads / 64 : 1;
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

template <int TY, int GATE>
void launch_backward(const BlockNormArgs& a, int sets, hipStream_t s) {
  const int D = a.D;
  if (D <= 512)
    block_norm_backward_kernel<TY, 64, GATE><<<dim3(sets / 4), dim3(kThreads), 0, s>>>(a);
  else if (D <= 2048)
    block_norm_backward_kernel<TY, 256, GATE><<<dim3(sets), dim3(256), 0, s>>>(a);
  else if (D <= 4096)
    block_norm_backward_kernel<TY, 512, GATE><<<dim3(sets), dim3(512), 0, s>>>(a);
  else if (D <= 8192)
    block_norm_backward_kernel<TY, 1024, GATE><<<dim3(sets), dim3(1024), 0, s>>>(a);
  else
    block_norm_backward_long_kernel<TY, GATE == kGateChannel ? 3 : 2><<<dim3(sets), dim3(kThreads), 0, s>>>(a);
}

template <int TY>
hipError_t backward(const BlockNormArgs& a, hipStream_t s) {
  const int sets = partial_sets(a.T, a.D), S = a.gate_kind == kGateChannel ? 3 : 2;
  if (a.T > 0) {
    switch (a.gate_kind) {
      case kGateNone: launch_backward<TY, kGateNone>(a, sets, s); break;
      case kGateToken: launch_backward<TY, kGateToken>(a, sets, s); break;
      case kGateChannel: launch_backward<TY, kGateChannel>(a, sets, s); break;
      default: launch_backward<TY, kGateFull>(a, sets, s);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  block_norm_columns_kernel<TY><<<dim3((unsigned)((a.D + 63) / 64), S), dim3(1024), 0, s>>>(a, a.T > 0 ? sets : 0, S);
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
  return a.type == DSMOE_F32 ? backward<DSMOE_F32>(a, s) : a.type == DSMOE_BF16 ? backward<DSMOE_BF16>(a, s) : backward<DSMOE_F16>(a, s);
}

}  // namespace dsmoe
