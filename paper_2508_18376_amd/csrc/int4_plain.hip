// Products with weights in 4 bits, for every type, alignment and number of rows: the tiles of 128 x 128 of grouped_plain.h, whose weights are widened on their way
// from registers to LDS.  16-bit types: (q - z) s is rounded to x's type once, which is what the matrix instructions take; fp32 products are fp32.
// Sums of fp32 go in parts (see Parts); as one chain 4096 rows of 4096 x 14336 took 4030 us, 17 of 14336 x 4096 1135 instead of 1195.
// Bound by the matrix instructions in fp32 (4096 rows of 4096 x 14336 4134 us, 116 of 153 TFLOP/s; few rows are tiles of 128 all the same, 342 us), by the way
// through registers in 16 bits: weights that start off 16 bytes 1088 us, 442 TFLOP/s, where int4_tiles.hip takes 471.
#include "grouped_plain.h"
#include "int4_matmul.h"

namespace dsmoe {

namespace {

// A stage's tile of weights: 128 output channels by 128 bytes of the contraction, as Operand<TY, false> has it in LDS.  A thread widens four chunks of
// 16 bytes (8 values of 16 bits, 4 of fp32): never across two blocks.
template <int TY>
struct Weights4 {
  using E = Elem<TY>;
  static constexpr int VALUES = E::per_chunk, BYTES = VALUES / 2;
  const uint8_t* p[kChunks];
  int64_t s_at[kChunks], z_at[kChunks];
  int first, column, row_bytes, exponent[kChunks];
  // (z: in fp32 the third byte of q, whose weights are two; the register more each would not leave those that Parts takes)
  struct Stage {
    uint32_t q[kChunks], z[TY == kElemF32 ? 1 : kChunks];
    float s[kChunks];
  };

  // n0: first output channel, of which `edge` exist; the last one again behind them
  __device__ __forceinline__ void init(const Int4Args& a, int group, int n0, int edge) {
    const int t = threadIdx.x;
    first = t >> 3;
    column = (t & 7) * VALUES;
    row_bytes = (a.K + 1) / 2;
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      const int64_t c = n0 + min(first + i * 32, edge - 1);
      p[i] = a.w + group * a.w_group + c * a.w_row;
      s_at[i] = group * a.s_group + c * a.s_row;
      z_at[i] = group * a.z_group + c * a.z_row;
      exponent[i] = 0;
      if (TY == kElemF16) {  // eight threads a channel
        uint32_t top = 0;
        for (int j = t & 7; j < a.blocks; j += 8) top = max(top, __float_as_uint(int4_scale(a, s_at[i] + j)) & 0x7fffffffu);
#pragma unroll
        for (int m = 1; m < 8; m <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m));
        exponent[i] = int4_exponent(top);
      }
    }
  }
  __device__ __forceinline__ void load(const Int4Args& a, Stage& v, int k0) const {
    const int k = k0 + column, at = k >> 1, left = row_bytes - at, block = min(k >> a.shift, a.blocks - 1);
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      v.q[i] = 0;
      if (left >= BYTES) {
        __builtin_memcpy(&v.q[i], p[i] + at, BYTES);
      } else {
#pragma unroll
        for (int b = 0; b < BYTES; ++b)
          if (b < left) v.q[i] |= (uint32_t)p[i][at + b] << (8 * b);
      }
      v.s[i] = int4_scale(a, s_at[i] + block);
      const uint32_t z = a.zero ? a.zero[z_at[i] + block] : 8;
      if (TY == kElemF32)
        v.q[i] |= z << 16;
      else
        v.z[TY == kElemF32 ? 0 : i] = z;
    }
  }
  __device__ __forceinline__ void store(char* tile, const Stage& v) const {
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      const float s = TY == kElemF16 ? ldexpf(v.s[i], -exponent[i]) : v.s[i];
      const float z = (float)(TY == kElemF32 ? v.q[i] >> 16 : v.z[TY == kElemF32 ? 0 : i]);
      float f[VALUES];
#pragma unroll
      for (int e = 0; e < VALUES; ++e) f[e] = ((float)(v.q[i] >> (4 * e) & 15) - z) * s;
      pi32x4 out;
#pragma unroll
      for (int d = 0; d < 4; ++d)
        out[d] = TY == kElemF32 ? (int)__float_as_uint(f[d])
                                : (int)((uint32_t)f32_to_16(f[2 * d % VALUES], TY) | (uint32_t)f32_to_16(f[(2 * d + 1) % VALUES], TY) << 16);
      const int r = first + i * 32;
      *(pi32x4*)(tile + r * kStageK + swz_wide(r, column / VALUES) * 16) = out;
    }
  }
};

template <int TY>
__global__ __launch_bounds__(256, 2) void int4_plain_kernel(Int4Args a) {
  using E = Elem<TY>;
  __shared__ __align__(16) char lds[4 * kTileBytes];
  __shared__ float unit[kPT];  // what the channels' sums are taken times
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, NT = (a.N + kPT - 1) / kPT;
  Segments all;
  all.init(a.off, a.G, a.R);
  all.zero_others(a.y, a.y_row, a.N * E::bytes);
  Segment s;
  int piece, rt, nt;
  if (!all.find(kPT, NT, [](int n) { return piece_of(blockIdx.x, n); }, piece, s)) return;
  band_tile(piece - s.base, (s.rows + kPT - 1) / kPT, NT, rt, nt);
  const int m0 = rt * kPT, n0 = nt * kPT, m_edge = min(kPT, s.rows - m0), n_edge = min(kPT, a.N - n0), K = a.K;

  Acc<TY> acc[2][2];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int q = 0; q < 16; ++q) acc[i >> 1][i & 1].v[q] = 0;
  Parts<TY == kElemF32> parts;
  Operand<TY, false> oa;
  Weights4<TY> ob;
  oa.init(a.x + (int64_t)(s.row0 + m0) * a.x_row, a.x_row, m_edge, 0);
  ob.init(a, s.group, n0, n_edge);
  if ((threadIdx.x & 7) == 0) {
#pragma unroll
    for (int i = 0; i < kChunks; ++i) unit[ob.first + i * 32] = ldexpf(1.f, ob.exponent[i]);
  }
  const int mw = (w & 1) * 64, nw = (w >> 1) * 64;
  pi32x4 va[2][kChunks];
  typename Weights4<TY>::Stage vb[2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (i * E::k_stage < K) {
      oa.load(va[i], K - i * E::k_stage);
      ob.load(a, vb[i], i * E::k_stage);
    }
  for (int k = 0; k < K; k += 2 * E::k_stage) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int at = k + i * E::k_stage, left = K - at;
      if (left <= 0) break;
      char *ta = lds + i * 2 * kTileBytes, *tb = ta + kTileBytes;
      oa.store(ta, va[i]);
      ob.store(tb, vb[i]);
      __syncthreads();  // (this buffer's last readers passed the barrier of the stage before)
      if (left > 2 * E::k_stage) {
        oa.load(va[i], left - 2 * E::k_stage);
        ob.load(a, vb[i], at + 2 * E::k_stage);
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        pi32x4 fa[2], fb[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          fa[j] = oa.read(ta, mw + 32 * j, q, lane);
          fb[j] = oa.read(tb, nw + 32 * j, q, lane);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j >> 1][j & 1].mac(fb[j & 1], fa[j >> 1]);
      }
    }
    parts.step(acc);
  }
  parts.end(acc);
  __syncthreads();

  // as grouped_plain_kernel stores its tile
  char* turn = lds + w * (32 * 272);
  constexpr int ob_ = E::bytes, per16 = 16 / ob_, lanes = 64 / per16;
  const int r32 = lane & 31;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int c = j * 32 + 8 * q + 4 * (lane >> 5);
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = acc[i][j].get(4 * q + e) * (TY == kElemF16 ? unit[nw + c + e] : 1.f);
        if (TY == kElemF32) {
          *(pf32x4*)(turn + r32 * 272 + c * 4) = pf32x4{v[0], v[1], v[2], v[3]};
        } else {
          uint2 h;
          h.x = (uint32_t)f32_to_16(v[0], TY) | (uint32_t)f32_to_16(v[1], TY) << 16;
          h.y = (uint32_t)f32_to_16(v[2], TY) | (uint32_t)f32_to_16(v[3], TY) << 16;
          *(uint2*)(turn + r32 * 272 + c * 2) = h;
        }
      }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const int c = nw + lane % lanes * per16;
    for (int r0 = 0; r0 < 32; r0 += 64 / lanes) {
      const int rr = r0 + lane / lanes;
      if (mw + i * 32 + rr >= m_edge || c >= n_edge) continue;
      const pi32x4 v = *(const pi32x4*)(turn + rr * 272 + (c - nw) * ob_);
      char* to = a.y + (int64_t)(s.row0 + m0 + mw + i * 32 + rr) * a.y_row + (int64_t)(n0 + c) * ob_;
      if (c + per16 <= n_edge) {
        __builtin_memcpy(to, &v, 16);
      } else {
        const uint32_t words[4] = {(uint32_t)v[0], (uint32_t)v[1], (uint32_t)v[2], (uint32_t)v[3]};
#pragma unroll
        for (int e = 0; e < 7; ++e)
          if (c + e < n_edge) {
            if (ob_ == 4 && e < 3) ((uint32_t*)to)[e] = words[e & 3];
            if (ob_ == 2) ((uint16_t*)to)[e] = (uint16_t)(words[e >> 1] >> (16 * (e & 1)));
          }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

}  // namespace

hipError_t launch_int4_plain(const Int4Args& a, hipStream_t s) {
  const int64_t blocks = row_tiles_bound(a.R, a.G, a.off != nullptr, kPT) * ((a.N + kPT - 1) / kPT);
  if (blocks == 0) return hipSuccess;
  const dim3 grid((unsigned)blocks), threads(256);
  switch (a.type) {
    case kElemF32: int4_plain_kernel<kElemF32><<<grid, threads, 0, s>>>(a); break;
    case kElemBF16: int4_plain_kernel<kElemBF16><<<grid, threads, 0, s>>>(a); break;
    default: int4_plain_kernel<kElemF16><<<grid, threads, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace dsmoe
