// Products with weights in 4 bits for few rows and few output channels, any alignment, 16-bit x: the weights go straight into registers, and the contraction is
// dealt out among the wavefronts of a workgroup, each with two of its steps under way (one, for more than 16 rows).  Bound by latency: a launch, rounds of loads and the
// sums' way through LDS.  One row of 4096 x 14336 takes 13 us, 30 MB at 2.3 TB/s: a wavefront has four steps there, so that half of the weights are asked for at first
// and the others as those have come, and 224 workgroups leave 32 compute units without one.  16 rows 15 us; from elsewhere than 16 bytes 23 and 25.
//
// A workgroup takes 64 output channels for up to 32 rows of a group.  Its wavefronts take steps of 128 values of the contraction in turn and add their sums up
// through LDS at the end.  A step is spans of SPAN = 128, 64 or 32 values that lie in one block each: lane 16 q + i has channel i of sixteen, and of a span its
// q-th quarter, so that its weights of a span are one load (16, 8 or 4 bytes).
#include <type_traits>

#include "int4_widen.h"

namespace dsmoe {

namespace {

struct Yes {
  static constexpr bool value = true;
};
struct No {
  static constexpr bool value = false;
};

constexpr int kCols4 = 64, kJ4 = kCols4 / 16, kRowFloats4 = kCols4 + 4;

// Loads go through buffers: a base in scalar registers, an offset of 32 bits in each lane and a scalar one.  (From pointers the compiler keeps a 64-bit
// address in each lane for each load of the loop, which leaves no registers for the loads.)  An offset from kBeyond on is out of bounds: it loads zero.
constexpr uint32_t kBeyond = 0x80000000u;
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_at(const void* p) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)(kBeyond - 1), 0x00020000);
}
template <int BYTES>
__device__ __forceinline__ void load_bytes(uint32_t* v, __amdgpu_buffer_rsrc_t b, uint32_t at, int scalar) {
  if constexpr (BYTES == 1) {
    v[0] = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(b, (int)at, scalar, 0);
  } else if constexpr (BYTES == 2) {
    v[0] = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(b, (int)at, scalar, 0);
  } else if constexpr (BYTES == 4) {
    v[0] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(b, (int)at, scalar, 0);
  } else if constexpr (BYTES == 8) {
    const auto x = __builtin_amdgcn_raw_buffer_load_b64(b, (int)at, scalar, 0);
    __builtin_memcpy(v, &x, 8);
  } else {
    const auto x = __builtin_amdgcn_raw_buffer_load_b128(b, (int)at, scalar, 0);
    __builtin_memcpy(v, &x, 16);
  }
}

// What a lane holds of a step, as it lies in memory.  S32: scales in fp32.
template <int SPAN_, int STEP_, int NR, bool S32>
struct Step4 {
  static constexpr int SPAN = SPAN_, STEP = STEP_, SPANS = STEP / SPAN, WORDS = SPAN / 32;  // words of a span's weights in a lane
  static constexpr int SB = SPANS * (S32 ? 4 : 2), ZB = SPANS;    // bytes of a channel's scales and zero points
  uint32_t w[kJ4][SPANS][WORDS], x[NR][SPANS][WORDS][4], s[kJ4][SB < 4 ? 1 : SB / 4], z[kJ4];
};

template <int TY, int SPAN, int NR, int W, bool S32>
__global__ __launch_bounds__(64 * W, 2) void int4_stream_kernel(Int4Args a) {
  extern __shared__ __align__(16) char lds[];
  constexpr int J = kJ4;
  // whole steps, and what is left behind them in steps of 32 values, guarded
  constexpr int kStep4 = SPAN == 32 && NR == 2 ? 64 : 128;  // (128: more registers than there are)
  typedef Step4<SPAN, kStep4, NR, S32> S;
  typedef Step4<32, 32, NR, S32> Rest;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, q = lane >> 4;
  const int NT = (a.N + kCols4 - 1) / kCols4;
  Segments all;
  all.init(a.off, a.G, a.R);
  all.zero_others(a.y, a.y_row, a.N * 2);
  Segment seg;
  int piece, rt, nt;
  if (!all.find(16 * NR, NT, [](int n) { return piece_of(blockIdx.x, n); }, piece, seg)) return;
  band_tile(piece - seg.base, (seg.rows + 16 * NR - 1) / (16 * NR), NT, rt, nt);
  const int m0 = rt * 16 * NR, n0 = nt * kCols4, rows = min(16 * NR, seg.rows - m0), cols = min(kCols4, a.N - n0), K = a.K;
  const int row_bytes = (K + 1) / 2;
  // (the launch checks that offsets from here on fit)
  const char* px = a.x + (int64_t)(seg.row0 + m0) * a.x_row;
  const char* pw = (const char*)a.w + seg.group * a.w_group + n0 * a.w_row;
  const char* ps = a.scale + (seg.group * a.s_group + n0 * a.s_row) * (S32 ? 4 : 2);
  const char* pz = (const char*)a.zero + seg.group * a.z_group + n0 * a.z_row;
  uint32_t x_at[NR], w_at[J], s_at[J], z_at[J];
#pragma unroll
  for (int r = 0; r < NR; ++r) x_at[r] = (uint32_t)min(r * 16 + i, rows - 1) * (uint32_t)a.x_row;
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const uint32_t c = min(16 * j + i, cols - 1);
    w_at[j] = c * (uint32_t)a.w_row;
    s_at[j] = c * (uint32_t)a.s_row * (S32 ? 4 : 2);
    z_at[j] = a.zero ? c * (uint32_t)a.z_row : kBeyond;
  }

  const uint32_t no_zeros = a.zero ? 0 : 0x08080808u;  // (without zero points their loads are out of bounds and give zeros: no branch in the loop)
  const __amdgpu_buffer_rsrc_t bx = buffer_at(px), bw = buffer_at(pw), bs = buffer_at(ps), bz = buffer_at(pz);
  // guard: the last step, whose values beyond K are zeros in x (what the weights hold there does not matter)
  auto load = [&](auto& t, int k0, auto guard) __attribute__((always_inline)) {
    typedef std::remove_reference_t<decltype(t)> T;
    constexpr bool GUARD = decltype(guard)::value;
    constexpr int SP = T::SPAN, EB = S32 ? 4 : 2;
    const int block = k0 >> a.shift;
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int p = 0; p < T::SPANS; ++p) {
        const uint32_t at = w_at[j] + q * (SP / 8) + p * (SP / 2);
        if constexpr (GUARD) {
          static_assert(SP == 32, "four bytes a lane");
          t.w[j][p][0] = 0;
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            uint32_t v;
            load_bytes<1>(&v, bw, k0 / 2 + q * 4 + b < row_bytes ? at + b : kBeyond, k0 / 2);
            t.w[j][p][0] |= v << (8 * b);
          }
        } else {
          load_bytes<T::WORDS * 4>(t.w[j][p], bw, at, k0 / 2);
        }
      }
#pragma unroll
    for (int j = 0; j < J; ++j) load_bytes<T::SB>(t.s[j], bs, s_at[j], block * EB);
#pragma unroll
    for (int j = 0; j < J; ++j) load_bytes<T::ZB>(&t.z[j], bz, z_at[j], block);
#pragma unroll
    for (int r = 0; r < NR; ++r)
#pragma unroll
      for (int p = 0; p < T::SPANS; ++p)
#pragma unroll
        for (int m = 0; m < T::WORDS; ++m) {
          const int k = q * (SP / 4) + p * SP + m * 8;
          if constexpr (GUARD) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              uint32_t v;
              load_bytes<2>(&v, bx, k0 + k + e < K ? x_at[r] + (k + e) * 2 : kBeyond, k0 * 2);
              t.x[r][p][m][e >> 1] = e & 1 ? t.x[r][p][m][e >> 1] | v << 16 : v;
            }
          } else {
            load_bytes<16>(t.x[r][p][m], bx, x_at[r] + k * 2, k0 * 2);
          }
        }
  };
  qf32x4 total[NR][J];  // sixteenths
#pragma unroll
  for (int r = 0; r < NR; ++r)
#pragma unroll
    for (int j = 0; j < J; ++j) total[r][j] = qf32x4{0, 0, 0, 0};
  auto multiply = [&](const auto& t) __attribute__((always_inline)) {
    typedef std::remove_const_t<std::remove_reference_t<decltype(t)>> T;
    const uint32_t one = one_of<TY>();
    const qi32x4 ones = {(int)one, (int)one, (int)one, (int)one};
#pragma unroll
    for (int p = 0; p < T::SPANS; ++p) {
      qf32x4 sum[NR], acc[NR][J];
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        sum[r] = qf32x4{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < J; ++j) acc[r][j] = qf32x4{0, 0, 0, 0};
      }
#pragma unroll
      for (int m = 0; m < T::WORDS; ++m) {
        qi32x4 x[NR];
#pragma unroll
        for (int r = 0; r < NR; ++r) {
          x[r] = paired(qi32x4{(int)t.x[r][p][m][0], (int)t.x[r][p][m][1], (int)t.x[r][p][m][2], (int)t.x[r][p][m][3]});
          mac4<TY>(sum[r], x[r], ones);
        }
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const qi32x4 w = widened<TY>(t.w[j][p][m], one);
#pragma unroll
          for (int r = 0; r < NR; ++r) mac4<TY>(acc[r][j], x[r], w);
        }
      }
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const float s = scale_of<TY, S32>(S32 ? t.s[j][p] : t.s[j][p / 2] >> (16 * (p & 1)) & 0xffff);
        const float z = zero_of((t.z[j] | no_zeros) >> (8 * p) & 0xff);
#pragma unroll
        for (int r = 0; r < NR; ++r)
#pragma unroll
          for (int v = 0; v < 4; ++v) total[r][j][v] += s * (acc[r][j][v] - z * sum[r][v]);
      }
      __builtin_amdgcn_sched_barrier(0);  // (one span's sums at a time: those of several do not fit the registers)
    }
  };
  const int whole = K / kStep4, n = whole > wave ? (whole - wave + W - 1) / W : 0;
  constexpr int DEPTH = NR == 1 ? 2 : 1;  // steps under way
  S st[DEPTH];
#pragma unroll
  for (int d = 0; d < DEPTH; ++d)
    if (d < n) load(st[d], (wave + d * W) * kStep4, No());
  int t = 0;
  for (; t + 2 * DEPTH <= n; t += DEPTH) {
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      multiply(st[d]);
      load(st[d], (wave + (t + DEPTH + d) * W) * kStep4, No());
    }
  }
  for (; t < n; t += DEPTH) {
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
      if (t + d < n) {
        multiply(st[d]);
        if (t + DEPTH + d < n) load(st[d], (wave + (t + DEPTH + d) * W) * kStep4, No());
      }
  }
  if (wave == W - 1) {
#pragma unroll 1
    for (int k0 = whole * kStep4; k0 < K; k0 += 32) {
      Rest rest;
      load(rest, k0, Yes());
      multiply(rest);
    }
  }

  // a lane's sums: rows 4 q .. + 3 of sixteen, channel 16 j + i
  float* mine = (float*)lds + wave * (16 * kRowFloats4);
  constexpr int PT = 16 * kCols4 / (64 * W);
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    if (r > 0) __syncthreads();
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int v = 0; v < 4; ++v) mine[(4 * q + v) * kRowFloats4 + 16 * j + i] = total[r][j][v];
    __syncthreads();
    const int o = threadIdx.x * PT, row = o / kCols4, col = o % kCols4, rr = r * 16 + row;
    if (rr < rows) {
      uint16_t* y = (uint16_t*)(a.y + (int64_t)(seg.row0 + m0 + rr) * a.y_row) + n0 + col;
#pragma unroll
      for (int p = 0; p < PT; ++p) {
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) v += ((const float*)lds)[w * (16 * kRowFloats4) + row * kRowFloats4 + col + p];
        v *= 16.f;
        if (col + p < cols) y[p] = f32_to_16(__builtin_isfinite(v) ? v : sum_again<TY>(a, seg.group, seg.row0 + m0 + rr, n0 + col + p, 0, K), TY);
      }
    }
  }
}

template <int TY, int SPAN, int NR, int W, bool S32>
hipError_t launch(const Int4Args& a, hipStream_t s) {
  constexpr int bytes = W * 16 * kRowFloats4 * 4;
  const int64_t pieces = row_tiles_bound(a.R, a.G, a.off != nullptr, 16 * NR) * ((a.N + kCols4 - 1) / kCols4);
  int4_stream_kernel<TY, SPAN, NR, W, S32><<<dim3((unsigned)pieces), dim3(64 * W), bytes, s>>>(a);
  return hipGetLastError();
}

template <int TY, int SPAN>
hipError_t launch_span(const Int4Args& a, hipStream_t s) {
  const bool one = a.R <= 16 * (int64_t)a.G;
  if (a.scale_type == kElemF32) return one ? launch<TY, SPAN, 1, 8, true>(a, s) : launch<TY, SPAN, 2, 8, true>(a, s);
  return one ? launch<TY, SPAN, 1, 8, false>(a, s) : launch<TY, SPAN, 2, 8, false>(a, s);
}
template <int TY>
hipError_t launch_type(const Int4Args& a, hipStream_t s) {
  return a.shift == 5 ? launch_span<TY, 32>(a, s) : a.shift == 6 ? launch_span<TY, 64>(a, s) : launch_span<TY, 128>(a, s);
}

}  // namespace

// A launch of 2^32 threads and more is silently cut short: a workgroup of 512 threads for 16 rows and 64 channels.
bool int4_stream_fits(const Int4Args& a) {
  if (a.type == kElemF32) return false;
  const int64_t most = (int64_t)1 << 24;  // 64 rows of it are below 2^32
  if (a.x_row > most || a.w_row > most || a.s_row * 4 > most || (a.zero && a.z_row > most)) return false;
  return row_tiles_bound(a.R, a.G, a.off != nullptr, 16) * ((a.N + kCols4 - 1) / kCols4) * 512 < (int64_t)1 << 32 && a.R <= 32 * (int64_t)a.G;
}
hipError_t launch_int4_stream(const Int4Args& a, hipStream_t s) { return a.type == kElemBF16 ? launch_type<kElemBF16>(a, s) : launch_type<kElemF16>(a, s); }

}  // namespace dsmoe
