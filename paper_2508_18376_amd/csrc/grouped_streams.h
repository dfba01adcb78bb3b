// Products over groups of few rows (decode steps, short prompts): the weights' stream is all there is, so this path loads each weight
// once, straight into registers, with as many loads under way as fit, and does the rest in the shadow of that.
//
// A workgroup of 8 or 16 wavefronts takes 64 columns of C for up to 32 rows of a group.  The wavefronts deal the contraction out among
// themselves in steps of 32 values (8-bit: 64) and add their sums up through LDS at the end.  Products are 16 x 16 matrix instructions with the
// weights as the first operand:
//   along   (the weights of a column follow each other along the contraction: gradients of x, 8 bits) a lane's 16 bytes of a column are
//           what the instruction takes
//   across  (y = x W) lane i of sixteen loads columns 4 i .. 4 i + 3 of eight contraction rows; instruction j takes the j-th of the four
//           columns from each lane, i.e. columns j, 4 + j, 8 + j ..: the turning around is one byte permutation for two values
// Both operands may start on any value.  Rows past the last one are the last one again (their sums are not stored).
#pragma once
#include "grouped.h"

namespace dsmoe {

namespace {

typedef __bf16 sbf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 sf16x8 __attribute__((ext_vector_type(8)));
typedef int si32x4 __attribute__((ext_vector_type(4)));
typedef float sf32x4 __attribute__((ext_vector_type(4)));

constexpr int kStreamTile = 32;  // rows of a workgroup
// a row of sums in LDS, for J x 16 columns: the four extra ones keep sixteen rows out of each other's banks
constexpr int row_floats(int J) { return 16 * J + 4; }

constexpr int kWordsAhead = 76;  // registers of a lane for the loads under way

// A step is 32 values of the contraction across, and 128 bytes of it along: whole lines.
template <int TY, bool BX>
struct SElem {
  static constexpr int bytes = TY == kElemF32 ? 4 : TY == kElemI8 ? 1 : 2;
  static constexpr int parts = BX || TY == kElemF32 ? 1 : 2;              // matrix instructions a step (fp32: 8, of one part)
  static constexpr int step = parts * (TY == kElemI8 ? 64 : 32);          // values a step
  static constexpr int lane = step / 4 / parts;                           // ... of a lane and part, one after the other in memory
  static constexpr int words = lane * bytes / 4, lane_words = parts * words;  // 32-bit words of these
};
template <int TY>
struct SAcc {
  typedef sf32x4 type;
};
template <>
struct SAcc<kElemI8> {
  typedef si32x4 type;
};

struct Yes {
  static constexpr bool value = true;
};
struct No {
  static constexpr bool value = false;
};

// W (a power of two) words from p, of which `left` values of SZ bytes exist (zeros behind them); `before`: values of the row in front of p.
// A part of them is loaded up to its end and shifted down; only rows shorter than that are loaded value by value.
template <int W, int SZ, bool GUARD, bool ONCE>
__device__ __forceinline__ void load_words(uint32_t* v, const char* p, int left, int before) {
  typedef uint32_t words_t __attribute__((ext_vector_type(W < 4 ? W : 4), aligned(1)));
  constexpr int FULL = W * 4 / SZ;
  if (GUARD && left <= 0) {
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = 0;
    return;
  }
  const int missing = GUARD && left < FULL ? FULL - left : 0;
  if (!GUARD || missing <= before) {
    if (GUARD) p -= missing * SZ;
#pragma unroll
    for (int i = 0; i < W; i += 4) {
      const words_t x = ONCE ? __builtin_nontemporal_load((const words_t*)(p + 4 * i)) : *(const words_t*)(p + 4 * i);
      __builtin_memcpy(v + i, &x, sizeof(x));
    }
    if (GUARD) {
      const int bytes = missing * SZ;
#pragma unroll
      for (int s = W / 2; s > 0; s >>= 1)  // whole words, in powers of two
        if (bytes / 4 & s) {
#pragma unroll
          for (int i = 0; i < W; ++i) v[i] = i + s < W ? v[i + s] : 0;
        }
#pragma unroll
      for (int i = 0; i < W; ++i) v[i] = (uint32_t)(((uint64_t)(i + 1 < W ? v[i + 1] : 0) << 32 | v[i]) >> (bytes % 4 * 8));
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < W; ++i) {
    v[i] = 0;
#pragma unroll
    for (int b = 0; b < 4 / SZ; ++b) {
      const int e = i * (4 / SZ) + b;
      if (e < left) {
        uint32_t x;
        if (SZ == 4) x = *(const uint32_t*)(p + 4 * e);
        if (SZ == 2) x = *(const uint16_t*)(p + 2 * e);
        if (SZ == 1) x = *(const uint8_t*)(p + e);
        v[i] |= x << (8 * SZ * b);
      }
    }
  }
}

// What a lane holds of one step: the weights as they lie in memory, and its part of NR x 16 rows of A.
template <int TY, bool BX, int NR, int J>
struct Step {
  using E = SElem<TY, BX>;
  // along: J columns' chunks; across: 8 contraction rows of J columns
  static constexpr int RW = J * E::bytes / 4, WW = BX ? 8 * RW : J * E::lane_words;
  uint32_t w[WW], a[NR][E::lane_words];
};

template <int TY, bool BX, int NR, int J, int W, bool ONCE>
__device__ __forceinline__ void stream_tile(const GroupedArgs& g, const char* pa, const char* pb, int rows, int n0, int cols, int K,
                                            int wave, typename SAcc<TY>::type (&acc)[NR][J]) {
  using E = SElem<TY, BX>;
  using S = Step<TY, BX, NR, J>;
  const int lane = threadIdx.x & 63, i = lane & 15, q = lane >> 4;
  // offsets from bases that are the same for the whole wavefront (the launch checks that they fit)
  uint32_t a_at[NR], b_at[BX ? 1 : J];
#pragma unroll
  for (int r = 0; r < NR; ++r) a_at[r] = (uint32_t)min(r * 16 + i, rows - 1) * (uint32_t)g.a_row + q * (E::lane * E::bytes);
#pragma unroll
  for (int j = 0; j < (BX ? 1 : J); ++j)
    b_at[j] = BX ? (uint32_t)(q * 8) * (uint32_t)g.b_row + i * (J * E::bytes) : (uint32_t)min(16 * j + i, cols - 1) * (uint32_t)g.b_row + q * (E::lane * E::bytes);

  auto load = [&](S& s, int step, auto guard) __attribute__((always_inline)) {
    constexpr bool GUARD = decltype(guard)::value;
    const int k0 = step * E::step;
    const int left = K - k0 - q * E::lane;  // values of the contraction from the lane's first on
    if (BX) {
      const char* p = pb + k0 * g.b_row;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        load_words<S::RW, E::bytes, GUARD, ONCE>(s.w + e * S::RW, p + b_at[0], e < left ? cols - J * i : 0, n0 + J * i);
        p += g.b_row;
      }
    } else {
      const char* p = pb + (int64_t)k0 * E::bytes;
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int h = 0; h < E::parts; ++h)
          load_words<E::words, E::bytes, GUARD, ONCE>(s.w + j * E::lane_words + h * E::words, p + b_at[j] + h * 64, left - h * (E::step / 2), K - left + h * (E::step / 2));
    }
    const char* p = pa + (int64_t)k0 * E::bytes;
#pragma unroll
    for (int r = 0; r < NR; ++r)
#pragma unroll
      for (int h = 0; h < E::parts; ++h) load_words<E::words, E::bytes, GUARD, false>(s.a[r] + h * E::words, p + a_at[r] + h * 64, left - h * (E::step / 2), K - left + h * (E::step / 2));
  };
  auto multiply = [&](const S& s) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < J; ++j) {
      if constexpr (TY == kElemF32) {
        // 8 instructions of 4 contraction values, each lane's e-th
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
          for (int r = 0; r < NR; ++r)
            acc[r][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(BX ? s.w[e * S::RW + j] : s.w[j * 8 + e]), __uint_as_float(s.a[r][e]), acc[r][j], 0, 0, 0);
      } else {
#pragma unroll
        for (int h = 0; h < E::parts; ++h) {
          si32x4 f;
#pragma unroll
          for (int d = 0; d < 4; ++d)
            f[d] = BX ? (int)__builtin_amdgcn_perm(s.w[(2 * d + 1) * S::RW + (j >> 1)], s.w[2 * d * S::RW + (j >> 1)], j & 1 ? 0x07060302u : 0x05040100u)
                      : (int)s.w[j * E::lane_words + h * 4 + d];
#pragma unroll
          for (int r = 0; r < NR; ++r) {
            const si32x4 x = {(int)s.a[r][h * 4], (int)s.a[r][h * 4 + 1], (int)s.a[r][h * 4 + 2], (int)s.a[r][h * 4 + 3]};
            if constexpr (TY == kElemBF16)
              acc[r][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(sbf16x8, f), __builtin_bit_cast(sbf16x8, x), acc[r][j], 0, 0, 0);
            if constexpr (TY == kElemF16)
              acc[r][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(sf16x8, f), __builtin_bit_cast(sf16x8, x), acc[r][j], 0, 0, 0);
            if constexpr (TY == kElemI8) acc[r][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(f, x, acc[r][j], 0, 0, 0);
          }
        }
      }
    }
  };
  const int whole = K / E::step;
  if (!BX || cols == 16 * J) {
    // the wavefronts deal the steps out among themselves, DEPTH of each under way
    constexpr int DEPTH = kWordsAhead * (J / 4) / (S::WW + NR * E::lane_words) > 1 ? kWordsAhead * (J / 4) / (S::WW + NR * E::lane_words) : 1;
    const int n = whole > wave ? (whole - wave + W - 1) / W : 0;
    S s[DEPTH];
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
      if (d < n) load(s[d], wave + d * W, No());
    int t = 0;
    for (; t + 2 * DEPTH <= n; t += DEPTH) {
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) {
        multiply(s[d]);
        load(s[d], wave + (t + DEPTH + d) * W, No());
      }
    }
    for (; t < n; t += DEPTH) {
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) {
        if (t + d < n) {
          multiply(s[d]);
          if (t + DEPTH + d < n) load(s[d], wave + (t + DEPTH + d) * W, No());
        }
      }
    }
    if (K % E::step != 0 && wave == W - 1) {
      S s1;
      load(s1, whole, Yes());
      multiply(s1);
    }
  } else {
    for (int t = wave; t * E::step < K; t += W) {  // columns past the last one
      S s1;
      load(s1, t, Yes());
      multiply(s1);
    }
  }
}

// MODE: a gated pair and a sum of two deal their two products out to the two halves of the wavefronts.
template <int TY, int OUT, bool BX, int NR, int J, int W, bool ONCE, int MODE>
__device__ __forceinline__ void stream_rows(const GroupedArgs& g, char* lds, const char* pa, const char* pb, char* pc, const float* as,
                                            const float* bs, int64_t row0, int rows, int n0, int cols, int K) {
  constexpr int WP = MODE == kOneProduct ? W : W / 2;  // wavefronts of a product
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, q = lane >> 4;
  typedef typename SAcc<TY>::type acc_t;
  acc_t acc[NR][J];
#pragma unroll
  for (int r = 0; r < NR; ++r)
#pragma unroll
    for (int j = 0; j < J; ++j) acc[r][j] = acc_t{0, 0, 0, 0};
  const int wv = __builtin_amdgcn_readfirstlane(wave), other = MODE == kOneProduct ? 0 : wv / WP;
  stream_tile<TY, BX, NR, J, WP, ONCE>(g, MODE == kSumOfTwo && other ? g.a2 + (pa - g.a) : pa, other ? g.b2 + (pb - g.b) : pb, rows, n0, cols, K, wv - other * WP, acc);
  // A lane's sums: row lane % 16 of sixteen; along: columns 16 j + 4 q .. + 3 from acc[.][j]; across: columns J (4 q + v) + j from acc[.][j][v].
  typedef uint32_t word4 __attribute__((ext_vector_type(4)));
  constexpr int COLS = 16 * J, RF = row_floats(J);
  uint32_t* mine = (uint32_t*)lds + wave * (16 * RF);
  constexpr int OB = OUT == kElemF32 ? 4 : 2, PT = 16 * COLS / (64 * W);  // outputs a thread
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    if (r > 0) __syncthreads();
#pragma unroll
    for (int j = 0; j < J; ++j) {
      word4 v;  // j-th of the lane's quadruples of columns
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int ja = BX ? j % (J / 4) * 4 + e : j, va = BX ? j / (J / 4) : e;
        if constexpr (TY == kElemI8)
          v[e] = (uint32_t)acc[r][ja][va];
        else
          v[e] = __float_as_uint(acc[r][ja][va]);
      }
      *(word4*)(mine + i * RF + (BX ? J * (4 * q + j / (J / 4)) + j % (J / 4) * 4 : 16 * j + 4 * q)) = v;
    }
    __syncthreads();
    const int o = threadIdx.x * PT, row = o / COLS, col = o % COLS, rr = r * 16 + row;
    float out[PT];
#pragma unroll
    for (int p = 0; p < PT; ++p) {
      const uint32_t* at = (const uint32_t*)lds + row * RF + col + p;
      if constexpr (TY == kElemI8) {
        int sum = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) sum += (int)at[w * (16 * RF)];
        out[p] = rr < rows && col + p < cols ? (float)sum * as[rr] * bs[col + p] : 0.f;
      } else {
        out[p] = 0.f;
#pragma unroll
        for (int w = 0; w < (MODE == kGatedPair ? WP : W); ++w) out[p] += __uint_as_float(at[w * (16 * RF)]);
        if constexpr (MODE == kGatedPair) {
          float up = 0.f;
#pragma unroll
          for (int w = WP; w < W; ++w) up += __uint_as_float(at[w * (16 * RF)]);
          if (g.sums != nullptr && rr < rows && col + p < cols) {
            float* to = g.sums + (row0 + rr) * g.N + n0 + col + p;
            to[0] = out[p];
            to[(int64_t)g.R * g.N] = up;
          }
          out[p] = activation(g.act, out[p]) * up;
        }
      }
    }
    if (rr < rows) {
      char* c = pc + rr * g.c_row + (int64_t)col * OB;
#pragma unroll
      for (int p = 0; p < PT; ++p)
        if (col + p < cols) {
          if (OUT == kElemF32)
            ((float*)c)[p] = out[p];
          else
            ((uint16_t*)c)[p] = f32_to_16(out[p], OUT);
        }
    }
  }
}

template <int TY, int OUT, bool BX, int J, int W, bool ONCE, int MODE>
__global__ __launch_bounds__(64 * W, J == 8 ? 2 : 4) void grouped_stream_kernel(GroupedArgs g) {
  extern __shared__ __align__(16) char lds[];
  using E = SElem<TY, BX>;
  constexpr int COLS = 16 * J;
  const int NT = (g.N + COLS - 1) / COLS;
  int piece;
  Segment s;
  Segments all;
  all.init(g.off, g.G, g.R);
  all.zero_others(g.c, g.c_row, g.N * (OUT == kElemF32 ? 4 : 2));
  if (!all.find(kStreamTile, NT, [](int n) { return piece_of(blockIdx.x, n); }, piece, s)) return;
  int rt, nt;
  band_tile(piece - s.base, (s.rows + kStreamTile - 1) / kStreamTile, NT, rt, nt);
  const int m0 = rt * kStreamTile, n0 = nt * COLS, grp = s.group;
  const int64_t row = s.row0 + m0;
  const char* pa = g.a + row * g.a_row;
  const char* pb = g.b + grp * g.b_group + (BX ? (int64_t)n0 * E::bytes : n0 * g.b_row);
  char* pc = g.c + row * g.c_row + (int64_t)n0 * (OUT == kElemF32 ? 4 : 2);
  const float* as = TY == kElemI8 ? g.a_scale + row : nullptr;
  const float* bs = TY == kElemI8 ? g.b_scale + grp * g.bs_group + n0 : nullptr;
  const int rows = min(kStreamTile, s.rows - m0), cols = min(COLS, g.N - n0), K = g.K;
  if (rows <= 16)
    stream_rows<TY, OUT, BX, 1, J, W, ONCE, MODE>(g, lds, pa, pb, pc, as, bs, row, rows, n0, cols, K);
  else
    stream_rows<TY, OUT, BX, 2, J, W, ONCE, MODE>(g, lds, pa, pb, pc, as, bs, row, rows, n0, cols, K);
}

template <int TY, int OUT, bool BX, int J, int W, bool ONCE, int MODE>
hipError_t launch(const GroupedArgs& g, hipStream_t s) {
  constexpr int bytes = W * 16 * row_floats(J) * 4;
  if (bytes > 64 * 1024) {
    static PerDeviceOnce once;
    const hipError_t e =
        once.run([] { return hipFuncSetAttribute((const void*)grouped_stream_kernel<TY, OUT, BX, J, W, ONCE, MODE>, hipFuncAttributeMaxDynamicSharedMemorySize, bytes); });
    if (e != hipSuccess) return e;
  }
  const int64_t pieces = row_tiles_bound(g.R, g.G, g.off != nullptr, kStreamTile) * ((g.N + 16 * J - 1) / (16 * J));
  grouped_stream_kernel<TY, OUT, BX, J, W, ONCE, MODE><<<dim3((unsigned)pieces), dim3(64 * W), bytes, s>>>(g);
  return hipGetLastError();
}

// The weights that a call can touch against the last-level cache (256 MiB): those that do not fit are loaded past it.
// 64 tokens on 8 experts of 4096 x 14336 (0.94 GB) 179 -> 167 us; one token on 64 experts of 2048 x 1024 (34 MB, again and again) would lose, 9.8 ->
// 12.4, as would 333 on 64 of 2048 x 1408 in 8 bits.
constexpr int64_t kLastLevelBytes = 256ll << 20;
// Few pieces: 16 wavefronts to each, so that all of the weights are under way at once (one token on 64 experts of 2048 x 1024, 128 pieces:
// 9.8 us).  Many: whole 256-byte rows of 128 columns across the contraction, in workgroups of 4 wavefronts of which two share a
// compute unit, so that one's beginning and end lie in the other's stream (64 tokens on 8 of 4096 x 14336: 8 wavefronts 171, 4 167; 64
// columns 176).
// Rows that do not start on 16 bytes, of either weight (b2: nullptr for one product), keep to 64 columns, 8 bytes a lane: loads of 16 bytes from elsewhere are slow
// (a gated pair's weights as halves of rows of 2824 values, 64 tokens on 64 experts of 2048 x 1412: 259 us, like this 178).
template <int TY, int OUT, bool BX, int MODE = kOneProduct>
hipError_t launch_w(const GroupedArgs& g, hipStream_t s) {
  const int64_t pieces = row_tiles_bound(g.R, g.G, g.off != nullptr, kStreamTile) * ((g.N + 63) / 64);
  // (a gated pair in fp32 has no registers left for 16)
  if (pieces < 512) return launch<TY, OUT, BX, 4, MODE == kGatedPair && TY == kElemF32 ? 8 : 16, false, MODE>(g, s);
  constexpr bool WIDE = BX && TY != kElemF32;
  if (WIDE && (((uintptr_t)g.b | (uintptr_t)g.b2 | g.b_row | g.b_group) & 15) != 0) return launch<TY, OUT, BX, 4, 8, false, MODE>(g, s);
  const bool once = (int64_t)(g.G < g.R ? g.G : g.R) * g.K * g.N * SElem<TY, BX>::bytes > kLastLevelBytes;
  return once ? launch<TY, OUT, BX, WIDE ? 8 : 4, WIDE ? 4 : 8, true, MODE>(g, s) : launch<TY, OUT, BX, WIDE ? 8 : 4, WIDE ? 4 : 8, false, MODE>(g, s);
}

// Threads of the launch, a workgroup for each piece: few rows of very many columns reach 2^32, where a launch is silently cut short (64 groups of a row each
// and 2^23 columns: 2^23 pieces of 512 threads).  The other paths take those calls: their launches are bounded by the checks at the C boundary.
// aligned: the weights' rows start on 16 bytes (see launch_w).
inline bool launch_holds(const GroupedArgs& g, int type, bool b_along, bool aligned) {
  const int64_t row_tiles = row_tiles_bound(g.R, g.G, g.off != nullptr, kStreamTile);
  const bool wide = !b_along && type != kElemF32 && aligned;
  const int64_t threads = wide ? row_tiles * ((g.N + 127) / 128) * 256 : row_tiles * ((g.N + 63) / 64) * 512;
  return threads < (int64_t)1 << 32;
}

}  // namespace

}  // namespace dsmoe
