// Products with weights in 4 bits for groups of few rows (16-bit x, rows on 16 bytes): tiles of 16, 32 or 64 rows by 256 output channels.
//
// Bound by memory where blocks are long (128 rows on 8 groups of 4096 x 14336, scales in fp32 74 us of kernel, 5.1 TB/s; a third of the bytes are lines of scales
// fetched again stage by stage, without which it takes 64), else by the chains of products and sums of the two wavefronts that a SIMD holds (1998 rows on 64
// groups of 2048 x 1408 60 us; without loads 54, without products 34): one reads while the other multiplies.
//
// A workgroup of 4 wavefronts, 64 channels each, goes through the contraction in stages of 128 values.  A stage's weights (64 bytes a channel), x (256 bytes a
// row), scales and zero points all come to LDS by loads without registers in between, two workgroups to a compute unit, 64 to 96 KiB under way.  The detour
// is for the addresses: neighbouring lanes load neighbouring bytes here, while a lane that loads what the matrix instructions want of it has a
// line of its own, and a compute unit looks up one line a clock (straight into registers, 64 tokens on 8 experts of 4096 x 14336 took 174 us, 77 million
// lookups).
//
// In LDS a channel's 64 bytes have their four 16-byte chunks rotated by a quarter of the channel, a row's 256 bytes theirs by the row (exclusive or), so that the
// lanes of a read lie in different banks.  A stage is spans of SPAN = 128, 64 or 32 values that lie in one block each.
#include "int4_widen.h"

namespace dsmoe {

namespace {

constexpr int kCols = 256, kStage = 128, kWeights = kCols * kStage / 2;
constexpr uint32_t kBeyond = 0x80000000u;

template <int SPAN, int NR>
struct Shape {
  static constexpr int SPANS = kStage / SPAN, WORDS = SPAN / 32, ROWS = 16 * NR;
  static constexpr int x_at = kWeights, s_at = x_at + ROWS * kStage * 2, bytes = s_at + SPANS * 2 * kCols * 4;
  static constexpr int room = 160 * 1024 / (NR == 1 ? 3 : 2);              // of a workgroup in LDS: three (two) to a compute unit
  static constexpr int ring = room / bytes < 2 ? 2 : room / bytes < 4 ? room / bytes : 4;  // stages
  static constexpr int loads = 4 + NR + 2 * SPANS;                    // of a wavefront and stage
};

// BYTES (1, 2, 4 or 16) a lane to LDS: at lds + 4 (16) times the lane, of values of less than 4 bytes widened
template <int BYTES>
__device__ __forceinline__ void to_lds(const qi32x4& rsrc, uint32_t lds, uint32_t at) {
  if constexpr (BYTES == 16)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(at), "s"(rsrc) : "memory");
  if constexpr (BYTES == 4)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(lds), "v"(at), "s"(rsrc) : "memory");
  if constexpr (BYTES == 2)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_ushort %1, %2, 0 offen lds" ::"s"(lds), "v"(at), "s"(rsrc) : "memory");
  if constexpr (BYTES == 1)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_ubyte %1, %2, 0 offen lds" ::"s"(lds), "v"(at), "s"(rsrc) : "memory");
}
__device__ __forceinline__ qi32x4 buffer(const void* p, int64_t extent) {
  const uint64_t base = (uint64_t)(uintptr_t)p;
  return qi32x4{__builtin_amdgcn_readfirstlane((int)(uint32_t)base), __builtin_amdgcn_readfirstlane((int)(uint32_t)(base >> 32)),
                __builtin_amdgcn_readfirstlane((int)extent), 0x00020000};
}
template <int N>
__device__ __forceinline__ void loads_but() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Where piece `piece` of all lies: `parts` pieces a tile, neighbours in the contraction.
struct Place {
  Segment seg;
  int m0, n0, rows, cols, part;
};
__device__ __forceinline__ bool place_of(const Int4Args& a, const Segments& all, int BM, int piece, Place& p) {
  const int NT = (a.N + kCols - 1) / kCols;
  int found;
  if (!all.find(BM, NT * a.parts, [&](int n) { return piece < n ? piece : n; }, found, p.seg)) return false;
  const int id = found - p.seg.base, tile = id / a.parts;
  p.part = id - tile * a.parts;
  int rt, nt;
  band_tile(tile, (p.seg.rows + BM - 1) / BM, NT, rt, nt);
  p.m0 = rt * BM;
  p.n0 = nt * kCols;
  p.rows = min(BM, p.seg.rows - p.m0);
  p.cols = min(kCols, a.N - p.n0);
  return true;
}

template <int TY, int SPAN, int NR, bool S32>
__global__ __launch_bounds__(256, NR == 1 ? 3 : 2) void int4_short_kernel(Int4Args a) {
  extern __shared__ __align__(16) char ring[];
  typedef Shape<SPAN, NR> Sh;
  constexpr int J = 4, EB = S32 ? 4 : 2, RING = Sh::ring;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, q = lane >> 4;
  Segments all;
  all.init(a.off, a.G, a.R);
  all.zero_others(a.y, a.y_row, a.N * 2);
  Place p;
  {
    int total;
    Segment s;
    const int NT = (a.N + kCols - 1) / kCols * a.parts;
    if (!all.find(Sh::ROWS, NT, [](int n) { return piece_of(blockIdx.x, n); }, total, s)) return;
    if (!place_of(a, all, Sh::ROWS, total, p)) return;
    total = __builtin_amdgcn_readfirstlane(total);
    p.seg.total = total;  // (this piece's number: where its sums go, if they are not all)
  }
  const int stages = (a.K + kStage - 1) / kStage, first = (int)((int64_t)stages * p.part / a.parts), n = (int)((int64_t)stages * (p.part + 1) / a.parts) - first;
  const char* px = a.x + (int64_t)(p.seg.row0 + p.m0) * a.x_row;
  const char* pw = (const char*)a.w + p.seg.group * a.w_group + p.n0 * a.w_row;
  const char* ps = a.scale + (p.seg.group * a.s_group + p.n0 * a.s_row) * EB;
  const char* pz = (const char*)a.zero + p.seg.group * a.z_group + p.n0 * a.z_row;
  // a lane's offsets: channel lane / 4 of sixteen and one of its chunks; row lane / 16 of four; channel `lane` of 64
  uint32_t w_off[4], x_off[NR], x_chunk[NR], s_off, z_off;
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const int c = t * 16 + (lane >> 2);
    w_off[t] = (uint32_t)min(w * 64 + c, p.cols - 1) * (uint32_t)a.w_row + ((lane & 3) ^ (c >> 2 & 3)) * 16;
  }
#pragma unroll
  for (int t = 0; t < NR; ++t) {
    const int r = (w * NR + t) * 4 + (lane >> 4);
    x_chunk[t] = (lane & 15) ^ (r & 15);
    x_off[t] = r < p.rows ? (uint32_t)r * (uint32_t)a.x_row + x_chunk[t] * 16 : kBeyond;
  }
  s_off = (uint32_t)min(w * 64 + lane, p.cols - 1) * (uint32_t)a.s_row * EB;
  z_off = (uint32_t)min(w * 64 + lane, p.cols - 1) * (uint32_t)a.z_row;
  const uint32_t lds = (uint32_t)(uintptr_t)((__attribute__((address_space(3))) const char*)ring);

  auto load = [&](int st) __attribute__((always_inline)) {  // stage st of the piece, into its place
    const int k0 = (first + st) * kStage, left = min(a.K - k0, kStage);  // values of the contraction that exist (K is a multiple of 8)
    const uint32_t to = lds + (uint32_t)(st % RING) * Sh::bytes;
    const qi32x4 bw = buffer(pw + k0 / 2, (p.cols - 1) * a.w_row + left / 2), bx = buffer(px + (int64_t)k0 * 2, (p.rows - 1) * a.x_row + left * 2);
#pragma unroll
    for (int t = 0; t < 4; ++t) to_lds<16>(bw, to + w * 4096 + t * 1024, w_off[t]);
#pragma unroll
    for (int t = 0; t < NR; ++t) to_lds<16>(bx, to + Sh::x_at + (w * NR + t) * 1024, (int)x_chunk[t] * 8 < left ? x_off[t] : kBeyond);
#pragma unroll
    for (int s = 0; s < Sh::SPANS; ++s) {
      const int block = min((k0 + s * SPAN) >> a.shift, a.blocks - 1);
      const qi32x4 bs = buffer(ps + (int64_t)block * EB, ((p.cols - 1) * a.s_row + 1) * EB);
      // (without zero points the buffer is empty, and gives zeros)
      const qi32x4 bz = buffer(pz + block, a.zero ? (p.cols - 1) * a.z_row + 1 : 0);
      to_lds<EB>(bs, to + Sh::s_at + (s * 2 * kCols + w * 64) * 4, s_off);
      to_lds<1>(bz, to + Sh::s_at + ((s * 2 + 1) * kCols + w * 64) * 4, z_off);
    }
  };
  qf32x4 total[NR][J];  // sixteenths
#pragma unroll
  for (int r = 0; r < NR; ++r)
#pragma unroll
    for (int j = 0; j < J; ++j) total[r][j] = qf32x4{0, 0, 0, 0};
  // What is taken off for the zero points, the sum of x times (16 + z) s, is a product over the spans itself: of four spans at a time, the q-th one's factors in
  // lanes 16 q .., by the fp32 matrix instructions (by the vector units it is a quarter of their instructions: 1998 rows on 64 groups of 2048 x 1408 60.5 us
  // instead of 58.5).
  float xs[NR], zs[J];
#pragma unroll
  for (int r = 0; r < NR; ++r) xs[r] = 0;
#pragma unroll
  for (int j = 0; j < J; ++j) zs[j] = 0;
  const uint32_t no_zeros = a.zero ? 0 : 8, one = one_of<TY>();
  // BLOCKS of sixteen rows
  auto multiply = [&](const char* at, int st, auto blocks) __attribute__((always_inline)) {
    constexpr int BLOCKS = decltype(blocks)::value;
    const qi32x4 ones = {(int)one, (int)one, (int)one, (int)one};
    constexpr int WORDS = Sh::WORDS;
#pragma unroll
    for (int s = 0; s < Sh::SPANS; ++s) {
      const int place = (st * Sh::SPANS + s) & 3;
      const float mine = q == place ? 1.f : 0.f;
      qf32x4 sum[BLOCKS], acc[BLOCKS][J];
#pragma unroll
      for (int r = 0; r < BLOCKS; ++r) {
        sum[r] = qf32x4{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < J; ++j) acc[r][j] = qf32x4{0, 0, 0, 0};
      }
      uint32_t wd[J][WORDS];
      const int o = s * (SPAN / 2) + q * (SPAN / 8);
#pragma unroll
      for (int j = 0; j < J; ++j)
        __builtin_memcpy(wd[j], __builtin_assume_aligned(at + w * 4096 + (16 * j + i) * 64 + ((o >> 4) ^ (i >> 2)) * 16 + (o & 15), WORDS * 4), WORDS * 4);
#pragma unroll
      for (int m = 0; m < WORDS; ++m) {
        qi32x4 x[BLOCKS];
#pragma unroll
        for (int r = 0; r < BLOCKS; ++r) {
          x[r] = paired(*(const qi32x4*)(at + Sh::x_at + (16 * r + i) * 256 + ((s * (SPAN / 8) + q * WORDS + m) ^ i) * 16));
          mac4<TY>(sum[r], ones, x[r]);
        }
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const qi32x4 v = widened<TY>(wd[j][m], one);
#pragma unroll
          for (int r = 0; r < BLOCKS; ++r) mac4<TY>(acc[r][j], x[r], v);
        }
      }
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const uint32_t* sz = (const uint32_t*)(at + Sh::s_at) + s * 2 * kCols + w * 64 + 16 * j + i;
        const float f = scale_of<TY, S32>(sz[0]), z = zero_of(sz[kCols] | no_zeros);
        zs[j] = fmaf(-f * z, mine, zs[j]);
#pragma unroll
        for (int r = 0; r < BLOCKS; ++r)
#pragma unroll
          for (int v = 0; v < 4; ++v) total[r][j][v] = fmaf(f, acc[r][j][v], total[r][j][v]);
      }
#pragma unroll
      for (int r = 0; r < BLOCKS; ++r)
        xs[r] = fmaf(sum[r][0], mine, xs[r]);
      if (place == 3 || (s == Sh::SPANS - 1 && st == n - 1)) {
#pragma unroll
        for (int j = 0; j < J; ++j) {
#pragma unroll
          for (int r = 0; r < BLOCKS; ++r) total[r][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(xs[r], zs[j], total[r][j], 0, 0, 0);
          zs[j] = 0;
        }
#pragma unroll
        for (int r = 0; r < BLOCKS; ++r) xs[r] = 0;
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
#pragma unroll
  for (int st = 0; st < RING - 1; ++st)
    if (st < n) load(st);
  auto stages_of = [&](auto blocks) __attribute__((always_inline)) {
    for (int st = 0; st < n; ++st) {
      // stage st is there for every wavefront, and every wavefront has read the one before, whose place stage st + RING - 1 takes
      const int behind = min(RING - 2, n - 1 - st);
      if (behind >= 2)
        loads_but<2 * Sh::loads>();
      else if (behind == 1)
        loads_but<Sh::loads>();
      else
        loads_but<0>();
      meet();
      if (st + RING - 1 < n) load(st + RING - 1);
      if (w * 64 < p.cols) multiply(ring + (st % RING) * Sh::bytes, st, blocks);
    }
  };
  const int blocks = (p.rows + 15) / 16;
  if constexpr (NR >= 4) {
    if (blocks == 4) stages_of(std::integral_constant<int, 4>());
    if (blocks == 3) stages_of(std::integral_constant<int, 3>());
  }
  if constexpr (NR >= 2)
    if (blocks == 2) stages_of(std::integral_constant<int, 2>());
  if (blocks == 1) stages_of(std::integral_constant<int, 1>());
  meet();

  // The wavefront turns sixteen rows of its 64 channels around in LDS at a time: rows of 256 bytes whose 64-byte blocks are rotated by a quarter of the row.
  char* turn = ring + w * 4096;
  char* sums = a.partial + (int64_t)p.seg.total * (Sh::ROWS * kCols * 4);
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    bool finite = true;
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const float sum = 16.f * total[r][j][v];
        finite = finite && __builtin_isfinite(sum);
        *(float*)(turn + (4 * q + v) * 256 + ((j ^ q) * 16 + i) * 4) = sum;
      }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (__any(!finite)) {
#pragma unroll 1
      for (int row = 0; row < 16; ++row) {  // the lane's channel of each row
        float* at = (float*)(turn + row * 256 + ((q ^ (row >> 2)) * 16 + i) * 4);
        if (!__builtin_isfinite(*at) && r * 16 + row < p.rows && w * 64 + lane < p.cols)
          *at = sum_again<TY>(a, p.seg.group, p.seg.row0 + p.m0 + r * 16 + row, p.n0 + w * 64 + lane, first * kStage, min(a.K, (first + n) * kStage));
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int row = h * 8 + (lane >> 3), c = (lane & 7) * 8, rr = r * 16 + row;
      const char* from = turn + row * 256 + ((c >> 4) ^ (row >> 2)) * 64 + (c & 15) * 4;
      const qf32x4 lo = *(const qf32x4*)from, hi = *(const qf32x4*)(from + 16);
      if (rr < p.rows && w * 64 + c < p.cols) {
        if (a.parts > 1) {
          qf32x4* to = (qf32x4*)(sums + (rr * kCols + w * 64 + c) * 4);
          to[0] = lo;
          to[1] = hi;
        } else {
          uint32_t out[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float u = e < 2 ? lo[2 * e] : hi[2 * e - 4], v = e < 2 ? lo[2 * e + 1] : hi[2 * e - 3];
            out[e] = (uint32_t)f32_to_16(u, TY) | (uint32_t)f32_to_16(v, TY) << 16;
          }
          *(uint4*)(a.y + (int64_t)(p.seg.row0 + p.m0 + rr) * a.y_row + (int64_t)(p.n0 + w * 64 + c) * 2) = make_uint4(out[0], out[1], out[2], out[3]);
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

// Adds up a tile's parts, in order: a thread eight channels of a row (blockIdx.x: the tile; blockIdx.y: eight of its rows).
template <int TY, int ROWS>
__global__ __launch_bounds__(256) void int4_join_kernel(Int4Args a) {
  Segments all;
  all.init(a.off, a.G, a.R);
  Place p;
  const int piece = blockIdx.x * a.parts;
  if (!place_of(a, all, ROWS, piece, p)) return;
  const int r = blockIdx.y * 8 + (threadIdx.x >> 5), c = (threadIdx.x & 31) * 8;
  if (r >= p.rows || c >= p.cols) return;
  const char* from = a.partial + (int64_t)piece * (ROWS * kCols * 4) + (r * kCols + c) * 4;
  qf32x4 lo = *(const qf32x4*)from, hi = *(const qf32x4*)(from + 16);
  for (int s = 1; s < a.parts; ++s) {
    from += ROWS * kCols * 4;
    lo += *(const qf32x4*)from;
    hi += *(const qf32x4*)(from + 16);
  }
  uint32_t out[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float u = e < 2 ? lo[2 * e] : hi[2 * e - 4], v = e < 2 ? lo[2 * e + 1] : hi[2 * e - 3];
    out[e] = (uint32_t)f32_to_16(u, TY) | (uint32_t)f32_to_16(v, TY) << 16;
  }
  *(uint4*)(a.y + (int64_t)(p.seg.row0 + p.m0 + r) * a.y_row + (int64_t)(p.n0 + c) * 2) = make_uint4(out[0], out[1], out[2], out[3]);
}

inline int64_t most_tiles(const Int4Args& a, int rows) { return row_tiles_bound(a.R, a.G, a.off != nullptr, rows) * ((a.N + kCols - 1) / kCols); }

// Rows of a tile, by the groups' mean.
inline int tile_rows(const Int4Args& a) { return a.R <= 8 * (int64_t)a.G ? 16 : a.R <= 24 * (int64_t)a.G ? 32 : 64; }

// Parts of the contraction: enough for two workgroups to a compute unit, of four stages at least.
inline int parts_of(const Int4Args& a) {
  const int64_t tiles = most_tiles(a, tile_rows(a));
  const int stages = (a.K + kStage - 1) / kStage;
  int parts = 1;
  while (parts < 16 && 2 * parts * tiles <= 512 && stages >= 8 * parts) parts *= 2;
  return parts;
}

template <int TY, int SPAN, int NR, bool S32>
hipError_t launch(const Int4Args& a, hipStream_t s) {
  constexpr int bytes = Shape<SPAN, NR>::ring * Shape<SPAN, NR>::bytes;
  static PerDeviceOnce once;
  hipError_t e = once.run([] { return hipFuncSetAttribute((const void*)int4_short_kernel<TY, SPAN, NR, S32>, hipFuncAttributeMaxDynamicSharedMemorySize, bytes); });
  if (e != hipSuccess) return e;
  const int64_t tiles = most_tiles(a, 16 * NR);
  int4_short_kernel<TY, SPAN, NR, S32><<<dim3((unsigned)(tiles * a.parts)), dim3(256), bytes, s>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess || a.parts == 1) return e;
  int4_join_kernel<TY, 16 * NR><<<dim3((unsigned)tiles, 2 * NR), dim3(256), 0, s>>>(a);
  return hipGetLastError();
}
template <int TY, int SPAN, int NR>
hipError_t launch_scale(const Int4Args& a, hipStream_t s) {
  return a.scale_type == kElemF32 ? launch<TY, SPAN, NR, true>(a, s) : launch<TY, SPAN, NR, false>(a, s);
}
template <int TY, int SPAN>
hipError_t launch_rows(const Int4Args& a, hipStream_t s) {
  const int rows = tile_rows(a);
  return rows == 16 ? launch_scale<TY, SPAN, 1>(a, s) : rows == 32 ? launch_scale<TY, SPAN, 2>(a, s) : launch_scale<TY, SPAN, 4>(a, s);
}
template <int TY>
hipError_t launch_type(const Int4Args& a, hipStream_t s) {
  return a.shift == 5 ? launch_rows<TY, 32>(a, s) : a.shift == 6 ? launch_rows<TY, 64>(a, s) : launch_rows<TY, 128>(a, s);
}

}  // namespace

bool int4_short_fits(const Int4Args& a) {
  const int64_t most = (int64_t)1 << 22;
  if (a.type == kElemF32 || a.K % 8 != 0 || a.N % 8 != 0) return false;
  if ((((uintptr_t)a.x | a.x_row | (uintptr_t)a.y | a.y_row | (uintptr_t)a.w | a.w_row | a.w_group) & 15) != 0) return false;
  return a.x_row <= most && a.w_row <= most && a.s_row * 4 <= most && (!a.zero || a.z_row <= most);
}
size_t int4_short_bytes(const Int4Args& a) {
  const int rows = tile_rows(a), parts = parts_of(a);
  return parts == 1 ? 0 : (size_t)(most_tiles(a, rows) * parts) * (rows * kCols * 4);
}
hipError_t launch_int4_short(Int4Args a, hipStream_t s) {
  a.parts = a.partial != nullptr ? parts_of(a) : 1;
  return a.type == kElemBF16 ? launch_type<kElemBF16>(a, s) : launch_type<kElemF16>(a, s);
}

}  // namespace dsmoe
