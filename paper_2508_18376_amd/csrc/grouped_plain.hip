// Products over groups of rows, for every type, alignment and stride: the path of operands whose rows do not start on 16 bytes, and
// of fp32.  C tile of 128 x 128 a workgroup of 4 wavefronts (2 x 2, 64 x 64 each), 128 bytes of the contraction a stage, staged through
// registers into two LDS buffers, so that the next stage's loads are in flight under this stage's matrix instructions.
// fp32 products are exact fp32 (v_mfma_f32_32x32x2_f32), 8-bit ones exact int32, 16-bit ones accumulate in fp32.
#include "grouped.h"

namespace dsmoe {

namespace {

typedef __bf16 pbf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 pf16x8 __attribute__((ext_vector_type(8)));
typedef short ps16x4 __attribute__((ext_vector_type(4)));
typedef int pi32x4 __attribute__((ext_vector_type(4)));
typedef float pf32x4 __attribute__((ext_vector_type(4)));
typedef float pf32x16 __attribute__((ext_vector_type(16)));
typedef int pi32x16 __attribute__((ext_vector_type(16)));

constexpr int kPT = 128;                // tile edge
constexpr int kStageK = 128;            // bytes of the contraction a stage
constexpr int kTileBytes = kPT * kStageK;
constexpr int kChunks = kTileBytes / 16 / 256;  // of a thread, operand and stage

template <int TY>
struct Elem {
  static constexpr int bytes = TY == kElemF32 ? 4 : TY == kElemI8 ? 1 : 2;
  static constexpr int per_chunk = 16 / bytes;
  static constexpr int k_stage = kStageK / bytes;
};

// n (<= 16 / SZ) values from p, zeros behind them; `before`: values of the row in front of p.  p has the alignment of a value only: a whole
// chunk is one 16-byte load wherever it starts (unaligned access is on for global memory), and so is a part of one, loaded up to its end and
// shifted down (value by value the last column tile of 2047 columns held up all others: 4096 rows in 4 groups of 2047 x 2047 took 200 us for y = x W and
// 246 for dW, 109 and 85 once it was loaded like this).  Only rows
// shorter than a chunk are loaded value by value.
template <int SZ>
__device__ __forceinline__ pi32x4 load_chunk(const char* p, int n, int before) {
  constexpr int FULL = 16 / SZ;
  pi32x4 v = {0, 0, 0, 0};
  if (n <= 0) return v;
  const int missing = n < FULL ? FULL - n : 0;
  if (missing <= before) {
    __builtin_memcpy(&v, p - missing * SZ, 16);
    if (missing) {
      const int bits = missing * SZ * 8;
      uint64_t lo, hi;
      __builtin_memcpy(&lo, &v, 8);
      __builtin_memcpy(&hi, (char*)&v + 8, 8);
      const uint64_t l = bits < 64 ? lo >> bits | hi << 1 << (63 - bits) : hi >> (bits - 64), h = bits < 64 ? hi >> bits : 0;
      __builtin_memcpy(&v, &l, 8);
      __builtin_memcpy((char*)&v + 8, &h, 8);
    }
  } else {
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < FULL; ++i) {
      if (i >= n) continue;
      uint32_t e;
      if (SZ == 4) e = *(const uint32_t*)(p + 4 * i);
      if (SZ == 2) e = *(const uint16_t*)(p + 2 * i);
      if (SZ == 1) e = *(const uint8_t*)(p + i);
      w[i * SZ / 4] |= e << (i * SZ % 4 * 8);
    }
    v = pi32x4{(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
  }
  return v;
}

// One operand tile: 128 rows (rows or columns of C) by a stage of the contraction.
//   along   the values of a row lie along the contraction in memory: [128][128 bytes] in LDS, chunks rotated by the row (swz_wide)
//   across  the contraction strides over rows of memory: [k_stage][128 values] in LDS; 16-bit values are turned around by the transposing
//           LDS read, whose 16 lanes take 4 rows: their 64-byte blocks are rotated by the row so that the 4 rows lie in different banks
template <int TY, bool ACROSS>
struct Operand {
  using E = Elem<TY>;
  static constexpr int row_chunks = kPT * E::bytes / 16;  // across
  const char* p[kChunks];  // the thread's chunks of the next stage
  int64_t step;
  int first, column, edge, done;  // its first row (along) or contraction row (across), its values' place in the row; columns that exist (across)
  static constexpr int rows_apart = ACROSS ? 256 / row_chunks : 32;

  // origin: first value of the tile; across: of its first contraction row.  edge: rows (along) / columns (across) of the tile that exist;
  // before: columns in front of the tile (across)
  __device__ __forceinline__ void init(const char* origin, int64_t row_bytes, int edge_, int before) {
    const int t = threadIdx.x, ch = ACROSS ? t % row_chunks : t & 7;
    first = ACROSS ? t / row_chunks : t >> 3;
    column = ch * E::per_chunk;
    edge = ACROSS ? edge_ : kPT;
    done = ACROSS ? before : 0;
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {  // (along, rows past the last one: the last one again, whose products are not stored)
      const int r = first + i * rows_apart;
      p[i] = origin + (ACROSS ? r : min(r, edge_ - 1)) * row_bytes + ch * 16;
    }
    step = ACROSS ? row_bytes * E::k_stage : kStageK;
  }
  // the next stage; k_left: values of the contraction from the stage's start on
  __device__ __forceinline__ void load(pi32x4 (&v)[kChunks], int k_left) {
    if (edge == kPT && k_left >= E::k_stage) {  // (the same for all threads)
#pragma unroll
      for (int i = 0; i < kChunks; ++i) __builtin_memcpy(&v[i], p[i], 16);
    } else {
#pragma unroll
      for (int i = 0; i < kChunks; ++i)
        v[i] = load_chunk<E::bytes>(p[i], ACROSS ? (first + i * rows_apart < k_left ? edge - column : 0) : k_left - column, done + column);
    }
#pragma unroll
    for (int i = 0; i < kChunks; ++i) p[i] += step;
    if (!ACROSS) done += E::k_stage;
  }
  __device__ __forceinline__ void store(char* tile, const pi32x4 (&v)[kChunks]) const {
    const int ch = column / E::per_chunk;
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      const int r = first + i * rows_apart;
      *(pi32x4*)(tile + (ACROSS ? r * (kPT * E::bytes) + (E::bytes == 2 ? ch ^ ((r & 3) << 2) : ch) * 16 : r * kStageK + swz_wide(r, ch) * 16)) = v[i];
    }
  }
  // fragment of rows r0 .. r0 + 31 for substep s (a quarter of a stage): lane l holds row r0 + l % 32 and 16 bytes of the contraction
  static __device__ __forceinline__ pi32x4 read(const char* tile, int r0, int s, int lane) {
    const int r = r0 + (lane & 31), half = lane >> 5;
    if (!ACROSS) return *(const pi32x4*)(tile + r * kStageK + swz_wide(r, 2 * s + half) * 16);
    if (E::bytes == 4) {
      pi32x4 v;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = *(const int*)(tile + ((8 * s + 4 * half + j) * kPT + r) * 4);
      return v;
    }
    const int g = lane >> 4, i = lane & 15, col = r0 + 16 * (g & 1) + 4 * (i & 3);
    const int chunk = (col >> 3) ^ ((i >> 2) << 2);
    const char* q = tile + (16 * s + 8 * half + (i >> 2)) * (kPT * 2) + chunk * 16 + (col & 7) * 2;
    typedef __attribute__((address_space(3))) ps16x4* lp;
    const ps16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(uintptr_t)(uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)q);
    const ps16x4 hi =
        __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(uintptr_t)(uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)(q + 4 * kPT * 2));
    pi32x4 v;
    __builtin_memcpy(&v, &lo, 8);
    __builtin_memcpy((char*)&v + 8, &hi, 8);
    return v;
  }
};

template <int TY>
struct Acc {
  pf32x16 v;
  __device__ __forceinline__ void mac(const pi32x4& a, const pi32x4& b) {
    if (TY == kElemBF16) v = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(pbf16x8, a), __builtin_bit_cast(pbf16x8, b), v, 0, 0, 0);
    if (TY == kElemF16) v = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(pf16x8, a), __builtin_bit_cast(pf16x8, b), v, 0, 0, 0);
    if (TY == kElemF32) {  // lane half h holds contraction values 4h .. 4h + 3 of each 8: any order will do that both operands have
      const pf32x4 fa = __builtin_bit_cast(pf32x4, a), fb = __builtin_bit_cast(pf32x4, b);
#pragma unroll
      for (int j = 0; j < 4; ++j) v = __builtin_amdgcn_mfma_f32_32x32x2f32(fa[j], fb[j], v, 0, 0, 0);
    }
  }
  __device__ __forceinline__ float get(int i) const { return v[i]; }
};
template <>
struct Acc<kElemI8> {
  pi32x16 v;
  __device__ __forceinline__ void mac(const pi32x4& a, const pi32x4& b) { v = __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, v, 0, 0, 0); }
  __device__ __forceinline__ float get(int i) const { return (float)v[i]; }
};

// Where tile t of `width` columns that lie across the contraction begins: the last one ends with the columns, so that no stage of it has to watch for
// their end (its first columns are the tile's before it too, which come out the same).
__device__ __forceinline__ int last_tile(int t, int width) { return width >= kPT ? min(t * kPT, width - kPT) : 0; }

// DW: both operands across the contraction, which runs over the group's rows; else A along it, and B across (BX) or along.
template <int TY, bool BX, bool DW>
__global__ __launch_bounds__(256, 2) void grouped_plain_kernel(GroupedArgs g) {
  using E = Elem<TY>;
  __shared__ __align__(16) char lds[4 * kTileBytes];  // 64 KiB: two workgroups to a compute unit
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int NT = (g.N + kPT - 1) / kPT;
  int piece, m0, n0, m_edge, n_edge, K;
  int64_t c_row0 = 0;
  const char *pa, *pb;
  char* pc;
  const float* b_scale = nullptr;
  if (DW) {
    const int MT = (g.M + kPT - 1) / kPT;
    piece = blockIdx.x;
    const int grp = piece / (MT * NT), id = piece - grp * MT * NT;
    int mt, nt, row0;
    band_tile(id, MT, NT, mt, nt);
    Segments all;
    all.init(g.off, g.G, g.R);
    all.group(grp, row0, K);
    m0 = last_tile(mt, g.M);
    n0 = last_tile(nt, g.N);
    m_edge = min(kPT, g.M - m0);
    pa = g.a + (int64_t)row0 * g.a_row + (int64_t)m0 * E::bytes;
    pb = g.b + (int64_t)row0 * g.b_row + (int64_t)n0 * E::bytes;
    pc = g.c + grp * g.c_group;
  } else {
    Segment s;
    Segments all;
    all.init(g.off, g.G, g.R);
    all.zero_others(g.c, g.c_row, g.N * elem_bytes(TY == kElemI8 ? g.out_type : TY));
    if (!all.find(kPT, NT, [](int n) { return piece_of(blockIdx.x, n); }, piece, s)) return;
    int rt, nt;
    band_tile(piece - s.base, (s.rows + kPT - 1) / kPT, NT, rt, nt);
    m0 = rt * kPT;
    n0 = BX ? last_tile(nt, g.N) : nt * kPT;
    m_edge = min(kPT, s.rows - m0);
    K = g.K;
    const int grp = s.group;
    pa = g.a + (int64_t)(s.row0 + m0) * g.a_row;
    pb = g.b + grp * g.b_group + (BX ? (int64_t)n0 * E::bytes : n0 * g.b_row);
    pc = g.c;
    c_row0 = s.row0;
    if (TY == kElemI8) b_scale = g.b_scale + grp * g.bs_group;
  }
  n_edge = min(kPT, g.N - n0);

  Acc<TY> acc[2][2];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int q = 0; q < 16; ++q) acc[i >> 1][i & 1].v[q] = 0;

  if (K > 0) {
    Operand<TY, DW> oa;
    Operand<TY, BX || DW> ob;
    oa.init(pa, g.a_row, m_edge, m0);
    ob.init(pb, g.b_row, n_edge, n0);
    const int mw = (w & 1) * 64, nw = (w >> 1) * 64;
    // two stages are under way: while one is multiplied, the next one's loads have that time, and the one's behind it too
    pi32x4 va[2][kChunks], vb[2][kChunks];
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (i * E::k_stage < K) {
        oa.load(va[i], K - i * E::k_stage);
        ob.load(vb[i], K - i * E::k_stage);
      }
    for (int k = 0; k < K; k += 2 * E::k_stage) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int left = K - k - i * E::k_stage;
        if (left <= 0) break;
        char *ta = lds + i * 2 * kTileBytes, *tb = ta + kTileBytes;
        oa.store(ta, va[i]);
        ob.store(tb, vb[i]);
        __syncthreads();  // (this buffer's last readers passed the barrier of the stage before)
        if (left > 2 * E::k_stage) {
          oa.load(va[i], left - 2 * E::k_stage);
          ob.load(vb[i], left - 2 * E::k_stage);
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          pi32x4 fa[2], fb[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            fa[j] = oa.read(ta, mw + 32 * j, s, lane);
            fb[j] = ob.read(tb, nw + 32 * j, s, lane);
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[j >> 1][j & 1].mac(fb[j & 1], fa[j >> 1]);
        }
      }
    }
    __syncthreads();
  }

  // A lane holds row lane % 32 of the block and, for q = 0 .. 3, the four columns 8 q + 4 (lane / 32) ..: a wavefront turns 32 rows of its 64 columns
  // around in LDS and stores them 16 bytes a lane (straight from the registers, 8 bytes of a row each, a dW of 33 x 1001 x 1409 took 81 us instead of 50).
  const int out = TY == kElemI8 ? g.out_type : TY, ob = elem_bytes(out);
  char* turn = lds + w * (32 * 272);
  const int r32 = lane & 31, mw = (w & 1) * 64, nw = (w >> 1) * 64, per16 = 16 / ob, lanes = 64 / per16;  // lanes of a row
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = mw + i * 32 + r32;
    const float as = TY == kElemI8 && r < m_edge ? g.a_scale[c_row0 + m0 + r] : 1.f;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int c = j * 32 + 8 * q + 4 * (lane >> 5);
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[e] = acc[i][j].get(4 * q + e);
          if (TY == kElemI8) v[e] = nw + c + e < n_edge ? v[e] * as * b_scale[n0 + nw + c + e] : 0.f;
        }
        if (out == kElemF32) {
          *(pf32x4*)(turn + r32 * 272 + c * 4) = pf32x4{v[0], v[1], v[2], v[3]};
        } else {
          uint2 h;
          h.x = (uint32_t)f32_to_16(v[0], out) | (uint32_t)f32_to_16(v[1], out) << 16;
          h.y = (uint32_t)f32_to_16(v[2], out) | (uint32_t)f32_to_16(v[3], out) << 16;
          *(uint2*)(turn + r32 * 272 + c * 2) = h;
        }
      }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const int c = nw + lane % lanes * per16;
    for (int r0 = 0; r0 < 32; r0 += 64 / lanes) {
      const int rr = r0 + lane / lanes;
      if (mw + i * 32 + rr >= m_edge || c >= n_edge) continue;
      const pi32x4 v = *(const pi32x4*)(turn + rr * 272 + (c - nw) * ob);
      char* to = pc + (c_row0 + m0 + mw + i * 32 + rr) * g.c_row + (int64_t)(n0 + c) * ob;
      if (c + per16 <= n_edge) {
        __builtin_memcpy(to, &v, 16);
      } else {
        const uint32_t words[4] = {(uint32_t)v[0], (uint32_t)v[1], (uint32_t)v[2], (uint32_t)v[3]};
#pragma unroll
        for (int e = 0; e < 7; ++e)
          if (c + e < n_edge) {
            if (ob == 4 && e < 3) ((uint32_t*)to)[e] = words[e & 3];
            if (ob == 2) ((uint16_t*)to)[e] = (uint16_t)(words[e >> 1] >> (16 * (e & 1)));
          }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

template <int TY, bool BX, bool DW>
hipError_t launch(const GroupedArgs& g, int64_t blocks, hipStream_t s) {
  if (blocks > 0) grouped_plain_kernel<TY, BX, DW><<<dim3((unsigned)blocks), dim3(256), 0, s>>>(g);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_grouped_plain(const GroupedArgs& g, int type, bool b_along, hipStream_t s) {
  const int64_t blocks = row_tiles_bound(g.R, g.G, g.off != nullptr, kPT) * ((g.N + kPT - 1) / kPT);
  switch (type) {
    case kElemF32: return b_along ? launch<kElemF32, false, false>(g, blocks, s) : launch<kElemF32, true, false>(g, blocks, s);
    case kElemBF16: return b_along ? launch<kElemBF16, false, false>(g, blocks, s) : launch<kElemBF16, true, false>(g, blocks, s);
    case kElemF16: return b_along ? launch<kElemF16, false, false>(g, blocks, s) : launch<kElemF16, true, false>(g, blocks, s);
    default: return launch<kElemI8, false, false>(g, blocks, s);
  }
}

hipError_t launch_grouped_dw_plain(const GroupedArgs& g, int type, hipStream_t s) {
  const int64_t blocks = (int64_t)g.G * ((g.M + kPT - 1) / kPT) * ((g.N + kPT - 1) / kPT);
  switch (type) {
    case kElemF32: return launch<kElemF32, true, true>(g, blocks, s);
    case kElemBF16: return launch<kElemBF16, true, true>(g, blocks, s);
    default: return launch<kElemF16, true, true>(g, blocks, s);
  }
}

}  // namespace dsmoe
