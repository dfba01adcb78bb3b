// Products over groups of rows, for every type, alignment and stride: the path of operands whose rows do not start on 16 bytes, and
// of fp32.  C tile of 128 x 128 a workgroup of 4 wavefronts (2 x 2, 64 x 64 each), 64 bytes of the contraction a stage, staged through
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
constexpr int kStageK = 64;             // bytes of the contraction a stage
constexpr int kTileBytes = kPT * kStageK;

template <int TY>
struct Elem {
  static constexpr int bytes = TY == kElemF32 ? 4 : TY == kElemI8 ? 1 : 2;
  static constexpr int per_chunk = 16 / bytes;
  static constexpr int k_stage = kStageK / bytes;
};

// n (<= 16 / SZ) values from p, zeros behind them.  p has the alignment of a value only: a whole chunk is one 16-byte load wherever it
// starts (unaligned access is on for global memory).
template <int SZ>
__device__ __forceinline__ pi32x4 load_chunk(const char* p, int n) {
  pi32x4 v = {0, 0, 0, 0};
  if (n >= 16 / SZ) {
    __builtin_memcpy(&v, p, 16);
  } else if (n > 0) {
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 16 / SZ; ++i) {
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
//   along   the values of a row lie along the contraction in memory: [128][64 bytes] in LDS, chunks rotated as everywhere (swz_chunk)
//   across  the contraction strides over rows of memory: [k_stage][128 values] in LDS; 16-bit values are turned around by the transposing
//           LDS read, whose 16 lanes take 4 rows: their 64-byte blocks are rotated by the row so that the 4 rows lie in different banks
template <int TY, bool ACROSS>
struct Operand {
  using E = Elem<TY>;
  static constexpr int row_chunks = kPT * E::bytes / 16;  // across
  const char* p[2];
  int lds[2], at[2], left[2];  // left: values of the chunk that exist (across)
  int64_t step;

  // origin: first value of the tile; across: of its first contraction row.  edge: rows (along) / columns (across) of the tile that exist
  __device__ __forceinline__ void init(const char* origin, int64_t row_bytes, int edge) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int c = threadIdx.x + i * 256;
      if (!ACROSS) {
        const int r = c >> 2, ch = c & 3;
        p[i] = origin + (int64_t)min(r, edge - 1) * row_bytes + ch * 16;
        at[i] = ch * E::per_chunk;
        left[i] = r < edge ? 1 : 0;
        lds[i] = r * kStageK + swz_chunk(r, ch) * 16;
      } else {
        const int r = c / row_chunks, ch = c % row_chunks;
        p[i] = origin + r * row_bytes + ch * 16;
        at[i] = r;
        left[i] = min(E::per_chunk, edge - ch * E::per_chunk);
        lds[i] = r * (kPT * E::bytes) + (E::bytes == 2 ? ch ^ ((r & 3) << 2) : ch) * 16;
      }
    }
    step = ACROSS ? row_bytes * E::k_stage : kStageK;
  }
  // the next stage; k_left: values of the contraction from the stage's start on
  __device__ __forceinline__ void load(pi32x4 (&v)[2], int k_left) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      v[i] = load_chunk<E::bytes>(p[i], ACROSS ? (at[i] < k_left ? left[i] : 0) : (left[i] ? k_left - at[i] : 0));
      p[i] += step;
    }
  }
  __device__ __forceinline__ void store(char* tile, const pi32x4 (&v)[2]) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) *(pi32x4*)(tile + lds[i]) = v[i];
  }
  // fragment of rows r0 .. r0 + 31 for substep s (half a stage): lane l holds row r0 + l % 32 and 16 bytes of the contraction
  static __device__ __forceinline__ pi32x4 read(const char* tile, int r0, int s, int lane) {
    const int r = r0 + (lane & 31), half = lane >> 5;
    if (!ACROSS) return *(const pi32x4*)(tile + r * kStageK + swz_chunk(r, 2 * s + half) * 16);
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

// n (1..4) values to p, which has the alignment of a value only
__device__ __forceinline__ void store4(char* p, const float (&v)[4], int n, int type) {
  if (type == kElemF32) {
    if (n >= 4)
      __builtin_memcpy(p, v, 16);
    else
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if (i < n) ((float*)p)[i] = v[i];
    return;
  }
  uint16_t h[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = f32_to_16(v[i], type);
  if (n >= 4) {
    __builtin_memcpy(p, h, 8);
  } else {
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (i < n) ((uint16_t*)p)[i] = h[i];
  }
}

// DW: both operands across the contraction, which runs over the group's rows; else A along it, and B across (BX) or along.
template <int TY, bool BX, bool DW>
__global__ __launch_bounds__(256, 2) void grouped_plain_kernel(GroupedArgs g) {
  using E = Elem<TY>;
  __shared__ __align__(16) char lds[4 * kTileBytes];
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
    group_rows(g.off, g.G, g.R, grp, row0, K);
    m0 = mt * kPT;
    n0 = nt * kPT;
    m_edge = min(kPT, g.M - m0);
    pa = g.a + (int64_t)row0 * g.a_row + (int64_t)m0 * E::bytes;
    pb = g.b + (int64_t)row0 * g.b_row + (int64_t)n0 * E::bytes;
    pc = g.c + grp * g.c_group;
  } else {
    Segment s;
    if (!find_segment(g.off, g.G, g.R, kPT, NT, [](int n) { return take_piece<false>(n, nullptr, nullptr); }, piece, s)) return;
    int rt, nt;
    band_tile(piece - s.base, (s.rows + kPT - 1) / kPT, NT, rt, nt);
    m0 = rt * kPT;
    n0 = nt * kPT;
    m_edge = min(kPT, s.rows - m0);
    K = s.group < 0 ? 0 : g.K;
    const int grp = max(s.group, 0);
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
    oa.init(pa, g.a_row, m_edge);
    ob.init(pb, g.b_row, n_edge);
    pi32x4 va[2], vb[2];
    oa.load(va, K);
    ob.load(vb, K);
    const int mw = (w & 1) * 64, nw = (w >> 1) * 64;
    int buf = 0;
    for (int k = 0; k < K; k += E::k_stage) {
      char *ta = lds + buf * 2 * kTileBytes, *tb = ta + kTileBytes;
      oa.store(ta, va);
      ob.store(tb, vb);
      __syncthreads();  // (the other buffer's readers passed it one stage ago)
      if (k + E::k_stage < K) {
        oa.load(va, K - k - E::k_stage);
        ob.load(vb, K - k - E::k_stage);
      }
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        pi32x4 fa[2], fb[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          fa[i] = oa.read(ta, mw + 32 * i, s, lane);
          fb[i] = ob.read(tb, nw + 32 * i, s, lane);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) acc[i][j].mac(fb[j], fa[i]);
      }
      buf ^= 1;
    }
  }

  // a lane holds row lane % 32 of the block and, for q = 0 .. 3, the four columns 8 q + 4 (lane / 32) ..
  const int out = TY == kElemI8 ? g.out_type : TY, ob = elem_bytes(out);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = (w & 1) * 64 + i * 32 + (lane & 31);
    if (r >= m_edge) continue;
    char* row = pc + (c_row0 + m0 + r) * g.c_row;
    const float as = TY == kElemI8 ? g.a_scale[c_row0 + m0 + r] : 1.f;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int c = (w >> 1) * 64 + j * 32 + 8 * q + 4 * (lane >> 5);
        if (c >= n_edge) continue;
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[e] = acc[i][j].get(4 * q + e);
          if (TY == kElemI8) v[e] = K > 0 ? v[e] * as * (c + e < n_edge ? b_scale[n0 + c + e] : 0.f) : 0.f;
        }
        store4(row + (int64_t)(n0 + c) * ob, v, n_edge - c, out);
      }
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
